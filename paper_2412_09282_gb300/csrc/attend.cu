// Attention over the paged 8-bit cache: o = sum_j p_j V_j / sum_j p_j with p_j = exp(scale q . K_j - max),
// K_j = c_j s^k, V_j = c'_j s^v (one scale per 16 tokens and head).
//
// Form. A warp takes one block of 16 tokens at a time: S^T (16 tokens x 8 columns) = K Q^T on
// mma.sync.m16n8k16 with the codes as the A operand, O^T += V^T P^T with V^T as A and the weights as
// B. A column is one (query token, query head) pair; a unit is up to 8 NT columns of one kv head, so
// query heads that share a kv head (and a few drafted tokens) share every code that is read. The
// contraction index of either product may be taken in any order, so each lane's operand pieces are
// chosen as 16 consecutive codes of one token row: the codes come straight from global memory in
// 16-byte loads, one block ahead, and become fp16 by byte permutes (int8: 1024 + code + 128, less
// 1152; exact) or by one conversion per pair (e4m3; exact).
//   The key scale multiplies the block's scores in fp32. The value scale multiplies the weights,
// relative to the largest scale so far (a power of two), so that a weight in fp16 is at most 2^14
// whatever the scales are; weights below 2^-38 of that vanish. Running maxima and sums are fp32. From
// fp32 queries both q and the weights are two fp16 operands each.
//
// Split. The work is every (sequence, kv head, column group)'s tiles of 64 tokens in one line, of which
// each CTA takes an equal share, whatever the lengths are: they are read on the device. A unit that
// lies within a share is written at once; the others' parts (maximum, sum, unnormalised output) go to
// scratch and are joined in order by a second kernel, so results do not depend on timing.
#include "cache.cuh"

#include "kernels.h"

namespace crvq {

namespace {

constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
// Blocks that a warp takes at a time (two: twice the independent work, and one maximum for both)
template <int D>
constexpr int kBlocks = D == 256 ? 1 : 2;
template <int D>
constexpr int kTile = kCacheBlock * kBlocks<D> * kWarps;  // tokens of a CTA at a time
constexpr float kWeight = 16384.f;           // weights are scaled into fp16's range
constexpr float kLog2e = 1.4426950408889634f;

// 2^x (within 2 ulp; results below 2^-126 are 0)
__device__ __forceinline__ float pow2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

struct AttendArgs {
  CacheView c;
  HeadsView q, o;
  RowsView rows;
  int group;        // query heads per kv head
  float scale;      // times log2(e)
  bool causal;
  int window;
  bool vec_q;
  float* lse;
  float* part;      // 2 slots per CTA: [cols][D] outputs, [cols] maxima, [cols] sums
  int shares;
  unsigned* err;
};

// A sequence's work.
struct Seq {
  int len, n;       // tokens in the cache, queries
  int64_t first;    // first query row
  int lo, tiles;    // tiles that some query sees (at least one, so that outputs are written)
  int groups;       // column groups
};

template <int D, int COLS>
__device__ __forceinline__ Seq load_seq(const AttendArgs& a, int b) {
  Seq s;
  seq_rows(a.rows, b, &s.first, &s.n, a.err);
  s.len = seq_len(a.c, b, a.err);
  const int begin = a.window > 0 ? max(0, s.len - s.n - a.window + 1) : 0;
  s.lo = min(begin, s.len) / kTile<D>;
  s.tiles = max(1, (s.len + kTile<D> - 1) / kTile<D> - s.lo);
  s.groups = (int)(((int64_t)s.n * a.group + COLS - 1) / COLS);
  return s;
}

struct Unit {
  Seq s;
  int b, h, cg;
  int tile;         // of the position that was looked for
  int64_t begin;    // the unit's first tile in the line
};

// Tiles of all units (warp-wide).
template <int D, int COLS>
__device__ int64_t total_tiles(const AttendArgs& a) {
  const int lane = threadIdx.x & 31;
  int64_t sum = 0;
  for (int b = lane; b < a.c.n_seq; b += 32) {
    const Seq s = load_seq<D, COLS>(a, b);
    sum += (int64_t)s.groups * s.tiles;
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  return sum * a.c.n_kv;
}

// The unit that holds position w of the line, 0 <= w < total (warp-wide).
template <int D, int COLS>
__device__ Unit locate(const AttendArgs& a, int64_t w) {
  const int lane = threadIdx.x & 31;
  int64_t base = 0;
  Unit u;
  u.b = 0;
  for (int b0 = 0; b0 < a.c.n_seq; b0 += 32) {
    int64_t cost = 0;
    if (b0 + lane < a.c.n_seq) {
      const Seq s = load_seq<D, COLS>(a, b0 + lane);
      cost = (int64_t)s.groups * s.tiles * a.c.n_kv;
    }
    int64_t incl = cost;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int64_t v = __shfl_up_sync(0xffffffffu, incl, d);
      if (lane >= d) incl += v;
    }
    const unsigned hit = __ballot_sync(0xffffffffu, base + incl > w);
    if (hit) {
      const int src = __ffs(hit) - 1;
      base += __shfl_sync(0xffffffffu, incl - cost, src);
      u.b = b0 + src;
      break;
    }
    base += __shfl_sync(0xffffffffu, incl, 31);
  }
  u.s = load_seq<D, COLS>(a, u.b);
  const int64_t rem = w - base;
  const int64_t idx = rem / u.s.tiles;
  u.tile = (int)(rem - idx * u.s.tiles);
  u.h = (int)(idx / u.s.groups);
  u.cg = (int)(idx - (int64_t)u.h * u.s.groups);
  u.begin = w - u.tile;
  return u;
}

__device__ __forceinline__ int64_t share_begin(int64_t total, int i, int shares) {
  return total * i / shares;
}

__device__ __forceinline__ void mma_f16(float d[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                        uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
      "{%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

// Codes 0, 1 (half 0) or 2, 3 (half 1) of a word as fp16.
template <int FMT, int HALF>
__device__ __forceinline__ uint32_t codes2(uint32_t w) {
  if constexpr (FMT == CRVQ_KV_INT8) {
    const uint32_t u = __byte_perm(w ^ 0x80808080u, 0x64646464u, HALF ? 0x4342 : 0x4140);
    const __half2 v = __hsub2(*reinterpret_cast<const __half2*>(&u), __half2half2(__ushort_as_half(0x6480)));
    return *reinterpret_cast<const uint32_t*>(&v);
  } else {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)(HALF ? w >> 16 : w)));
    return r;
  }
}

__device__ __forceinline__ uint32_t half2_bits(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// a - fp16(a) for the pair, as fp16
__device__ __forceinline__ uint32_t half2_rest(float a, float b, uint32_t hi) {
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&hi));
  return half2_bits(a - f.x, b - f.y);
}

__device__ __forceinline__ int word(const uint4& u, int i) {
  return i == 0 ? u.x : i == 1 ? u.y : i == 2 ? u.z : u.w;
}

// The pieces of one block that a lane needs: K rows key_row and key_row + 8 (16 codes from every 64), V rows
// 2 tig, 2 tig + 1, + 8, + 9 (16 codes, 8 of 64). Every lane copies its own pieces to shared memory,
// piece by piece with the lanes side by side: no bank conflicts, and no lane waits for another's copy.
template <int D>
struct Pieces {
  static constexpr int kChunks = D / 64;                  // 16-byte pieces of a key row
  static constexpr int kKeys = 2 * kChunks;
  static constexpr int kValues = D == 64 ? 2 : D / 32;    // 16-byte units: D = 64 has two 8-byte pieces in one
  static constexpr int kBytes = (kKeys + kValues) * 512;  // of a warp and block
};

__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy8(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(src) : "memory");
}

// Starts the copies of the block whose codes begin at byte `at` of K and V; dst: this warp's stage.
template <int D>
__device__ __forceinline__ void start_block(const CacheView& c, int64_t at, uint32_t dst) {
  const int lane = threadIdx.x & 31, gid = lane >> 2, tig = lane & 3;
  const uint8_t* k = c.K + at + gid * D + 16 * tig;
  dst += lane * 16;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < Pieces<D>::kChunks; ++j) copy16(dst + (i * Pieces<D>::kChunks + j) * 512, k + 8 * i * D + 64 * j);
  dst += Pieces<D>::kKeys * 512;
  const uint8_t* v = c.V + at + 2 * tig * D + (D == 64 ? 8 : 16) * gid;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint8_t* row = v + ((i & 1) + 8 * (i >> 1)) * D;
    if constexpr (D == 64) {
      copy8(dst + (i >> 1) * 512 + (i & 1) * 8, row);
    } else {
#pragma unroll
      for (int j = 0; j < D / 128; ++j) copy16(dst + (i * (D / 128) + j) * 512, row + 128 * j);
    }
  }
}

template <int D, int NT, int FMT, bool SPLIT>
struct Shape {
  static constexpr int kCols = 8 * NT;
  static constexpr int kQRow = D + 8;  // halves per query row, padded against bank conflicts
  static constexpr size_t kQ = (size_t)kCols * kQRow * 2 * (SPLIT ? 2 : 1);
  // the ring of blocks on their way; at a unit's end each warp's outputs [kCols][D] lie in its own part
  static constexpr int kStages = D == 128 ? 2 : 3;
  static constexpr int kRing = Pieces<D>::kBytes * kBlocks<D> * kStages;
  static_assert(kRing >= kCols * D * 4, "outputs fit the ring");
  static constexpr size_t kSmem = kQ + (size_t)kWarps * kRing + 3 * kCols * 4 + 3 * kWarps * kCols * 4;
  // CTAs per SM, by registers (128 threads of 128 or 168) and shared memory
  static constexpr int kPerSm = D == 64 ? (NT == 1 ? 4 : 3) : (D == 128 ? 3 : 2);
  static constexpr int kSlot = kCols * (D + 2);  // floats of a part
};

template <int D, int NT, int FMT, bool SPLIT>
__global__ void __launch_bounds__(kThreads, Shape<D, NT, FMT, SPLIT>::kPerSm)
attend_kernel(const __grid_constant__ AttendArgs a) {
  using S = Shape<D, NT, FMT, SPLIT>;
  constexpr int COLS = S::kCols;
  extern __shared__ __align__(16) char sm[];
  __half* q_s = reinterpret_cast<__half*>(sm);                       // [split][COLS][kQRow]
  char* ring = sm + S::kQ;                                           // [kWarps][kStages][pieces][lane]
  float* f_s = reinterpret_cast<float*>(ring + kWarps * S::kRing);   // [COLS] score factor
  int* beg_s = reinterpret_cast<int*>(f_s + COLS);                   // [COLS] first and last + 1 key seen
  int* end_s = beg_s + COLS;
  float* m_s = reinterpret_cast<float*>(end_s + COLS);               // [kWarps][COLS]
  float* l_s = m_s + kWarps * COLS;
  float* r_s = l_s + kWarps * COLS;                                  // value reference of a warp
  pdl_wait();  // (no early trigger: waiting blocks of the next kernels would take this one's places)
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, gid = lane >> 2, tig = lane & 3;
  const int64_t total = total_tiles<D, COLS>(a);
  const int shares = (int)min((int64_t)a.shares, total);
  if ((int)blockIdx.x >= shares) return;
  const int64_t w1 = share_begin(total, blockIdx.x + 1, shares);
  char* mine = ring + warp * S::kRing;
  const uint32_t mine_u = (uint32_t)__cvta_generic_to_shared(mine);

  for (int64_t w = share_begin(total, blockIdx.x, shares); w < w1;) {
    const Unit u = locate<D, COLS>(a, w);
    const int64_t unit_end = u.begin + u.s.tiles;
    const int t_end = (int)(min(unit_end, w1) - u.begin);
    const int len = u.s.len, group = a.group;
    const int col0 = u.cg * COLS, n_cols = min(COLS, u.s.n * group - col0);
    __syncthreads();  // the previous unit's shared memory has been read

    // A lane looks up the place and the scales of every 32nd of this warp's blocks; the copies of
    // kStages - 1 blocks are on their way ahead of the one in work.
    const int reach = u.s.len - u.s.n + (col0 + n_cols - 1) / group + 1;  // past the last column's place
    const int some_e = a.causal ? min(len, reach) : len;
    const int some_b = a.window > 0 ? max(0, len - u.s.n + col0 / group - a.window + 1) : 0;
    int64_t at_l = -1;
    float sk_l = 0.f, sv_l = 0.f, sk_old = 0.f, sv_old = 0.f;
    uint32_t has = 0, has_old = 0;  // blocks of the present 32 and of those before that some query sees
    constexpr int NB = kBlocks<D>;
    auto start = [&](int i) {       // the warp's i-th blocks NB i .., counted from the part's first tile
      if (u.tile + i < t_end) {
        const int i0 = i * NB;
        if ((i0 & 31) == 0) {
          sk_old = sk_l;
          sv_old = sv_l;
          has_old = has;
          const int tl = u.tile + (i0 + lane) / NB;
          const int tok = (u.s.lo + tl) * kTile<D> + (warp * NB + lane % NB) * kCacheBlock;
          at_l = -1;
          if (tl < t_end && tok < some_e && tok + kCacheBlock > some_b) {
            const int64_t page = seq_page(a.c, u.b, tok / a.c.page, a.err);
            if (page >= 0) {
              const int in = tok % a.c.page;
              at_l = page * a.c.page_stride + ((int64_t)u.h * a.c.page + in) * D;
              const int64_t at_s = (page * a.c.n_kv + u.h) * (a.c.page / kCacheBlock) + in / kCacheBlock;
              sk_l = __ldg(a.c.ks + at_s);
              sv_l = __ldg(a.c.vs + at_s);
            }
          }
          has = __ballot_sync(0xffffffffu, at_l >= 0);
        }
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          const int64_t at = __shfl_sync(0xffffffffu, at_l, (i0 + b) & 31);
          if (at >= 0) start_block<D>(a.c, at, mine_u + ((i % S::kStages) * NB + b) * Pieces<D>::kBytes);
        }
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int i = 0; i < S::kStages - 1; ++i) start(i);

    // queries: a warp per column, relative to the power of two at its largest element
    for (int col = warp; col < COLS; col += kWarps) {
      float x[D / 32];
      float top = 0.f;
      const int j = (col0 + col) / group, h = u.h * group + (col0 + col) % group;
#pragma unroll
      for (int e = 0; e < D / 32; ++e) {
        x[e] = col < n_cols ? load_elem(a.q.data, (u.s.first + j) * a.q.ld_tok + h * a.q.ld_head + lane + 32 * e,
                                        a.q.type)
                            : 0.f;
        top = fmaxf(top, fabsf(x[e]));
      }
      top = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top)));
      // 2^-e for a top in [2^e, 2^(e + 1)); 1 for zeros, subnormals and infinities
      const uint32_t ex = __float_as_uint(top) >> 23;
      const bool plain = ex == 0 || ex == 255;
      const float inv = plain ? 1.f : __uint_as_float(ex == 254 ? 0x00400000u : (254u - ex) << 23);
      const float back = plain ? 1.f : __uint_as_float(ex << 23);
#pragma unroll
      for (int e = 0; e < D / 32; ++e) {
        const float v = x[e] * inv;
        const __half hi = __float2half_rn(v);
        q_s[col * S::kQRow + lane + 32 * e] = hi;
        if constexpr (SPLIT)
          q_s[(COLS + col) * S::kQRow + lane + 32 * e] = __float2half_rn(v - __half2float(hi));
      }
      if (lane == 0) {
        f_s[col] = back * a.scale;
        const int pos = len - u.s.n + j;
        beg_s[col] = a.window > 0 ? max(0, pos - a.window + 1) : 0;
        end_s[col] = a.causal ? min(len, pos + 1) : len;
      }
    }
    __syncthreads();
    float f[NT][2];
    int kb[NT][2], ke[NT][2];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        f[t][e] = f_s[8 * t + 2 * tig + e];
        kb[t][e] = beg_s[8 * t + 2 * tig + e];
        ke[t][e] = end_s[8 * t + 2 * tig + e];
      }
    // keys that every column sees (positions do not fall from column to column)
    const int every_b = beg_s[n_cols - 1], every_e = end_s[0];

    float o[D / 16][NT][4];
    float m[NT][2], l[NT][2], ref = 0.f, inv_ref = 0.f;
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[i][t][e] = 0.f;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        m[t][e] = -INFINITY;
        l[t][e] = 0.f;
      }

    const int n_tiles = t_end - u.tile;
    for (int i = 0; i < n_tiles; ++i) {
      start(i + S::kStages - 1);
      asm volatile("cp.async.wait_group %0;" ::"n"(S::kStages - 1) : "memory");
      const bool old = (i * NB >> 5) != (min(i + S::kStages - 1, n_tiles - 1) * NB >> 5);
      const uint32_t live = (old ? has_old : has) >> (i * NB & 31);
      if ((live & ((1u << NB) - 1)) == 0) continue;
      float sk[NB], sv[NB];
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        sk[b] = __shfl_sync(0xffffffffu, old ? sk_old : sk_l, (i * NB + b) & 31);
        sv[b] = __shfl_sync(0xffffffffu, old ? sv_old : sv_l, (i * NB + b) & 31);
      }
      const int tok = (u.s.lo + u.tile + i) * kTile<D> + warp * NB * kCacheBlock;
      const uint4* stage = reinterpret_cast<const uint4*>(mine + (i % S::kStages) * NB * Pieces<D>::kBytes) + lane;
      constexpr int kUnits = Pieces<D>::kBytes / 16;

      float s[NB][NT][4];
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[b][n][e] = 0.f;
#pragma unroll
      for (int j = 0; j < D / 64; ++j) {
        uint32_t qv[SPLIT ? 2 : 1][NT][8];
#pragma unroll
        for (int z = 0; z < (SPLIT ? 2 : 1); ++z)
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            const uint4* p = reinterpret_cast<const uint4*>(
                q_s + (z * COLS + 8 * n + gid) * S::kQRow + 64 * j + 16 * tig);
            const uint4 x = p[0], y = p[1];
            qv[z][n][0] = x.x; qv[z][n][1] = x.y; qv[z][n][2] = x.z; qv[z][n][3] = x.w;
            qv[z][n][4] = y.x; qv[z][n][5] = y.y; qv[z][n][6] = y.z; qv[z][n][7] = y.w;
          }
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          const uint4 k0 = stage[b * kUnits + j * 32], k1 = stage[b * kUnits + (D / 64 + j) * 32];
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const uint32_t x = word(k0, w), y = word(k1, w);
            const uint32_t a0 = codes2<FMT, 0>(x), a2 = codes2<FMT, 1>(x);
            const uint32_t a1 = codes2<FMT, 0>(y), a3 = codes2<FMT, 1>(y);
#pragma unroll
            for (int z = 0; z < (SPLIT ? 2 : 1); ++z)
#pragma unroll
              for (int n = 0; n < NT; ++n) mma_f16(s[b][n], a0, a1, a2, a3, qv[z][n][2 * w], qv[z][n][2 * w + 1]);
          }
        }
      }
      // scores in units of log2, masked (a block that no query sees: all of it); their maxima
      const bool whole = tok >= every_b && tok + NB * kCacheBlock <= every_e && (live & ((1u << NB) - 1)) == (1u << NB) - 1;
      float top[NT][2];
      bool grew = false;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float v = -INFINITY;
#pragma unroll
          for (int b = 0; b < NB; ++b) {
            const float g = f[n][e] * sk[b];
            s[b][n][e] *= g;
            s[b][n][e + 2] *= g;
            if (!whole) {
              const int t0 = tok + b * kCacheBlock + gid;
              const bool in = live >> b & 1;
              if (!in || t0 < kb[n][e] || t0 >= ke[n][e]) s[b][n][e] = -INFINITY;
              if (!in || t0 + 8 < kb[n][e] || t0 + 8 >= ke[n][e]) s[b][n][e + 2] = -INFINITY;
            }
            v = fmaxf(v, fmaxf(s[b][n][e], s[b][n][e + 2]));
          }
          v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 4));
          v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 8));
          v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 16));
          top[n][e] = v;
          grew = grew || v > m[n][e];
        }
      float sv_top = 0.f;
#pragma unroll
      for (int b = 0; b < NB; ++b)
        if (live >> b & 1) sv_top = fmaxf(sv_top, sv[b]);
      if (sv_top > ref || __any_sync(0xffffffffu, grew)) {
        float r = 1.f;
        if (sv_top > ref) {
          // the power of two at or above, within 2^-110 .. 2^127 (its reciprocal times kWeight is finite)
          const float up = fmaxf(__uint_as_float(min((__float_as_uint(sv_top) + 0x7fffffu) & 0x7f800000u,
                                                     0x7f000000u)), 7.7037197775489434e-34f);
          r = ref / up;
          ref = up;
          inv_ref = 1.f / up * kWeight;
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float mn = fmaxf(m[n][e], top[n][e]);
            const float fac = m[n][e] == mn ? 1.f : pow2(m[n][e] - mn);
            m[n][e] = mn;
            l[n][e] *= fac;
#pragma unroll
            for (int d = 0; d < D / 16; ++d) {
              o[d][n][e] *= fac * r;
              o[d][n][e + 2] *= fac * r;
            }
          }
      }
      uint32_t pb[NB][2][NT][2];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const float m0 = m[n][0] == -INFINITY ? 0.f : m[n][0], m1 = m[n][1] == -INFINITY ? 0.f : m[n][1];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          const float wv = sv[b] * inv_ref;
          float p0 = pow2(s[b][n][0] - m0), p1 = pow2(s[b][n][1] - m1);
          float p2 = pow2(s[b][n][2] - m0), p3 = pow2(s[b][n][3] - m1);
          l[n][0] += p0 + p2;
          l[n][1] += p1 + p3;
          p0 *= wv; p1 *= wv; p2 *= wv; p3 *= wv;
          const uint32_t h0 = half2_bits(p0, p1), h1 = half2_bits(p2, p3);
          pb[b][0][n][0] = transpose8(h0);
          pb[b][0][n][1] = transpose8(h1);
          pb[b][1][n][0] = transpose8(half2_rest(p0, p1, h0));
          pb[b][1][n][1] = transpose8(half2_rest(p2, p3, h1));
        }
      }
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        if (!(live >> b & 1)) continue;  // (its place in shared memory holds anything)
        const int t0 = tok + b * kCacheBlock;
        const uint4* stage_v = stage + b * kUnits + Pieces<D>::kKeys * 32;
#pragma unroll
        for (int j = 0; j < (D == 64 ? 1 : D / 128); ++j) {
          uint4 v[4];
          if constexpr (D == 64) {
            const uint4 x = stage_v[0], y = stage_v[32];
            v[0] = make_uint4(x.x, x.y, 0, 0);
            v[1] = make_uint4(x.z, x.w, 0, 0);
            v[2] = make_uint4(y.x, y.y, 0, 0);
            v[3] = make_uint4(y.z, y.w, 0, 0);
          } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = stage_v[(k * (D / 128) + j) * 32];
          }
          if (t0 + kCacheBlock > len) {  // places past the end hold anything: taken as codes of 0
#pragma unroll
            for (int k = 0; k < 4; ++k)
              if (t0 + 2 * tig + (k & 1) + 8 * (k >> 1) >= len) v[k] = make_uint4(0, 0, 0, 0);
          }
#pragma unroll
          for (int w = 0; w < (D == 64 ? 2 : 4); ++w) {
            // tokens 2 tig, 2 tig + 1 side by side, channel by channel; then + 8, + 9
            const uint32_t x0 = word(v[0], w), x1 = word(v[1], w);
            const uint32_t y0 = word(v[2], w), y1 = word(v[3], w);
            const uint32_t xl = __byte_perm(x0, x1, 0x5140), xh = __byte_perm(x0, x1, 0x7362);
            const uint32_t yl = __byte_perm(y0, y1, 0x5140), yh = __byte_perm(y0, y1, 0x7362);
            const uint32_t a0 = codes2<FMT, 0>(xl), a1 = codes2<FMT, 1>(xl);
            const uint32_t a2 = codes2<FMT, 0>(yl), a3 = codes2<FMT, 1>(yl);
            const uint32_t c0 = codes2<FMT, 0>(xh), c1 = codes2<FMT, 1>(xh);
            const uint32_t c2 = codes2<FMT, 0>(yh), c3 = codes2<FMT, 1>(yh);
            const int mt = 8 * j + 2 * w;
#pragma unroll
            for (int z = 0; z < 2; ++z)
#pragma unroll
              for (int n = 0; n < NT; ++n) {
                mma_f16(o[mt][n], a0, a1, a2, a3, pb[b][z][n][0], pb[b][z][n][1]);
                mma_f16(o[mt + 1][n], c0, c1, c2, c3, pb[b][z][n][0], pb[b][z][n][1]);
              }
          }
        }
      }
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncwarp();  // every lane has read its pieces: the ring takes the outputs
    float* o_s = reinterpret_cast<float*>(mine);

    // join the warps
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float v = l[n][e];
        v += __shfl_xor_sync(0xffffffffu, v, 4);
        v += __shfl_xor_sync(0xffffffffu, v, 8);
        v += __shfl_xor_sync(0xffffffffu, v, 16);
        const int col = 8 * n + 2 * tig + e;
        if (gid == 0) {
          m_s[warp * COLS + col] = m[n][e];
          l_s[warp * COLS + col] = v;
          r_s[warp * COLS + col] = ref;
        }
        float* row = o_s + col * D;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
          // m-tile i: channels 2 i and 2 i + 1 of the lane's piece
          const int d = D == 64 ? 8 * gid + 2 * i : 128 * (i / 8) + 16 * gid + 2 * (i % 8);
          *reinterpret_cast<float2*>(row + d) = make_float2(o[i][n][e], o[i][n][e + 2]);
        }
      }
    __syncthreads();
    const bool complete = w == u.begin && u.begin + t_end == unit_end;
    float* part = a.part + (int64_t)(2 * blockIdx.x + (w == u.begin ? 1 : 0)) * S::kSlot;
    for (int col = warp; col < n_cols; col += kWarps) {
      float M = -INFINITY, L = 0.f;
#pragma unroll
      for (int i = 0; i < kWarps; ++i) M = fmaxf(M, m_s[i * COLS + col]);
      const float mm = M == -INFINITY ? 0.f : M;
      float fac[kWarps];
#pragma unroll
      for (int i = 0; i < kWarps; ++i) {
        const float x = pow2(m_s[i * COLS + col] - mm);
        L += l_s[i * COLS + col] * x;
        fac[i] = x * r_s[i * COLS + col] * (1.f / kWeight);
      }
      const int j = (col0 + col) / group, h = u.h * group + (col0 + col) % group;
      const float inv = L > 0.f ? 1.f / L : (L == 0.f ? 0.f : L);
#pragma unroll
      for (int e = 0; e < D / 32; ++e) {
        const int d = lane + 32 * e;
        float v = 0.f;
#pragma unroll
        for (int i = 0; i < kWarps; ++i) v += reinterpret_cast<const float*>(ring + i * S::kRing)[col * D + d] * fac[i];
        if (complete)
          store_elem(a.o.data, (u.s.first + j) * a.o.ld_tok + h * a.o.ld_head + d, a.o.type, v * inv);
        else
          part[col * D + d] = v;
      }
      if (lane == 0) {
        if (!complete) {
          part[COLS * D + col] = M;
          part[COLS * D + COLS + col] = L;
        } else if (a.lse) {
          a.lse[(u.s.first + j) * a.q.heads + h] = L > 0.f ? (M + log2f(L)) / kLog2e : (L == 0.f ? -INFINITY : L);
        }
      }
    }
    w = u.begin + t_end;
  }
}

// Joins the parts of the unit that the boundary between shares blockIdx.x and blockIdx.x + 1 cuts, if
// it is the first that does: a warp per column, the parts in the order of the shares.
template <int D, int COLS>
__global__ void __launch_bounds__(32 * COLS)
attend_join_kernel(const __grid_constant__ AttendArgs a) {
  pdl_trigger();
  pdl_wait();
  const int lane = threadIdx.x & 31, col = threadIdx.x >> 5;
  const int64_t total = total_tiles<D, COLS>(a);
  const int shares = (int)min((int64_t)a.shares, total), i0 = blockIdx.x;
  if (i0 + 1 >= shares) return;
  const int64_t cut = share_begin(total, i0 + 1, shares);
  const Unit u = locate<D, COLS>(a, cut);
  if (u.begin == cut || u.begin < share_begin(total, i0, shares)) return;
  const int64_t end = u.begin + u.s.tiles;
  constexpr int kSlot = COLS * (D + 2);
  const int col0 = u.cg * COLS;
  if (col0 + col >= u.s.n * a.group) return;
  int n = 1;  // shares that hold a part
  while (i0 + n < shares && share_begin(total, i0 + n, shares) < end) ++n;
  // slot of part 0: the share's last unit; of the others: their first (the unit began before them)
  const float* part = a.part + (int64_t)2 * i0 * kSlot;
  float M = -INFINITY, L = 0.f, o[D / 32];
#pragma unroll
  for (int e = 0; e < D / 32; ++e) o[e] = 0.f;
  for (int p0 = 0; p0 < n; p0 += 32) {
    const int p = p0 + lane;
    const float* pl = part + (int64_t)(2 * p + (p == 0 ? 1 : 0)) * kSlot + COLS * D + col;
    const float mp = p < n ? pl[0] : -INFINITY, lp = p < n ? pl[COLS] : 0.f;
    float mn = fmaxf(M, mp);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) mn = fmaxf(mn, __shfl_xor_sync(0xffffffffu, mn, d));
    const float mm = mn == -INFINITY ? 0.f : mn;
    const float f = pow2(mp - mm), back = pow2(M - mm);
    float sum = lp * f;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    L = L * back + sum;
    M = mn;
#pragma unroll
    for (int e = 0; e < D / 32; ++e) o[e] *= back;
    const int k = min(32, n - p0);
#pragma unroll 8
    for (int q = 0; q < k; ++q) {
      const float fq = __shfl_sync(0xffffffffu, f, q);
      const float* src = part + (int64_t)(2 * (p0 + q) + (p0 + q == 0 ? 1 : 0)) * kSlot + col * D + lane;
#pragma unroll
      for (int e = 0; e < D / 32; ++e) o[e] += src[32 * e] * fq;
    }
  }
  const int j = (col0 + col) / a.group, h = u.h * a.group + (col0 + col) % a.group;
  const float inv = L > 0.f ? 1.f / L : (L == 0.f ? 0.f : L);
#pragma unroll
  for (int e = 0; e < D / 32; ++e)
    store_elem(a.o.data, (u.s.first + j) * a.o.ld_tok + h * a.o.ld_head + lane + 32 * e, a.o.type, o[e] * inv);
  if (lane == 0 && a.lse)
    a.lse[(u.s.first + j) * a.q.heads + h] = L > 0.f ? (M + log2f(L)) / kLog2e : (L == 0.f ? -INFINITY : L);
}

template <int D, int NT, int FMT, bool SPLIT>
crvq_status launch_attend(AttendArgs& a, cudaStream_t stream) {
  using S = Shape<D, NT, FMT, SPLIT>;
  auto kernel = attend_kernel<D, NT, FMT, SPLIT>;
  CRVQ_TRY(smem_limit((const void*)kernel, S::kSmem));
  a.shares = sm_count() * S::kPerSm;
  Scratch mem;
  CRVQ_TRY(mem.alloc((size_t)2 * a.shares * S::kSlot * sizeof(float), stream));
  a.part = mem.as<float>();
  ProfScope ps("cache_attention", stream, (double)a.rows.n_tok * a.q.heads * D);
  CRVQ_CUDA(launch_pdl(kernel, dim3((unsigned)a.shares), dim3(kThreads), S::kSmem, stream, a));
  CRVQ_LAUNCHED();
  CRVQ_CUDA(launch_pdl(attend_join_kernel<D, S::kCols>, dim3((unsigned)a.shares - 1), dim3(32 * S::kCols), 0, stream, a));
  CRVQ_LAUNCHED();
  return CRVQ_OK;
}

template <int D, int FMT, bool SPLIT>
crvq_status pick_columns(AttendArgs& a, cudaStream_t stream) {
  // 16 columns where a sequence has more than 8 (by the average: the rows' offsets are on the device)
  const bool wide = a.rows.n_tok * a.group > 8 * (int64_t)a.c.n_seq;
  if constexpr (D == 256)
    return launch_attend<D, 1, FMT, SPLIT>(a, stream);
  else
    return wide ? launch_attend<D, 2, FMT, SPLIT>(a, stream) : launch_attend<D, 1, FMT, SPLIT>(a, stream);
}

template <int D>
crvq_status pick_format(AttendArgs& a, int format, cudaStream_t stream) {
  const bool split = a.q.type == CRVQ_F32;
  if (format == CRVQ_KV_INT8)
    return split ? pick_columns<D, CRVQ_KV_INT8, true>(a, stream) : pick_columns<D, CRVQ_KV_INT8, false>(a, stream);
  return split ? pick_columns<D, CRVQ_KV_E4M3, true>(a, stream) : pick_columns<D, CRVQ_KV_E4M3, false>(a, stream);
}

crvq_status attention(const crvq_kv_cache* cache, const crvq_heads* q, int64_t n_tok, const int32_t* q_off,
                      float scale, int32_t causal, int32_t window, const crvq_heads* out, float* lse,
                      cudaStream_t stream) {
  AttendArgs a{};
  CRVQ_TRY(make_cache(cache, &a.c));
  const int D = cache->head_dim;
  CRVQ_TRY(make_rows(q_off, n_tok, a.c.n_seq, &a.rows));
  CRVQ_TRY(make_heads(q, "q", D, n_tok, &a.q));
  CRVQ_TRY(make_heads(out, "out", D, n_tok, &a.o));
  CRVQ_CHECK_ARG(a.q.heads == a.o.heads && a.q.type == a.o.type, "q and out differ in heads or type");
  CRVQ_CHECK_ARG(a.q.heads % a.c.n_kv == 0, "q->heads (%d) must be a multiple of n_kv (%d)", a.q.heads, a.c.n_kv);
  CRVQ_CHECK_ARG(window >= 0, "window must be >= 0");
  CRVQ_CHECK_ARG(scale == scale && fabsf(scale) <= 3.402823466e38f, "scale must be finite");
  CRVQ_CHECK_ARG(((uintptr_t)lse & 3u) == 0, "lse is not aligned");
  CRVQ_TRY(check_dev({{lse, "lse"}}));
  a.group = a.q.heads / a.c.n_kv;
  CRVQ_CHECK_ARG(n_tok * a.group < (int64_t)1 << 31, "too many queries in one call");
  if (n_tok == 0) return CRVQ_OK;
  a.scale = scale * kLog2e;
  a.causal = causal != 0;
  a.window = window < (1 << 30) ? window : (1 << 30);
  a.lse = lse;
  CRVQ_TRY(device_error_word(&a.err));
  if (D == 64) return pick_format<64>(a, cache->format, stream);
  if (D == 128) return pick_format<128>(a, cache->format, stream);
  return pick_format<256>(a, cache->format, stream);
}

}  // namespace

}  // namespace crvq

extern "C" {

crvq_status crvq_cache_attention(const crvq_kv_cache* cache, const crvq_heads* q, int64_t n_tok,
                                 const int32_t* q_off, float scale, int32_t causal, int32_t window,
                                 const crvq_heads* out, float* lse, crvq_stream_t stream) {
  CRVQ_ENTRY({
    return crvq::attention(cache, q, n_tok, q_off, scale, causal, window, out, lse, (cudaStream_t)stream);
  })
}

}  // extern "C"
