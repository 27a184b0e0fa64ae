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
constexpr int kTile = kCacheBlock * kWarps;  // tokens
constexpr float kWeight = 16384.f;           // weights are scaled into fp16's range
constexpr float kLog2e = 1.4426950408889634f;

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

template <int COLS>
__device__ __forceinline__ Seq load_seq(const AttendArgs& a, int b) {
  Seq s;
  seq_rows(a.rows, b, &s.first, &s.n, a.err);
  s.len = seq_len(a.c, b, a.err);
  const int begin = a.window > 0 ? max(0, s.len - s.n - a.window + 1) : 0;
  s.lo = min(begin, s.len) / kTile;
  s.tiles = max(1, (s.len + kTile - 1) / kTile - s.lo);
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
template <int COLS>
__device__ int64_t total_tiles(const AttendArgs& a) {
  const int lane = threadIdx.x & 31;
  int64_t sum = 0;
  for (int b = lane; b < a.c.n_seq; b += 32) {
    const Seq s = load_seq<COLS>(a, b);
    sum += (int64_t)s.groups * s.tiles;
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  return sum * a.c.n_kv;
}

// The unit that holds position w of the line, 0 <= w < total (warp-wide).
template <int COLS>
__device__ Unit locate(const AttendArgs& a, int64_t w) {
  const int lane = threadIdx.x & 31;
  int64_t base = 0;
  Unit u;
  u.b = 0;
  for (int b0 = 0; b0 < a.c.n_seq; b0 += 32) {
    int64_t cost = 0;
    if (b0 + lane < a.c.n_seq) {
      const Seq s = load_seq<COLS>(a, b0 + lane);
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
  u.s = load_seq<COLS>(a, u.b);
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

// Codes of one block that a lane holds: K rows gid and gid + 8, V rows 2 tig, 2 tig + 1, + 8, + 9.
template <int D>
struct BlockRegs {
  static constexpr int kChunks = D / 64;                // 16-byte pieces of a key row per lane
  static constexpr int kPieces = D >= 128 ? D / 128 : 1;  // 16-byte (D = 64: 8-byte) pieces of a value row
  uint4 k[2][kChunks];
  uint4 v[4][kPieces];
};

template <int D>
__device__ __forceinline__ void load_block(const CacheView& c, int64_t at, BlockRegs<D>& r) {
  const int lane = threadIdx.x & 31, gid = lane >> 2, tig = lane & 3;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < BlockRegs<D>::kChunks; ++j)
      r.k[i][j] = __ldg(reinterpret_cast<const uint4*>(c.K + at + (gid + 8 * i) * D + 64 * j + 16 * tig));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint8_t* row = c.V + at + (2 * tig + (i & 1) + 8 * (i >> 1)) * D;
#pragma unroll
    for (int j = 0; j < BlockRegs<D>::kPieces; ++j) {
      if constexpr (D == 64) {
        const uint2 u = __ldg(reinterpret_cast<const uint2*>(row + 8 * gid));
        r.v[i][j] = make_uint4(u.x, u.y, 0, 0);
      } else {
        r.v[i][j] = __ldg(reinterpret_cast<const uint4*>(row + 128 * j + 16 * gid));
      }
    }
  }
}

template <int D, int NT, int FMT, bool SPLIT>
struct Shape {
  static constexpr int kCols = 8 * NT;
  static constexpr int kQRow = D + 8;  // halves per query row, padded against bank conflicts
  static constexpr size_t kQ = (size_t)kCols * kQRow * 2 * (SPLIT ? 2 : 1);
  static constexpr size_t kO = (size_t)kWarps * kCols * D * 4;
  static constexpr size_t kSmem = kQ + kO + 4 * kCols * 4 + 3 * kWarps * kCols * 4;
  static constexpr int kSlot = kCols * (D + 2);  // floats of a part
};

template <int D, int NT, int FMT, bool SPLIT>
__global__ void __launch_bounds__(kThreads)
attend_kernel(const __grid_constant__ AttendArgs a) {
  using S = Shape<D, NT, FMT, SPLIT>;
  constexpr int COLS = S::kCols;
  extern __shared__ __align__(16) char sm[];
  __half* q_s = reinterpret_cast<__half*>(sm);                       // [split][COLS][kQRow]
  float* o_s = reinterpret_cast<float*>(sm + S::kQ);                 // [kWarps][COLS][D]
  float* f_s = o_s + kWarps * COLS * D;                              // [COLS] score factor
  int* beg_s = reinterpret_cast<int*>(f_s + COLS);                   // [COLS] first and last + 1 key seen
  int* end_s = beg_s + COLS;
  float* m_s = reinterpret_cast<float*>(end_s + COLS) + COLS;        // [kWarps][COLS]
  float* l_s = m_s + kWarps * COLS;
  float* r_s = l_s + kWarps * COLS;                                  // value reference of a warp
  pdl_trigger();
  pdl_wait();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, gid = lane >> 2, tig = lane & 3;
  const int64_t total = total_tiles<COLS>(a);
  const int64_t w0 = share_begin(total, blockIdx.x, a.shares);
  const int64_t w1 = share_begin(total, blockIdx.x + 1, a.shares);

  for (int64_t w = w0; w < w1;) {
    const Unit u = locate<COLS>(a, w);
    const int64_t unit_end = u.begin + u.s.tiles;
    const int t_end = (int)(min(unit_end, w1) - u.begin);
    const int len = u.s.len, group = a.group;
    const int col0 = u.cg * COLS, n_cols = min(COLS, u.s.n * group - col0);
    __syncthreads();  // the previous unit's shared memory has been read
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
    // keys that some / every column sees (positions do not fall from column to column)
    const int some_b = beg_s[0], some_e = end_s[n_cols - 1];
    const int every_b = beg_s[n_cols - 1], every_e = end_s[0];

    float o[D / 16][NT][4];
    float m[NT][2], l[NT][2], ref = 0.f;
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

    // A lane looks up the place and the scales of every 32nd of this warp's blocks.
    int64_t at_l = -1;
    float sk_l = 0.f, sv_l = 0.f;
    auto look_up = [&](int t0) {
      const int t = t0 + lane;
      const int tok = (u.s.lo + t) * kTile + warp * kCacheBlock;
      at_l = -1;
      if (t < t_end && tok < some_e && tok + kCacheBlock > some_b) {
        const int64_t page = seq_page(a.c, u.b, tok / a.c.page, a.err);
        if (page >= 0) {
          const int in = tok % a.c.page;
          at_l = page * a.c.page_stride + ((int64_t)u.h * a.c.page + in) * D;
          const int64_t at_s = (page * a.c.n_kv + u.h) * (a.c.page / kCacheBlock) + in / kCacheBlock;
          sk_l = __ldg(a.c.ks + at_s);
          sv_l = __ldg(a.c.vs + at_s);
        }
      }
    };
    BlockRegs<D> cur, nxt;
    look_up(u.tile);
    int64_t at = __shfl_sync(0xffffffffu, at_l, 0);
    float sk = __shfl_sync(0xffffffffu, sk_l, 0), sv = __shfl_sync(0xffffffffu, sv_l, 0);
    if (at >= 0) load_block<D>(a.c, at, cur);
    for (int t = u.tile; t < t_end; ++t) {
      const int step = (t + 1 - u.tile) & 31;
      if (step == 0) look_up(t + 1);
      const int64_t at_n = t + 1 < t_end ? __shfl_sync(0xffffffffu, at_l, step) : -1;
      const float sk_n = __shfl_sync(0xffffffffu, sk_l, step), sv_n = __shfl_sync(0xffffffffu, sv_l, step);
      if (at_n >= 0) load_block<D>(a.c, at_n, nxt);
      if (at >= 0) {
        const int tok = (u.s.lo + t) * kTile + warp * kCacheBlock;
        float s[NT][4];
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[i][e] = 0.f;
#pragma unroll
        for (int j = 0; j < D / 64; ++j) {
          uint32_t qv[SPLIT ? 2 : 1][NT][8];
#pragma unroll
          for (int z = 0; z < (SPLIT ? 2 : 1); ++z)
#pragma unroll
            for (int i = 0; i < NT; ++i) {
              const uint4* p = reinterpret_cast<const uint4*>(
                  q_s + (z * COLS + 8 * i + gid) * S::kQRow + 64 * j + 16 * tig);
              const uint4 x = p[0], y = p[1];
              qv[z][i][0] = x.x; qv[z][i][1] = x.y; qv[z][i][2] = x.z; qv[z][i][3] = x.w;
              qv[z][i][4] = y.x; qv[z][i][5] = y.y; qv[z][i][6] = y.z; qv[z][i][7] = y.w;
            }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t x = word(cur.k[0][j], i), y = word(cur.k[1][j], i);
            const uint32_t a0 = codes2<FMT, 0>(x), a2 = codes2<FMT, 1>(x);
            const uint32_t a1 = codes2<FMT, 0>(y), a3 = codes2<FMT, 1>(y);
#pragma unroll
            for (int z = 0; z < (SPLIT ? 2 : 1); ++z)
#pragma unroll
              for (int n = 0; n < NT; ++n) mma_f16(s[n], a0, a1, a2, a3, qv[z][n][2 * i], qv[z][n][2 * i + 1]);
          }
        }
        // scores in units of log2, masked; the block's maxima
        const bool whole = tok >= every_b && tok + kCacheBlock <= every_e;
        float top[NT][2];
        bool grew = false;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float g = f[n][e] * sk;
            s[n][e] *= g;
            s[n][e + 2] *= g;
            if (!whole) {
              const int t0 = tok + gid;
              if (t0 < kb[n][e] || t0 >= ke[n][e]) s[n][e] = -INFINITY;
              if (t0 + 8 < kb[n][e] || t0 + 8 >= ke[n][e]) s[n][e + 2] = -INFINITY;
            }
            float v = fmaxf(s[n][e], s[n][e + 2]);
            v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 4));
            v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 8));
            v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 16));
            top[n][e] = v;
            grew = grew || v > m[n][e];
          }
        if (sv > ref || __any_sync(0xffffffffu, grew)) {
          const float old = ref;
          if (sv > ref) ref = __uint_as_float((__float_as_uint(sv) + 0x7fffffu) & 0x7f800000u);
          const float r = old == ref ? 1.f : old / ref;
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float mn = fmaxf(m[n][e], top[n][e]);
              const float fac = m[n][e] == mn ? 1.f : exp2f(m[n][e] - mn);
              m[n][e] = mn;
              l[n][e] *= fac;
#pragma unroll
              for (int i = 0; i < D / 16; ++i) {
                o[i][n][e] *= fac * r;
                o[i][n][e + 2] *= fac * r;
              }
            }
        }
        const float wv = ref > 0.f ? sv / ref * kWeight : 0.f;
        uint32_t pb[SPLIT ? 2 : 1][NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float p[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float mm = m[n][e & 1] == -INFINITY ? 0.f : m[n][e & 1];
            p[e] = exp2f(s[n][e] - mm);
          }
          l[n][0] += p[0] + p[2];
          l[n][1] += p[1] + p[3];
#pragma unroll
          for (int e = 0; e < 4; ++e) p[e] *= wv;
          const uint32_t h0 = half2_bits(p[0], p[1]), h1 = half2_bits(p[2], p[3]);
          pb[0][n][0] = transpose8(h0);
          pb[0][n][1] = transpose8(h1);
          if constexpr (SPLIT) {
            pb[1][n][0] = transpose8(half2_rest(p[0], p[1], h0));
            pb[1][n][1] = transpose8(half2_rest(p[2], p[3], h1));
          }
        }
        if (tok + kCacheBlock > len) {  // places past the end hold anything: as codes of 0
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (tok + 2 * tig + (i & 1) + 8 * (i >> 1) >= len)
#pragma unroll
              for (int j = 0; j < BlockRegs<D>::kPieces; ++j) cur.v[i][j] = make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int j = 0; j < BlockRegs<D>::kPieces; ++j)
#pragma unroll
          for (int i = 0; i < (D == 64 ? 2 : 4); ++i) {
            // tokens 2 tig, 2 tig + 1 side by side, channel by channel; then + 8, + 9
            const uint32_t x0 = word(cur.v[0][j], i), x1 = word(cur.v[1][j], i);
            const uint32_t y0 = word(cur.v[2][j], i), y1 = word(cur.v[3][j], i);
            const uint32_t xl = __byte_perm(x0, x1, 0x5140), xh = __byte_perm(x0, x1, 0x7362);
            const uint32_t yl = __byte_perm(y0, y1, 0x5140), yh = __byte_perm(y0, y1, 0x7362);
            const uint32_t a0 = codes2<FMT, 0>(xl), a1 = codes2<FMT, 1>(xl);
            const uint32_t a2 = codes2<FMT, 0>(yl), a3 = codes2<FMT, 1>(yl);
            const uint32_t c0 = codes2<FMT, 0>(xh), c1 = codes2<FMT, 1>(xh);
            const uint32_t c2 = codes2<FMT, 0>(yh), c3 = codes2<FMT, 1>(yh);
            const int mt = 8 * j + 2 * i;
#pragma unroll
            for (int z = 0; z < (SPLIT ? 2 : 1); ++z)
#pragma unroll
              for (int n = 0; n < NT; ++n) {
                mma_f16(o[mt][n], a0, a1, a2, a3, pb[z][n][0], pb[z][n][1]);
                mma_f16(o[mt + 1][n], c0, c1, c2, c3, pb[z][n][0], pb[z][n][1]);
              }
          }
      }
      cur = nxt;
      at = at_n;
      sk = sk_n;
      sv = sv_n;
    }

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
        float* row = o_s + ((size_t)warp * COLS + col) * D;
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
        const float x = exp2f(m_s[i * COLS + col] - mm);
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
        for (int i = 0; i < kWarps; ++i) v += o_s[((size_t)i * COLS + col) * D + d] * fac[i];
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
// it is the first that does; the parts are added in the order of the shares.
template <int D, int COLS>
__global__ void __launch_bounds__(kThreads)
attend_join_kernel(const __grid_constant__ AttendArgs a) {
  pdl_trigger();
  pdl_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t total = total_tiles<COLS>(a);
  const int i0 = blockIdx.x;
  const int64_t before = share_begin(total, i0, a.shares), cut = share_begin(total, i0 + 1, a.shares);
  if (before == cut || cut >= total) return;
  const Unit u = locate<COLS>(a, cut);
  if (u.begin == cut || u.begin < before) return;
  const int64_t end = u.begin + u.s.tiles;
  constexpr int kSlot = COLS * (D + 2);
  const int col0 = u.cg * COLS, n_cols = min(COLS, u.s.n * a.group - col0);
  for (int col = warp; col < n_cols; col += kWarps) {
    float M = -INFINITY, L = 0.f, o[D / 32];
#pragma unroll
    for (int e = 0; e < D / 32; ++e) o[e] = 0.f;
    for (int i = i0; i < a.shares; ++i) {
      const int64_t b = share_begin(total, i, a.shares);
      if (b >= end) break;
      if (b == share_begin(total, i + 1, a.shares)) continue;
      const float* part = a.part + (int64_t)(2 * i + (u.begin >= b ? 1 : 0)) * kSlot;
      const float mi = part[COLS * D + col], li = part[COLS * D + COLS + col];
      const float mn = fmaxf(M, mi), mm = mn == -INFINITY ? 0.f : mn;
      const float fo = exp2f(M - mm), fi = exp2f(mi - mm);
      L = L * fo + li * fi;
#pragma unroll
      for (int e = 0; e < D / 32; ++e) o[e] = o[e] * fo + part[col * D + lane + 32 * e] * fi;
      M = mn;
    }
    const int j = (col0 + col) / a.group, h = u.h * a.group + (col0 + col) % a.group;
    const float inv = L > 0.f ? 1.f / L : (L == 0.f ? 0.f : L);
#pragma unroll
    for (int e = 0; e < D / 32; ++e)
      store_elem(a.o.data, (u.s.first + j) * a.o.ld_tok + h * a.o.ld_head + lane + 32 * e, a.o.type, o[e] * inv);
    if (lane == 0 && a.lse)
      a.lse[(u.s.first + j) * a.q.heads + h] = L > 0.f ? (M + log2f(L)) / kLog2e : (L == 0.f ? -INFINITY : L);
  }
}

template <int D, int NT, int FMT, bool SPLIT>
crvq_status launch_attend(AttendArgs& a, cudaStream_t stream) {
  using S = Shape<D, NT, FMT, SPLIT>;
  auto kernel = attend_kernel<D, NT, FMT, SPLIT>;
  CRVQ_TRY(smem_limit((const void*)kernel, S::kSmem));
  // CTAs that an SM holds, by registers: 16 warps of 128, fewer with wide accumulators
  constexpr int kPerSm = D == 256 ? 2 : (NT == 1 ? 4 : 3);
  a.shares = sm_count() * kPerSm;
  Scratch mem;
  CRVQ_TRY(mem.alloc((size_t)2 * a.shares * S::kSlot * sizeof(float), stream));
  a.part = mem.as<float>();
  ProfScope ps("cache_attention", stream, (double)a.rows.n_tok * a.q.heads * D);
  CRVQ_CUDA(launch_pdl(kernel, dim3((unsigned)a.shares), dim3(kThreads), S::kSmem, stream, a));
  CRVQ_LAUNCHED();
  CRVQ_CUDA(launch_pdl(attend_join_kernel<D, S::kCols>, dim3((unsigned)a.shares - 1), dim3(kThreads), 0, stream, a));
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
