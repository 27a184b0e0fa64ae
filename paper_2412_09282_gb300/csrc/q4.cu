// Matrices with 4-bit weights and a scale per group of 32, 64 or 128 inputs: quantizing by rounding,
// and the product with 1 to 32 inputs,
//   y_b[i] = sum_groups s_ig sum_{j in group} (code_ij - zero_ig) x_bj.
//
// Product. code - zero is an integer of at most 15, exact in fp16, so the inner sums run on
// mma.sync.m16n8k16 with the weights as A (16 rows) and up to 8 NT inputs as B. fp16 inputs go as they are;
// bf16 inputs are taken relative to a power of two per group and input (exact but for elements below 2^-14 of
// the group's largest), fp32 inputs so in two pieces (22 bits). A group's sum is scaled once, in fp32. The
// order of the inner index is free: a lane holds 32 (16, 8) consecutive codes of a row and pairs nibbles
// e and e + 4 of a word; one shift and four masks turn a word into fp16 pairs 1024 + code or 1024 + 16 code, one
// fp16 operation each into code - zero. The lane's piece of the inputs is laid out in the same order.
//
// Split. One CTA per SM owns an equal run of tiles (16 RT rows). It lays the inputs out in operand order in
// shared memory once (or in chunks, where they do not fit), and each of its warps takes an equal share of the
// line of all (tile, step) pairs, a step being 256 inputs: 128 bytes of a row's codes, copied ahead to the
// warp's own ring, every copy instruction four whole 128-byte lines; the scales follow in registers. A warp
// whose share begins inside a tile leaves that tile's sum in a slot of its own; the slots are added in warp
// order. Where there are fewer tiles than SMs the inputs are sliced over a cluster, whose sums meet in
// distributed shared memory. One launch, no scratch, sums in a fixed order. (A CTA per tile spent
// most of its time on laying out inputs and on its own start: 28672 x 8192, one input, 73 us.)
//
// What bounds it: instructions. A step of 16 rows takes about 390 (9 per word of 8 codes into operands; the rest
// products, input reads, scales and places), 0.6 per cycle and scheduler, and a call starts and ends with some 6000 cycles of code
// that runs once (places, layout, joins). One input, matrices that are not in L2: 28672 x 8192 28.0 us,
// 4.3 TB/s; 11008 x 4096 9.9 us (9.0 from L2). From L2: 512 x 512 3.6 us. 16 inputs, 28672 x 8192: 45.8 us.
#include <cooperative_groups.h>

#include <algorithm>

#include "cache.cuh"

#include "kernels.h"

namespace crvq {

namespace {

constexpr int kStep = 256;       // inputs per warp step: 128 bytes of a row's codes
constexpr int kTileBytes = 16 * kStep / 2;
constexpr int kMaxInputs = 32;
constexpr int kMaxSlices = 8;

struct Q4View {
  uint8_t* codes;
  __nv_bfloat16* scales;
  uint8_t* zeros;
  int64_t M, N, ld_codes, ld_scales;
};

struct MatvecQ4 {
  Q4View m;
  const void* X;
  int64_t ldx;
  void* Y;
  int64_t ldy;
  int b;
  bool vec_w, vec_x;
  int cols;           // columns laid out: b, or 8 NT
  int chunk;          // steps laid out at a time
  int group;          // tiles whose sums are held at a time
  int log_slices;     // slices of the inputs: CTAs of a cluster
  int tiles_each, tiles_more, steps_each, steps_more;  // of a cluster and of a slice; the first `more` have one more
};

__device__ __forceinline__ void mma16(float d[4], const uint32_t a[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
      "{%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// The same into zeros (no registers are cleared for it).
__device__ __forceinline__ void mma16_first(float d[4], const uint32_t a[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
      "{%10,%10,%10,%10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}

__device__ __forceinline__ __half2 as_half2(uint32_t x) { return *reinterpret_cast<const __half2*>(&x); }
__device__ __forceinline__ uint32_t bits(__half2 x) { return *reinterpret_cast<const uint32_t*>(&x); }

// Codes e and e + 4 of a word (e = 0 .. 3) less the zero point z; lo: 1024 + z twice, hi: -(64 + z) twice. The
// integers' low bits are the mantissa's, so both forms are exact: (1024 + c) - (1024 + z), (1024 + 16 c) / 16 - (64 + z).
__device__ __forceinline__ uint32_t take(uint32_t v, uint32_t mask) {  // (v & mask) | 1024 twice, in one operation
  uint32_t u;
  asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(u) : "r"(v), "r"(mask), "r"(0x64006400u));
  return u;
}

__device__ __forceinline__ uint32_t codes_pair(uint32_t w, int e, uint32_t lo, uint32_t hi) {
  const uint32_t v = e >= 2 ? w >> 8 : w;
  if (e & 1) return bits(__hfma2(as_half2(take(v, 0x00f000f0u)), as_half2(0x2c002c00u), as_half2(hi)));
  return bits(__hsub2(as_half2(take(v, 0x000f000fu)), as_half2(lo)));
}

// The inputs k .. k + 7 of row `row` of X (zeros past N), unless fp16 as fp32.
template <int TYPE>
__device__ __forceinline__ void load_x(const MatvecQ4& a, int64_t row, int64_t k, float x[8]) {
  const char* p = static_cast<const char*>(a.X) + row * a.ldx * (TYPE == CRVQ_F32 ? 4 : 2);
  if (k + 8 <= a.m.N) {
    load8(p, k, TYPE, a.vec_x, x);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = k + j < a.m.N ? load_elem(p, k + j, TYPE) : 0.f;
  }
}

// Eight inputs as fp16 B operand pairs (0, 4), (1, 5), (2, 6), (3, 7); rest: what the pairs leave over, or null.
__device__ __forceinline__ uint4 operand_pairs(const float x[8], uint4* rest) {
  uint32_t v[4], r[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const __half2 h = __floats2half2_rn(x[e], x[e + 4]);
    v[e] = bits(h);
    if (rest) {
      const float2 f = __half22float2(h);
      r[e] = bits(__floats2half2_rn(fabsf(f.x) == INFINITY ? 0.f : x[e] - f.x,
                                    fabsf(f.y) == INFINITY ? 0.f : x[e + 4] - f.y));
    }
  }
  if (rest) *rest = make_uint4(r[0], r[1], r[2], r[3]);
  return make_uint4(v[0], v[1], v[2], v[3]);
}

// A row's 128 bytes in shared memory: eight 16-byte units, exchanged by the row so that eight lanes (two rows, four
// neighbouring units) read without bank conflicts.
__device__ __forceinline__ uint32_t unit_at(int r, int c) {
  return (uint32_t)(r * 8 + (c ^ ((r & 6) ^ ((r & 1) << 2)))) * 16;
}

// Offset of lane (row r, tig) in a tile's rows; the words of half j (128 inputs, 64 bytes) follow by exchanging
// bits of it (load_words): of each group of 4 x 8 WORDS inputs, lane tig holds the tig-th WORDS words, so
// that the four lanes of a row hold one group at a time.
template <int GROUP>
__device__ __forceinline__ uint32_t words_at(int r, int tig) {
  return GROUP == 128 ? unit_at(r, tig) : GROUP == 64 ? unit_at(r, tig >> 1) + (tig & 1) * 8 : unit_at(r, 0) + tig * 4;
}

template <int GROUP>
__device__ __forceinline__ void load_words(const char* tile, uint32_t at, int j, uint32_t w[4]) {
  at ^= 64 * j;
  if constexpr (GROUP == 128) {
    const uint4 u = *reinterpret_cast<const uint4*>(tile + at);
    w[0] = u.x; w[1] = u.y; w[2] = u.z; w[3] = u.w;
  } else if constexpr (GROUP == 64) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const uint2 u = *reinterpret_cast<const uint2*>(tile + (at ^ 32 * s));
      w[2 * s] = u.x; w[2 * s + 1] = u.y;
    }
  } else {
#pragma unroll
    for (int s = 0; s < 4; ++s) w[s] = *reinterpret_cast<const uint32_t*>(tile + (at ^ 16 * s));
  }
}

__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}

// Copies 16 rows' codes of one step to a tile where rows or inputs may end in it, or rows are not aligned.
__device__ __noinline__ void start_tile_edge(const MatvecQ4& a, int64_t row0, int64_t k, char* tile) {
  const int lane = threadIdx.x & 31;
  const int64_t bytes = (a.m.N + 1) / 2, at = k / 2 + (lane & 7) * 16;
#pragma unroll 1
  for (int i = 0; i < 4; ++i) {
    const int r = 4 * i + (lane >> 3);
    const uint8_t* src = a.m.codes + min(row0 + r, a.m.M - 1) * a.m.ld_codes;
    const int n = (int)max((int64_t)0, min((int64_t)16, bytes - at));
    char* dst = tile + unit_at(r, lane & 7);
    if (a.vec_w) {
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)),
                   "l"(src + (n > 0 ? at : 0)), "r"(n)
                   : "memory");
    } else {
      uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < 16; ++j)
        if (j < n) w[j / 4] |= (uint32_t)__ldg(src + at + j) << (8 * (j % 4));
      *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
}

template <int TYPE, int GROUP, int NT, int RT>
struct MatvecShape {
  static constexpr int kPieces = TYPE == CRVQ_F32 ? 2 : 1;
  static constexpr bool kScaled = TYPE != CRVQ_F16;           // inputs relative to a power of two per group
  // (32 fp32 inputs need 203 to 255 registers; 8, 14 and 16 warps elsewhere: 10, 4 and 0 to 10 % slower)
  static constexpr int kWarps = NT == 4 && TYPE == CRVQ_F32 ? 8 : 12;
  static constexpr int kStages = 2;                           // (3: 3 % slower, and less room for inputs)

  static constexpr int kGroups = kStep / GROUP;               // groups in a step
  static constexpr int kScales = 16 * RT * kGroups;           // scales of a step's rows, with zero points, 4 bytes
  static constexpr int kStage = RT * kTileBytes + kScales * 4;
  static constexpr int kRing = kStages * kStage;
  static constexpr int kSums = 8 * NT * 16 * RT;              // outputs of a tile
  static constexpr size_t kFixed = (size_t)kWarps * kRing + (size_t)kWarps * kSums * 4 + 16;
  // a step's inputs, and their powers of two; the steps that fit beside the rest
  static int step_bytes(int cols) { return cols * (kPieces * 2 * kStep + (kScaled ? 4 * kGroups : 0)); }
  static size_t smem(int chunk, int group, int cols) {
    return kFixed + (size_t)group * kSums * 4 + (size_t)step_bytes(cols) * chunk;
  }
  static int64_t chunk(int64_t group, int cols) {
    return ((int64_t)(225 * 1024 - kFixed) - group * kSums * 4) / step_bytes(cols);
  }
};

template <int TYPE, int GROUP, int NT, int RT>
__global__ void __launch_bounds__(32 * MatvecShape<TYPE, GROUP, NT, RT>::kWarps, 1)
q4_matvec_kernel(const __grid_constant__ MatvecQ4 a) {
  namespace cg = cooperative_groups;
  using S = MatvecShape<TYPE, GROUP, NT, RT>;
  constexpr int W = S::kWarps, kThreads = 32 * W, R = 16 * RT, COLS = 8 * NT, WORDS = GROUP / 32;
  extern __shared__ __align__(128) char sm[];
  __shared__ int slot_tile[W];
  pdl_trigger();
  pdl_wait();
  cg::cluster_group cluster = cg::this_cluster();
  const int slices = 1 << a.log_slices, rank = blockIdx.x & (slices - 1), me = blockIdx.x >> a.log_slices;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, gid = lane >> 2, tig = lane & 3;
  const Q4View& m = a.m;
  // this CTA's tiles and steps
  const int tile0 = me * a.tiles_each + min(me, a.tiles_more);
  const int n_tiles = a.tiles_each + (me < a.tiles_more);
  const int step0 = rank * a.steps_each + min(rank, a.steps_more), n_steps = a.steps_each + (rank < a.steps_more);

  const int ring = warp * S::kRing;  // (offsets from sm: 32-bit shared-memory addresses)
  float* slots = reinterpret_cast<float*>(sm + W * S::kRing);  // [W][COLS][R]
  float* sums = slots + W * S::kSums;                          // [group][COLS][R]
  uint4* none = reinterpret_cast<uint4*>(sums + a.group * S::kSums);  // zeros, for columns past the inputs
  uint4* xs = none + 1;                                        // [pieces][half step][word][cols][4]
  const int cols = NT > 1 ? COLS : a.cols;
  float* xf = reinterpret_cast<float*>(xs + S::kPieces * a.chunk * 32 * cols);  // [group][cols] powers of two
  if (tid == 0) *none = make_uint4(0, 0, 0, 0);
  // this lane's column of the inputs: its first word's place, and how far the next word's is
  const bool laid = gid < cols;
  const int x_lane = (int)(laid ? reinterpret_cast<char*>(xs + gid * 4 + tig) - sm : reinterpret_cast<char*>(none) - sm);
  const int x_word = laid ? 64 * cols : 0, x_piece = laid ? a.chunk * 512 * cols : 0;
  const int xf_lane = (int)(reinterpret_cast<char*>(xf + 2 * tig) - sm);
  const uint32_t w_lane = words_at<GROUP>(gid, tig);

  // A place on this warp's way: tiles t0 .. of the present group, the chunk from step c0 on, and in it the
  // share [i, end) of the line of (tile, step) pairs.
  struct Place {
    int t0, c0, i, end, tile, st, nst;
  };
  auto enter = [&](Place& p) {  // the first place of the group and chunk that t0 and c0 name
    const int nt = min(a.group, n_tiles - p.t0);
    p.nst = min(a.chunk, n_steps - p.c0);
    const int line = nt * p.nst;
    p.i = line * warp / W;
    p.end = line * (warp + 1) / W;
    p.tile = p.i / p.nst;
    p.st = p.i - p.tile * p.nst;
  };
  auto leave = [&](Place& p) {  // to the next chunk or group that has a share; false past the last
    while (p.i >= p.end) {
      p.c0 += a.chunk;
      if (p.c0 >= n_steps) {
        p.c0 = 0;
        p.t0 += a.group;
        if (p.t0 >= n_tiles) return false;
      }
      enter(p);
    }
    return true;
  };
  auto next = [&](Place& p) {
    ++p.i;
    if (++p.st == p.nst) {
      p.st = 0;
      ++p.tile;
    }
  };

  // Copies ahead: a step's codes, and its scales and zero points, which wait in registers until the step
  // after (lane: row lane / 2 of each 16, half of its groups).
  constexpr int kMine = S::kGroups / 2;
  uint32_t held[RT][kMine];
  int held_slot = -1;
  Place ahead = {0, 0, 0, 0, 0, 0, 0};
  bool more = n_tiles > 0 && n_steps > 0, inside = false;
  const uint8_t* codes = nullptr;  // this lane's first 16 bytes of the step ahead, and its first scale there
  const __nv_bfloat16* scales = nullptr;
  int64_t zeros = 0;               // (the zero points' offset)
  auto point = [&]() {             // after a tile's or a chunk's first place
    const int64_t k = (int64_t)(step0 + ahead.c0 + ahead.st) * kStep, row0 = (int64_t)(tile0 + ahead.t0 + ahead.tile) * R;
    inside = a.vec_w && row0 + R <= m.M;
    codes = m.codes + (row0 + (lane >> 3)) * m.ld_codes + k / 2 + (lane & 7) * 16;
    zeros = (row0 + (lane >> 1)) * m.ld_scales + k / GROUP + (lane & 1) * kMine;
    scales = m.scales + zeros;
  };
  if (more) {
    enter(ahead);
    more = leave(ahead);
    if (more) point();
  }
  const int64_t ld4 = 4 * m.ld_codes, ld16 = 16 * m.ld_scales;
  const uint32_t ring_u = (uint32_t)__cvta_generic_to_shared(sm + ring), dst0 = unit_at(lane >> 3, lane & 7);
  auto start = [&](int slot) {
    if (held_slot >= 0) {
      uint32_t* sc = reinterpret_cast<uint32_t*>(sm + ring + held_slot * S::kStage + RT * kTileBytes);
#pragma unroll
      for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int e = 0; e < kMine; ++e) sc[((lane & 1) * kMine + e) * R + 16 * t + (lane >> 1)] = held[t][e];
      held_slot = -1;
    }
    if (more) {
      const int step = step0 + ahead.c0 + ahead.st;
      if (inside && (int64_t)(step + 1) * kStep <= m.N) {
        const uint8_t* src = codes;
        const uint32_t dst = ring_u + slot * S::kStage;
#pragma unroll
        for (int i = 0; i < 4 * RT; ++i) {
          // (rows 4 i on: the unit's exchange differs in one bit for odd i)
          copy16(dst + (dst0 ^ (i & 1) * 64) + i * 512, src);
          src += ld4;
        }
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
          for (int e = 0; e < kMine; ++e) {
            const uint32_t s = __bfloat16_as_ushort(scales[t * ld16 + e]);
            held[t][e] = s << 16 | (m.zeros ? __ldg(m.zeros + zeros + t * ld16 + e) & 15u : 8u);
          }
      } else {
        const int64_t k = (int64_t)step * kStep, row0 = (int64_t)(tile0 + ahead.t0 + ahead.tile) * R;
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          start_tile_edge(a, row0 + 16 * t, k, sm + ring + slot * S::kStage + t * kTileBytes);
          const int64_t row = min(row0 + 16 * t + (lane >> 1), m.M - 1) * m.ld_scales;
#pragma unroll
          for (int e = 0; e < kMine; ++e) {
            const int64_t g = k / GROUP + (lane & 1) * kMine + e;
            const bool in = g * GROUP < m.N;  // (past N: 0)
            const uint32_t s = in ? __bfloat16_as_ushort(m.scales[row + g]) : 0u;
            held[t][e] = s << 16 | (in && m.zeros ? __ldg(m.zeros + row + g) & 15u : 8u);
          }
        }
      }
      held_slot = slot;
      const int tile = ahead.tile, c0 = ahead.c0, group0 = ahead.t0;
      next(ahead);
      codes += kStep / 2;
      scales += S::kGroups;
      zeros += S::kGroups;
      more = leave(ahead);
      if (more && (ahead.tile != tile || ahead.c0 != c0 || ahead.t0 != group0)) point();
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int i = 0; i < S::kStages - 1; ++i) start(i);

  int slot = 0;
  for (int t0 = 0; t0 < n_tiles; t0 += a.group) {
    const int nt = min(a.group, n_tiles - t0);
    if (t0) __syncthreads();  // the previous group's sums have been read
    for (int e = tid; e < nt * S::kSums; e += kThreads) sums[e] = 0.f;
    for (int c0 = 0; c0 < n_steps; c0 += a.chunk) {
      Place p = {t0, c0, 0, 0, 0, 0, 0};
      enter(p);
      if (n_steps > a.chunk || t0 == 0) {
        __syncthreads();  // the inputs before these have been read
        const int cn = p.nst * (kStep / 8);  // eights of inputs
        const int all = cn * cols;
        // loads on their way together (few inputs: what counts is that code that runs once is short; 4: 2 % slower)
        constexpr int kAhead = NT == 1 ? 1 : TYPE == CRVQ_F32 ? 2 : 4;
        for (int e0 = 0; e0 < all; e0 += kThreads * kAhead) {  // (whole warps: 32 eights of one column)
          float xa[kAhead][8];
#pragma unroll
          for (int u = 0; u < kAhead; ++u) {
            const int e = e0 + u * kThreads + tid, col = e / cn, o = e - col * cn;
            if (e < all && col < a.b) {  // neighbouring threads read neighbouring inputs
              load_x<TYPE>(a, col, (int64_t)(step0 + p.c0) * kStep + 8 * o, xa[u]);
            } else {
#pragma unroll
              for (int z = 0; z < 8; ++z) xa[u][z] = 0.f;
            }
          }
#pragma unroll
          for (int u = 0; u < kAhead; ++u) {
            const int e = e0 + u * kThreads + tid, col = e / cn, o = e - col * cn;
            if (e >= all) break;
            // the half step, and the word and lane that want it: of each group, lane t the t-th quarter
            const int j = o / 16, in = o % 16 * 8, sub = in / GROUP, rest = in % GROUP;
            const int t = rest / (GROUP / 4), i = sub * WORDS + rest % (GROUP / 4) / 8;
            uint4* dst = xs + ((j * 4 + i) * cols + col) * 4 + t;
            float* x = xa[u];
            if constexpr (S::kScaled) {
              float top = 0.f;
#pragma unroll
              for (int z = 0; z < 8; ++z) top = fmaxf(top, fabsf(x[z]));
#pragma unroll
              for (int d = GROUP / 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
              // 2^-e for a top in [2^e, 2^(e + 1)); 1 for zeros, subnormals and infinities
              const uint32_t ex = __float_as_uint(top) >> 23;
              const bool plain = ex == 0 || ex == 255;
              const float inv = plain ? 1.f : __uint_as_float(ex == 254 ? 0x00400000u : (254u - ex) << 23);
#pragma unroll
              for (int z = 0; z < 8; ++z) x[z] *= inv;
              if (rest == 0) xf[(j * (128 / GROUP) + sub) * cols + col] = plain ? 1.f : __uint_as_float(ex << 23);
            }
            if constexpr (S::kPieces == 2)
              *dst = operand_pairs(x, dst + a.chunk * 32 * cols);
            else
              *dst = operand_pairs(x, nullptr);
          }
        }
      }
      if (tid < W) slot_tile[tid] = -1;
      __syncthreads();

      float acc[RT][NT][4];
      bool fresh = true, first = false;  // at a new tile; its sum begins with this warp
      while (p.i < p.end) {
        if (fresh) {
          first = p.st == 0;
#pragma unroll
          for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
              for (int e = 0; e < 4; ++e) acc[t][n][e] = 0.f;
        }
        __syncwarp();  // every lane has read the stage that these copies overwrite
        start(slot == 0 ? S::kStages - 1 : slot - 1);
        asm volatile("cp.async.wait_group %0;" ::"n"(S::kStages - 1) : "memory");
        __syncwarp();
        const int stage = ring + slot * S::kStage, sc = stage + RT * kTileBytes + gid * 4;
        int xp = x_lane + p.st * 8 * x_word;
        const int xfp = xf_lane + p.st * S::kGroups * cols * 4;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          uint32_t w[RT][2][4];
#pragma unroll
          for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int h = 0; h < 2; ++h) load_words<GROUP>(sm + stage + t * kTileBytes + h * 1024, w_lane, j, w[t][h]);
#pragma unroll
          for (int sub = 0; sub < 128 / GROUP; ++sub) {
            uint32_t sz[RT][2], lo[RT][2], hi[RT][2];
            float part[RT][NT][4];
#pragma unroll
            for (int t = 0; t < RT; ++t) {
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                sz[t][h] = *reinterpret_cast<const uint32_t*>(sm + sc + ((j * (128 / GROUP) + sub) * R + 16 * t + 8 * h) * 4);
                const uint32_t z = sz[t][h] & 15u;
                lo[t][h] = z * 0x10001u + 0x64006400u;
                hi[t][h] = z * 0x100010u + 0xd400d400u;
              }
            }
#pragma unroll
            for (int i = sub * WORDS; i < (sub + 1) * WORDS; ++i) {
              uint4 x[NT][S::kPieces];
#pragma unroll
              for (int z = 0; z < S::kPieces; ++z)
#pragma unroll
                for (int n = 0; n < NT; ++n) x[n][z] = *reinterpret_cast<const uint4*>(sm + xp + z * x_piece + 512 * n);
              xp += x_word;
#pragma unroll
              for (int t = 0; t < RT; ++t) {
                uint32_t A[4];
#pragma unroll
                for (int e = 0; e < 4; e += 2) {
                  A[0] = codes_pair(w[t][0][i], e, lo[t][0], hi[t][0]);
                  A[1] = codes_pair(w[t][1][i], e, lo[t][1], hi[t][1]);
                  A[2] = codes_pair(w[t][0][i], e + 1, lo[t][0], hi[t][0]);
                  A[3] = codes_pair(w[t][1][i], e + 1, lo[t][1], hi[t][1]);
#pragma unroll
                  for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int z = 0; z < S::kPieces; ++z)
                      if (i == sub * WORDS && z == 0 && e == 0)
                        mma16_first(part[t][n], A, x[n][z].x, x[n][z].y);
                      else
                        mma16(part[t][n], A, e ? x[n][z].z : x[n][z].x, e ? x[n][z].w : x[n][z].y);
                }
              }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              float f[2] = {1.f, 1.f};
              if constexpr (S::kScaled) {
#pragma unroll
                for (int e = 0; e < 2; ++e)
                  f[e] = NT > 1 || 2 * tig + e < cols
                             ? *reinterpret_cast<const float*>(sm + xfp + ((j * (128 / GROUP) + sub) * cols + 8 * n + e) * 4)
                             : 0.f;
              }
#pragma unroll
              for (int t = 0; t < RT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  const float s = __uint_as_float(sz[t][e >> 1] & 0xffff0000u);
                  acc[t][n][e] = fmaf(S::kScaled ? s * f[e & 1] : s, part[t][n][e], acc[t][n][e]);
                }
            }
          }
        }
        slot = slot + 1 == S::kStages ? 0 : slot + 1;
        const int tile = p.tile;
        next(p);
        fresh = p.tile != tile;
        if (fresh || p.i == p.end) {
          // the tile's sum of this chunk begins here: to the sums themselves; else to this warp's slot
          float* dst = first ? sums + tile * S::kSums : slots + warp * S::kSums;
          if (!first && lane == 0) slot_tile[warp] = tile;
#pragma unroll
          for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                float* q = dst + (8 * n + 2 * tig + (e & 1)) * R + 16 * t + gid + 8 * (e >> 1);
                *q = first ? *q + acc[t][n][e] : acc[t][n][e];
              }
        }
      }
      __syncthreads();
      for (int e = tid; e < S::kSums; e += kThreads) {
        float v[W];
        int t[W];
#pragma unroll
        for (int i = 0; i < W; ++i) {
          t[i] = slot_tile[i];
          v[i] = t[i] >= 0 ? slots[i * S::kSums + e] : 0.f;
        }
#pragma unroll
        for (int i = 0; i < W; ++i)
          if (t[i] >= 0) sums[t[i] * S::kSums + e] += v[i];
      }
    }
    const int64_t r0 = (int64_t)(tile0 + t0) * R;
    if (slices == 1) {
      for (int e = tid; e < S::kSums; e += kThreads) {
        const int col = e / R, r = e - col * R;
        if (col >= a.b) break;
        for (int t = 0; t < nt; ++t)
          if (r0 + t * R + r < m.M) store_elem(a.Y, col * a.ldy + r0 + t * R + r, TYPE, sums[t * S::kSums + e]);
      }
    } else {
      cluster.sync();
      constexpr int kJoin = 4;  // outputs whose parts are on their way together
      for (int e0 = rank * kThreads + tid; e0 < nt * S::kSums; e0 += kJoin * slices * kThreads) {
        float v[kJoin] = {};
#pragma unroll 2
        for (int i = 0; i < slices; ++i) {
          const float* part = cluster.map_shared_rank(sums, i);
#pragma unroll
          for (int u = 0; u < kJoin; ++u) {
            const int e = e0 + u * slices * kThreads;
            if (e < nt * S::kSums) v[u] += part[e];
          }
        }
#pragma unroll
        for (int u = 0; u < kJoin; ++u) {
          const int e = e0 + u * slices * kThreads, t = e / S::kSums, col = (e - t * S::kSums) / R, r = e % R;
          if (t < nt && col < a.b && r0 + t * R + r < m.M) store_elem(a.Y, col * a.ldy + r0 + t * R + r, TYPE, v[u]);
        }
      }
      cluster.sync();  // nobody's sums are read any more
    }
  }
}

// A thread takes eight consecutive weights; the GROUP / 8 threads of a group find its range by shuffles. 16.8 M fp32
// weights with their values: 26.5 us, 5.4 TB/s; 40 instructions per weight issue 0.72 of the time (with CUDA's division
// and 64-bit places 54, 30.3 us).
struct QuantizeArgs {
  Q4View m;
  const void* W;
  int64_t ldw;
  int type;
  bool vec_w, vec_c, vec_h;
  float* W_hat;
  Divisor by_row;  // threads per row, whole groups
  unsigned* err;
};

template <int GROUP>
__global__ void __launch_bounds__(256) q4_quantize_kernel(const __grid_constant__ QuantizeArgs a) {
  constexpr int kLanes = GROUP / 8;
  pdl_trigger();
  pdl_wait();
  const int at = (int)blockIdx.x * 256 + threadIdx.x, row_i = a.by_row.div(at);
  const int64_t row = row_i, j0 = (int64_t)(at - row_i * (int)a.by_row.d) * 8, g = j0 / GROUP;
  const bool live = row < a.m.M;  // whole groups of lanes
  const int64_t N = a.m.N;
  const int n = live ? (int)max((int64_t)0, min((int64_t)8, N - j0)) : 0;
  float w[8];
  if (n == 8) {
    load8(a.W, row * a.ldw + j0, a.type, a.vec_w, w);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = e < n ? load_elem(a.W, row * a.ldw + j0 + e, a.type) : 0.f;
  }
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(w[e]) & 0x7fffffffu);
  if (top >= 0x7f800000u) {
    raise_error(a.err, ERRBIT_NUMERIC);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (!(fabsf(w[e]) <= 3.402823466e38f)) w[e] = 0.f;
  }
  float lo = 0.f, hi = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    lo = fminf(lo, w[e]);
    hi = fmaxf(hi, w[e]);
  }
#pragma unroll
  for (int d = kLanes / 2; d > 0; d >>= 1) {
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, d));
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, d));
  }
  constexpr float k7 = (float)(1.0 / 7.0), k15 = (float)(1.0 / 15.0);
  float range = __fmul_rn(__fsub_rn(hi, lo), k15);
  if (range == INFINITY) range = __fsub_rn(__fmul_rn(hi, k15), __fmul_rn(lo, k15));  // (hi - lo is above fp32's numbers)
  const __nv_bfloat16 s16 = __float2bfloat16_rn(a.m.zeros ? range : __fmul_rn(fmaxf(hi, -lo), k7));
  const float s = __bfloat162float(s16);
  float z = 8.f;
  if (a.m.zeros) z = s > 0.f ? fminf(fmaxf(rintf(__fdiv_rn(-lo, s)), 0.f), 15.f) : 0.f;
  if (plain_divisor(s)) {
    const float inv = __frcp_rn(s);
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = quotient(w[e], s, inv);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = s > 0.f ? fminf(fmaxf(__fdiv_rn(w[e], s), -64.f), 64.f) : 0.f;
  }
  // Adding 1.5 * 2^23 rounds to an integer, which the sum's low bits are (quotients by a normal scale are below 16.1).
  constexpr float kRound = 12582912.f;
  float v[8];
  uint32_t codes = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float q = fminf(fmaxf(__fsub_rn(__fadd_rn(w[e], kRound), kRound) + z, 0.f), 15.f);
    v[e] = (q - z) * s;
    codes |= (__float_as_uint(__fadd_rn(q, kRound)) & 15u) << (4 * e);
  }
  if (s > 0x1p120f) {  // a nearest level may be above fp32's numbers: then the one before it (rare: apart from the loop)
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (fabsf(v[e]) == INFINITY) {
        codes = v[e] > 0.f ? codes - (1u << 4 * e) : codes + (1u << 4 * e);
        v[e] = ((float)(codes >> 4 * e & 15u) - z) * s;
      }
  }
  if (n == 0) return;
  if (n < 8) codes &= (1u << (4 * n)) - 1u;
  uint8_t* c = a.m.codes + row * a.m.ld_codes + j0 / 2;
  if (a.vec_c && n == 8) {
    *reinterpret_cast<uint32_t*>(c) = codes;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (2 * e < n) c[e] = (uint8_t)(codes >> (8 * e));
  }
  if (j0 % GROUP == 0) {
    a.m.scales[row * a.m.ld_scales + g] = s16;
    if (a.m.zeros) a.m.zeros[row * a.m.ld_scales + g] = (uint8_t)z;
  }
  if (a.W_hat) {
    float* h = a.W_hat + row * N + j0;
    if (n == 8) {
      store8(h, 0, CRVQ_F32, a.vec_h, v);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < n) h[e] = v[e];
    }
  }
}

crvq_status make_q4(const crvq_q4_matrix* m, Q4View* out) {
  CRVQ_CHECK_ARG(m != nullptr && m->codes && m->scales, "the 4-bit matrix, its codes or scales are NULL");
  CRVQ_CHECK_ARG(m->M >= 1 && m->N >= 1, "need M, N >= 1");
  if (m->group != 32 && m->group != 64 && m->group != 128)
    return fail(CRVQ_ERR_UNSUPPORTED, "groups of %d inputs: 32, 64 and 128 are implemented", m->group);
  CRVQ_CHECK_ARG(m->ld_codes >= ceil_div(m->N, 2), "ld_codes < ceil(N / 2)");
  CRVQ_CHECK_ARG(m->ld_scales >= ceil_div(m->N, m->group), "ld_scales < ceil(N / group)");
  CRVQ_CHECK_ARG(((uintptr_t)m->scales & 1u) == 0, "scales are not aligned");
  CRVQ_TRY(check_dev({{m->codes, "codes"}, {m->scales, "scales"}, {m->zeros, "zeros"}}));
  *out = Q4View{m->codes, static_cast<__nv_bfloat16*>(m->scales), m->zeros, m->M, m->N, m->ld_codes, m->ld_scales};
  return CRVQ_OK;
}

template <int TYPE, int GROUP, int NT, int RT>
crvq_status launch_matvec(MatvecQ4& a, cudaStream_t stream) {
  using S = MatvecShape<TYPE, GROUP, NT, RT>;
  auto kernel = q4_matvec_kernel<TYPE, GROUP, NT, RT>;
  a.cols = a.b <= 8 ? a.b : 8 * NT;
  const int64_t tiles = ceil_div(a.m.M, 16 * RT), sms = sm_count();
  const int64_t steps = ceil_div(a.m.N, kStep);
  if (tiles >= (int64_t)1 << 31) return fail(CRVQ_ERR_UNSUPPORTED, "M = %lld is too large", (long long)a.m.M);
  if (steps > (1 << 24)) return fail(CRVQ_ERR_UNSUPPORTED, "N = %lld is too large", (long long)a.m.N);
  // Slices, and the tiles whose sums are held at a time: the choice with the least (tile, step) pairs of one row
  // tile on the busiest SM, with what else costs time in such pairs (about 50 ns): laying out inputs a
  // third per step and column, ten per chunk and group, 20 per group of a cluster. Clusters that are resident
  // at one CTA per SM: 152, 76, 36 and 15 (of 1, 2, 4 and 8). Us with 1, 2, 4 and 8 slices, the choice in brackets: one
  // bf16 input, 4096 x 4096 [5.5], 5.9, 6.0, 7.3; 11008 x 4096 [9.0], 8.9, 9.2, 10.8; 4096 x 11008 [9.6], 9.9, 9.2, 11.5;
  // 28672 x 8192 [27.6], 27.8, 29.0, 36.0; 8192 x 28672 34.5, 32.1, [30.9], 34.1; 16 inputs, 4096 x 4096 16.6, 11.9, 9.9,
  // [9.5]; 28672 x 8192 59.8, 49.1, [44.5], 53.1; 32 fp32 inputs of it 161, 131, [124], 151.
  int slices = 1;
  int64_t clusters = 0;
  double best = 0;
  for (int n = 1; n <= kMaxSlices && n <= steps; n *= 2) {
    const int64_t slots = std::max<int64_t>(1, n == 8 ? sms * 4 / 5 / 8 : n == 4 ? sms * 18 / 19 / 4 : sms / n);
    const int64_t own = ceil_div(tiles, slots), st = ceil_div(steps, n);
    for (int64_t parts = 1; parts <= own; parts = parts < 8 ? parts + 1 : 2 * parts) {
      const int64_t group = ceil_div(own, parts), chunk = std::min(st, S::chunk(group, a.cols));
      if (chunk < 1) continue;
      const int64_t chunks = ceil_div(st, chunk), groups = ceil_div(own, group);
      const double pairs = (double)ceil_div(group * chunk, S::kWarps) * S::kWarps * RT * (double)(chunks * groups);
      const double cost = pairs + 0.33 * (double)st * a.cols * (chunks > 1 ? (double)groups : 1.0) +
                          10.0 * (double)(chunks * groups) + (n > 1 ? 20.0 * (double)groups : 0.0);
      if (clusters == 0 || cost < best) {
        best = cost;
        slices = n;
        clusters = std::min(tiles, slots);
        a.group = (int)group;
        a.chunk = (int)chunk;
      }
    }
  }
  if (clusters == 0) return fail(CRVQ_ERR_UNSUPPORTED, "matrix too large");
  a.log_slices = slices == 8 ? 3 : slices == 4 ? 2 : slices == 2 ? 1 : 0;
  a.tiles_each = (int)(tiles / clusters);
  a.tiles_more = (int)(tiles % clusters);
  a.steps_each = (int)(steps / slices);
  a.steps_more = (int)(steps % slices);
  const size_t smem = S::smem(a.chunk, a.group, a.cols);
  CRVQ_TRY(smem_limit((const void*)kernel, smem));
  ProfScope ps("q4_matvec", stream, (double)a.m.M * a.m.N * a.b);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(clusters * slices));
  cfg.blockDim = dim3(32 * S::kWarps);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)slices;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = slices > 1 ? 2 : 1;
  CRVQ_CUDA(cudaLaunchKernelEx(&cfg, kernel, a));
  CRVQ_LAUNCHED();
  return CRVQ_OK;
}

template <int TYPE, int GROUP>
crvq_status pick_inputs(MatvecQ4& a, cudaStream_t stream) {
  // Row tiles of a step: 2 share what is read of the inputs; with more than 8 of those one leaves registers for the
  // products of a group on their way (28672 x 8192, us with 2 and 1: 16 bf16 inputs 48.5, 45.8; 32 97.5, 77.3; 32 fp32
  // 155, 126; one input 28.7, 30.9)
  if (a.b <= 8) return launch_matvec<TYPE, GROUP, 1, 2>(a, stream);
  if (a.b <= 16) return launch_matvec<TYPE, GROUP, 2, 1>(a, stream);
  return launch_matvec<TYPE, GROUP, 4, 1>(a, stream);
}

template <int TYPE>
crvq_status pick_group(MatvecQ4& a, int group, cudaStream_t stream) {
  if (group == 32) return pick_inputs<TYPE, 32>(a, stream);
  if (group == 64) return pick_inputs<TYPE, 64>(a, stream);
  return pick_inputs<TYPE, 128>(a, stream);
}

crvq_status matvec(const crvq_q4_matrix* m, const void* X, int64_t ldx, int64_t b, int type, void* Y,
                   int64_t ldy, cudaStream_t stream) {
  MatvecQ4 a{};
  CRVQ_TRY(make_q4(m, &a.m));
  CRVQ_CHECK_ARG(X && Y, "X and Y must not be NULL");
  CRVQ_CHECK_ARG(type >= CRVQ_F32 && type <= CRVQ_F16, "unknown type %d", type);
  CRVQ_CHECK_ARG(b >= 1, "need b >= 1");
  if (b > kMaxInputs) return fail(CRVQ_ERR_UNSUPPORTED, "batches of more than %d inputs are not implemented", kMaxInputs);
  CRVQ_CHECK_ARG(ldx >= m->N && ldy >= m->M, "need ldx >= N, ldy >= M");
  const size_t wide = type_bytes(type);
  CRVQ_CHECK_ARG((uintptr_t)X % wide == 0 && (uintptr_t)Y % wide == 0, "X or Y is not aligned to its type");
  CRVQ_TRY(check_dev({{X, "X"}, {Y, "Y"}}));
  a.X = X;
  a.ldx = ldx;
  a.Y = Y;
  a.ldy = ldy;
  a.b = (int)b;
  a.vec_w = ((uintptr_t)m->codes & 15u) == 0 && m->ld_codes % 16 == 0;
  a.vec_x = ((uintptr_t)X & 15u) == 0 && (b == 1 || ldx * (int64_t)wide % 16 == 0);
  if (type == CRVQ_F32) return pick_group<CRVQ_F32>(a, m->group, stream);
  if (type == CRVQ_BF16) return pick_group<CRVQ_BF16>(a, m->group, stream);
  return pick_group<CRVQ_F16>(a, m->group, stream);
}

crvq_status quantize(const void* W, int64_t ldw, int type, const crvq_q4_matrix* m, float* W_hat,
                     cudaStream_t stream) {
  QuantizeArgs a{};
  CRVQ_TRY(make_q4(m, &a.m));
  CRVQ_CHECK_ARG(W != nullptr, "W is NULL");
  CRVQ_CHECK_ARG(type >= CRVQ_F32 && type <= CRVQ_F16, "unknown type %d", type);
  CRVQ_CHECK_ARG(ldw >= m->N, "need ldw >= N");
  const size_t wide = type_bytes(type);
  CRVQ_CHECK_ARG((uintptr_t)W % wide == 0 && ((uintptr_t)W_hat & 3u) == 0, "W or W_hat is not aligned to its type");
  CRVQ_TRY(check_dev({{W, "W"}, {W_hat, "W_hat"}}));
  CRVQ_TRY(device_error_word(&a.err));
  a.W = W;
  a.ldw = ldw;
  a.type = type;
  a.vec_w = ((uintptr_t)W & 15u) == 0 && ldw * (int64_t)wide % 16 == 0;
  a.vec_c = ((uintptr_t)m->codes & 3u) == 0 && m->ld_codes % 4 == 0;
  a.vec_h = ((uintptr_t)W_hat & 15u) == 0 && m->N % 4 == 0;
  a.W_hat = W_hat;
  const int64_t per_row = ceil_div(m->N, m->group) * (m->group / 8), most = ((int64_t)1 << 31) - 256;
  if (per_row > most) return fail(CRVQ_ERR_UNSUPPORTED, "rows of %lld inputs are too long", (long long)m->N);
  a.by_row = Divisor(per_row);
  ProfScope ps("q4_quantize", stream, (double)m->M * m->N);
  const int64_t rows = most / per_row;  // of a launch: thread indices have 31 bits
  for (int64_t r0 = 0; r0 < m->M; r0 += rows) {
    a.m.M = std::min(rows, m->M - r0);
    const dim3 g((unsigned)ceil_div(a.m.M * per_row, 256)), t(256);
    if (m->group == 32)
      CRVQ_CUDA(launch_pdl(q4_quantize_kernel<32>, g, t, 0, stream, a));
    else if (m->group == 64)
      CRVQ_CUDA(launch_pdl(q4_quantize_kernel<64>, g, t, 0, stream, a));
    else
      CRVQ_CUDA(launch_pdl(q4_quantize_kernel<128>, g, t, 0, stream, a));
    CRVQ_LAUNCHED();
    a.W = static_cast<const char*>(a.W) + rows * ldw * (int64_t)wide;
    a.m.codes += rows * m->ld_codes;
    a.m.scales += rows * m->ld_scales;
    if (a.m.zeros) a.m.zeros += rows * m->ld_scales;
    if (a.W_hat) a.W_hat += rows * m->N;
  }
  return CRVQ_OK;
}

}  // namespace

}  // namespace crvq

extern "C" {

crvq_status crvq_q4_quantize(const void* W, int64_t ldw, int32_t type, const crvq_q4_matrix* m, float* W_hat,
                             crvq_stream_t stream) {
  CRVQ_ENTRY({ return crvq::quantize(W, ldw, type, m, W_hat, (cudaStream_t)stream); })
}

crvq_status crvq_q4_matvec(const crvq_q4_matrix* m, const void* X, int64_t ldx, int64_t b, int32_t type,
                           void* Y, int64_t ldy, crvq_stream_t stream) {
  CRVQ_ENTRY({ return crvq::matvec(m, X, ldx, b, type, Y, ldy, (cudaStream_t)stream); })
}

}  // extern "C"
