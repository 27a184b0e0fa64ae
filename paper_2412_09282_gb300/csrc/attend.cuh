// Attention over the paged 8-bit cache: what the kernels share (attend_mma.cuh: few queries per sequence
// on mma.sync; attend_tc.cu: many on tcgen05). Arguments, the split of the work into equal shares of one
// line, code conversion, and the joining of units that lie in several shares (latency: where 16 sequences with up to
// five queries go by shares, 8.3 us of 25; the parts are in L2).
#pragma once

#include "cache.cuh"
#include "kernels.h"

namespace crvq {

struct AttendArgs {
  CacheView c;
  HeadsView q, o;
  RowsView rows;
  int group;        // query heads per kv head
  float scale;      // times log2(e)
  bool causal;
  int window;
  bool vec_q, vec_o;  // 16-byte rows
  float* lse;
  float* part;      // 2 slots per CTA: [cols][D] outputs, [cols] maxima, [cols] sums
  int shares;
  int cluster;      // CTAs of a unit that join it among themselves, a power of two (0: shares of the line)
  int log_cluster;
  unsigned* err;
};

// Few queries, short sequences (attend_cluster.cu): `size` CTAs (2, 4 or 8) per unit of 8 NT columns.
crvq_status launch_attend_clusters(AttendArgs& a, int D, int NT, int format, int64_t units, int size,
                                   cudaStream_t stream);
// Many queries per sequence (attend_tc.cu): 16-bit queries, 64 or 128 channels.
crvq_status launch_attend_many(AttendArgs& a, int D, int format, cudaStream_t stream);

namespace {

constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
// Blocks that a warp takes at a time (two: twice the independent work, and one maximum for both)
template <int D>
constexpr int kBlocks = D == 256 ? 1 : 2;
template <int D>
constexpr int kTile = kCacheBlock * kBlocks<D> * kWarps;  // tokens of a CTA at a time
constexpr float kLogWeight = 14.f;           // weights are scaled by 2^14 into fp16's range
constexpr float kLog2e = 1.4426950408889634f;

// 2^x (within 2 ulp; results below 2^-126 are 0)
__device__ __forceinline__ float pow2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}


// What a unit costs beside its tiles (its start, and joining its warps), in tiles: the first kStart places
// of a unit on the line hold no tile.
constexpr int kStart = 3;

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
  int tile;         // at the place that was looked for (0 before the first tile)
  int64_t begin;    // the unit's first place on the line; its tiles begin kStart later
};

__device__ __forceinline__ int64_t divide(int64_t x, int y) {  // x >= 0, y > 0
  return x >> 32 ? x / y : (int64_t)((uint32_t)x / (uint32_t)y);
}

__device__ __forceinline__ int64_t share_begin(int64_t total, int i, int shares) {
  return divide(total * i, shares);
}

// The line of all units' tiles, warp-wide: every lane holds a sequence's end of the first 32.
template <int D, int COLS>
struct Line {
  int64_t cost, end;  // of sequence `lane`
  int64_t total;

  Line() = default;
  static __device__ __forceinline__ int64_t cost_of(const AttendArgs& a, int b) {
    if (b >= a.c.n_seq) return 0;
    const Seq s = load_seq<D, COLS>(a, b);
    return (int64_t)s.groups * (s.tiles + kStart) * a.c.n_kv;
  }
  static __device__ __forceinline__ int64_t scan(int64_t v) {
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int64_t x = __shfl_up_sync(0xffffffffu, v, d);
      if ((int)(threadIdx.x & 31) >= d) v += x;
    }
    return v;
  }
  __device__ explicit Line(const AttendArgs& a) {
    const int lane = threadIdx.x & 31;
    cost = cost_of(a, lane);
    end = scan(cost);
    int64_t more = 0;
    for (int b = 32 + lane; b < a.c.n_seq; b += 32) more += cost_of(a, b);
    total = __shfl_sync(0xffffffffu, end, 31);
    if (a.c.n_seq > 32) total += __shfl_sync(0xffffffffu, scan(more), 31);
  }
  // Unit number i (sequence by sequence, head by head); false past the last.
  static __device__ bool unit(const AttendArgs& a, int64_t i, Unit* u) {
    const int lane = threadIdx.x & 31;
    int64_t base = 0;
    for (int b0 = 0; b0 < a.c.n_seq; b0 += 32) {
      int64_t units = 0, places = 0;
      if (b0 + lane < a.c.n_seq) {
        const Seq s = load_seq<D, COLS>(a, b0 + lane);
        units = (int64_t)s.groups * a.c.n_kv;
        places = units * (s.tiles + kStart);
      }
      const int64_t e = scan(units), pe = scan(places);
      const unsigned hit = __ballot_sync(0xffffffffu, e > i);
      if (hit) {
        const int src = __ffs(hit) - 1;
        i -= __shfl_sync(0xffffffffu, e - units, src);
        u->b = b0 + src;
        u->s = load_seq<D, COLS>(a, u->b);
        u->begin = base + __shfl_sync(0xffffffffu, pe - places, src) + i * (u->s.tiles + kStart);
        u->h = (int)divide(i, u->s.groups);
        u->cg = (int)(i - (int64_t)u->h * u->s.groups);
        u->tile = 0;
        return true;
      }
      i -= __shfl_sync(0xffffffffu, e, 31);
      base += __shfl_sync(0xffffffffu, pe, 31);
    }
    return false;
  }
  // The same for counts below 2^31, without the unit's places on the line.
  static __device__ bool unit_only(const AttendArgs& a, int i, Unit* u) {
    const int lane = threadIdx.x & 31;
    for (int b0 = 0; b0 < a.c.n_seq; b0 += 32) {
      Seq s;
      s.groups = 0;
      if (b0 + lane < a.c.n_seq) s = load_seq<D, COLS>(a, b0 + lane);
      const int units = s.groups * a.c.n_kv;
      int e = units;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, e, d);
        if (lane >= d) e += x;
      }
      const unsigned hit = __ballot_sync(0xffffffffu, e > i);
      if (hit) {
        const int src = __ffs(hit) - 1;
        i -= __shfl_sync(0xffffffffu, e - units, src);
        u->b = b0 + src;
        u->s = load_seq<D, COLS>(a, u->b);
        u->h = i / u->s.groups;
        u->cg = i - u->h * u->s.groups;
        return true;
      }
      i -= __shfl_sync(0xffffffffu, e, 31);
    }
    return false;
  }
  // The unit that holds position w, 0 <= w < total.
  __device__ Unit locate(const AttendArgs& a, int64_t w) const {
    const int lane = threadIdx.x & 31;
    int64_t base = 0, c = cost, e = end;
    Unit u;
    u.b = 0;
    for (int b0 = 0; b0 < a.c.n_seq; b0 += 32) {
      if (b0) {
        c = cost_of(a, b0 + lane);
        e = scan(c);
      }
      const unsigned hit = __ballot_sync(0xffffffffu, base + e > w);
      if (hit) {
        const int src = __ffs(hit) - 1;
        base += __shfl_sync(0xffffffffu, e - c, src);
        u.b = b0 + src;
        break;
      }
      base += __shfl_sync(0xffffffffu, e, 31);
    }
    u.s = load_seq<D, COLS>(a, u.b);
    const int places = u.s.tiles + kStart;
    const int64_t rem = w - base, idx = divide(rem, places);
    const int at = (int)(rem - idx * places);
    u.tile = max(0, at - kStart);
    u.h = (int)divide(idx, u.s.groups);
    u.cg = (int)(idx - (int64_t)u.h * u.s.groups);
    u.begin = w - at;
    return u;
  }
};

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

// Joins the parts of units that lie in several shares, in the order of the shares. Two forms:
//   BY_UNIT (few units, so many parts each): a block per unit (x) and column (y), whose warps take every
//     eighth part;
//   otherwise (few parts each): blocks (y: some of the columns each) per boundary between shares x and x + 1, if
//     it is the first that cuts its unit; a warp per column.
constexpr int kJoinWarps = 8;

template <int D, int COLS, bool BY_UNIT>
__global__ void __launch_bounds__(32 * kJoinWarps)
attend_join_kernel(const __grid_constant__ AttendArgs a) {
  __shared__ float m_s[kJoinWarps], l_s[kJoinWarps], o_s[BY_UNIT ? kJoinWarps * D : 1];
  pdl_trigger();
  pdl_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const Line<D, COLS> line(a);
  const int64_t total = line.total;
  const int shares = (int)min((int64_t)a.shares, total);
  Unit u;
  int i0;  // the share that holds the unit's first tile
  if constexpr (BY_UNIT) {
    if (!Line<D, COLS>::unit(a, blockIdx.x, &u)) return;
    const int64_t first = u.begin + kStart;
    i0 = (int)min((int64_t)shares - 1, divide(first * shares, total));  // within one of it
    while (i0 + 1 < shares && share_begin(total, i0 + 1, shares) <= first) ++i0;
    while (i0 > 0 && share_begin(total, i0, shares) > first) --i0;
  } else {
    i0 = blockIdx.x;
    if (i0 + 1 >= shares) return;
    u = line.locate(a, share_begin(total, i0 + 1, shares));
    if (u.tile == 0 || share_begin(total, i0, shares) > u.begin + kStart) return;
  }
  const int64_t end = u.begin + kStart + u.s.tiles;
  constexpr int kSlot = COLS * (D + 2);
  const int col0 = u.cg * COLS, n_cols = min(COLS, u.s.n * a.group - col0);
  int n = 1;  // shares that hold a part
  while (i0 + n < shares && share_begin(total, i0 + n, shares) < end) ++n;
  if (n == 1) return;  // (written whole)
  constexpr int kPer = D / 32;  // neighbouring channels of a lane
  const float* part = a.part + (int64_t)2 * i0 * kSlot;
  // part p: its share's last unit (p = 0), or its first
  auto slot = [&](int p) { return part + (int64_t)(2 * p + (p == 0 ? 1 : 0)) * kSlot; };

  for (int col = BY_UNIT ? (int)blockIdx.y : (int)blockIdx.y * kJoinWarps + warp; col < n_cols;
       col += BY_UNIT ? COLS : (int)gridDim.y * kJoinWarps) {
    float M = -INFINITY, L = 0.f, o[kPer];
#pragma unroll
    for (int e = 0; e < kPer; ++e) o[e] = 0.f;
    constexpr int kBatch = 8;
    for (int p0 = BY_UNIT ? warp : 0; p0 < n; p0 += kBatch * (BY_UNIT ? kJoinWarps : 1)) {
      float mp[kBatch], lp[kBatch], v[kBatch][kPer];
#pragma unroll
      for (int q = 0; q < kBatch; ++q) {
        const int p = p0 + q * (BY_UNIT ? kJoinWarps : 1);
        mp[q] = -INFINITY;
        lp[q] = 0.f;
#pragma unroll
        for (int e = 0; e < kPer; ++e) v[q][e] = 0.f;
        if (p >= n) continue;
        const float* src = slot(p);
        mp[q] = src[COLS * D + col];
        lp[q] = src[COLS * D + COLS + col];
        if constexpr (D == 64) {
          const float2 x = reinterpret_cast<const float2*>(src + col * D)[lane];
          v[q][0] = x.x; v[q][1] = x.y;
        } else {
#pragma unroll
          for (int e = 0; e < kPer / 4; ++e) {
            const float4 x = reinterpret_cast<const float4*>(src + col * D)[lane * (kPer / 4) + e];
            v[q][4 * e] = x.x; v[q][4 * e + 1] = x.y; v[q][4 * e + 2] = x.z; v[q][4 * e + 3] = x.w;
          }
        }
      }
      float mn = M;
#pragma unroll
      for (int q = 0; q < kBatch; ++q) mn = fmaxf(mn, mp[q]);
      const float mm = mn == -INFINITY ? 0.f : mn, back = pow2(M - mm);
      M = mn;
      L *= back;
#pragma unroll
      for (int e = 0; e < kPer; ++e) o[e] *= back;
#pragma unroll
      for (int q = 0; q < kBatch; ++q) {
        const float f = pow2(mp[q] - mm);
        L += lp[q] * f;
#pragma unroll
        for (int e = 0; e < kPer; ++e) o[e] += v[q][e] * f;
      }
    }
    if constexpr (BY_UNIT) {  // the warps' shares of the parts
      if (lane == 0) {
        m_s[warp] = M;
        l_s[warp] = L;
      }
#pragma unroll
      for (int e = 0; e < kPer; ++e) o_s[warp * D + lane * kPer + e] = o[e];
      __syncthreads();
      if (warp > 0) return;
      M = -INFINITY;
#pragma unroll
      for (int i = 0; i < kJoinWarps; ++i) M = fmaxf(M, m_s[i]);
      const float mm = M == -INFINITY ? 0.f : M;
      L = 0.f;
#pragma unroll
      for (int e = 0; e < kPer; ++e) o[e] = 0.f;
#pragma unroll
      for (int i = 0; i < kJoinWarps; ++i) {
        const float f = pow2(m_s[i] - mm);
        L += l_s[i] * f;
#pragma unroll
        for (int e = 0; e < kPer; ++e) o[e] += o_s[i * D + lane * kPer + e] * f;
      }
    }
    const int j = (col0 + col) / a.group, h = u.h * a.group + (col0 + col) % a.group;
    const float inv = L > 0.f ? 1.f / L : (L == 0.f ? 0.f : L);
#pragma unroll
    for (int e = 0; e < kPer; ++e)
      store_elem(a.o.data, (u.s.first + j) * a.o.ld_tok + h * a.o.ld_head + lane * kPer + e, a.o.type, o[e] * inv);
    if (lane == 0 && a.lse)
      a.lse[(u.s.first + j) * a.q.heads + h] = L > 0.f ? (M + log2f(L)) / kLog2e : (L == 0.f ? -INFINITY : L);
  }
}

// An upper bound of the units: every sequence's columns, rounded up to whole groups.
template <int COLS>
int64_t most_units(const AttendArgs& a) {
  return (a.rows.n_tok * a.group / COLS + a.c.n_seq) * a.c.n_kv;
}

template <int D, int COLS>
crvq_status launch_join(const AttendArgs& a, cudaStream_t stream) {
  const int64_t units = most_units<COLS>(a);
  const dim3 threads(32 * kJoinWarps);
  // 8 units of 40 parts, 8 columns: 24 us by boundaries, 18 by units; 64 units of 7 parts: 16.5 and 20.5; 16 units of
  // 9 parts, 256 columns: 41 and 58.
  if constexpr (COLS <= 16)
    if (units * kJoinWarps <= a.shares) {
      CRVQ_CUDA(launch_pdl(attend_join_kernel<D, COLS, true>, dim3((unsigned)units, COLS), threads, 0, stream, a));
      CRVQ_LAUNCHED();
      return CRVQ_OK;
    }
  CRVQ_CUDA(launch_pdl(attend_join_kernel<D, COLS, false>, dim3((unsigned)a.shares - 1, COLS > 32 ? 8 : COLS / kJoinWarps),
                       threads, 0, stream, a));
  CRVQ_LAUNCHED();
  return CRVQ_OK;
}

}  // namespace

}  // namespace crvq
