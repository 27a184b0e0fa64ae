// Attention over the paged 8-bit cache for many queries per sequence (chunks of prompts), on tcgen05.
//
// A unit is 256 columns (query token, query head) of one kv head: two groups of 128 rows, the lanes of
// tensor memory. Per tile of 128 tokens and group X:
//   S_X = Q_X K^T (fp16 x fp16 codes, fp32 in tensor memory), softmax in registers, P_X = weights in fp16 over
//   S_X's own columns, O_X += P_X V (P_X read from tensor memory).
// Twelve warps and one: two softmax groups of four warps (thread = row), four warps that turn the tile's codes into
// fp16 operands (exact), one that issues the products. While one group's softmax runs, the other group's
// products do.
//   Keys and values have one layout, core matrices of 8 tokens x 8 channels: K-major for Q K^T, and
// MN-major (channels along N) for P V, so values need no transposition.
//   The key scales multiply scores in the softmax. A value scale s is an addend log2(s) in the weights' exponent,
// from which the sum takes it out again. Weights are relative to a power of two of their row, at the largest p s of
// the tokens that the row sees: fp16 has 2^-24 to 2^16, and a common reference (the largest scale of a tile, say) would
// leave nothing of a row that does not see the token with that scale, or gives it no weight. O is rescaled
// only when that of a warp's rows grows by more than 2^8 (weights are at most 2^14 in fp16), and then to every row's
// present one; a score's maximum that grows rescales the sum alone. fp16 outputs take the weights in two pieces, side
// by side over S's columns.
// Work is split like attend_mma.cuh's line: equal shares, a CTA per SM; units that lie in two shares are joined.
//
// What bounds it: a chain of about 5000 cycles per tile and group (waits, row maxima, weights, products), which two
// groups do not hide: the tensor pipe is active 35 % of the time, 0.44 instructions issue per cycle and scheduler, and
// no one of maxima, exponentials, operand stores and products takes more than a sixth of the time when left out.
// Two prompts of up to 1024 tokens over 8192, 64 heads on 8: 414 us, 751 TFLOP/s (39 % of the measured bf16 rate).
// Steps of 64 keys with scores two steps ahead were slower (520 when this form took 410), as were an issuing warp per
// group (413) and 16 softmax warps (spills).
#pragma once

#include "attend.cuh"
#include "tc_ops.cuh"

namespace crvq {

namespace {

constexpr int kRows = 128;                // rows of a group
constexpr int kUnit = 2 * kRows;          // columns of a unit
constexpr int kKeys = 128;                // tokens of a tile
constexpr int kTcThreads = 13 * 32;
constexpr float kTcLogWeight = 6.f;       // weights are scaled by 2^6, and up to 2^8 more before a rescale
constexpr float kLazy = 8.f;
constexpr uint32_t kTmemCols = 512;       // S_0, S_1 at 0, 128; O_0, O_1 at 256, 384

template <int D>
struct TcShape {
  static_assert(kTile<D> == kKeys, "the line's tiles are this kernel's");
  static constexpr int kQ = kRows * D * 2;
  static constexpr int kSide = kKeys * D * 2;  // keys or values of a tile
  static constexpr uint32_t kBand = D * 16;    // bytes of 8 tokens (rows)
  static constexpr size_t kSmem = 2 * kQ + 4 * kSide + 128;
  static constexpr int kSlot = kUnit * (D + 2);
};

// Byte offset of the 16-byte piece c (8 channels) of row r.
template <int D>
__device__ __forceinline__ uint32_t piece(int r, int c) {
  return (uint32_t)(r >> 3) * TcShape<D>::kBand + c * 128 + (r & 7) * 16;
}

// kind::f16, fp16 operands, fp32 accumulator; bn: B is MN-major.
constexpr uint32_t idesc_f16(int M, int N, bool bn) {
  return (1u << 4) | ((bn ? 1u : 0u) << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

// Issued by one lane of a whole warp (always the same): the operands are then the warp's, in uniform registers. From
// a branch that only lane 0 took, an issue cost about 100 cycles, more than the product itself.
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p, e;\n setp.ne.b32 p, %4, 0;\n elect.sync _|e, 0xffffffff;\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}

__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p, e;\n setp.ne.b32 p, %4, 0;\n elect.sync _|e, 0xffffffff;\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}

__device__ __forceinline__ void commit(uint64_t* bar) {
  asm volatile(
      "{\n .reg .pred e;\n elect.sync _|e, 0xffffffff;\n"
      " @e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}\n" ::"r"(tc::smem_u32(bar))
      : "memory");
}

// Two fp32 numbers at once.
__device__ __forceinline__ uint64_t pair(float x, float y) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
  return r;
}
__device__ __forceinline__ void halves(uint64_t v, float& x, float& y) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v));
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// Bounded wait; false once any wait of the CTA has run out. (Out of line but for the first look: the roles' code
// together overflowed the instruction caches.)
__device__ __noinline__ bool wait_longer(uint32_t bar, uint32_t parity, volatile int* dead, unsigned* err) {
  const unsigned long long t0 = tc::globaltimer();
  while (!tc::mbar_try_wait(bar, parity)) {
    if (*dead) return false;
    if (tc::globaltimer() - t0 > tc::kWaitNs) {
      raise_error(err, ERRBIT_TIMEOUT);
      *dead = 1;
      return false;
    }
  }
  return true;
}

__device__ __forceinline__ bool wait_for(uint64_t* bar, uint32_t parity, volatile int* dead, unsigned* err) {
  const uint32_t b = tc::smem_u32(bar);
  return tc::mbar_try_wait(b, parity) || wait_longer(b, parity, dead, err);
}

// Sixteen codes of a token as fp16, to two neighbouring pieces.
template <int FMT>
__device__ __forceinline__ void store_codes(char* dst, const uint4& u) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
  uint32_t h[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    h[2 * i] = codes2<FMT, 0>(w[i]);
    h[2 * i + 1] = codes2<FMT, 1>(w[i]);
  }
  *reinterpret_cast<uint4*>(dst) = make_uint4(h[0], h[1], h[2], h[3]);
  *reinterpret_cast<uint4*>(dst + 128) = make_uint4(h[4], h[5], h[6], h[7]);
}

__device__ __forceinline__ float4 four(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ float of(const float4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// Which of the 32 tokens from t0 on (two blocks) a row sees, as bits.
__device__ __forceinline__ uint32_t seen32(int t0, const int* live, int kb, int ke) {
  return range32(t0, kb, ke) & ((live[0] ? 0xffffu : 0u) | (live[1] ? 0xffff0000u : 0u));
}
// The same of a drafted token, by its row of bits.
__device__ __forceinline__ uint32_t seen32(const AttendArgs& a, int64_t row, int t0, const int* live, int kb, int held, int len) {
  return tree32(a, row, t0, kb, held, len) & ((live[0] ? 0xffffu : 0u) | (live[1] ? 0xffff0000u : 0u));
}

// Stores 16 consecutive columns of this thread's lane (waited for by tcgen05.wait::st).
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t r[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}

// A share's part of a unit.
struct Part {
  Unit u;
  int t_end;
  int col0, n_cols;
  int some_b, some_e;   // keys that some column sees
  int every_b, every_e; // keys that every column sees
  int first, n;         // tokens before the first tile that holds such a key; tiles
};

// The next part of a share whose places [*w, w1) are left; false past the last (whole warps, out of line).
template <int D, bool TREE>
__device__ __noinline__ bool find_part(const AttendArgs& a, const Line<D, kUnit>& line, int64_t* w, int64_t w1, Part* part) {
  Part& p = *part;
  while (*w < w1) {
    p.u = line.locate(a, *w);
    const Seq& s = p.u.s;
    const int64_t tile0 = p.u.begin + kStart, unit_end = tile0 + s.tiles;
    p.t_end = (int)max((int64_t)0, min(unit_end, w1) - tile0);
    *w = min(unit_end, w1);
    if (p.u.tile >= p.t_end) continue;
    p.col0 = p.u.cg * kUnit;
    p.n_cols = min(kUnit, s.n * a.group - p.col0);
    const int pos0 = s.len - s.n + p.col0 / a.group, pos1 = s.len - s.n + (p.col0 + p.n_cols - 1) / a.group;
    p.some_e = a.causal ? min(s.len, pos1 + 1) : s.len;
    p.some_b = a.window > 0 ? max(0, pos0 - a.window + 1) : 0;
    p.every_e = a.causal ? min(s.len, pos0 + 1) : s.len;
    p.every_b = a.window > 0 ? max(0, pos1 - a.window + 1) : 0;
    if constexpr (TREE) {  // (positions in any order among the sequence's last n places)
      p.some_e = s.len;
      p.some_b = a.window > 0 ? max(0, s.len - s.n - a.window + 1) : 0;
      p.every_e = min(s.len, s.len - s.n);
      p.every_b = a.window > 0 ? max(0, s.len - a.window) : 0;
    }
    const int t0 = max(p.u.tile, p.some_b / kKeys - s.lo);
    const int t1 = min(p.t_end, (max(0, p.some_e) + kKeys - 1) / kKeys - s.lo);
    p.first = (s.lo + t0) * kKeys;
    p.n = p.some_b < p.some_e ? max(0, t1 - t0) : 0;
    return true;
  }
  return false;
}

// TWO: weights in two fp16 pieces (22 bits), for outputs that a single piece's 11 bits would show in.
// TREE: the queries are trees of drafted tokens (AttendArgs::tree).
template <int D, int FMT, bool TWO, bool TREE = false>
__global__ void __launch_bounds__(kTcThreads, 1)
attend_tc_kernel(const __grid_constant__ AttendArgs a) {
  using S = TcShape<D>;
  extern __shared__ __align__(128) char sm[];
  __shared__ __align__(8) uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2], s_full[2], p_full[2], pv_done[2],
      q_full[2], all_done;
  __shared__ __align__(16) float sk_s[2][8], lg_s[2][8];  // key scales of a tile's blocks, log2 of the values'
  __shared__ __align__(16) int live_s[2][8];
  __shared__ uint32_t tmem_slot;
  __shared__ int dead_s;
  volatile int* dead = &dead_s;
  pdl_wait();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const Line<D, kUnit> line(a);
  const int64_t total = line.total;
  const int shares = (int)min((int64_t)a.shares, total);
  if ((int)blockIdx.x >= shares) return;
  const int64_t w1 = share_begin(total, blockIdx.x + 1, shares);

  if (warp == 12) tc::tmem_alloc(&tmem_slot, kTmemCols);
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      tc::mbar_init(tc::smem_u32(&k_full[i]), 128);
      tc::mbar_init(tc::smem_u32(&k_empty[i]), 1 + 8);  // the products, and every softmax warp (scales)
      tc::mbar_init(tc::smem_u32(&v_full[i]), 128);
      tc::mbar_init(tc::smem_u32(&v_empty[i]), 1);
      tc::mbar_init(tc::smem_u32(&s_full[i]), 1);
      tc::mbar_init(tc::smem_u32(&p_full[i]), 128);
      tc::mbar_init(tc::smem_u32(&pv_done[i]), 1);
      tc::mbar_init(tc::smem_u32(&q_full[i]), 128);
    }
    tc::mbar_init(tc::smem_u32(&all_done), 1);
    dead_s = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  const uint32_t tmem = tmem_slot;
  char* q_sm = sm;
  char* k_sm = sm + 2 * S::kQ;
  char* v_sm = k_sm + 2 * S::kSide;

  int64_t w = share_begin(total, blockIdx.x, shares);
  Part found;
  auto next_part = [&]() { return find_part<D, TREE>(a, line, &w, w1, &found); };
  bool ok = true;

  if (warp < 8) {
    // ------------------------------------------------------------------ softmax: thread = row of group X
    const int X = warp >> 2, row = tid & (kRows - 1);
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t s_at = tmem + lanes + X * 128, o_at = tmem + lanes + 256 + X * 128;
    char* q_mine = q_sm + X * S::kQ;
    uint32_t tile_no = 0, mine_no = 0;  // tiles of the share; of those that this group works on
    while (ok && next_part()) {
      const Part p = found;  // (in registers)
      const int r = X * kRows + row, c = p.col0 + r;
      const bool valid = r < p.n_cols, active = X == 0 || p.n_cols > kRows;
      const int j = valid ? c / a.group : 0, h = p.u.h * a.group + (valid ? c % a.group : 0);
      const int pos = p.u.s.len - p.u.s.n + j;
      const int kb = TREE ? tree_begin(a, p.u.s.first + j, p.u.s.len - p.u.s.n, p.u.s.len) : a.window > 0 ? max(0, pos - a.window + 1) : 0;
      const int ke = a.causal ? min(p.u.s.len, pos + 1) : p.u.s.len;
      auto sees = [&](int t0, const int* live) {
        if constexpr (TREE)
          return seen32(a, p.u.s.first + j, t0, live, kb, p.u.s.len - p.u.s.n, p.u.s.len);
        else
          return seen32(t0, live, kb, ke);
      };
      float f = 0.f;
      if (active && p.n > 0) {
        // the row of Q relative to the power of two at its largest element, in fp16 (sign of the scale included)
        const int64_t src = (p.u.s.first + j) * a.q.ld_tok + h * a.q.ld_head;
        uint4 raw[D / 8];
        if (valid && a.vec_q) {  // (all loads on their way before the first is used)
          const uint4* row_q = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.q.data) + src);
#pragma unroll
          for (int e = 0; e < D / 8; ++e) raw[e] = row_q[e];
        } else {
          const uint16_t* row_q = static_cast<const uint16_t*>(a.q.data) + src;
#pragma unroll
          for (int e = 0; e < D / 8; ++e) {
            uint32_t u[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
              u[i] = valid ? row_q[8 * e + 2 * i] | (uint32_t)row_q[8 * e + 2 * i + 1] << 16 : 0u;
            raw[e] = make_uint4(u[0], u[1], u[2], u[3]);
          }
        }
        // the largest magnitude, as bits (either type's order like integers); in fp32
        uint32_t top2 = 0;
#pragma unroll
        for (int e = 0; e < D / 8; ++e) {
          const uint32_t u[4] = {raw[e].x, raw[e].y, raw[e].z, raw[e].w};
#pragma unroll
          for (int i = 0; i < 4; ++i) top2 = __vmaxu2(top2, u[i] & 0x7fff7fffu);
        }
        const uint32_t top16 = max(top2 & 0xffffu, top2 >> 16);
        const float top = a.q.type == CRVQ_BF16 ? __uint_as_float(top16 << 16) : __half2float(__ushort_as_half((uint16_t)top16));
        const uint32_t ex = __float_as_uint(top) >> 23;
        const bool plain = ex == 0 || ex == 255;
        float inv = plain ? 1.f : __uint_as_float(ex == 254 ? 0x00400000u : (254u - ex) << 23);
        f = (plain ? 1.f : __uint_as_float(ex << 23)) * fabsf(a.scale);
        if (a.scale < 0.f) inv = -inv;
#pragma unroll
        for (int e = 0; e < D / 8; ++e) {
          const uint32_t u[4] = {raw[e].x, raw[e].y, raw[e].z, raw[e].w};
          uint32_t o[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float2 x;
            if (a.q.type == CRVQ_BF16)
              x = make_float2(__uint_as_float(u[i] << 16), __uint_as_float(u[i] & 0xffff0000u));
            else
              x = __half22float2(*reinterpret_cast<const __half2*>(&u[i]));
            o[i] = half2_bits(x.x * inv, x.y * inv);
          }
          *reinterpret_cast<uint4*>(q_mine + piece<D>(row, e)) = make_uint4(o[0], o[1], o[2], o[3]);
        }
        tc::fence_async_smem();
        tc::mbar_arrive(tc::smem_u32(&q_full[X]));
      }
      // All in log2: the score that the sum l is relative to, a whole number at the maximum or above; the weights'
      // reference and what it should be, the largest score + log2 s (whole numbers: rescales are exact).
      float m = -INFINITY, l = 0.f, ref = -INFINITY, top = -INFINITY;
      for (int i = 0; i < p.n && ok; ++i, ++tile_no) {
        const int buf = tile_no & 1;
        ok = wait_for(&k_full[buf], (tile_no >> 1) & 1, dead, a.err);
        if (active) {
          // (while the scores are on their way: what the blocks' scales say)
          const int tok = p.first + i * kKeys;
          const int4 lv0 = *reinterpret_cast<const int4*>(&live_s[buf][0]), lv1 = *reinterpret_cast<const int4*>(&live_s[buf][4]);
          const bool whole = (lv0.x & lv0.y & lv0.z & lv0.w & lv1.x & lv1.y & lv1.z & lv1.w) != 0 && tok >= p.every_b &&
                             tok + kKeys <= p.every_e;
          ok = ok && wait_for(&s_full[X], mine_no & 1, dead, a.err);
          tc::tc_fence_after();
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          // The row's maxima over the tile, then (after the rescale) its weights, half a tile at a time, in rolled
          // loops: unrolled, the warps' different code overflowed the instruction caches.
          float mt = -INFINITY, rt = -INFINITY;
          if (whole) {
#pragma unroll 1
            for (int half = 0; half < 2; ++half) {
              uint32_t u[64];
              tc::tmem_ld64_wait(s_at + half * 64, u);
              const float4 sk4 = four(&sk_s[buf][4 * half]), lg4 = four(&lg_s[buf][4 * half]);
#pragma unroll
              for (int b = 0; b < 4; ++b) {
                float t[8];
#pragma unroll
                for (int e = 0; e < 8; ++e)
                  t[e] = fmaxf(__uint_as_float(u[16 * b + e]), __uint_as_float(u[16 * b + 8 + e]));
#pragma unroll
                for (int w2 = 4; w2 > 0; w2 >>= 1)
#pragma unroll
                  for (int e = 0; e < w2; ++e) t[e] = fmaxf(t[e], t[e + w2]);
                const float best = t[0] * (of(sk4, b) * f);
                mt = fmaxf(mt, best);
                rt = fmaxf(rt, best + of(lg4, b));
              }
            }
          } else {
#pragma unroll 1
            for (int ch = 0; ch < 4; ++ch) {
              float v[32];
              tc::tmem_ld32(s_at + ch * 32, v);
              const uint32_t seen = sees(tok + 32 * ch, &live_s[buf][2 * ch]);
              const float s0 = sk_s[buf][2 * ch] * f, s1 = sk_s[buf][2 * ch + 1] * f;
              float best[2] = {-INFINITY, -INFINITY};
#pragma unroll
              for (int e = 0; e < 32; ++e)
                if (seen >> e & 1) best[e / 16] = fmaxf(best[e / 16], v[e] * (e < 16 ? s0 : s1));
              mt = fmaxf(mt, fmaxf(best[0], best[1]));
              rt = fmaxf(rt, fmaxf(best[0] + lg_s[buf][2 * ch], best[1] + lg_s[buf][2 * ch + 1]));
            }
          }
          const float mn = fmaxf(m, ceilf(mt));
          if (mn != m) l *= pow2(m - mn);
          m = mn;
          top = fmaxf(top, ceilf(rt));
          const bool need = top > ref + kLazy || (ref == -INFINITY && top > ref);
          if (i == 0) {
            ref = top;
          } else if (__any_sync(0xffffffffu, need)) {
            ok = wait_for(&pv_done[X], (mine_no - 1) & 1, dead, a.err);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            tc::tc_fence_after();
            const float fac = ref == top ? 1.f : pow2(ref - top);
            ref = top;  // (every row's: the warp's other rows will need it later)
#pragma unroll 1
            for (int ch = 0; ch < D / 32; ++ch) {
              float v[32];
              tc::tmem_ld32(o_at + ch * 32, v);
              uint32_t u[32];
#pragma unroll
              for (int e = 0; e < 32; ++e) u[e] = __float_as_uint(v[e] * fac);
              tc::tmem_st32_wait(o_at + ch * 32, u);
            }
          }
          // weights, over S's own columns (a half's scores are in registers before they are overwritten): in 32
          // columns each half's, second pieces in the next 32 where there are any
          const float mm = m == -INFINITY ? 0.f : m, rr = (ref == -INFINITY ? 0.f : ref) - kTcLogWeight;
          const float least = -54.f - mm;  // (2^-60 of the largest weight instead of less: the sum is taken from it, too)
#pragma unroll 1
          for (int half = 0; half < 2; ++half) {
            uint32_t u[64];
            tc::tmem_ld64_wait(s_at + half * 64, u);
            const uint32_t p_at = s_at + (TWO ? 64 : 32) * half;
            const float4 sk4 = four(&sk_s[buf][4 * half]), lg4 = four(&lg_s[buf][4 * half]);
            float bias[4], g[4];
#pragma unroll
            for (int b = 0; b < 4; ++b) {
              const float lw = of(lg4, b) - rr;
              bias[b] = lw < least ? least : lw;  // (a scale that is no number stays one)
              g[b] = of(sk4, b) * f;
            }
            if (whole) {
#pragma unroll
              for (int b = 0; b < 4; b += 2) {
                uint32_t hi[16], lo[TWO ? 16 : 1];
#pragma unroll
                for (int e0 = 0; e0 < 32; e0 += 16) {
                  const int bb = b + e0 / 16;
                  const uint64_t gg = pair(g[bb], g[bb]), bias2 = pair(bias[bb], bias[bb]);
                  uint64_t sum[4];
#pragma unroll
                  for (int e = 0; e < 16; e += 2) {
                    float x, y;
                    halves(fma2(pair(__uint_as_float(u[16 * bb + e]), __uint_as_float(u[16 * bb + e + 1])), gg, bias2), x, y);
                    x = pow2(x);
                    y = pow2(y);
                    sum[e / 2 & 3] = e < 8 ? pair(x, y) : add2(sum[e / 2 & 3], pair(x, y));
                    hi[(e0 + e) / 2] = half2_bits(x, y);
                    if constexpr (TWO) lo[(e0 + e) / 2] = half2_rest(x, y, hi[(e0 + e) / 2]);
                  }
                  float s0, s1;
                  halves(add2(add2(sum[0], sum[1]), add2(sum[2], sum[3])), s0, s1);
                  l = fmaf(s0 + s1, pow2(-mm - bias[bb]), l);
                }
                tmem_st16(p_at + b * 8, hi);
                if constexpr (TWO) tmem_st16(p_at + 32 + b * 8, lo);
              }
            } else {
#pragma unroll
              for (int b = 0; b < 4; b += 2) {
                uint32_t hi[16], lo[TWO ? 16 : 1];
                const uint32_t seen = sees(tok + 64 * half + 16 * b, &live_s[buf][4 * half + b]);
#pragma unroll
                for (int e0 = 0; e0 < 32; e0 += 16) {
                  const int bb = b + e0 / 16;
                  float sum = 0.f;
#pragma unroll
                  for (int e = 0; e < 16; e += 2) {
                    const float x = seen >> (e0 + e) & 1 ? pow2(fmaf(__uint_as_float(u[16 * bb + e]), g[bb], bias[bb])) : 0.f;
                    const float y = seen >> (e0 + e + 1) & 1 ? pow2(fmaf(__uint_as_float(u[16 * bb + e + 1]), g[bb], bias[bb])) : 0.f;
                    sum += x + y;
                    hi[(e0 + e) / 2] = half2_bits(x, y);
                    if constexpr (TWO) lo[(e0 + e) / 2] = half2_rest(x, y, hi[(e0 + e) / 2]);
                  }
                  if (sum != 0.f) l = fmaf(sum, pow2(-mm - bias[bb]), l);  // (an unseen scale may be anything)
                }
                tmem_st16(p_at + b * 8, hi);
                if constexpr (TWO) tmem_st16(p_at + 32 + b * 8, lo);
              }
            }
          }
          asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
          tc::tc_fence_before();
          tc::mbar_arrive(tc::smem_u32(&p_full[X]));
          ++mine_no;
        }
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        if (lane == 0) tc::mbar_arrive(tc::smem_u32(&k_empty[buf]));
      }
      if (!ok) break;
      // the part's rows
      const bool complete = p.u.tile == 0 && p.t_end == p.u.s.tiles;
      if (active && p.n > 0) {
        ok = wait_for(&pv_done[X], (mine_no - 1) & 1, dead, a.err);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        tc::tc_fence_after();
      }
      const float inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);
      const float fac = p.n > 0 ? pow2(ref - kTcLogWeight - (m == -INFINITY ? 0.f : m)) * (complete ? inv : 1.f) : 0.f;
      float* part = a.part + (int64_t)(2 * blockIdx.x + (p.u.tile == 0 ? 1 : 0)) * S::kSlot;
      if (active) {
        // 32 columns at a time through this warp's rows of Q's memory (read whole by now), then rows by neighbouring
        // lanes: a thread's own row, 16 bytes in each of 32 lines per store, took 9000 cycles
        float* stage = reinterpret_cast<float*>(q_mine + (warp & 3) * (S::kQ / 4));
        const int r0 = X * kRows + (warp & 3) * 32;  // this warp's first row
#pragma unroll 1
        for (int ch = 0; ch < D / 32; ++ch) {
          float v[32];
          if (p.n > 0) {
            tc::tmem_ld32(o_at + ch * 32, v);
#pragma unroll
            for (int e = 0; e < 32; ++e) v[e] *= fac;
          } else {
#pragma unroll
            for (int e = 0; e < 32; ++e) v[e] = 0.f;
          }
          __syncwarp();
#pragma unroll
          for (int e = 0; e < 8; ++e)  // (16-byte units exchanged by the row: no bank conflicts)
            *reinterpret_cast<float4*>(stage + lane * 32 + ((e ^ lane & 7) * 4)) =
                make_float4(v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]);
          __syncwarp();
          auto unit = [&](int rr, int e) {
            return *reinterpret_cast<const float4*>(stage + rr * 32 + ((e ^ rr & 7) * 4));
          };
          if (!complete) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              const int rr = 4 * k + (lane >> 3);
              if (r0 + rr < p.n_cols)
                *reinterpret_cast<float4*>(part + (r0 + rr) * D + ch * 32 + (lane & 7) * 4) = unit(rr, lane & 7);
            }
          } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const int rr = 8 * k + (lane >> 2), cc = p.col0 + r0 + rr;
              if (r0 + rr < p.n_cols) {
                const float4 x = unit(rr, 2 * (lane & 3)), y = unit(rr, 2 * (lane & 3) + 1);
                const float o[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
                store8(a.o.data, (p.u.s.first + cc / a.group) * a.o.ld_tok + (p.u.h * a.group + cc % a.group) * a.o.ld_head +
                                     ch * 32 + (lane & 3) * 8, a.o.type, a.vec_o, o);
              }
            }
          }
        }
        tc::tc_fence_before();  // (O is overwritten after this group's next arrival)
        if (valid) {
          if (!complete) {
            part[kUnit * D + r] = m;
            part[kUnit * D + kUnit + r] = l;
          } else if (a.lse) {
            a.lse[(p.u.s.first + j) * a.q.heads + h] = l > 0.f ? (m + log2f(l)) / kLog2e : (l == 0.f ? -INFINITY : l);
          }
        }
      }
    }
  } else if (warp < 12) {
    // ------------------------------------------------------------------ codes to operands: 32 tokens per warp
    const int cw = warp - 8;
    constexpr int UH = D / 64;
    uint4 kr[4][UH], vr[4][UH];
    int64_t at[2], at_n[2];
    float sk[2], sv[2], sk_n[2], sv_n[2];
    uint32_t tile_no = 0;
    while (ok && next_part()) {
      const Part p = found;  // (in registers)
      const int len = p.u.s.len, tok0 = p.first + 32 * cw;
      auto look_up = [&](int i) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const int tok = tok0 + i * kKeys + 16 * b;
          at_n[b] = -1;
          sk_n[b] = sv_n[b] = 0.f;
          if (i < p.n && tok < p.some_e && tok + kCacheBlock > p.some_b) {
            const int64_t page = seq_page(a.c, p.u.b, tok / a.c.page, a.err);
            if (page >= 0) {
              const int in = tok % a.c.page;
              at_n[b] = page * a.c.page_stride + ((int64_t)p.u.h * a.c.page + in) * D;
              const int64_t at_s = (page * a.c.n_kv + p.u.h) * (a.c.page / kCacheBlock) + in / kCacheBlock;
              sk_n[b] = __ldg(a.c.ks + at_s);
              sv_n[b] = __ldg(a.c.vs + at_s);
            }
          }
        }
      };
      // lane: rows (lane & 7) of each 8, 16-byte units (lane >> 3) of each 4
      auto load = [&](const uint8_t* base, int i, bool values, uint4 (&x)[4][UH]) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int r = 8 * g + (lane & 7);
          const bool in = at_n[g >> 1] >= 0 && !(values && tok0 + i * kKeys + r >= len);
#pragma unroll
          for (int u = 0; u < UH; ++u)
            x[g][u] = in ? __ldg(reinterpret_cast<const uint4*>(base + at_n[g >> 1] + (8 * (g & 1) + (lane & 7)) * D +
                                                                (4 * u + (lane >> 3)) * 16))
                         : make_uint4(0, 0, 0, 0);
        }
      };
      auto store = [&](char* dst, const uint4 (&x)[4][UH]) {
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
          for (int u = 0; u < UH; ++u)
            store_codes<FMT>(dst + piece<D>(32 * cw + 8 * g + (lane & 7), 2 * (4 * u + (lane >> 3))), x[g][u]);
      };
      auto take = [&]() {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          at[b] = at_n[b];
          sk[b] = sk_n[b];
          sv[b] = sv_n[b];
        }
      };
      if (p.n > 0) look_up(0);
      for (int i = -1; i < p.n && ok; ++i) {  // tile i's operands are written, tile i + 1's codes loaded
        const int buf = tile_no & 1;
        const uint32_t ph = ((tile_no >> 1) & 1) ^ 1;
        if (i >= 0) {
          ok = wait_for(&k_empty[buf], ph, dead, a.err);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          if (lane < 2) {
            sk_s[buf][2 * cw + lane] = lane ? sk[1] : sk[0];
            lg_s[buf][2 * cw + lane] = log2f(lane ? sv[1] : sv[0]);
            live_s[buf][2 * cw + lane] = (lane ? at[1] : at[0]) >= 0;
          }
          store(k_sm + buf * S::kSide, kr);
          tc::fence_async_smem();
          __syncwarp();
          tc::mbar_arrive(tc::smem_u32(&k_full[buf]));
        }
        if (i + 1 < p.n) load(a.c.K, i + 1, false, kr);
        if (i >= 0) {
          ok = wait_for(&v_empty[buf], ph, dead, a.err);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          store(v_sm + buf * S::kSide, vr);
          tc::fence_async_smem();
          tc::mbar_arrive(tc::smem_u32(&v_full[buf]));
          ++tile_no;
        }
        if (i + 1 < p.n) load(a.c.V, i + 1, true, vr);
        take();
        look_up(i + 2);
      }
    }
  } else {
    // ------------------------------------------------------------------ products (the whole warp, one lane issues)
    constexpr uint32_t kQk = idesc_f16(kRows, kKeys, false), kPv = idesc_f16(kRows, D, true);
    const uint64_t q_desc = tc::smem_desc(tc::smem_u32(q_sm), 128, S::kBand);
    const uint64_t k_desc = tc::smem_desc(tc::smem_u32(k_sm), 128, S::kBand);
    const uint64_t v_desc = tc::smem_desc(tc::smem_u32(v_sm), S::kBand, 128);
    uint32_t tile_no = 0, mine_no[2] = {0, 0}, q_no[2] = {0, 0};
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      ok = ok && wait_for(bar, parity, dead, a.err);
      ok = __all_sync(0xffffffffu, ok);
      return ok;
    };
    auto scores = [&](int X, int buf) {  // S_X = Q_X K^T (descriptors count 16 bytes)
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks)
        mma_ss(tmem + X * 128, q_desc + (X * S::kQ + ks * 256) / 16, k_desc + (buf * S::kSide + ks * 256) / 16, kQk, ks > 0);
      commit(&s_full[X]);
    };
    while (ok && next_part()) {
      const Part p = found;  // (in registers)
      if (p.n == 0) continue;
      const int groups = p.n_cols > kRows ? 2 : 1;
      for (int X = 0; X < groups; ++X) {
        if (!wait(&q_full[X], q_no[X] & 1)) break;
        ++q_no[X];
      }
      if (!wait(&k_full[tile_no & 1], (tile_no >> 1) & 1)) break;
      tc::tc_fence_after();
      for (int X = 0; X < groups; ++X) scores(X, tile_no & 1);
      commit(&k_empty[tile_no & 1]);
      for (int i = 0; i < p.n && ok; ++i, ++tile_no) {
        const int buf = tile_no & 1, nbuf = buf ^ 1;
        if (!wait(&v_full[buf], (tile_no >> 1) & 1)) break;
        for (int X = 0; X < groups; ++X) {
          if (!wait(&p_full[X], mine_no[X] & 1)) break;
          tc::tc_fence_after();
#pragma unroll
          for (int ks = 0; ks < kKeys / 16; ++ks)
#pragma unroll
            for (int z = 0; z < (TWO ? 2 : 1); ++z)
              mma_ts(tmem + 256 + X * 128, tmem + X * 128 + (TWO ? (ks >> 2) * 64 + z * 32 + (ks & 3) * 8 : ks * 8),
                     v_desc + (buf * S::kSide + ks * 2 * (int)S::kBand) / 16, kPv, i > 0 || ks > 0 || z > 0);
          commit(&pv_done[X]);
          if (X == groups - 1) commit(&v_empty[buf]);
          if (i + 1 < p.n) {
            if (X == 0 && !wait(&k_full[nbuf], ((tile_no + 1) >> 1) & 1)) break;
            // the weights lie where the next scores go
            if (!wait(&pv_done[X], mine_no[X] & 1)) break;
            tc::tc_fence_after();
            scores(X, nbuf);
            if (X == groups - 1) commit(&k_empty[nbuf]);
          }
          ++mine_no[X];
        }
      }
    }
    __syncwarp();
    commit(&all_done);  // whatever was issued has ended before tensor memory is freed
    tc::mbar_wait(tc::smem_u32(&all_done), 0, a.err);
    __syncwarp();
  }
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  if (warp == 12) tc::tmem_dealloc(tmem, kTmemCols);
}

template <int D, int FMT, bool TWO, bool TREE>
crvq_status launch_tc(AttendArgs& a, cudaStream_t stream) {
  using S = TcShape<D>;
  auto kernel = attend_tc_kernel<D, FMT, TWO, TREE>;
  CRVQ_TRY(smem_limit((const void*)kernel, S::kSmem));
  a.shares = sm_count();
  Scratch mem;
  CRVQ_TRY(mem.alloc((size_t)2 * a.shares * S::kSlot * sizeof(float), stream));
  a.part = mem.as<float>();
  ProfScope ps("cache_attention", stream, (double)a.rows.n_tok * a.q.heads * D);
  CRVQ_CUDA(launch_pdl(kernel, dim3((unsigned)a.shares), dim3(kTcThreads), S::kSmem, stream, a));
  CRVQ_LAUNCHED();
  return launch_join<D, kUnit>(a, stream);
}

// (bf16 outputs' own rounding is 8 times a single piece's error. fp16 outputs with a single piece were 1.4 to 1.5 times as
// far from exact as their rounding; the second one takes two prompts of up to 1024 tokens over 8192 from 414 to 487 us. Trees of 64
// tokens over two sequences of up to 65536 in bf16, one piece and two: 1.672e-3 and 1.659e-3 from exact, 340 and 371 us.)
template <int D, bool TREE>
crvq_status pick_tc(AttendArgs& a, int format, cudaStream_t stream) {
  const bool two = a.q.type == CRVQ_F16;
  if (format == CRVQ_KV_INT8)
    return two ? launch_tc<D, CRVQ_KV_INT8, true, TREE>(a, stream) : launch_tc<D, CRVQ_KV_INT8, false, TREE>(a, stream);
  return two ? launch_tc<D, CRVQ_KV_E4M3, true, TREE>(a, stream) : launch_tc<D, CRVQ_KV_E4M3, false, TREE>(a, stream);
}

}  // namespace

}  // namespace crvq
