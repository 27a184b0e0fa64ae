// Accumulated attention weights for many queries per sequence (see weights.cu for the formula), on tcgen05.
//
// S^T (128 tokens x up to 256 columns) = K Q^T: tokens are the lanes of tensor memory, so a thread has one token's scores, and
// its sum over the columns is its own: no maxima, no shuffles. All columns' queries (512 at a time, as they are) lie in shared
// memory while the tiles of a (sequence, kv head) pass. Codes become operands of the queries' type, exactly: no query needs
// a factor but bf16 ones so large that their sums could leave fp32's range where scores do not. Those are laid out relative to the
// power of two at their largest element, which joins a factor per column; all tiles then go by these factors, with the loop of
// tiles that some columns do not see, while this filling of Q's memory lasts. Looking for them takes 1.2 us of 90.
// Two groups of four warps take every other tile, each with its own half of tensor memory and its own issuing warp; four warps
// turn codes into operands. While one group's exponentials run, the other's products do, and its own next 128 columns' (two
// of 64 queries over up to 32768 tokens, 64 heads on 8: 92.8 -> 90.6 us).
// Work is split like attend_mma.cuh's line: equal shares of all tiles, a CTA per SM; while a filling of Q's memory lasts, every token
// is one thread's (the next filling's may be the other group's, which has waited for all to be done with the one before).
//   What bounds it: the chain from tensor memory to registers, exponentials and sums, 32 columns at a time, of two warps per scheduler
// (690 TFLOP/s of products; the tensor pipe is active 28% of the time). Slower, in us: four groups of 128 columns 128, loads in
// two buffers 112 (with 168 registers, and two converting warps for that, 97), an eighth of the exponentials by a polynomial 97,
// one power of two for all columns of fp16 operands 113.
#include "attend_tc.cuh"
#include "weights.cuh"

namespace crvq {

namespace {

constexpr int kMostCols = 512, kStepCols = 128;  // a group's two halves of its 256 columns of tensor memory
constexpr int kWtThreads = 14 * 32;

template <int D>
struct WtShape {
  static constexpr int kQ = kMostCols * D * 2;
  static constexpr int kSide = kKeys * D * 2;
  static constexpr size_t kSmem = kQ + 2 * kSide + kMostCols * 16;
};

// Queries of elements below 2^65 go as they are by a scale of up to 2^60: over 128 channels and codes up to 448 their sums stay
// below 2^81; where the scale times a key's scale has lost bits, below 2^-126, their scores are below 2^-45; and that product is
// beyond fp32's range for a key's scale above 2^67 alone. By a larger scale all queries are laid out with a factor.
constexpr float kNearScale = 0x1p60f;

__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// Codes 0, 1 (half 0) or 2, 3 (half 1) of a word as bf16: exact, both formats have 8 significant bits at most.
template <int FMT, int HALF>
__device__ __forceinline__ uint32_t codes2_bf16(uint32_t w) {
  if constexpr (FMT == CRVQ_KV_INT8) {
    // c = (128 + (u & 127)) - (u & 128 ? 128 : 256) for u = c + 128
    const uint32_t u = w ^ 0x80808080u;
    const uint32_t x = __byte_perm(u & 0x7f7f7f7fu, 0x43434343u, HALF ? 0x4342 : 0x4140);
    const uint32_t y = __byte_perm((u & 0x80808080u) ^ 0x80808080u, 0x43434343u, HALF ? 0x4342 : 0x4140);
    const __nv_bfloat162 v = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&x), *reinterpret_cast<const __nv_bfloat162*>(&y));
    return *reinterpret_cast<const uint32_t*>(&v);
  } else {
    const uint32_t h = codes2<FMT, HALF>(w);
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
    return __byte_perm(__float_as_uint(f.x), __float_as_uint(f.y), 0x7632);
  }
}

// Sixteen codes of a token as the queries' type, to two neighbouring pieces.
template <int FMT, bool BF16>
__device__ __forceinline__ void store_codes(char* dst, const uint4& u) {
  if constexpr (!BF16) {
    store_codes<FMT>(dst, u);
  } else {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
    uint32_t h[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      h[2 * i] = codes2_bf16<FMT, 0>(w[i]);
      h[2 * i + 1] = codes2_bf16<FMT, 1>(w[i]);
    }
    *reinterpret_cast<uint4*>(dst) = make_uint4(h[0], h[1], h[2], h[3]);
    *reinterpret_cast<uint4*>(dst + 128) = make_uint4(h[4], h[5], h[6], h[7]);
  }
}

// Lays column col of Q out relative to the power of two at its largest element, if that is 2^65 or more (or all are to be), with the
// power joined to its factor. Four lanes have every fourth piece each, e0 the first; a warp has eight columns.
template <int D>
__device__ __forceinline__ void far_column(char* q_sm, int col, int e0, bool all, float* f_s) {
  uint32_t top2 = 0;
  for (int i = 0; i < D / 32; ++i) {
    const uint4 x = *reinterpret_cast<const uint4*>(q_sm + piece<D>(col, 4 * i + e0));
    top2 = __vmaxu2(top2, __vmaxu2(__vmaxu2(x.x & 0x7fff7fffu, x.y & 0x7fff7fffu), __vmaxu2(x.z & 0x7fff7fffu, x.w & 0x7fff7fffu)));
  }
  top2 = __vmaxu2(top2, __shfl_xor_sync(0xffffffffu, top2, 8));
  top2 = __vmaxu2(top2, __shfl_xor_sync(0xffffffffu, top2, 16));
  const uint32_t ex = max(top2 & 0xffffu, top2 >> 16) >> 7;
  if (ex == 0 || ex == 255 || !(all || ex >= 192)) return;
  const float inv = __uint_as_float(ex == 254 ? 0x00400000u : (254u - ex) << 23);
  auto times = [&](uint32_t v) {  // (exact, but for elements below 2^-126 of the largest)
    return __byte_perm(__float_as_uint(__uint_as_float(v << 16) * inv), __float_as_uint(__uint_as_float(v & 0xffff0000u) * inv), 0x7632);
  };
  for (int i = 0; i < D / 32; ++i) {
    uint4& x = *reinterpret_cast<uint4*>(q_sm + piece<D>(col, 4 * i + e0));
    x = make_uint4(times(x.x), times(x.y), times(x.z), times(x.w));
  }
  if (e0 == 0) f_s[col] *= __uint_as_float(ex << 23);
}

// The same for all of this warp's columns; true if there were any. (Out of line: its registers are not the tiles'.)
template <int D>
__device__ __noinline__ bool far_columns(char* q_sm, int n_pad, bool all, float* f_s) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t large = all ? 0x40004000u : 0u;  // elements of 2^65 and more: exponents of 11......
#pragma unroll 2
  for (int col = 8 * warp + (lane & 7); col < n_pad; col += 64) {
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {  // (a lane looks at what it copied)
      const uint4 x = *reinterpret_cast<const uint4*>(q_sm + piece<D>(col, 4 * i + (lane >> 3)));
      large |= (x.x & x.x << 1) | (x.y & x.y << 1) | (x.z & x.z << 1) | (x.w & x.w << 1);
    }
  }
  if (!__any_sync(0xffffffffu, large & 0x40004000u)) return false;
  for (int col = 8 * warp + (lane & 7); col < n_pad; col += 64) far_column<D>(q_sm, col, lane >> 3, all, f_s);
  return true;
}

template <int D, int FMT, bool BF16>
__global__ void __launch_bounds__(kWtThreads, 1) weights_tc_kernel(const __grid_constant__ WeightArgs w) {
  using S = WtShape<D>;
  const AttendArgs& a = w.a;
  extern __shared__ __align__(128) char sm[];
  __shared__ __align__(8) uint64_t k_full[2], k_empty[2], s_full[2][2], s_empty[2][2], q_full, q_read, all_done[2];
  __shared__ float sk_s[2][8];
  __shared__ int live_s[2][8];
  __shared__ uint32_t far_s;  // number + 1 of the last filling with far queries
  __shared__ uint32_t tmem_slot;
  __shared__ int dead_s;
  volatile int* dead = &dead_s;
  pdl_wait();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const Line<D, kAllColumns> line(a);
  const int shares = (int)min((int64_t)a.shares, line.total);
  int64_t at = 0, at_end = 0;
  if ((int)blockIdx.x < shares) {
    at = share_begin(line.total, blockIdx.x, shares);
    at_end = share_begin(line.total, blockIdx.x + 1, shares);
  }
  char* q_sm = sm;
  char* k_sm = sm + S::kQ;
  float* l_s = reinterpret_cast<float*>(k_sm + 2 * S::kSide);  // [kMostCols] -lse, first and last + 1 key seen
  int* kb_s = reinterpret_cast<int*>(l_s + kMostCols);
  int* ke_s = kb_s + kMostCols;
  float* f_s = reinterpret_cast<float*>(ke_s + kMostCols);     // the scale, times the query's power of two if it is far
  if (warp == 12) tc::tmem_alloc(&tmem_slot, 4 * kStepCols);
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      tc::mbar_init(tc::smem_u32(&k_full[i]), 128);
      tc::mbar_init(tc::smem_u32(&k_empty[i]), 1 + 4);  // the products, and the group's warps (scales)
      for (int j = 0; j < 2; ++j) {
        tc::mbar_init(tc::smem_u32(&s_full[i][j]), 1);
        tc::mbar_init(tc::smem_u32(&s_empty[i][j]), 128);
      }
      tc::mbar_init(tc::smem_u32(&all_done[i]), 1);
    }
    tc::mbar_init(tc::smem_u32(&q_full), 256);
    tc::mbar_init(tc::smem_u32(&q_read), 256 + 2);  // (and the issuing warps, one of which may have no tile: neither falls a filling behind)
    dead_s = 0;
    far_s = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  const uint32_t tmem = tmem_slot;

  Unit u;
  int n_tiles = 0;      // of the part
  int64_t cols = 0;
  auto next_part = [&]() {
    while (at < at_end) {
      u = line.locate(a, at);
      const int64_t tile0 = u.begin + kStart, unit_end = tile0 + u.s.tiles;
      const int t_end = (int)max((int64_t)0, min(unit_end, at_end) - tile0);
      at = min(unit_end, at_end);
      n_tiles = t_end - u.tile;
      cols = (int64_t)u.s.n * a.group;
      if (n_tiles > 0) return true;
    }
    return false;
  };
  bool ok = true;
  uint32_t tile_no = 0, q_no = 0;  // tiles, and fillings of Q's memory, of this share
  auto wait = [&](uint64_t* bar, uint32_t parity) {
    ok = ok && wait_for(bar, parity, dead, a.err);
    ok = __all_sync(0xffffffffu, ok);
    return ok;
  };

  if (warp < 8) {
    // ------------------------------------------------------------------ exponentials: thread = token of every other tile
    const int X = warp >> 2, row = tid & (kKeys - 1);
    const uint32_t s_at = tmem + ((uint32_t)((warp & 3) * 32) << 16) + X * 2 * kStepCols;
    uint32_t s_no = 0;
    while (ok && next_part()) {
      const int len = u.s.len, held = len - u.s.n;
      float* out = w.out + u.b * w.out_seq + u.h * w.out_head;
      const float* before = w.before ? w.before + u.b * w.before_seq + u.h * w.before_head : nullptr;
      for (int64_t c0 = 0; c0 < cols && ok; c0 += kMostCols, ++q_no) {
        const int n_cols = (int)min((int64_t)kMostCols, cols - c0), n_pad = (n_cols + 31) / 32 * 32;
        // every thread has read what lay there before; products that read it have ended (their scores have been read)
        if (q_no > 0 && !wait(&q_read, (q_no - 1) & 1)) break;
        // a warp takes 8 columns at a time; lane: column (lane & 7), 16-byte pieces (lane >> 3) of each 4. All lse first.
        constexpr int kTimes = kMostCols / 64;
        float lse[kTimes];
        auto query = [&](int col, int* h) {  // (a padding column: any)
          const uint32_t c = (uint32_t)c0 + (col < n_cols ? col : 0), j = c / (uint32_t)a.group;
          *h = u.h * a.group + (int)(c - j * (uint32_t)a.group);
          return (int)j;
        };
#pragma unroll
        for (int k = 0; k < kTimes; ++k) {
          const int col = 64 * k + 8 * warp + (lane & 7);
          int h;
          const int j = query(col, &h);
          lse[k] = col < n_cols ? __ldg(w.lse + (u.s.first + j) * a.q.heads + h) : INFINITY;
        }
#pragma unroll
        for (int k = 0; k < kTimes; ++k) {
          const int col = 64 * k + 8 * warp + (lane & 7);
          if (col >= n_pad) break;
          int h;
          const int j = query(col, &h);
          const bool none = isinf(lse[k]);  // (such a query has no weights)
          const uint16_t* row_q = static_cast<const uint16_t*>(a.q.data) + (u.s.first + j) * a.q.ld_tok + h * a.q.ld_head;
#pragma unroll
          for (int i = 0; i < D / 32; ++i) {
            const int e = 4 * i + (lane >> 3);
            char* dst = q_sm + piece<D>(col, e);
            if (a.vec_q) {
              asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(tc::smem_u32(dst)), "l"(row_q + 8 * e), "r"(none ? 0 : 16) : "memory");
            } else {
              uint32_t x[4];
#pragma unroll
              for (int y = 0; y < 4; ++y) x[y] = none ? 0u : row_q[8 * e + 2 * y] | (uint32_t)row_q[8 * e + 2 * y + 1] << 16;
              *reinterpret_cast<uint4*>(dst) = make_uint4(x[0], x[1], x[2], x[3]);
            }
          }
          if (lane < 8) {
            const int pos = held + j;
            l_s[col] = none ? -INFINITY : -lse[k];
            kb_s[col] = a.window > 0 ? max(0, pos - a.window + 1) : 0;
            ke_s[col] = a.causal ? min(len, pos + 1) : len;
            f_s[col] = w.scale;
          }
        }
        asm volatile("cp.async.commit_group;\ncp.async.wait_group 0;" ::: "memory");
        if constexpr (BF16)
          if (far_columns<D>(q_sm, n_pad, fabsf(w.scale) > kNearScale, f_s)) far_s = q_no + 1;
        tc::fence_async_smem();
        tc::mbar_arrive(tc::smem_u32(&q_full));
        if (!wait(&q_full, q_no & 1)) break;
        // keys that every column sees (places do not fall from column to column)
        const int every_b = BF16 && far_s == q_no + 1 ? INT_MAX : kb_s[n_cols - 1], every_e = ke_s[0];
        for (int i = 0; i < n_tiles && ok; ++i, ++tile_no) {
          if ((int)(tile_no & 1) != X) continue;
          const int tok = (u.s.lo + u.tile + i) * kKeys, t = tok + row;
          if (!wait(&k_full[X], (tile_no >> 1) & 1)) break;
          const float sk = sk_s[X][row >> 4];
          const bool live = live_s[X][row >> 4] != 0;
          __syncwarp();
          if (lane == 0) tc::mbar_arrive(tc::smem_u32(&k_empty[X]));
          const bool writes = t < len && t < w.width;
          float base = 0.f;
          if (writes) {
            if (c0 > 0)
              base = out[t];
            else if (before)
              base = w.decay * before[t];
          }
          const bool whole = tok >= every_b && tok + kKeys <= every_e;
          const float g = w.scale * sk;
          const uint64_t g2 = pair(g, g), log2e = pair(kLog2e, kLog2e);
          uint64_t sum[4] = {0, 0, 0, 0};
          for (int h0 = 0; h0 < n_pad; h0 += kStepCols, ++s_no) {
            const int half = s_no & 1;
            if (!wait(&s_full[X][half], (s_no >> 1) & 1)) break;
            tc::tc_fence_after();
            const int n = min(kStepCols, n_pad - h0);
#pragma unroll 1
            for (int ch = 0; ch < n; ch += 32) {
              float v[32];
              tc::tmem_ld32(s_at + half * kStepCols + ch, v);
              const float* l = l_s + h0 + ch;
              if (whole) {
#pragma unroll
                for (int e = 0; e < 32; e += 4) {
                  const float4 l4 = four(l + e);
                  float x[4];
                  halves(mul2(fma2(pair(v[e], v[e + 1]), g2, pair(l4.x, l4.y)), log2e), x[0], x[1]);
                  halves(mul2(fma2(pair(v[e + 2], v[e + 3]), g2, pair(l4.z, l4.w)), log2e), x[2], x[3]);
                  sum[e / 2 & 3] = add2(sum[e / 2 & 3], pair(pow2(x[0]), pow2(x[1])));
                  sum[(e / 2 + 1) & 3] = add2(sum[(e / 2 + 1) & 3], pair(pow2(x[2]), pow2(x[3])));
                }
              } else {
                // (sixteen bytes at a time: number by number, with a factor, these few tiles took 2.5 us of 93)
                const int4* kb = reinterpret_cast<const int4*>(kb_s + h0 + ch);
                const int4* ke = reinterpret_cast<const int4*>(ke_s + h0 + ch);
                const float* f = f_s + h0 + ch;
                auto weight = [&](float s, float fc, float lc, int b, int e) {
                  const float x = pow2(fmaf(s, fc * sk, lc) * kLog2e);
                  return t >= b && t < e ? x : 0.f;
                };
#pragma unroll
                for (int e = 0; e < 32; e += 4) {
                  const float4 l4 = four(l + e), f4 = four(f + e);
                  const int4 b4 = kb[e / 4], e4 = ke[e / 4];
                  sum[e / 2 & 3] = add2(sum[e / 2 & 3], pair(weight(v[e], f4.x, l4.x, b4.x, e4.x), weight(v[e + 1], f4.y, l4.y, b4.y, e4.y)));
                  sum[(e / 2 + 1) & 3] =
                      add2(sum[(e / 2 + 1) & 3], pair(weight(v[e + 2], f4.z, l4.z, b4.z, e4.z), weight(v[e + 3], f4.w, l4.w, b4.w, e4.w)));
                }
              }
            }
            tc::tc_fence_before();
            tc::mbar_arrive(tc::smem_u32(&s_empty[X][half]));
          }
          float x, y;
          halves(add2(add2(sum[0], sum[1]), add2(sum[2], sum[3])), x, y);
          if (writes && ok) out[t] = base + (live ? x + y : 0.f);
        }
        tc::mbar_arrive(tc::smem_u32(&q_read));
      }
    }
  } else if (warp < 12) {
    // ------------------------------------------------------------------ codes to operands: 32 tokens per warp
    const int cw = warp - 8;
    constexpr int UH = D / 64;
    // codes of two tiles on their way, and places and scales of the one after them
    uint4 kr[2][4][UH];
    int64_t place[3][2];
    float sk[3][2];
    while (ok && next_part()) {
      const int len = u.s.len, tok0 = (u.s.lo + u.tile) * kKeys + 32 * cw;
      const int some_b = a.window > 0 ? max(0, len - u.s.n - a.window + 1) : 0;
      auto look_up = [&](int i, int64_t (&p)[2], float (&scale)[2]) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const int tok = tok0 + i * kKeys + 16 * b;
          p[b] = -1;
          scale[b] = 0.f;
          if (i < n_tiles && tok < len && tok + kCacheBlock > some_b) {
            const int64_t page = seq_page(a.c, u.b, tok / a.c.page, a.err);
            if (page >= 0) {
              const int in = tok % a.c.page;
              p[b] = page * a.c.page_stride + ((int64_t)u.h * a.c.page + in) * D;
              scale[b] = __ldg(a.c.ks + (page * a.c.n_kv + u.h) * (a.c.page / kCacheBlock) + in / kCacheBlock);
            }
          }
        }
      };
      // lane: rows (lane & 7) of each 8, 16-byte units (lane >> 3) of each 4
      auto load = [&](const int64_t (&p)[2], uint4 (&x)[4][UH]) {
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
          for (int e = 0; e < UH; ++e)
            x[g][e] = p[g >> 1] >= 0 ? __ldg(reinterpret_cast<const uint4*>(a.c.K + p[g >> 1] + (8 * (g & 1) + (lane & 7)) * D + (4 * e + (lane >> 3)) * 16))
                                     : make_uint4(0, 0, 0, 0);
      };
      auto store = [&](const int64_t (&p)[2], const float (&scale)[2], const uint4 (&x)[4][UH]) {
        const int buf = tile_no & 1;
        if (!wait(&k_empty[buf], ((tile_no >> 1) & 1) ^ 1)) return;
        if (lane < 2) {
          sk_s[buf][2 * cw + lane] = lane ? scale[1] : scale[0];
          live_s[buf][2 * cw + lane] = (lane ? p[1] : p[0]) >= 0;
        }
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
          for (int e = 0; e < UH; ++e)
            store_codes<FMT, BF16>(k_sm + buf * S::kSide + piece<D>(32 * cw + 8 * g + (lane & 7), 2 * (4 * e + (lane >> 3))), x[g][e]);
        tc::fence_async_smem();
        __syncwarp();
        tc::mbar_arrive(tc::smem_u32(&k_full[buf]));
        ++tile_no;
      };
      for (int64_t c0 = 0; c0 < cols && ok; c0 += kMostCols) {
        look_up(0, place[0], sk[0]);
        look_up(1, place[1], sk[1]);
        load(place[0], kr[0]);
        load(place[1], kr[1]);
        for (int i = 0; i < n_tiles && ok; i += 2) {
#pragma unroll
          for (int z = 0; z < 2; ++z) {
            look_up(i + z + 2, place[2], sk[2]);
            if (i + z < n_tiles && ok) store(place[z], sk[z], kr[z]);
#pragma unroll
            for (int b = 0; b < 2; ++b) {
              place[z][b] = place[2][b];
              sk[z][b] = sk[2][b];
            }
            load(place[z], kr[z]);
          }
        }
      }
    }
  } else {
    // ------------------------------------------------------------------ products of a group's tiles (one lane issues)
    const int X = warp - 12;
    const uint64_t q_desc = tc::smem_desc(tc::smem_u32(q_sm), 128, D * 16);
    const uint64_t k_desc = tc::smem_desc(tc::smem_u32(k_sm + X * S::kSide), 128, D * 16);
    uint32_t s_no = 0;
    while (ok && next_part()) {
      for (int64_t c0 = 0; c0 < cols && ok; c0 += kMostCols, ++q_no) {
        const int n_cols = (int)min((int64_t)kMostCols, cols - c0), n_pad = (n_cols + 31) / 32 * 32;
        if (!wait(&q_full, q_no & 1)) break;
        for (int i = 0; i < n_tiles && ok; ++i, ++tile_no) {
          if ((int)(tile_no & 1) != X) continue;
          if (!wait(&k_full[X], (tile_no >> 1) & 1)) break;
          for (int h0 = 0; h0 < n_pad; h0 += kStepCols, ++s_no) {
            const int half = s_no & 1;
            if (!wait(&s_empty[X][half], ((s_no >> 1) & 1) ^ 1)) break;
            tc::tc_fence_after();
            const uint32_t idesc = idesc_f16(kKeys, min(kStepCols, n_pad - h0), false) | (BF16 ? 1u << 7 | 1u << 10 : 0u);
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks)
              mma_ss(tmem + (2 * X + half) * kStepCols, k_desc + ks * 16, q_desc + (h0 * D * 2 + ks * 256) / 16, idesc, ks > 0);
            commit(&s_full[X][half]);
          }
          commit(&k_empty[X]);
        }
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(tc::smem_u32(&q_read));
      }
    }
    __syncwarp();
    commit(&all_done[X]);  // whatever was issued has ended before tensor memory is freed
    tc::mbar_wait(tc::smem_u32(&all_done[X]), 0, a.err);
    __syncwarp();
  }
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  if (warp == 12) tc::tmem_dealloc(tmem, 4 * kStepCols);
  unseen_places<D>(w);
}

template <int D, int FMT, bool BF16>
crvq_status launch_wt(WeightArgs& w, cudaStream_t stream) {
  using S = WtShape<D>;
  auto kernel = weights_tc_kernel<D, FMT, BF16>;
  CRVQ_TRY(smem_limit((const void*)kernel, S::kSmem));
  w.a.shares = sm_count();
  ProfScope ps("cache_weights", stream, (double)w.a.rows.n_tok * w.a.q.heads * D);
  CRVQ_CUDA(launch_pdl(kernel, dim3((unsigned)w.a.shares), dim3(kWtThreads), S::kSmem, stream, w));
  CRVQ_LAUNCHED();
  return CRVQ_OK;
}

}  // namespace

crvq_status launch_weights_many(WeightArgs& w, int D, int format, cudaStream_t stream) {
  const bool int8 = format == CRVQ_KV_INT8;
  if (w.a.q.type == CRVQ_BF16) {
    if (D == 64) return int8 ? launch_wt<64, CRVQ_KV_INT8, true>(w, stream) : launch_wt<64, CRVQ_KV_E4M3, true>(w, stream);
    return int8 ? launch_wt<128, CRVQ_KV_INT8, true>(w, stream) : launch_wt<128, CRVQ_KV_E4M3, true>(w, stream);
  }
  if (D == 64) return int8 ? launch_wt<64, CRVQ_KV_INT8, false>(w, stream) : launch_wt<64, CRVQ_KV_E4M3, false>(w, stream);
  return int8 ? launch_wt<128, CRVQ_KV_INT8, false>(w, stream) : launch_wt<128, CRVQ_KV_E4M3, false>(w, stream);
}

}  // namespace crvq
