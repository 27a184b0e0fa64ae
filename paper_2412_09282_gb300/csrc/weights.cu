// How much attention every cached token gets from a step's queries, added to what it had:
//   out[b][h][t] = decay * before[b][h][t] + sum over the sequence's queries i and the query heads g of kv head h of
//                  exp(scale q_ig . K_t - lse_ig).
// The softmax's sum is known (lse), so tokens do not depend on one another: no maxima, no rescaling, nothing to join, and
// every sum is one warp's, in a fixed order.
//
// Form. S^T (16 tokens x 8 columns, a column = a query token and head) = K Q^T on mma.sync.m16n8k16 with the codes as A
// operand, as attention does for few queries (attend_mma.cuh), and the weights summed over the columns: in a lane's
// registers, then over the four lanes that share a token. A warp takes two blocks of 16 tokens at a time (one of 256
// channels), turns their codes into operands once and goes over all columns with them; up to `chunk` columns' queries lie
// in shared memory as fp16 relative to a power of two each (two operands from fp32). Blocks are copied ahead into a ring
// per warp, four steps deep: only keys are read, half of what attention reads.
//   What bounds it: memory. One token of 64 sequences of up to 4096, 32 heads, e4m3: 113 us, 5.4 TB/s. Alone at 46% of the
// issue slots (373 instructions per warp and 32 tokens); page numbers looked up a step earlier, and warps without a barrier
// at a unit's start, left it there (113.5, 112).
#include "attend_mma.cuh"
#include "weights.cuh"

namespace crvq {

namespace {

template <int D>
struct WShape {
  static constexpr int kQRow = D + 8;  // halves per query row, padded against bank conflicts
  static constexpr int kStages = 4;
  static constexpr int kStage = Tile<D>::kBytes * kBlocks<D>;
  static constexpr int kRing = kStage * kStages;
  static constexpr int kHad = kStages * 32;  // floats per warp: what the ring's tokens had
  static constexpr size_t smem(int chunk, bool split) {
    return (size_t)kWarps * (kRing + kHad * 4) + (size_t)chunk * (kQRow * 2 * (split ? 2 : 1) + 16);
  }
  // columns at a time: 256, or what a CTA's 227 KB hold (152 of 256 channels, two operands each)
  static constexpr int most(bool split) {
    const size_t fit = (232448 - smem(0, split)) / (smem(1, split) - smem(0, split)) / 8 * 8;
    return fit < 256 ? (int)fit : 256;
  }
};

// ONE: sequences of up to 8 columns each: their queries stay in registers, and codes are used as they are converted.
template <int D, int FMT, bool SPLIT, bool ONE>
__global__ void __launch_bounds__(kThreads, D == 256 ? 2 : 3)
weights_kernel(const __grid_constant__ WeightArgs w) {
  using S = WShape<D>;
  constexpr int NB = kBlocks<D>;
  const AttendArgs& a = w.a;
  extern __shared__ __align__(16) char sm[];
  char* ring = sm;                                                  // [kWarps][kStages][blocks] tiles
  float* had_s = reinterpret_cast<float*>(sm + kWarps * S::kRing);  // [kWarps][kStages][32]
  __half* q_s = reinterpret_cast<__half*>(had_s + kWarps * S::kHad);  // [split][chunk][kQRow]
  float4* col_s = reinterpret_cast<float4*>(q_s + (size_t)(SPLIT ? 2 : 1) * w.chunk * S::kQRow);  // factor, -lse, first, end
  pdl_wait();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, gid = lane >> 2, tig = lane & 3;
  const Line<D, kAllColumns> line(a);
  const int shares = (int)min((int64_t)a.shares, line.total);
  int64_t at = 0, at_end = 0;
  if ((int)blockIdx.x < shares) {
    at = share_begin(line.total, blockIdx.x, shares);
    at_end = share_begin(line.total, blockIdx.x + 1, shares);
  }
  char* mine = ring + warp * S::kRing;
  const uint32_t mine_u = (uint32_t)__cvta_generic_to_shared(mine);
  const uint32_t key_at = Tile<D>::at(gid, tig);
  // a lane's sums are those of one token of a step: block tig / 2, row gid + 8 (tig % 2)
  const int own = (tig >> 1) * kCacheBlock + (tig & 1) * 8 + gid;
  const float* had = had_s + warp * S::kHad + lane;

  while (at < at_end) {
    const Unit u = line.locate(a, at);
    const int64_t tile0 = u.begin + kStart, unit_end = tile0 + u.s.tiles;
    const int t_end = (int)max((int64_t)0, min(unit_end, at_end) - tile0);
    at = min(unit_end, at_end);
    if (u.tile >= t_end) continue;
    const int len = u.s.len, held = len - u.s.n, group = a.group;
    const int64_t cols = (int64_t)u.s.n * group;
    const int some_b = a.window > 0 ? max(0, held - a.window + 1) : 0;
    const int n_tiles = t_end - u.tile;
    float* out = w.out + u.b * w.out_seq + u.h * w.out_head;
    const float* before = w.before ? w.before + u.b * w.before_seq + u.h * w.before_head : nullptr;

    const int last = (int)min((int64_t)len, w.width);
    auto token = [&](int i) { return (u.s.lo + u.tile + i) * kTile<D> + warp * NB * kCacheBlock + own; };
    auto writes = [&](int i) { return (tig >> 1) < NB && token(i) < last; };

    for (int64_t c0 = 0; c0 < cols; c0 += w.chunk) {
      const int n_cols = (int)min((int64_t)w.chunk, cols - c0), groups = (n_cols + 7) / 8;
      __syncthreads();  // the previous columns have been read
      // places: a lane looks up every 32nd of this warp's blocks (as attend_kernel does)
      int64_t at_l = -1, at_old = -1;
      float sk_l = 0.f, sk_old = 0.f;
      int batch = -1;
      auto look_up = [&](int i) {
        if (i >= n_tiles || (i * NB & 31) != 0) return;
        at_old = at_l;
        sk_old = sk_l;
        batch = i * NB >> 5;
        const int tl = u.tile + i + lane / NB;
        const int tok = (u.s.lo + tl) * kTile<D> + (warp * NB + lane % NB) * kCacheBlock;
        at_l = -1;
        if (tl < t_end && tok < len && tok + kCacheBlock > some_b) {
          const int64_t page = seq_page(a.c, u.b, tok / a.c.page, a.err);
          if (page >= 0) {
            const int in = tok % a.c.page;
            at_l = page * a.c.page_stride + ((int64_t)u.h * a.c.page + in) * D;
            sk_l = __ldg(a.c.ks + (page * a.c.n_kv + u.h) * (a.c.page / kCacheBlock) + in / kCacheBlock);
          }
        }
      };
      auto start = [&](int i) {
        if (i < n_tiles) {
          const bool old = (i * NB >> 5) != batch;
#pragma unroll
          for (int b = 0; b < NB; ++b) {
            const int64_t src = __shfl_sync(0xffffffffu, old ? at_old : at_l, (i * NB + b) & 31);
            if (src >= 0)
              start_block<D, false>(a.c.K + src, mine_u + (i % S::kStages) * S::kStage + b * Tile<D>::kBytes, kCacheBlock);
          }
          // what a token had comes with its keys (loaded in its own step, it was what the step waited for: 64 sequences of
          // up to 4096 tokens, 32 heads, 131 -> 113 us)
          if (before && c0 == 0 && writes(i))
            asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"((uint32_t)__cvta_generic_to_shared(had + 32 * (i % S::kStages))),
                         "l"(before + token(i))
                         : "memory");
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
      };
#pragma unroll
      for (int i = 0; i < S::kStages - 1; ++i) {
        look_up(i);
        start(i);
      }
      // queries: a warp per column, relative to the power of two at its largest element
      for (int col = warp; col < 8 * groups; col += kWarps) {
        const int64_t c = c0 + col;
        const bool valid = col < n_cols;
        const int j = valid ? (int)(c / group) : 0, h = u.h * group + (valid ? (int)(c % group) : 0);
        const float lse = valid ? __ldg(w.lse + (u.s.first + j) * a.q.heads + h) : INFINITY;
        const bool none = isinf(lse);  // (such a query has no weights)
        float x[D / 32];
        float top = 0.f;
#pragma unroll
        for (int e = 0; e < D / 32; ++e) {
          x[e] = none ? 0.f : load_elem(a.q.data, (u.s.first + j) * a.q.ld_tok + h * a.q.ld_head + lane + 32 * e, a.q.type);
          top = fmaxf(top, fabsf(x[e]));
        }
        top = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top)));
        const uint32_t ex = __float_as_uint(top) >> 23;
        const bool plain = ex == 0 || ex == 255;
        const float inv = plain ? 1.f : __uint_as_float(ex == 254 ? 0x00400000u : (254u - ex) << 23);
        const float back = plain ? 1.f : __uint_as_float(ex << 23);
#pragma unroll
        for (int e = 0; e < D / 32; ++e) {
          const float v = x[e] * inv;
          const __half hi = __float2half_rn(v);
          q_s[col * S::kQRow + lane + 32 * e] = hi;
          if constexpr (SPLIT) q_s[(w.chunk + col) * S::kQRow + lane + 32 * e] = __float2half_rn(v - __half2float(hi));
        }
        if (lane == 0) {
          const int pos = held + j;
          col_s[col] = make_float4(none ? 0.f : back * w.scale, none ? -INFINITY : -lse,
                                   __int_as_float(a.window > 0 ? max(0, pos - a.window + 1) : 0),
                                   __int_as_float(a.causal ? min(len, pos + 1) : len));
        }
      }
      __syncthreads();
      // keys that every column sees (places do not fall from column to column)
      const int every_b = __float_as_int(col_s[n_cols - 1].z), every_e = __float_as_int(col_s[0].w);

      uint4 q_one[ONE && SPLIT ? 2 : 1][ONE ? D / 64 : 1][2];
      if constexpr (ONE) {
#pragma unroll
        for (int z = 0; z < (SPLIT ? 2 : 1); ++z)
#pragma unroll
          for (int j = 0; j < D / 64; ++j) {
            const uint4* p = reinterpret_cast<const uint4*>(q_s + ((size_t)z * w.chunk + gid) * S::kQRow + 64 * j + 16 * tig);
            q_one[z][j][0] = p[0];
            q_one[z][j][1] = p[1];
          }
      }

      for (int i = 0; i < n_tiles; ++i) {
        const bool old = (i * NB >> 5) != batch;
        const int tok = (u.s.lo + u.tile + i) * kTile<D> + warp * NB * kCacheBlock;
        float sk[NB];
        bool live[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          sk[b] = __shfl_sync(0xffffffffu, old ? sk_old : sk_l, (i * NB + b) & 31);
          live[b] = __shfl_sync(0xffffffffu, old ? at_old : at_l, (i * NB + b) & 31) >= 0;
        }
        asm volatile("cp.async.wait_group %0;" ::"n"(S::kStages - 2) : "memory");
        __syncwarp();
        float base = 0.f;
        if (writes(i)) {
          if (c0 > 0)
            base = out[token(i)];
          else if (before)
            base = w.decay * *const_cast<const volatile float*>(had + 32 * (i % S::kStages));
        }
        const char* keys = mine + (i % S::kStages) * S::kStage;
        // 16 consecutive codes of rows gid and gid + 8 of a block: four steps of the product
        auto codes = [&](int b, int j, uint4* k0, uint4* k1) {
          const char* p = keys + b * Tile<D>::kBytes + (j >> 1) * 128;
          *k0 = *reinterpret_cast<const uint4*>(p + (key_at ^ (j & 1) * 64));
          *k1 = *reinterpret_cast<const uint4*>(p + 8 * D + (key_at ^ (j & 1) * 64));
        };
        auto operand = [&](const uint4& k0, const uint4& k1, int e, uint32_t (&f)[4]) {
          const uint32_t x = word(k0, e), y = word(k1, e);
          f[0] = codes2<FMT, 0>(x);
          f[1] = codes2<FMT, 0>(y);
          f[2] = codes2<FMT, 1>(x);
          f[3] = codes2<FMT, 1>(y);
        };
        auto next_copies = [&]() {
          __syncwarp();  // every lane has read what these copies overwrite
          look_up(i + S::kStages - 1);
          start(i + S::kStages - 1);
        };
        uint32_t k[ONE ? 1 : NB][ONE ? 1 : D / 16][4];
        if constexpr (!ONE) {
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int j = 0; j < D / 64; ++j) {
              uint4 k0, k1;
              codes(b, j, &k0, &k1);
#pragma unroll
              for (int e = 0; e < 4; ++e) operand(k0, k1, e, k[b][4 * j + e]);
            }
          next_copies();
        }
        const bool whole = tok >= every_b && tok + NB * kCacheBlock <= every_e;
        float sum[NB][2];
#pragma unroll
        for (int b = 0; b < NB; ++b) sum[b][0] = sum[b][1] = 0.f;
        for (int g = 0; g < (ONE ? 1 : groups); ++g) {
          // 64 channels' products at a time, second operands' apart, are added up in fp32: a tensor core's sums are cut off
          // towards zero where they are long or a small product meets a large sum (16 of both kinds in a chain: weights
          // 1e-6 too small on average; so, 2e-7)
          float s[NB][4];
#pragma unroll
          for (int j = 0; j < D / 64; ++j)
#pragma unroll
            for (int z = SPLIT ? 1 : 0; z >= 0; --z) {
              uint4 x, y;
              if constexpr (ONE) {
                x = q_one[z][j][0];
                y = q_one[z][j][1];
              } else {
                const uint4* p = reinterpret_cast<const uint4*>(q_s + ((size_t)z * w.chunk + 8 * g + gid) * S::kQRow + 64 * j + 16 * tig);
                x = p[0];
                y = p[1];
              }
              float part[NB][4];
#pragma unroll
              for (int b = 0; b < NB; ++b) {
                part[b][0] = part[b][1] = part[b][2] = part[b][3] = 0.f;
                uint4 k0, k1;
                if constexpr (ONE) codes(b, j, &k0, &k1);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  uint32_t f[4];
                  if constexpr (ONE)
                    operand(k0, k1, e, f);
                  else
                    f[0] = k[b][4 * j + e][0], f[1] = k[b][4 * j + e][1], f[2] = k[b][4 * j + e][2], f[3] = k[b][4 * j + e][3];
                  mma_f16(part[b], f[0], f[1], f[2], f[3], e < 2 ? word(x, 2 * e) : word(y, 2 * e - 4),
                          e < 2 ? word(x, 2 * e + 1) : word(y, 2 * e - 3));
                }
              }
#pragma unroll
              for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[b][e] = j == 0 && z == (SPLIT ? 1 : 0) ? part[b][e] : s[b][e] + part[b][e];
            }
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float4 c = col_s[8 * g + 2 * tig + e];
#pragma unroll
            for (int b = 0; b < NB; ++b) {
              const float f = c.x * sk[b];
              float p0 = pow2(fmaf(s[b][e], f, c.y) * kLog2e), p1 = pow2(fmaf(s[b][e + 2], f, c.y) * kLog2e);
              if (!whole) {
                const int t0 = tok + b * kCacheBlock + gid, kb = __float_as_int(c.z), ke = __float_as_int(c.w);
                if (t0 < kb || t0 >= ke) p0 = 0.f;
                if (t0 + 8 < kb || t0 + 8 >= ke) p1 = 0.f;
              }
              sum[b][0] += p0;
              sum[b][1] += p1;
            }
          }
        }
        if constexpr (ONE) next_copies();
        float v = 0.f;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float x = live[b] ? sum[b][e] : 0.f;
            x += __shfl_xor_sync(0xffffffffu, x, 1);
            x += __shfl_xor_sync(0xffffffffu, x, 2);
            if (tig == 2 * b + e) v = x;
          }
        if (writes(i)) out[token(i)] = base + v;
      }
      asm volatile("cp.async.wait_group 0;" ::: "memory");
    }
  }
  unseen_places<D>(w);
}

template <int D, int FMT, bool SPLIT, bool ONE>
crvq_status launch(WeightArgs& w, int64_t cols, cudaStream_t stream) {
  using S = WShape<D>;
  auto kernel = weights_kernel<D, FMT, SPLIT, ONE>;
  w.chunk = (int)min((int64_t)S::most(SPLIT), ceil_div(max(cols, (int64_t)1), 8) * 8);
  const size_t smem = S::smem(w.chunk, SPLIT);
  CRVQ_TRY(smem_limit((const void*)kernel, smem));
  const int per_sm = max(1, min(D == 256 ? 2 : 3, (int)(233472 / (smem + 1024))));
  w.a.shares = sm_count() * per_sm;
  ProfScope ps("cache_weights", stream, (double)w.a.rows.n_tok * w.a.q.heads * D);
  CRVQ_CUDA(launch_pdl(kernel, dim3((unsigned)w.a.shares), dim3(kThreads), smem, stream, w));
  CRVQ_LAUNCHED();
  return CRVQ_OK;
}

template <int D, int FMT, bool SPLIT>
crvq_status pick_columns(WeightArgs& w, cudaStream_t stream) {
  // columns of a sequence, by the average where the rows' offsets are on the device (a chunk then, several where there are more)
  const AttendArgs& a = w.a;
  const int64_t cols = a.rows.off ? 2 * ceil_div(a.rows.n_tok * a.group, a.c.n_seq) : (int64_t)a.rows.per * a.group;
  // Up to 8 columns on average: queries in registers. Against shared memory, us, for (sequences of up to this many tokens x kv heads,
  // columns): (64 of 4096 x 32, 1, e4m3) 112, 117; (64 of 4096 x 32, 1, int8) 117, 124; (16 of 8192 x 8, 8) 18.7, 19.7; (1 of 65536 x
  // 8, 8) 15.4, 16.2; (8 of 4096 x 32, 7) 20.5, 21.6; (8 of 4096 x 4, 8, fp32) 7.7, 8.0; (1 of 1001 x 8, 8) 5.4, 5.4.
  if (a.rows.n_tok * a.group <= 8 * (int64_t)a.c.n_seq) return launch<D, FMT, SPLIT, true>(w, min(cols, (int64_t)8), stream);
  return launch<D, FMT, SPLIT, false>(w, cols, stream);
}

// Columns per sequence, on average, from which tokens are the rows of tcgen05 tiles (weights_tc.cu). This form against that, us,
// for (sequences of up to this many tokens x kv heads, columns): (64 of 4096 x 32, 32) 256, 541; (64 of 4096 x 32, 64) 527, 555; (16 of
// 4096 x 8, 48) 32, 43; (16 of 4096 x 8, 64) 39, 44; (1 of 4096 x 8, 32) 9.3, 10.0; (1 of 4096 x 8, 64) 14.0, 10.3; (1 of 4096 x 8,
// 128) 24.0, 11.1; (1 of 32768 x 8, 64) 30.6, 31.9; (1 of 32768 x 8, 128) 52, 32; (2 of 32768 x 8, 64) 41, 43; (1 of 1000 x 1, 64)
// 12.3, 7.2.
constexpr int64_t kManyColumns = 64;

template <int D>
crvq_status pick(WeightArgs& w, int format, cudaStream_t stream) {
  const bool split = w.a.q.type == CRVQ_F32;
  if (format == CRVQ_KV_INT8)
    return split ? pick_columns<D, CRVQ_KV_INT8, true>(w, stream) : pick_columns<D, CRVQ_KV_INT8, false>(w, stream);
  return split ? pick_columns<D, CRVQ_KV_E4M3, true>(w, stream) : pick_columns<D, CRVQ_KV_E4M3, false>(w, stream);
}

crvq_status weights(const crvq_kv_cache* cache, const crvq_heads* q, int64_t n_tok, const int32_t* q_off, float scale,
                    int32_t causal, int32_t window, const float* lse, const crvq_token_sums* before, float decay,
                    const crvq_token_sums* out, cudaStream_t stream) {
  WeightArgs w{};
  CRVQ_TRY(attend_args(cache, q, n_tok, q_off, scale, window, q, nullptr, &w.a));
  CRVQ_TRY(check_sums(out, "out", w.a.c.n_seq, w.a.c.n_kv));
  CRVQ_CHECK_ARG(lse != nullptr || n_tok == 0, "lse is NULL");
  CRVQ_CHECK_ARG(((uintptr_t)lse & 3u) == 0, "lse is not aligned");
  CRVQ_TRY(check_dev({{lse, "lse"}}));
  CRVQ_CHECK_ARG(fabsf(decay) <= 3.402823466e38f, "decay must be finite");
  if (before) {
    CRVQ_TRY(check_sums(before, "before", w.a.c.n_seq, w.a.c.n_kv));
    CRVQ_CHECK_ARG(before->width == out->width, "before and out differ in width");
    const bool same = before->data == out->data && before->ld_seq == out->ld_seq && before->ld_head == out->ld_head;
    CRVQ_CHECK_ARG(same || !sums_overlap(before, out, w.a.c.n_seq, w.a.c.n_kv), "before and out share memory, but are not the same");
    w.before = before->data;
    w.before_seq = before->ld_seq;
    w.before_head = before->ld_head;
  }
  w.a.causal = causal != 0;
  w.lse = lse;
  w.out = out->data;
  w.out_seq = out->ld_seq;
  w.out_head = out->ld_head;
  w.width = out->width;
  w.decay = decay;
  w.scale = scale;
  const int D = cache->head_dim;
  if (D != 256 && w.a.q.type != CRVQ_F32 && n_tok * w.a.group >= kManyColumns * (int64_t)w.a.c.n_seq)
    return launch_weights_many(w, D, cache->format, stream);
  if (D == 64) return pick<64>(w, cache->format, stream);
  if (D == 128) return pick<128>(w, cache->format, stream);
  return pick<256>(w, cache->format, stream);
}

}  // namespace

bool sums_overlap(const crvq_token_sums* x, const crvq_token_sums* y, int n_seq, int n_kv) {
  auto end = [&](const crvq_token_sums* s) {
    return s->data + (n_seq > 1 ? (n_seq - 1) * s->ld_seq : 0) + (n_kv > 1 ? (n_kv - 1) * s->ld_head : 0) + s->width;
  };
  return x->data < end(y) && y->data < end(x);
}

crvq_status check_sums(const crvq_token_sums* s, const char* name, int n_seq, int n_kv) {
  CRVQ_CHECK_ARG(s != nullptr && s->data != nullptr, "%s is NULL", name);
  CRVQ_CHECK_ARG(((uintptr_t)s->data & 3u) == 0, "%s is not aligned", name);
  CRVQ_CHECK_ARG(s->width >= 1 && s->width < (int64_t)1 << 31, "%s: width must be in [1, 2^31)", name);
  // rows that do not overlap, in either order
  const int64_t row = s->width, by_head = s->ld_head, by_seq = s->ld_seq;
  const bool seq_outer = (n_kv == 1 || by_head >= row) && (n_seq == 1 || by_seq >= (n_kv == 1 ? row : by_head * (n_kv - 1) + row));
  const bool head_outer = (n_seq == 1 || by_seq >= row) && (n_kv == 1 || by_head >= (n_seq == 1 ? row : by_seq * (n_seq - 1) + row));
  CRVQ_CHECK_ARG(seq_outer || head_outer, "%s: rows overlap", name);
  return check_dev({{s->data, name}});
}

}  // namespace crvq

extern "C" {

crvq_status crvq_cache_weights(const crvq_kv_cache* cache, const crvq_heads* q, int64_t n_tok, const int32_t* q_off,
                               float scale, int32_t causal, int32_t window, const float* lse,
                               const crvq_token_sums* before, float decay, const crvq_token_sums* out,
                               crvq_stream_t stream) {
  CRVQ_ENTRY({
    return crvq::weights(cache, q, n_tok, q_off, scale, causal, window, lse, before, decay, out, (cudaStream_t)stream);
  })
}

}  // extern "C"
