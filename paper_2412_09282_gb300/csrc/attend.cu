// Attention over the paged 8-bit cache: checks, the choice among the forms (attend_mma.cuh by shares of a line or,
// in attend_cluster.cu, by clusters; attend_tc.cu), and the line's launches.
#include "attend_mma.cuh"

namespace crvq {

namespace {

// Clusters where a CTA then has no more than this many tiles, whatever the lengths are: by the page table's width, so a
// table for long contexts takes the line for short sequences, too. Line against clusters, us, for (units, tiles per
// CTA): (8, 1) 12.3, 8.4; (8, 4) 16.4, 11.6; (32, 2) 14.2, 9.2; (96, 1) 15.5, 8.3; (96, 5) 18.6, 14.0; (130, 8, of 64
// channels) 25.3, 21.4; (32, 8) 20.2, 15.5; (8, 16) 24.2, 24.0; (96, 12) 24.9, 25.5; (8, 32) 28.5, 39.6.
constexpr int kClusterTiles = 8;

template <int D, int NT, int FMT, bool SPLIT>
crvq_status launch_attend(AttendArgs& a, cudaStream_t stream) {
  using S = Shape<D, NT, FMT, SPLIT>;
  constexpr int COLS = S::kCols;
  auto kernel = attend_kernel<D, NT, FMT, SPLIT, false>;
  a.shares = sm_count() * S::kPerSm;
  // the most tokens that a unit's columns see, in tiles
  const int64_t held = (int64_t)a.c.max_pages * a.c.page, seen = a.window > 0 ? min(held, a.window + a.rows.n_tok) : held;
  const int64_t units = most_units<COLS>(a), most = seen / kTile<D>;
  for (int size = 8; size >= 2; size /= 2) {
    if (units * size > a.shares) continue;
    if (most > kClusterTiles * size) break;
    return launch_attend_clusters(a, D, NT, FMT, units, size, stream);
  }
  CRVQ_TRY(smem_limit((const void*)kernel, S::kSmem));
  ProfScope ps("cache_attention", stream, (double)a.rows.n_tok * a.q.heads * D);
  Scratch mem;
  CRVQ_TRY(mem.alloc((size_t)2 * a.shares * S::kSlot * sizeof(float), stream));
  a.part = mem.as<float>();
  CRVQ_CUDA(launch_pdl(kernel, dim3((unsigned)a.shares), dim3(kThreads), S::kSmem, stream, a));
  CRVQ_LAUNCHED();
  return launch_join<D, S::kCols>(a, stream);
}

// Columns per sequence, on average, from which tiles of 128 rows (attend_tc.cu) are taken. This form against that, us,
// for (sequences of up to 4096 tokens x kv heads, columns): (64 x 32, 32) 691, 853; (16 x 8, 32) 61, 68; (16 x 8, 48)
// 83, 69; (8 x 8, 64) 62, 44; (1 x 8, 64) 19, 28; (64 x 32, 64) 1359, 855; (1 x 8, 128) 27, 32; (1 x 8, 256) 52, 41.
constexpr int64_t kManyColumns = 64;

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
  // (above, scale log2(e) is not finite, and a key of zeros would score 0 * infinity)
  CRVQ_CHECK_ARG(fabsf(scale) <= 0x1p127f, "scale must be within -2^127 .. 2^127");
  CRVQ_CHECK_ARG(((uintptr_t)lse & 3u) == 0, "lse is not aligned");
  CRVQ_TRY(check_dev({{lse, "lse"}}));
  a.group = a.q.heads / a.c.n_kv;
  CRVQ_CHECK_ARG(n_tok * a.group < (int64_t)1 << 31, "too many queries in one call");
  if (n_tok == 0) return CRVQ_OK;
  a.scale = scale * kLog2e;
  a.causal = causal != 0;
  a.window = window < (1 << 30) ? window : (1 << 30);
  a.lse = lse;
  auto vec_ok = [](const HeadsView& h) {
    const int64_t per = 16 / (int64_t)type_bytes(h.type);
    return ((uintptr_t)h.data & 15u) == 0 && h.ld_tok % per == 0 && h.ld_head % per == 0;
  };
  a.vec_q = vec_ok(a.q);
  a.vec_o = vec_ok(a.o);
  CRVQ_TRY(device_error_word(&a.err));
  if (D != 256 && a.q.type != CRVQ_F32 && n_tok * a.group >= kManyColumns * (int64_t)a.c.n_seq)
    return launch_attend_many(a, D, cache->format, stream);
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
