// Attention over the paged 8-bit cache: checks and the C entry (attend_launch.cuh chooses among the forms).
#include "attend_launch.cuh"

namespace crvq {

crvq_status attend_args(const crvq_kv_cache* cache, const crvq_heads* q, int64_t n_tok, const int32_t* q_off,
                        float scale, int32_t window, const crvq_heads* out, float* lse, AttendArgs* args) {
  AttendArgs& a = *args;
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
  a.scale = scale * kLog2e;
  a.window = window < (1 << 30) ? window : (1 << 30);
  a.lse = lse;
  auto vec_ok = [](const HeadsView& h) {
    const int64_t per = 16 / (int64_t)type_bytes(h.type);
    return ((uintptr_t)h.data & 15u) == 0 && h.ld_tok % per == 0 && h.ld_head % per == 0;
  };
  a.vec_q = vec_ok(a.q);
  a.vec_o = vec_ok(a.o);
  CRVQ_TRY(device_error_word(&a.err));
  return CRVQ_OK;
}

namespace {

crvq_status attention(const crvq_kv_cache* cache, const crvq_heads* q, int64_t n_tok, const int32_t* q_off,
                      float scale, int32_t causal, int32_t window, const crvq_heads* out, float* lse,
                      cudaStream_t stream) {
  AttendArgs a{};
  CRVQ_TRY(attend_args(cache, q, n_tok, q_off, scale, window, out, lse, &a));
  if (n_tok == 0) return CRVQ_OK;
  a.causal = causal != 0;
  return launch_form<false>(a, cache->head_dim, cache->format, stream);
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
