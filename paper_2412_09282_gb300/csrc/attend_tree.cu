// Trees of drafted tokens over the paged 8-bit cache: the mask of a tree from its parents, and the entry of attention
// by it (the kernels of attend_mma.cuh and attend_tc.cuh, whose masked tiles take a query's bits; every tile but a
// sequence's last ones is seen whole by all queries, as without a tree). Two sequences of up to 65536 tokens, trees of 64, 64 heads
// on 8: 339 us with the mask, 760 TFLOP/s, as chunks of prompts.
#include "attend_launch.cuh"

namespace crvq {

namespace {

struct TreeArgs {
  RowsView rows;
  const int32_t* parents;
  const int32_t* lens;  // or null: positions count from 0
  uint32_t* mask;
  int32_t* positions;
  int n_seq, words, window;
  unsigned* err;
};

constexpr int kStaged = 4096;  // parents kept in shared memory
constexpr int kTreeThreads = 128;

// mask[i] = { j : j = i, or j an ancestor of i less than `window` generations before it }, as bits; position[i] = its
// generation (+ the cached tokens before the tree). A thread walks from its token up to the root. Parents come before
// their children, so indices fall on the way and every word of the row is finished before the next lower one begins. A
// chain of depth shared-memory reads per token; what bounds it is the launch.
__global__ void __launch_bounds__(kTreeThreads) tree_mask_kernel(const __grid_constant__ TreeArgs a) {
  __shared__ int32_t parent_s[kStaged];
  pdl_trigger();
  pdl_wait();
  const int b = blockIdx.x;
  int64_t first;
  int n;
  seq_rows(a.rows, b, &first, &n, a.err);
  const int32_t* parent = a.parents + first;
  const int begin = blockIdx.y * kTreeThreads;
  if (begin >= n) return;
  // (ancestors of this block's tokens lie before its end)
  const int32_t* look = parent;
  const int end = min(n, begin + kTreeThreads);
  if (end <= kStaged) {
    for (int i = threadIdx.x; i < end; i += kTreeThreads) parent_s[i] = __ldg(parent + i);
    __syncthreads();
    look = parent_s;
  }
  const int i = begin + threadIdx.x;
  if (i >= n) return;
  uint32_t* row = a.mask + (first + i) * a.words;
  if (i >= 32 * a.words) raise_error(a.err, ERRBIT_INDEX);
  int w = a.words - 1, depth = 0;
  uint32_t bits = 0;
  for (int j = i;;) {
    if (a.window == 0 || depth < a.window) {
      const int at = j >> 5;
      if (at < a.words) {
        for (; w > at; --w) {
          row[w] = bits;
          bits = 0;
        }
        bits |= 1u << (j & 31);
      }
    }
    int up = look[j];
    if (up >= j || up < -1) {  // (not a parent before it: taken as a root)
      raise_error(a.err, ERRBIT_INDEX);
      up = -1;
    }
    if (up < 0) break;
    j = up;
    ++depth;
  }
  for (; w >= 0; --w) {
    row[w] = bits;
    bits = 0;
  }
  if (a.positions) a.positions[first + i] = (a.lens ? __ldg(a.lens + b) - n : 0) + depth;
}

crvq_status tree_mask(const int32_t* parents, int64_t n_tok, const int32_t* off, int32_t n_seq, const int32_t* lens,
                      int32_t window, uint32_t* mask, int32_t words, int32_t* positions, cudaStream_t stream) {
  TreeArgs a{};
  CRVQ_CHECK_ARG(n_seq >= 1, "n_seq must be >= 1");
  CRVQ_CHECK_ARG(words >= 1 && words <= (1 << 20), "words must be in [1, 2^20]");
  CRVQ_CHECK_ARG(window >= 0, "window must be >= 0");
  CRVQ_TRY(make_rows(off, n_tok, n_seq, &a.rows));
  if (n_tok == 0) return CRVQ_OK;
  CRVQ_CHECK_ARG(parents && mask, "parents and mask must not be NULL");
  CRVQ_CHECK_ARG((((uintptr_t)parents | (uintptr_t)lens | (uintptr_t)mask | (uintptr_t)positions) & 3u) == 0,
                 "parents, lens, mask or positions is not aligned");
  CRVQ_TRY(check_dev({{parents, "parents"}, {lens, "lens"}, {mask, "mask"}, {positions, "positions"}}));
  const int64_t most = off ? n_tok : n_tok / n_seq, grid_y = ceil_div(most, kTreeThreads);
  if (grid_y > 65535) return fail(CRVQ_ERR_UNSUPPORTED, "too many drafted tokens in one call");
  a.parents = parents;
  a.lens = lens;
  a.mask = mask;
  a.positions = positions;
  a.n_seq = n_seq;
  a.words = words;
  a.window = window;
  CRVQ_TRY(device_error_word(&a.err));
  ProfScope ps("tree_mask", stream, (double)n_tok * words);
  CRVQ_CUDA(launch_pdl(tree_mask_kernel, dim3((unsigned)n_seq, (unsigned)grid_y), dim3(kTreeThreads), 0, stream, a));
  CRVQ_LAUNCHED();
  return CRVQ_OK;
}

crvq_status tree_attention(const crvq_kv_cache* cache, const crvq_heads* q, int64_t n_tok, const int32_t* q_off,
                           const uint32_t* mask, int32_t words, const int32_t* positions, float scale, int32_t window,
                           const crvq_heads* out, float* lse, cudaStream_t stream) {
  AttendArgs a{};
  CRVQ_TRY(attend_args(cache, q, n_tok, q_off, scale, window, out, lse, &a));
  CRVQ_CHECK_ARG(words >= 1 && words <= (1 << 20), "words must be in [1, 2^20]");
  CRVQ_CHECK_ARG(window == 0 || positions != nullptr || n_tok == 0, "a window needs the queries' positions");
  CRVQ_CHECK_ARG(q_off != nullptr || n_tok <= (int64_t)32 * words * a.c.n_seq, "mask: %d words hold fewer than %lld drafted tokens",
                 words, (long long)(n_tok / a.c.n_seq));
  if (n_tok == 0) return CRVQ_OK;
  CRVQ_CHECK_ARG(mask != nullptr, "mask is NULL");
  CRVQ_CHECK_ARG((((uintptr_t)mask | (uintptr_t)positions) & 3u) == 0, "mask or positions is not aligned");
  CRVQ_TRY(check_dev({{mask, "mask"}, {positions, "positions"}}));
  a.tree = mask;
  a.words = words;
  a.positions = positions;
  return launch_form<true>(a, cache->head_dim, cache->format, stream);
}

}  // namespace

}  // namespace crvq

extern "C" {

crvq_status crvq_tree_mask(const int32_t* parents, int64_t n_tok, const int32_t* off, int32_t n_seq, const int32_t* lens,
                           int32_t window, uint32_t* mask, int32_t words, int32_t* positions, crvq_stream_t stream) {
  CRVQ_ENTRY({
    return crvq::tree_mask(parents, n_tok, off, n_seq, lens, window, mask, words, positions, (cudaStream_t)stream);
  })
}

crvq_status crvq_cache_tree_attention(const crvq_kv_cache* cache, const crvq_heads* q, int64_t n_tok,
                                      const int32_t* q_off, const uint32_t* mask, int32_t words,
                                      const int32_t* positions, float scale, int32_t window, const crvq_heads* out,
                                      float* lse, crvq_stream_t stream) {
  CRVQ_ENTRY({
    return crvq::tree_attention(cache, q, n_tok, q_off, mask, words, positions, scale, window, out, lse,
                                (cudaStream_t)stream);
  })
}

}  // extern "C"
