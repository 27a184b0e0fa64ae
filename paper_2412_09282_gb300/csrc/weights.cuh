// How much attention cached tokens get (see crvq_cache_weights in crvq.h): arguments and what its kernels share.
#pragma once

#include "attend.cuh"

namespace crvq {

struct WeightArgs {
  AttendArgs a;         // cache, queries, rows, group, scale, causal, window, error word; shares of the line
  const float* lse;     // [n_tok x q heads]
  const float* before;  // or null: zeros
  float* out;
  int64_t before_seq, before_head, out_seq, out_head;  // strides
  int64_t width;        // places in a row of before and out
  float decay;
  float scale;          // (a's is in log2: there the difference of score and lse would be rounded at their size)
  int chunk;            // columns at a time
};

// Many columns per sequence (weights_tc.cu): 16-bit queries, 64 or 128 channels.
crvq_status launch_weights_many(WeightArgs& w, int D, int format, cudaStream_t stream);

namespace {

constexpr int kAllColumns = 1 << 30;  // a sequence's columns are one unit

// The places that no query sees: out = decay * before (0 behind the sequence's last token). A CTA takes every
// gridDim-th (sequence, kv head).
template <int D>
__device__ __forceinline__ void unseen_places(const WeightArgs& w) {
  const AttendArgs& a = w.a;
  for (int64_t row = blockIdx.x; row < (int64_t)a.c.n_seq * a.c.n_kv; row += gridDim.x) {
    const int b = (int)(row / a.c.n_kv), h = (int)(row - (int64_t)b * a.c.n_kv);
    const Seq s = load_seq<D, kAllColumns>(a, b);
    const int64_t len = min((int64_t)s.len, w.width);
    const int64_t seen_b = s.n > 0 ? min((int64_t)s.lo * kTile<D>, len) : len;
    float* out = w.out + b * w.out_seq + h * w.out_head;
    const float* before = w.before + b * w.before_seq + h * w.before_head;
    for (int64_t t = threadIdx.x; t < seen_b; t += blockDim.x) out[t] = w.before ? w.decay * before[t] : 0.f;
    for (int64_t t = len + threadIdx.x; t < w.width; t += blockDim.x) out[t] = 0.f;
    if (s.len > w.width && threadIdx.x == 0 && h == 0) raise_error(a.err, ERRBIT_INDEX);
  }
}

}  // namespace

}  // namespace crvq
