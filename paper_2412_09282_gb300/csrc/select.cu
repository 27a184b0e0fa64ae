// Which tokens of every (sequence, kv head) stay when a cache is cut down to a budget: the first, the most recent, and of
// those between them the ones with the largest weights, ties to the lowest place; their places and weights in order.
//
// A row's k-th largest weight is found digit by digit (11, 11 and 10 bits, from the top) over keys whose unsigned order
// is the weights': a histogram of the keys that agree so far, and the bin in which the count from the top passes k. The row
// is then gone through once more: a token stays when its key is above the threshold, or equal to it and among the first
// that are still needed; its new place is the number of such tokens before it. All counts are whole numbers, so results
// do not depend on timing.
//   A row is the work of a cluster of 1, 2, 4 or 8 CTAs, each of which holds an equal run of neighbouring tokens in shared
// memory (it is read from global memory once) and every warp of it an equal run of those: counts over a warp's 32 tokens
// are ballots. Histograms and counts are joined by adding them to every CTA's shared memory: one barrier a digit, and nothing is
// read across CTAs.
#include "cache.cuh"
#include "kernels.h"

namespace crvq {

namespace {

constexpr int kBins = 2048, kBinRows = kBins / 32;
constexpr int kMaxWarps = 32;
constexpr int kStageMax = 44 * 1024;  // weights that a CTA holds in shared memory (more are read again)

struct SelectArgs {
  const float* w;
  float* w_out;  // or null
  int64_t w_seq, w_head, width, out_seq, out_head, out_width;
  const int32_t* lens;
  int32_t* idx;
  int32_t* count;
  int n_kv, keep, first, recent;
  int log_cluster, staged;  // weights of a CTA in shared memory
  unsigned* err;
};

// Unsigned keys in the order of the weights; -0 is 0, and NaN is above infinity. kAlways is above all of them: the first and the
// most recent tokens are then selected as any others are. 0 is below all: the places behind the last token.
constexpr uint32_t kAlways = 0xffffffffu, kNan = 0xfffffffeu;
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);  // (-0 + 0 = 0)
  return x != x ? kNan : u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

// The place of *p in the shared memory of the cluster's CTA `rank`.
__device__ __forceinline__ uint32_t remote(const uint32_t* p, int rank) {
  uint32_t at;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
  return at;
}
__device__ __forceinline__ void add_remote(uint32_t at, uint32_t v) {
  asm volatile("red.relaxed.cluster.shared::cluster.add.u32 [%0], %1;" ::"r"(at), "r"(v) : "memory");
}
__device__ __forceinline__ void store_remote(uint32_t at, uint32_t v) {
  asm volatile("st.relaxed.cluster.shared::cluster.u32 [%0], %1;" ::"r"(at), "r"(v) : "memory");
}

struct SelectShared {
  uint32_t hist[3][kBins];           // the row's, once every CTA of the cluster has added its own
  uint32_t mine[kBins];              // this CTA's part of the present one, where the cluster has others
  uint32_t rows[kBinRows];           // sums of 32 bins
  uint32_t bin, above;               // the threshold's bin, and the keys above it
  uint32_t sure[8], equal[8];        // tokens of every CTA that stay for certain; equal to the threshold
  uint32_t warp_sure[kMaxWarps], warp_equal[kMaxWarps];
};

// One more key in a bin of the lanes that are `in`. Lanes in the same bin wait for one another; where all are (a row of equal
// weights) one adds for them.
__device__ __forceinline__ void count_key(uint32_t* hist, uint32_t bin, bool in) {
  const unsigned who = __ballot_sync(0xffffffffu, in);
  if (who == 0) return;
  const int first = __ffs(who) - 1;
  const uint32_t b0 = __shfl_sync(0xffffffffu, bin, first);
  if (__all_sync(0xffffffffu, !in || bin == b0)) {
    if ((int)(threadIdx.x & 31) == first) atomicAdd(hist + b0, (uint32_t)__popc(who));
  } else if (in) {
    atomicAdd(hist + bin, 1u);
  }
}

__global__ void __launch_bounds__(32 * kMaxWarps, 2) select_kernel(const __grid_constant__ SelectArgs a) {
  extern __shared__ __align__(16) char sm[];
  SelectShared& s = *reinterpret_cast<SelectShared*>(sm);
  uint32_t* keys = reinterpret_cast<uint32_t*>(sm + sizeof(SelectShared));
  pdl_wait();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
  const int size = 1 << a.log_cluster, rank = blockIdx.x & (size - 1), row = blockIdx.x >> a.log_cluster;
  const int b = row / a.n_kv, h = row - b * a.n_kv;
  auto sync_all = [&]() {
    if (size == 1)
      __syncthreads();
    else
      asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  };
  for (int i = tid; i < (size > 1 ? 4 : 3) * kBins; i += blockDim.x) (&s.hist[0][0])[i] = 0;
  int len = __ldg(a.lens + b);
  if (len < 0 || len > a.width) {
    raise_error(a.err, ERRBIT_INDEX);
    len = 0;
  }
  const int count = min(len, a.keep);
  const bool find = len > a.keep;  // (else all stay)
  const int lo = a.first, hi = len - a.recent;  // tokens [lo, hi) are those between the first and the most recent ones
  const float* w = a.w + b * a.w_seq + h * a.w_head;
  // this CTA's tokens, this warp's
  const int per_cta = (int)(((int64_t)len + 32 * size - 1) / (32 * size)) * 32;
  const int c_begin = (int)min((int64_t)len, (int64_t)rank * per_cta), c_end = min(len, c_begin + per_cta);
  const int per_warp = (c_end - c_begin + 32 * warps - 1) / (32 * warps) * 32;
  const int begin = min(c_end, c_begin + warp * per_warp), end = min(c_end, begin + per_warp);
  const bool staged = per_cta <= a.staged;
  __syncthreads();

  auto key_of = [&](int t, float x) { return t < lo || t >= hi || !find ? kAlways : order_key(x); };
  constexpr int kBatch = 8;
  for (int t0 = begin; t0 < end; t0 += 32 * kBatch) {
    float x[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int t = t0 + 32 * i + lane;
      x[i] = t < end ? __ldg(w + t) : 0.f;
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int t = t0 + 32 * i + lane;
      if (t0 + 32 * i >= end) break;
      const uint32_t key = t < end ? key_of(t, x[i]) : 0u;
      if (staged) keys[t - c_begin] = key;
      if (find) count_key(size > 1 ? s.mine : s.hist[0], key >> 21, t < end);
    }
  }
  // places behind the last token that stays
  if (a.w_out) {
    float* out = a.w_out + b * a.out_seq + h * a.out_head;
    for (int64_t t = count + rank * (int)blockDim.x + tid; t < a.out_width; t += size * (int)blockDim.x) out[t] = 0.f;
  }
  int32_t* idx = a.idx + (int64_t)row * a.keep;
  for (int t = count + rank * (int)blockDim.x + tid; t < a.keep; t += size * (int)blockDim.x) idx[t] = -1;
  if (h == 0 && rank == 0 && tid == 0) a.count[b] = count;

  // the keys of 32 tokens, a lane each
  auto at = [&](int t) { return staged ? keys[t - c_begin] : t < end ? key_of(t, __ldg(w + t)) : 0u; };
  uint32_t need = (uint32_t)a.keep, threshold = kAlways - 1;  // (all stay for certain)
  if (find) {
    uint32_t prefix = 0;
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, digits = pass == 2 ? 10 : 11;
      if (pass > 0)
        for (int t0 = begin; t0 < end; t0 += 32) {
          const uint32_t key = at(t0 + lane);
          count_key(size > 1 ? s.mine : s.hist[pass], key >> shift & ((1u << digits) - 1u), key >> (shift + digits) == prefix);
        }
      if (size > 1) {  // to everyone
        if (pass == 0) sync_all();  // (whose counts are zeros by then)
        else __syncthreads();
        for (int i = tid; i < kBins; i += blockDim.x) {
          const uint32_t v = s.mine[i];
          if (v) {
            s.mine[i] = 0;
            for (int c = 0; c < size; ++c) add_remote(remote(&s.hist[pass][i], c), v);
          }
        }
      }
      sync_all();
      for (int r = warp; r < kBinRows; r += warps) {
        const uint32_t v = __reduce_add_sync(0xffffffffu, s.hist[pass][32 * r + lane]);
        if (lane == 0) s.rows[r] = v;
      }
      __syncthreads();
      if (warp == 0) {
        // from the top: lane i holds rows 63 - 2 i and 62 - 2 i
        const int r1 = kBinRows - 1 - 2 * lane, r0 = r1 - 1;
        const uint32_t v1 = s.rows[r1], v0 = s.rows[r0];
        uint32_t sum = v1 + v0;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const uint32_t o = __shfl_up_sync(0xffffffffu, sum, d);
          if (lane >= d) sum += o;
        }
        const int hit = __ffs(__ballot_sync(0xffffffffu, sum >= need)) - 1;
        uint32_t above = sum - v1 - v0;
        const bool second = above + v1 < need;
        const int r = __shfl_sync(0xffffffffu, second ? r0 : r1, hit);
        above = __shfl_sync(0xffffffffu, second ? above + v1 : above, hit);
        const uint32_t v = s.hist[pass][32 * r + 31 - lane];
        sum = v;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const uint32_t o = __shfl_up_sync(0xffffffffu, sum, d);
          if (lane >= d) sum += o;
        }
        const int in_row = __ffs(__ballot_sync(0xffffffffu, above + sum >= need)) - 1;
        if (lane == in_row) {
          s.bin = 32 * r + 31 - lane;
          s.above = above + sum - v;
        }
      }
      __syncthreads();
      prefix = prefix << digits | s.bin;
      need -= s.above;
    }
    threshold = prefix;
  }

  if (size > 1 && !find) sync_all();  // (every CTA is there)
  // this warp's tokens that stay for certain, and those at the threshold
  uint32_t sure = 0, equal = 0;
  for (int t0 = begin; t0 < end; t0 += 32) {
    const uint32_t key = at(t0 + lane);
    sure += key > threshold;
    equal += key == threshold;
  }
  sure = __reduce_add_sync(0xffffffffu, sure);
  equal = __reduce_add_sync(0xffffffffu, equal);
  if (lane == 0) {
    s.warp_sure[warp] = sure;
    s.warp_equal[warp] = equal;
  }
  __syncthreads();
  if (warp == 0) {
    uint32_t vs = lane < warps ? s.warp_sure[lane] : 0u, ve = lane < warps ? s.warp_equal[lane] : 0u;
    const uint32_t ms = vs, me = ve;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const uint32_t os = __shfl_up_sync(0xffffffffu, vs, d), oe = __shfl_up_sync(0xffffffffu, ve, d);
      if (lane >= d) {
        vs += os;
        ve += oe;
      }
    }
    if (lane < warps) {
      s.warp_sure[lane] = vs - ms;
      s.warp_equal[lane] = ve - me;
    }
    vs = __shfl_sync(0xffffffffu, vs, 31);
    ve = __shfl_sync(0xffffffffu, ve, 31);
    if (size > 1 && lane < size) {  // to everyone; the last word between the CTAs
      store_remote(remote(&s.sure[rank], lane), vs);
      store_remote(remote(&s.equal[rank], lane), ve);
    }
  }
  sync_all();
  sure = s.warp_sure[warp];
  equal = s.warp_equal[warp];
  for (int c = 0; c < rank; ++c) {
    sure += s.sure[c];
    equal += s.equal[c];
  }
  float* out = a.w_out ? a.w_out + b * a.out_seq + h * a.out_head : nullptr;
  const unsigned before = (1u << lane) - 1u;
  for (int t0 = begin; t0 < end; t0 += 32) {
    const int t = t0 + lane;
    const uint32_t key = at(t);
    const bool is_sure = key > threshold, is_equal = key == threshold;
    const unsigned ms = __ballot_sync(0xffffffffu, is_sure), me = __ballot_sync(0xffffffffu, is_equal);
    if ((ms | me) == 0) continue;
    const uint32_t my_equal = equal + __popc(me & before);
    const uint32_t place = sure + __popc(ms & before) + min(my_equal, need);
    if ((is_sure || (is_equal && my_equal < need)) && place < (uint32_t)count) {
      idx[place] = t;
      if (out) out[place] = __ldg(w + t);
    }
    sure += __popc(ms);
    equal += __popc(me);
  }
}

crvq_status select(const crvq_token_sums* weights, const int32_t* lens, int32_t n_seq, int32_t n_kv, int32_t keep,
                   int32_t first, int32_t recent, int32_t* idx, int32_t* count, const crvq_token_sums* weights_out,
                   cudaStream_t stream) {
  SelectArgs a{};
  CRVQ_CHECK_ARG(n_seq >= 1 && n_kv >= 1, "need n_seq, n_kv >= 1");
  CRVQ_TRY(check_sums(weights, "weights", n_seq, n_kv));
  CRVQ_CHECK_ARG(keep >= 1, "keep must be >= 1");
  CRVQ_CHECK_ARG(first >= 0 && recent >= 0 && (int64_t)first + recent <= keep, "first and recent must be >= 0 and fit in keep");
  CRVQ_CHECK_ARG(lens && idx && count, "lens, idx and count must not be NULL");
  CRVQ_CHECK_ARG((((uintptr_t)lens | (uintptr_t)idx | (uintptr_t)count) & 3u) == 0, "lens, idx or count is not aligned");
  CRVQ_TRY(check_dev({{lens, "lens"}, {idx, "idx"}, {count, "count"}}));
  if (weights_out) {
    CRVQ_TRY(check_sums(weights_out, "weights_out", n_seq, n_kv));
    CRVQ_CHECK_ARG(weights_out->width >= min((int64_t)keep, weights->width), "weights_out is too narrow for keep weights a row");
    auto end = [&](const crvq_token_sums* s) {
      return s->data + (n_seq > 1 ? (n_seq - 1) * s->ld_seq : 0) + (n_kv > 1 ? (n_kv - 1) * s->ld_head : 0) + s->width;
    };
    CRVQ_CHECK_ARG(end(weights_out) <= weights->data || end(weights) <= weights_out->data, "weights_out and weights share memory");
    a.w_out = weights_out->data;
    a.out_seq = weights_out->ld_seq;
    a.out_head = weights_out->ld_head;
    a.out_width = weights_out->width;
  }
  a.w = weights->data;
  a.w_seq = weights->ld_seq;
  a.w_head = weights->ld_head;
  a.width = weights->width;
  a.lens = lens;
  a.idx = idx;
  a.count = count;
  a.n_kv = n_kv;
  a.keep = keep;
  a.first = first;
  a.recent = recent;
  CRVQ_TRY(device_error_word(&a.err));
  const int64_t units = (int64_t)n_seq * n_kv;
  int size = 1;
  while (size < 8 && a.width > (int64_t)4096 * size) {
    size *= 2;
    ++a.log_cluster;
  }
  if (units * size >= (int64_t)1 << 31) return fail(CRVQ_ERR_UNSUPPORTED, "too many sequences and heads in one call");
  const int64_t per_cta = ceil_div(a.width, 32 * size) * 32;
  const int threads = 32 * (int)min((int64_t)kMaxWarps, max((int64_t)4, ceil_div(per_cta, 128)));
  a.staged = (int)min(per_cta, (int64_t)kStageMax);
  const size_t smem = sizeof(SelectShared) + (size_t)a.staged * sizeof(float);
  CRVQ_TRY(smem_limit((const void*)select_kernel, smem));
  ProfScope ps("cache_select", stream, (double)units * a.width);
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = size;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(units * size));
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  CRVQ_CUDA(cudaLaunchKernelEx(&cfg, select_kernel, a));
  CRVQ_LAUNCHED();
  return CRVQ_OK;
}

}  // namespace

}  // namespace crvq

extern "C" {

crvq_status crvq_cache_select(const crvq_token_sums* weights, const int32_t* lens, int32_t n_seq, int32_t n_kv,
                              int32_t keep, int32_t first, int32_t recent, int32_t* idx, int32_t* count,
                              const crvq_token_sums* weights_out, crvq_stream_t stream) {
  CRVQ_ENTRY({
    return crvq::select(weights, lens, n_seq, n_kv, keep, first, recent, idx, count, weights_out, (cudaStream_t)stream);
  })
}

}  // extern "C"
