// Which tokens of every (sequence, kv head) stay when a cache is cut down to a budget: the first, the most recent, and of
// those between them the ones with the largest weights, ties to the lowest place; their places and weights in order.
//
// A row's k-th largest weight is found digit by digit (11, 7, 7 and 7 bits, from the top) over keys whose unsigned order
// is the weights': a histogram of the keys that agree so far, and the bin in which the count from the top passes k. (The
// first digit splits a row's few powers of two. After it every bin would be in use; adding 2048 of them to the other CTAs'
// takes as long as one more digit.) Every warp lists its keys in the first digit's bin, a few in a hundred, and goes by its
// list from there on. The row is then gone through once more: a token stays when its key is above the threshold, or equal to
// it and among the first that are still needed; its new place is the number of such tokens before it. All counts are
// whole numbers, so results do not depend on timing.
//   A row is the work of a cluster of 1, 2, 4 or 8 CTAs, each of which holds an equal run of neighbouring tokens in shared
// memory (it is read from global memory once) and every warp of it an equal run of those, 128 tokens at a time. Histograms
// and counts are joined by adding them to every CTA's shared memory: one barrier a digit, and nothing is read across CTAs.
//   What bounds it: 32 rows of 131072 tokens take 22 us, of which reading and writing are 5. A CTA's 40000 cycles are, by
// clocks read in the kernel, 15% loading, 15% the first histogram, 15% the lists, 35% joining and searching four digits (six
// barriers of the cluster), 20% the last pass: instructions of 32 warps, and barriers.
#include "cache.cuh"
#include "kernels.h"

namespace crvq {

namespace {

constexpr int kBins = 2048, kBinRows = kBins / 32;  // of the first digit
constexpr int kFew = 128;                           // of the others
constexpr int kMaxWarps = 32;
constexpr int kLogStep = 7, kStep = 1 << kLogStep;  // tokens of a warp at a time, a lane's four neighbours
constexpr int kStageMax = 44 * 1024;  // weights that a CTA holds in shared memory (more are read again)
constexpr int kCandidates = 128;      // of a warp, in shared memory (a warp with more goes through all its tokens)

struct SelectArgs {
  const float* w;
  float* w_out;  // or null
  int64_t w_seq, w_head, width, out_seq, out_head, out_width;
  const int32_t* lens;
  int32_t* idx;
  int32_t* count;
  int n_kv, keep, first, recent;
  int log_cluster, staged;  // weights of a CTA in shared memory
  bool vec;                 // rows of 16-byte groups of weights
  unsigned* err;
};

// Unsigned keys in the order of the weights; -0 is 0, and NaN is above infinity. kAlways is above all of them: the first and the
// most recent tokens are then selected as any others are. 0 is below all: the places behind the last token.
constexpr uint32_t kAlways = 0xffffffffu, kNan = 0xfffffffeu;
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);  // (-0 + 0 = 0)
  return x != x ? kNan : u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

__device__ __forceinline__ float weight_of(uint32_t key) { return __uint_as_float(key >> 31 ? key ^ 0x80000000u : ~key); }

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

struct alignas(16) SelectShared {
  // the row's counts, once every CTA of the cluster has added its own, and this CTA's (where there are others)
  uint32_t hist[kBins], few[3][kFew];
  uint32_t mine[kBins], mine_few[3][kFew];
  uint32_t rows[kBinRows];           // sums of 32 bins
  uint32_t sure[8], equal[8];        // tokens of every CTA that stay for certain; equal to the threshold
  uint32_t warp_sure[kMaxWarps], warp_equal[kMaxWarps];
};

// Counts a lane's four keys in their bins, those that are `in`. Lanes in the same bin wait for one another; where all keys are (a
// row of equal weights) one lane adds for them.
__device__ __forceinline__ void count_keys(uint32_t* hist, const uint32_t bin[4], const bool in[4]) {
  const uint32_t b0 = __shfl_sync(0xffffffffu, bin[0], 0);
  if (__all_sync(0xffffffffu, in[0] && bin[0] == b0)) {
    bool same = true;
#pragma unroll
    for (int e = 1; e < 4; ++e) same = same && in[e] && bin[e] == b0;
    if (__all_sync(0xffffffffu, same)) {
      if ((threadIdx.x & 31) == 0) atomicAdd(hist + b0, 128u);
      return;
    }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (in[e]) atomicAdd(hist + bin[e], 1u);
}

__global__ void __launch_bounds__(32 * kMaxWarps, 2) select_kernel(const __grid_constant__ SelectArgs a) {
  extern __shared__ __align__(16) char sm[];
  SelectShared& s = *reinterpret_cast<SelectShared*>(sm);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
  uint32_t* cand = reinterpret_cast<uint32_t*>(sm + sizeof(SelectShared)) + warp * kCandidates;
  uint32_t* keys = reinterpret_cast<uint32_t*>(sm + sizeof(SelectShared)) + warps * kCandidates;
  pdl_wait();
  const int size = 1 << a.log_cluster, rank = blockIdx.x & (size - 1), row = blockIdx.x >> a.log_cluster;
  const int b = row / a.n_kv, h = row - b * a.n_kv;
  auto scan = [&](uint32_t v) {  // sums of the lanes up to this one
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const uint32_t o = __shfl_up_sync(0xffffffffu, v, d);
      if (lane >= d) v += o;
    }
    return v;
  };
  auto sync_all = [&]() {
    if (size == 1)
      __syncthreads();
    else
      asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  };
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
  const int per_cta = (int)(((uint32_t)len + (uint32_t)(kStep * size) - 1) >> (kLogStep + a.log_cluster)) * kStep;
  const int c_begin = (int)min((int64_t)len, (int64_t)rank * per_cta), c_end = min(len, c_begin + per_cta);
  const int per_warp = (c_end - c_begin + kStep * warps - 1) / (kStep * warps) * kStep;
  const int begin = min(c_end, c_begin + warp * per_warp), end = min(c_end, begin + per_warp);
  const bool staged = per_cta <= a.staged;
  // all of a warp's weights on their way at once
  if (staged) {
    for (int t = begin + 4 * lane; t < end; t += kStep) {
      const uint32_t dst = (uint32_t)__cvta_generic_to_shared(keys + (t - c_begin));
      if (a.vec && t + 3 < end) {
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(w + t) : "memory");
      } else {
        for (int e = 0; e < 4 && t + e < end; ++e)
          asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst + 4 * e), "l"(w + t + e) : "memory");
      }
    }
  }
  asm volatile("cp.async.commit_group;" ::: "memory");
  for (int i = tid; i < (size > 1 ? 2 : 1) * (kBins + 3 * kFew); i += blockDim.x) s.hist[i] = 0;

  // keys of a warp's tokens t0 .. t0 + 127, four of a lane; 0 behind the last
  auto load_keys = [&](int t0, uint32_t key[4]) {
    const int t = t0 + 4 * lane;
    float x[4] = {0.f, 0.f, 0.f, 0.f};
    if (staged) {  // (each lane reads what it copied; behind `end` anything)
      const float4 v = *reinterpret_cast<const float4*>(keys + (t - c_begin));
      x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
    } else if (a.vec && t + 3 < end) {
      const float4 v = __ldg(reinterpret_cast<const float4*>(w + t));
      x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (t + e < end) x[e] = __ldg(w + t + e);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) key[e] = order_key(x[e]);
    if (find && t0 >= lo && t0 + kStep <= min(hi, end)) return;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (t + e < lo || t + e >= hi || !find) key[e] = kAlways;
      if (t + e >= end) key[e] = 0;
    }
  };
  auto at = [&](int t0, uint32_t key[4]) {
    if (staged) {
      const uint4 v = *reinterpret_cast<const uint4*>(keys + (t0 + 4 * lane - c_begin));
      key[0] = v.x; key[1] = v.y; key[2] = v.z; key[3] = v.w;
    } else {
      load_keys(t0, key);
    }
  };
  // places behind the last token that stays
  if (a.w_out) {
    float* out = a.w_out + b * a.out_seq + h * a.out_head;
    int64_t t = (int64_t)count + rank * (int)blockDim.x + tid;
    if ((reinterpret_cast<uintptr_t>(out) & 15u) == 0) {  // (up to three before the first group of 16 bytes, and behind the last)
      const int64_t a0 = ((int64_t)count + 3) / 4, a1 = a.out_width / 4;
      for (int64_t g = a0 + rank * (int)blockDim.x + tid; g < a1; g += size * (int)blockDim.x)
        reinterpret_cast<float4*>(out)[g] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (rank == 0 && tid < 4 && count + tid < min(4 * a0, a.out_width)) out[count + tid] = 0.f;
      t = max(4 * a0, 4 * a1) + (rank == 0 ? tid : a.out_width);
    }
    for (; t < a.out_width; t += size * (int)blockDim.x) out[t] = 0.f;
  }
  int32_t* idx = a.idx + (int64_t)row * a.keep;
  for (int64_t t = (int64_t)count + rank * (int)blockDim.x + tid; t < a.keep; t += size * (int)blockDim.x) idx[t] = -1;
  if (h == 0 && rank == 0 && tid == 0) a.count[b] = count;

  asm volatile("cp.async.wait_group 0;" ::: "memory");
  __syncthreads();  // (counts are zeros)
  for (int t0 = begin; t0 < end; t0 += kStep) {
    uint32_t key[4], bin[4];
    bool in[4];
    load_keys(t0, key);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      bin[e] = key[e] >> 21;
      in[e] = key[e] != 0;
    }
    if (staged) *reinterpret_cast<uint4*>(keys + (t0 + 4 * lane - c_begin)) = make_uint4(key[0], key[1], key[2], key[3]);
    if (find) count_keys(size > 1 ? s.mine : s.hist, bin, in);
  }

  uint32_t need = (uint32_t)a.keep, threshold = kAlways - 1;  // (all stay for certain)
  uint32_t sure = 0, equal = 0;  // this warp's tokens that stay for certain, and those at the threshold (of a lane, at first)
  bool listed = false;           // all of this warp's tokens in the first digit's bin are in its list
  const uint32_t below = (1u << lane) - 1;
  if (find) {
    if (size > 1) {  // to everyone
      sync_all();    // (whose counts are zeros by then)
      for (int i = tid; i < kBins; i += blockDim.x) {
        const uint32_t v = s.mine[i];
        if (v)
          for (int c = 0; c < size; ++c) add_remote(remote(&s.hist[i], c), v);
      }
    }
    sync_all();
    for (int r = warp; r < kBinRows; r += warps) {
      const uint32_t v = __reduce_add_sync(0xffffffffu, s.hist[32 * r + lane]);
      if (lane == 0) s.rows[r] = v;
    }
    __syncthreads();
    // every warp finds the bin: first the row of 32, from the top (lane i holds rows 63 - 2 i and 62 - 2 i)
    uint32_t prefix;
    {
      const int r1 = kBinRows - 1 - 2 * lane, r0 = r1 - 1;
      const uint32_t v1 = s.rows[r1], v0 = s.rows[r0], sum = scan(v1 + v0);
      const int hit = __ffs(__ballot_sync(0xffffffffu, sum >= need)) - 1;
      const uint32_t above = sum - v1 - v0;
      const bool second = above + v1 < need;
      const int r = __shfl_sync(0xffffffffu, second ? r0 : r1, hit);
      need -= __shfl_sync(0xffffffffu, second ? above + v1 : above, hit);
      const uint32_t v = s.hist[32 * r + 31 - lane], in_row = scan(v);
      const int at_lane = __ffs(__ballot_sync(0xffffffffu, in_row >= need)) - 1;
      prefix = 32 * r + 31 - at_lane;
      need -= __shfl_sync(0xffffffffu, in_row - v, at_lane);
    }
    // the other digits go by the tokens in that bin alone, a few in a hundred: their keys, in any order
    int n_cand = 0;
    for (int t0 = begin; t0 < end; t0 += kStep) {
      uint32_t key[4];
      at(t0, key);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t digit = key[e] >> 21;
        sure += digit > prefix;
        const uint32_t all = __ballot_sync(0xffffffffu, digit == prefix && key[e] != 0);
        const int place = n_cand + __popc(all & below);
        if ((all >> lane & 1) && place < kCandidates) cand[place] = key[e];
        n_cand += __popc(all);
      }
    }
    listed = n_cand <= kCandidates;
    __syncwarp();
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = 14 - 7 * pass;
      uint32_t* few = size > 1 ? s.mine_few[pass] : s.few[pass];
      if (listed)
        for (int i = lane; i < n_cand; i += 32)
          if (cand[i] >> (shift + 7) == prefix) atomicAdd(few + (cand[i] >> shift & (kFew - 1)), 1u);
      for (int t0 = listed ? end : begin; t0 < end; t0 += kStep) {
        uint32_t key[4], bin[4];
        bool in[4];
        at(t0, key);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          in[e] = key[e] >> (shift + 7) == prefix && key[e] != 0;
          bin[e] = key[e] >> shift & (kFew - 1);
        }
        if (__any_sync(0xffffffffu, in[0] || in[1] || in[2] || in[3])) count_keys(few, bin, in);
      }
      if (size > 1) {
        __syncthreads();
        for (int i = tid; i < kFew * size; i += blockDim.x) {
          const uint32_t v = few[i % kFew];
          if (v) add_remote(remote(&s.few[pass][i % kFew], i / kFew), v);
        }
      }
      sync_all();
      // lane i holds bins 127 - 4 i .. 124 - 4 i
      const uint4 v = *reinterpret_cast<const uint4*>(&s.few[pass][kFew - 4 - 4 * lane]);
      const uint32_t mine = v.x + v.y + v.z + v.w, sum = scan(mine);
      const int hit = __ffs(__ballot_sync(0xffffffffu, sum >= need)) - 1;
      uint32_t above = sum - mine;
      uint32_t bin = kFew - 1 - 4 * lane;
      const uint32_t from_top[3] = {v.w, v.z, v.y};
      bool done = false;
#pragma unroll
      for (int e = 0; e < 3; ++e) {
        done = done || above + from_top[e] >= need;
        if (!done) {
          above += from_top[e];
          --bin;
        }
      }
      prefix = prefix << 7 | __shfl_sync(0xffffffffu, bin, hit);
      need -= __shfl_sync(0xffffffffu, above, hit);
    }
    threshold = prefix;
    for (int i = lane; listed && i < n_cand; i += 32) {
      sure += cand[i] > threshold;
      equal += cand[i] == threshold;
    }
  }

  if (size > 1 && !find) sync_all();  // (every CTA is there)
  if (!listed) sure = 0;
  for (int t0 = listed ? end : begin; t0 < end; t0 += kStep) {
    uint32_t key[4];
    at(t0, key);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      sure += key[e] > threshold;
      equal += key[e] == threshold;
    }
  }
  sure = __reduce_add_sync(0xffffffffu, sure);
  equal = __reduce_add_sync(0xffffffffu, equal);
  if (lane == 0) {
    s.warp_sure[warp] = sure;
    s.warp_equal[warp] = equal;
  }
  __syncthreads();
  if (warp == 0) {
    const uint32_t ms = lane < warps ? s.warp_sure[lane] : 0u, me = lane < warps ? s.warp_equal[lane] : 0u;
    uint32_t vs = scan(ms), ve = scan(me);
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
  uint32_t staying = sure + min(equal, need);  // before the warp's next tokens
  for (int t0 = begin; t0 < end; t0 += kStep) {
    const int t = t0 + 4 * lane;
    uint32_t key[4], flags = 0, equals = 0;  // a bit per token of this lane
    at(t0, key);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      flags |= key[e] > threshold ? 1u << e : 0u;
      equals |= key[e] == threshold ? 1u << e : 0u;
    }
    if (__any_sync(0xffffffffu, equals != 0)) {  // the first of them stay, too
      uint32_t mine = equal;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t all = __ballot_sync(0xffffffffu, equals >> e & 1);
        mine += __popc(all & below);
        equal += __popc(all);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (equals >> e & 1 && mine++ < need) flags |= 1u << e;
    }
    uint32_t place = staying;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t all = __ballot_sync(0xffffffffu, flags >> e & 1);
      place += __popc(all & below);
      staying += __popc(all);
    }
    for (; flags; flags &= flags - 1, ++place) {  // (few tokens stay: most lanes have none or one)
      const int e = __ffs(flags) - 1;
      const uint32_t k = e < 2 ? (e ? key[1] : key[0]) : (e == 2 ? key[2] : key[3]);
      if (place >= (uint32_t)count) break;
      idx[place] = t + e;
      if (out) out[place] = k < kNan ? weight_of(k) : __ldg(w + t + e);
    }
  }
}

crvq_status select(const crvq_token_sums* weights, const int32_t* lens, int32_t n_seq, int32_t n_kv, int32_t keep,
                   int32_t first, int32_t recent, int32_t* idx, int32_t* count, const crvq_token_sums* weights_out,
                   cudaStream_t stream) {
  SelectArgs a{};
  CRVQ_CHECK_ARG(n_seq >= 1 && n_kv >= 1, "need n_seq, n_kv >= 1");
  CRVQ_TRY(check_sums(weights, "weights", n_seq, n_kv));
  CRVQ_CHECK_ARG(weights->width < ((int64_t)1 << 31) - (1 << 16), "weights: width must be below 2^31 - 2^16");
  CRVQ_CHECK_ARG(keep >= 1, "keep must be >= 1");
  CRVQ_CHECK_ARG(first >= 0 && recent >= 0 && (int64_t)first + recent <= keep, "first and recent must be >= 0 and fit in keep");
  CRVQ_CHECK_ARG(lens && idx && count, "lens, idx and count must not be NULL");
  CRVQ_CHECK_ARG((((uintptr_t)lens | (uintptr_t)idx | (uintptr_t)count) & 3u) == 0, "lens, idx or count is not aligned");
  CRVQ_TRY(check_dev({{lens, "lens"}, {idx, "idx"}, {count, "count"}}));
  if (weights_out) {
    CRVQ_TRY(check_sums(weights_out, "weights_out", n_seq, n_kv));
    CRVQ_CHECK_ARG(weights_out->width >= min((int64_t)keep, weights->width), "weights_out is too narrow for keep weights a row");
    CRVQ_CHECK_ARG(!sums_overlap(weights, weights_out, n_seq, n_kv), "weights_out and weights share memory");
    a.w_out = weights_out->data;
    a.out_seq = weights_out->ld_seq;
    a.out_head = weights_out->ld_head;
    a.out_width = weights_out->width;
  }
  a.w = weights->data;
  a.w_seq = weights->ld_seq;
  a.w_head = weights->ld_head;
  a.width = weights->width;
  a.vec = ((uintptr_t)a.w & 15u) == 0 && (n_seq == 1 || a.w_seq % 4 == 0) && (n_kv == 1 || a.w_head % 4 == 0);
  a.lens = lens;
  a.idx = idx;
  a.count = count;
  a.n_kv = n_kv;
  a.keep = keep;
  a.first = first;
  a.recent = recent;
  CRVQ_TRY(device_error_word(&a.err));
  const int64_t units = (int64_t)n_seq * n_kv;
  // CTAs of a row: as many as hold it in shared memory; twice as many while each is left an SM of its own and 2048 tokens
  // (1, 2, 4, 8 CTAs, us: 32 rows of 131072 tokens 79, 46, 22, 33; 8 such rows 79, 46, 23, 16; 64 of 16384 14, 13, 17, 19;
  // 512 of 16384 46, 66, 108, 118; 8 of 8192 10.2, 11.0, 9.1, 9.6; 8 of 4096 8.3, 8.8, 8.9, 11.0)
  int size = 1;
  while (size < 8 && (a.width > (int64_t)kStageMax * size ||
                      (units * size * 2 <= sm_count() && a.width > 4096 && a.width > (int64_t)2048 * size))) {
    size *= 2;
    ++a.log_cluster;
  }
  if (units * size >= (int64_t)1 << 31) return fail(CRVQ_ERR_UNSUPPORTED, "too many sequences and heads in one call");
  const int64_t per_cta = ceil_div(a.width, kStep * size) * kStep;
  // 128 tokens a warp, or 512 where SMs have several CTAs, one after another: every warp searches the digits' counts (128, 256,
  // 512, 1024 tokens a warp, us: 2048 rows of 4096 tokens 81, 52, 41, 42; 512 of 4096 25, 17, 14, 15; 8 of 1001 6.1, 7.5)
  const int steps = units * size > sm_count() ? 4 : 1;
  const int threads = 32 * (int)min((int64_t)kMaxWarps, max((int64_t)4, ceil_div(per_cta, kStep * steps)));
  a.staged = (int)min(per_cta, (int64_t)kStageMax);
  const size_t smem = sizeof(SelectShared) + (size_t)(threads * (kCandidates / 32) + a.staged) * sizeof(float);
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
