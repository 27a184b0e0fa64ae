// Moving kept tokens together in a paged 8-bit cache: token idx[b][h][r] of the source goes to place start[b] + r of the
// destination. Per block of 16 places of a head's keys or values that tokens c_i at scales s_i come to (with those tokens
// before start[b] that the block holds already),
//   s = max_i s_i,   c_i <- round(c_i * (s_i / s)),
// each operation rounded to fp32: codes that keep their scale keep their bits.
//
// A CTA takes tiles of a few blocks of one head's keys or values: it looks up where every token of the tile lies (one thread a
// token), then each thread moves 16 codes at a time, a block's scale found by every thread that writes to it.
//   In place the tiles of a (sequence, head) are dealt out to the CTAs of a cluster, round by round: a round's codes and
// scales are read by all of them before any is written. Tokens only move towards the front there (idx >= place), so what a
// later round reads lies behind all that earlier ones have written.
//   What bounds it: loads in flight, and the instructions that turn codes into others (4 per code). 2047 of up to 8192 tokens of 8
// sequences, 32 heads, e4m3, into other pages: 60 us, 4.5 TB/s. 16384 of up to 65536 of 2, 8 heads, int8, in place: 42 us,
// 3.2 TB/s, eight rounds of 5 us (46 before a round's codes were on their way beside the writes of the one before).
#include "cache.cuh"
#include "kernels.h"

namespace crvq {

namespace {

constexpr int kKeepThreads = 256;

struct KeepArgs {
  CacheView from, to;
  const int32_t* idx;
  const int32_t* count;
  const int32_t* start;  // or null: 0
  int64_t ld_seq, ld_head;
  int most;              // columns of idx
  int tiles;             // grid: CTAs per (sequence, head, keys or values)
  bool same_pool;        // (then written pages must be others than those read at the same places)
  Divisor from_page, to_page;
  unsigned* err;
};

template <int D>
struct KeepShape {
  static constexpr int kRow = D / 16;                     // threads per token
  static constexpr int kSlots = kKeepThreads / kRow;      // tokens at a time: 64, 32 or 16
  static constexpr int kTimes = D == 64 ? 4 : 8;
  static constexpr int kTokens = kSlots * kTimes;         // of a tile: 256, 256 or 128
  static_assert(kTokens <= kKeepThreads, "a thread looks up one token");
};

// Where a tile's tokens lie and go (dst -1: nowhere).
template <int D>
struct KeepTile {
  static constexpr int kTokens = KeepShape<D>::kTokens;
  const uint8_t* src[kTokens];            // a token's codes, or null
  int64_t dst[kTokens / kCacheBlock], dst_scale[kTokens / kCacheBlock];
  float ratio[kTokens];                   // its scale / its new block's
  float scale[kTokens / kCacheBlock];
};

// (x - 8388736) * ratio + 12582912 of two numbers, each operation rounded, as bits. (The last one number by number: a product
// and a sum of two numbers at a time became one operation with one rounding.)
__device__ __forceinline__ void scale2(uint32_t x, uint32_t y, float ratio, uint32_t& rx, uint32_t& ry) {
  float vx, vy;
  asm("{\n.reg .b64 v, f, c;\n"
      "mov.b64 v, {%2, %3};\n"
      "mov.b64 f, {%4, %4};\n"
      "mov.b64 c, {%5, %5};\n"
      "add.rn.f32x2 v, v, c;\n"
      "mul.rn.f32x2 v, v, f;\n"
      "mov.b64 {%0, %1}, v;\n}"
      : "=f"(vx), "=f"(vy)
      : "r"(x), "r"(y), "f"(ratio), "f"(-8388736.f));
  rx = __float_as_uint(__fadd_rn(vx, 12582912.f));
  ry = __float_as_uint(__fadd_rn(vy, 12582912.f));
}

// Looking a token up takes three loads one after another (its place, its page, its scale), so a tile's begin three rounds ahead:
// in every round one step of three tiles is on its way beside the present tile's codes.
template <int D, int FMT, bool IN_PLACE>
__global__ void __launch_bounds__(kKeepThreads, IN_PLACE ? 2 : 3) keep_kernel(const __grid_constant__ KeepArgs a) {
  using S = KeepShape<D>;
  constexpr int kAhead = IN_PLACE ? 1 : 0;  // rounds whose codes are on their way beside a round's writes
  __shared__ KeepTile<D> tile_s[2 + kAhead];
  pdl_wait();
  const int tid = threadIdx.x;
  const int unit = blockIdx.x / a.tiles, rank = blockIdx.x - unit * a.tiles;
  const bool is_key = !(unit & 1);
  const int b = (unit >> 1) / a.from.n_kv, h = (unit >> 1) - b * a.from.n_kv;
  int n = __ldg(a.count + b);
  const int start = a.start ? __ldg(a.start + b) : 0;
  if (n < 0 || n > a.most || start < 0 || (int64_t)start + n > (int64_t)a.to.max_pages * a.to.page) {
    raise_error(a.err, ERRBIT_INDEX);
    n = 0;
  }
  if (n == 0) return;  // (with its whole cluster)
  const int len = seq_len(a.from, b, a.err);
  const int base = start / kCacheBlock * kCacheBlock, end = start + n;
  const int n_tiles = (int)(((uint32_t)(end - base) + S::kTokens - 1) / S::kTokens);
  // (in place, every CTA of a cluster takes part in every round)
  const int rounds = IN_PLACE ? (n_tiles + a.tiles - 1) / a.tiles : max(0, n_tiles - rank + a.tiles - 1) / a.tiles;
  const int32_t* idx = a.idx + b * a.ld_seq + h * a.ld_head;
  const uint8_t* from = is_key ? a.from.K : a.from.V;
  uint8_t* to = is_key ? a.to.K : a.to.V;
  const float* from_scale = is_key ? a.from.ks : a.from.vs;
  float* to_scale = is_key ? a.to.ks : a.to.vs;
  const int from_blocks = (unsigned)a.from.page / kCacheBlock, to_blocks = (unsigned)a.to.page / kCacheBlock;
  const int col = tid % S::kRow, slot = tid / S::kRow;
  // (places go up to 2^31 - 16)
  auto place0 = [&](int round) { return (int)min((int64_t)end, base + (int64_t)(rank + round * a.tiles) * S::kTokens); };
  // the place that this thread looks up for a round; `end` where there is none
  auto place = [&](int round) {
    const int p0 = place0(round);
    return tid < S::kTokens && round < rounds && tid < end - p0 ? p0 + tid : end;
  };

  auto find_token = [&](int round) {
    const int p = place(round);
    return p >= start && p < end ? __ldg(idx + (p - start)) : 0;
  };
  struct Pages {
    int64_t from, to;
  };
  auto find_pages = [&](int round, int t) {
    const int p = place(round);
    Pages g{-1, -1};
    if (p < end) {
      const int entry = a.to_page.div(p);
      g.to = seq_page(a.to, b, entry, a.err);
      if (p >= start) {
        if (t < 0 || t >= len || (IN_PLACE && t < p))
          raise_error(a.err, ERRBIT_INDEX);
        else
          g.from = seq_page(a.from, b, a.from_page.div(t), a.err);
      }
      if (!IN_PLACE && a.same_pool && g.to >= 0 && p < len && g.to == seq_page(a.from, b, entry, a.err)) {
        raise_error(a.err, ERRBIT_INDEX);  // (in place, unsaid: the order of reads and writes would be open)
        g.to = -1;
      }
    }
    return g;
  };
  struct Found {
    const uint8_t* src;
    int64_t dst, at_scale;
    float scale;
  };
  auto find_scale = [&](int round, int t, const Pages& g) {
    const int p = place(round);
    Found f{nullptr, -1, 0, 0.f};
    if (g.to >= 0) {  // (p < end)
      const int in = p - a.to_page.div(p) * a.to.page;
      f.dst = g.to * a.to.page_stride + ((int64_t)h * a.to.page + in) * D;
      f.at_scale = (g.to * a.to.n_kv + h) * to_blocks + in / kCacheBlock;
      if (p < start) {
        f.src = to + f.dst;
        f.scale = to_scale[f.at_scale];
      }
    }
    if (g.from >= 0) {
      const int in = t - a.from_page.div(t) * a.from.page;
      f.src = from + g.from * a.from.page_stride + ((int64_t)h * a.from.page + in) * D;
      f.scale = from_scale[(g.from * a.from.n_kv + h) * from_blocks + in / kCacheBlock];
    }
    return f;
  };
  auto put = [&](int round, const Found& f) {
    if (tid >= S::kTokens) return;  // (whole warps)
    KeepTile<D>& tile = tile_s[round % (2 + kAhead)];
    float s = f.scale;  // of a block, 16 lanes
#pragma unroll
    for (int d = kCacheBlock / 2; d > 0; d >>= 1) s = fmaxf(s, __shfl_xor_sync(0xffffffffu, s, d));
    if (tid % kCacheBlock == 0) {
      tile.dst[tid / kCacheBlock] = f.dst;
      tile.dst_scale[tid / kCacheBlock] = f.at_scale;
      tile.scale[tid / kCacheBlock] = s;
    }
    tile.src[tid] = f.src;
    tile.ratio[tid] = s > 0.f ? __fdiv_rn(f.scale, s) : 0.f;
  };
  auto load_codes = [&](int round, uint4 (&codes)[S::kTimes]) {
    const KeepTile<D>& tile = tile_s[round % (2 + kAhead)];
#pragma unroll
    for (int u = 0; u < S::kTimes; ++u) {
      const uint8_t* src = round < rounds ? tile.src[u * S::kSlots + slot] : nullptr;
      codes[u] = make_uint4(0, 0, 0, 0);
      if (src) codes[u] = *reinterpret_cast<const uint4*>(src + 16 * col);
    }
  };
  int t1, t2 = find_token(0), t3 = find_token(1);
  Pages g1, g2 = find_pages(0, t2);
#pragma unroll
  for (int i = 0; i <= kAhead; ++i) {
    t1 = t2;
    g1 = g2;
    t2 = t3;
    g2 = find_pages(i + 1, t2);
    t3 = find_token(i + 2);
    put(i, find_scale(i, t1, g1));
  }
  t1 = t2;
  t2 = t3;
  g1 = g2;  // (t1, g1: of the round whose scale is next to be looked up; t2: of the one after that)
  uint4 codes[S::kTimes], later[S::kTimes];
  if (kAhead) {
    __syncthreads();
    load_codes(0, codes);
  }
  for (int round = 0; round < rounds; ++round) {
    // In place: no CTA goes past the wait before all have this round's codes. The next round's, which lie behind all that this
    // one writes, are loaded meanwhile.
    if (IN_PLACE && a.tiles > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    __syncthreads();  // the places that the next codes go by are there, and those that are put next have been read
    const KeepTile<D>& tile = tile_s[round % (2 + kAhead)];
    load_codes(round + kAhead, kAhead ? later : codes);
    const Found next = find_scale(round + kAhead + 1, t1, g1);
    g2 = find_pages(round + kAhead + 2, t2);
    t3 = find_token(round + kAhead + 3);
    if (IN_PLACE && a.tiles > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    const int p0 = place0(round);
#pragma unroll
    for (int u = 0; u < S::kTimes; ++u) {
      const int i = u * S::kSlots + slot, block = i / kCacheBlock;
      if (i >= end - p0 || tile.dst[block] < 0) continue;
      const float ratio = tile.ratio[i];  // (at most 1; 0 for a token that is none)
      uint32_t w[4] = {codes[u].x, codes[u].y, codes[u].z, codes[u].w};
      if (ratio == 0.f) {
        w[0] = w[1] = w[2] = w[3] = 0;
      } else if (ratio != 1.f) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if constexpr (FMT == CRVQ_KV_INT8) {
            // 2^23 + code + 128, less 2^23 + 128: exact, without conversions; adding 1.5 * 2^23 rounds to an integer
            const uint32_t x = w[e] ^ 0x80808080u;
            uint32_t r[4];
#pragma unroll
            for (int k = 0; k < 4; k += 2)
              scale2(__byte_perm(x, 0x4b000000u, 0x7440 + k), __byte_perm(x, 0x4b000000u, 0x7441 + k), ratio, r[k], r[k + 1]);
            w[e] = __byte_perm(__byte_perm(r[0], r[1], 0x0040), __byte_perm(r[2], r[3], 0x0040), 0x5410);
          } else {
            float v[4];
            decode4<FMT>(w[e], v);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = __fmul_rn(v[k], ratio);
            w[e] = encode4<FMT, true>(v);
          }
        }
      }
      *reinterpret_cast<uint4*>(to + tile.dst[block] + (i % kCacheBlock) * D + 16 * col) = make_uint4(w[0], w[1], w[2], w[3]);
      if (i % kCacheBlock == 0 && col == 0) to_scale[tile.dst_scale[block]] = tile.scale[block];
    }
    put(round + kAhead + 1, next);
    t1 = t2;
    t2 = t3;
    g1 = g2;
    if (kAhead) {
#pragma unroll
      for (int u = 0; u < S::kTimes; ++u) codes[u] = later[u];
    }
  }
}

template <int D, int FMT>
crvq_status launch_keep(KeepArgs& a, bool in_place, cudaStream_t stream) {
  // tiles that n tokens can touch, from any start
  const int64_t tiles = ceil_div((int64_t)a.most + kCacheBlock - 1, KeepShape<D>::kTokens);
  const int64_t units = (int64_t)a.from.n_seq * a.from.n_kv * 2;
  int size = 1;
  while (in_place && size < 8 && size < tiles) size *= 2;
  // Into other pages: two waves of CTAs, so that each has tiles to look up while one is on its way. One wave, two, four, a CTA per
  // tile, us, for (sequences x kv heads, tokens of a sequence): (8 x 32, 2047, e4m3) 71, 59, 55, 56; (2 x 8, 16384) 38, 30, 30, 29; (64 x
  // 32, 300) 74, 74, 74, 83; (16 x 8, 1000) 13.8, 13.0, 13.1, 13.0; (8 x 8, 4000, 64 channels) 18.2, 16.9, 18.8, 17.7.
  a.tiles = in_place ? size : (int)min(tiles, ceil_div((int64_t)6 * sm_count(), units));
  if (units * a.tiles >= (int64_t)1 << 31) return fail(CRVQ_ERR_UNSUPPORTED, "too many tokens in one call");
  const dim3 grid((unsigned)(units * a.tiles)), threads(kKeepThreads);
  if (!in_place) {
    CRVQ_CUDA(launch_pdl(keep_kernel<D, FMT, false>, grid, threads, 0, stream, a));
  } else {
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = size;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = threads;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    CRVQ_CUDA(cudaLaunchKernelEx(&cfg, keep_kernel<D, FMT, true>, a));
  }
  CRVQ_LAUNCHED();
  return CRVQ_OK;
}

template <int D>
crvq_status pick_format(KeepArgs& a, int format, bool in_place, cudaStream_t stream) {
  return format == CRVQ_KV_INT8 ? launch_keep<D, CRVQ_KV_INT8>(a, in_place, stream)
                                : launch_keep<D, CRVQ_KV_E4M3>(a, in_place, stream);
}

crvq_status keep(const crvq_kv_cache* cache, const int32_t* idx, int64_t ld_seq, int64_t ld_head, int32_t most,
                 const int32_t* count, const int32_t* start, const crvq_kv_cache* out, cudaStream_t stream) {
  KeepArgs a{};
  CRVQ_TRY(make_cache(cache, &a.from));
  if (out == cache)
    a.to = a.from;
  else
    CRVQ_TRY(make_cache(out, &a.to));
  CRVQ_CHECK_ARG(a.from.n_seq == a.to.n_seq && a.from.n_kv == a.to.n_kv && cache->head_dim == out->head_dim &&
                     cache->format == out->format,
                 "cache and out differ in sequences, kv heads, head_dim or format");
  CRVQ_CHECK_ARG(most >= 0, "most must be >= 0");
  CRVQ_CHECK_ARG(ld_head == 0 || ld_head >= most, "idx: rows of heads overlap");
  CRVQ_CHECK_ARG(count != nullptr, "count is NULL");
  CRVQ_CHECK_ARG((((uintptr_t)idx | (uintptr_t)count | (uintptr_t)start) & 3u) == 0, "idx, count or start is not aligned");
  CRVQ_TRY(check_dev({{idx, "idx"}, {count, "count"}, {start, "start"}}));
  if (most == 0) return CRVQ_OK;
  CRVQ_CHECK_ARG(idx != nullptr, "idx is NULL");
  CRVQ_CHECK_ARG((cache->K == out->K) == (cache->V == out->V) && (cache->K == out->K) == (cache->k_scale == out->k_scale) &&
                     (cache->K == out->K) == (cache->v_scale == out->v_scale),
                 "cache and out share some arrays of a pool, not all");
  a.same_pool = cache->K == out->K;
  const bool in_place = a.same_pool && cache->pages == out->pages && cache->ld_pages == out->ld_pages;
  CRVQ_CHECK_ARG(!in_place || cache->page == out->page, "in place, cache and out differ in page");
  CRVQ_CHECK_ARG(!a.same_pool || (cache->page == out->page && cache->page_stride == out->page_stride), "cache and out share a pool of different pages");
  a.idx = idx;
  a.ld_seq = ld_seq;
  a.ld_head = ld_head;
  a.most = most;
  a.count = count;
  a.start = start;
  a.from_page = Divisor(a.from.page);
  a.to_page = Divisor(a.to.page);
  CRVQ_TRY(device_error_word(&a.err));
  ProfScope ps("cache_keep", stream, (double)a.from.n_seq * a.from.n_kv * most * cache->head_dim * 4);
  if (cache->head_dim == 64) return pick_format<64>(a, cache->format, in_place, stream);
  if (cache->head_dim == 128) return pick_format<128>(a, cache->format, in_place, stream);
  return pick_format<256>(a, cache->format, in_place, stream);
}

}  // namespace

}  // namespace crvq

extern "C" {

crvq_status crvq_cache_keep(const crvq_kv_cache* cache, const int32_t* idx, int64_t ld_seq, int64_t ld_head, int32_t most,
                            const int32_t* count, const int32_t* start, const crvq_kv_cache* out,
                            crvq_stream_t stream) {
  CRVQ_ENTRY({
    return crvq::keep(cache, idx, ld_seq, ld_head, most, count, start, out, (cudaStream_t)stream);
  })
}

}  // extern "C"
