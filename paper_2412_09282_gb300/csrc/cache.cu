// The paged 8-bit key/value cache: appending rotated keys and values, and reading ranges back.
//
// Append. Per touched block (16 tokens of one kv head, keys or values) with old tokens c_i at scale
// s0 and new values x_i:
//   s = max(max_i |x_i| * (1 / Q), s0 if there are old tokens),  Q = 127 or 448,
//   c_i <- round(c_i * (s0 / s)) for the old,  c_i = round(x_i / s) for the new,
// with x the rotated key (a cos - b sin, b cos + a sin) or the value. One CTA owns one block of one
// head's keys and values, so a scale is found and every code written by the same threads: no atomics,
// no second pass over the inputs. A thread holds 16 channels of a token's key and of its value, four at
// 4 c + k D / 4, k = 0 .. 3: a rotation pair of either form is one thread's, and every load of a row covers
// whole lines. What does not wait for another lookup is loaded first (the new rows beside the page).
// The grid has a slot for every block that could be touched (the lengths are on the device); the ones
// that are not leave at once. Each product, difference and quotient is rounded to fp32 by itself (no
// fused multiply-add): codes do not depend on how the compiler contracts.
//
// What bounds it: memory, with the lookups' latency between a CTA's start and its loads. Three fp32 prompts of up to
// 4091 tokens, 32 heads, queries rotated: 104 us for 544 MB (5.2 TB/s; 30000 CTAs of one block and head each, 12 per
// SM). Reading them back: 47 us, 302 MB (6.4 TB/s). One thread for K and V both took 179 us (registers); 64-bit
// divisions for the places and CUDA's division per element, 145.
#include "cache.cuh"

#include "kernels.h"

namespace crvq {

namespace {

constexpr int kOffShared = 1024;  // row offsets staged in shared memory up to this many sequences

struct AppendArgs {
  CacheView c;
  HeadsView k, v, q, qo;
  RowsView rows;
  const float* cos;
  const float* sin;
  const int32_t* positions;
  int64_t n_pos, ld_rot;
  int half;          // rotated pairs (0: none)
  bool interleaved;
  bool pair_regs;    // a rotation pair lies within a thread's 16 channels, read whole from the tables
  bool vec_k, vec_v, vec_q, vec_qo, vec_rot;
  int64_t slots;     // block slots of all sequences
  int per_seq;       // slots per sequence (rows.off null)
  int n_append;      // CTAs of the append; the rest rotate queries
  int n_rows;        // (token, head) rows of queries
  Divisor by_kv, by_page, by_heads, by_per, by_slots;  // n_kv, page, query heads, rows.per, per_seq
  unsigned* err;
};

__device__ __forceinline__ bool finite(float x) { return fabsf(x) <= 3.402823466e38f; }

// The 16 channels of a thread, c the thread's index in its row (0 .. D/16 - 1): channel of element e.
template <int D>
__device__ __forceinline__ int channel(int c, int e) {
  return 4 * c + (e >> 2) * (D / 4) + (e & 3);
}

__device__ __forceinline__ void turn(float& u, float& w, float c, float s) {
  const float x = u;
  u = __fsub_rn(__fmul_rn(u, c), __fmul_rn(w, s));
  w = __fadd_rn(__fmul_rn(w, c), __fmul_rn(x, s));
}

// Four consecutive fp32 elements (vec: 16-byte aligned).
__device__ __forceinline__ void load4(const float* p, bool vec, float v[4]) {
  if (vec) {
    const float4 a = __ldg(reinterpret_cast<const float4*>(p));
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = __ldg(p + j);
  }
}

__device__ __forceinline__ void store4(void* p, int64_t i, int type, bool vec, const float v[4]) {
  if (!vec) {
#pragma unroll
    for (int j = 0; j < 4; ++j) store_elem(p, i + j, type, v[j]);
  } else if (type == CRVQ_F32) {
    *reinterpret_cast<float4*>(static_cast<float*>(p) + i) = make_float4(v[0], v[1], v[2], v[3]);
  } else {
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p) + i) = make_uint2(pack2(v[0], v[1], type), pack2(v[2], v[3], type));
  }
}

// A thread's 16 channels of (token row t, head h).
template <int D>
__device__ __forceinline__ void load_row(const HeadsView& src, bool vec, int64_t t, int h, int c, float x[16]) {
  const int64_t row = t * src.ld_tok + h * src.ld_head;
  if (!vec) {
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = load_elem(src.data, row + channel<D>(c, e), src.type);
  } else if (src.type == CRVQ_F32) {
    const float* p = static_cast<const float*>(src.data) + row + 4 * c;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float4 a = *reinterpret_cast<const float4*>(p + k * (D / 4));
      x[4 * k] = a.x; x[4 * k + 1] = a.y; x[4 * k + 2] = a.z; x[4 * k + 3] = a.w;
    }
  } else {
    const uint16_t* p = static_cast<const uint16_t*>(src.data) + row + 4 * c;
    uint2 u[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) u[k] = *reinterpret_cast<const uint2*>(p + k * (D / 4));
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      float* v = x + 4 * k;
      if (src.type == CRVQ_BF16) {
        v[0] = __uint_as_float(u[k].x << 16); v[1] = __uint_as_float(u[k].x & 0xffff0000u);
        v[2] = __uint_as_float(u[k].y << 16); v[3] = __uint_as_float(u[k].y & 0xffff0000u);
      } else {
        const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&u[k].x));
        const float2 b = __half22float2(*reinterpret_cast<const __half2*>(&u[k].y));
        v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y;
      }
    }
  }
}

// The same, turned by the tables' row `pos` (-1: not).
template <int D>
__device__ __forceinline__ void rotate_row(const AppendArgs& a, const HeadsView& src, int64_t t, int h, int c,
                                           int64_t pos, float x[16]) {
  if (pos < 0) return;
  const float* cs = a.cos + pos * a.ld_rot;
  const float* sn = a.sin + pos * a.ld_rot;
  if (a.pair_regs && a.interleaved) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int i = channel<D>(c, 4 * k) / 2;  // (even: pairs i and i + 1)
      float* v = x + 4 * k;
      if (a.vec_rot && i + 1 < a.half) {
        const float2 cv = __ldg(reinterpret_cast<const float2*>(cs + i));
        const float2 sv = __ldg(reinterpret_cast<const float2*>(sn + i));
        turn(v[0], v[1], cv.x, sv.x);
        turn(v[2], v[3], cv.y, sv.y);
      } else {  // (an unrotated channel keeps its bits)
        if (i < a.half) turn(v[0], v[1], __ldg(cs + i), __ldg(sn + i));
        if (i + 1 < a.half) turn(v[2], v[3], __ldg(cs + i + 1), __ldg(sn + i + 1));
      }
    }
  } else if (a.pair_regs) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      float cv[4], sv[4];
      load4(cs + channel<D>(c, 4 * k), a.vec_rot, cv);
      load4(sn + channel<D>(c, 4 * k), a.vec_rot, sv);
#pragma unroll
      for (int j = 0; j < 4; ++j) turn(x[4 * k + j], x[4 * k + 8 + j], cv[j], sv[j]);
    }
  } else {
    // pairs (i, i + half) with half < D/2: the partner is another thread's, read again
    const int64_t row = t * src.ld_tok + h * src.ld_head;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int ch = channel<D>(c, e);
      if (ch >= 2 * a.half) continue;
      const bool first = ch < a.half;
      const int i = first ? ch : ch - a.half;
      const float other = load_elem(src.data, row + (first ? ch + a.half : i), src.type);
      const float cv = __ldg(cs + i), sv = __ldg(sn + i);
      x[e] = first ? __fsub_rn(__fmul_rn(x[e], cv), __fmul_rn(other, sv))
                   : __fadd_rn(__fmul_rn(x[e], cv), __fmul_rn(other, sv));
    }
  }
}

// Row of the rotation tables of token row t that lands at place p of its sequence; -1: none.
__device__ __forceinline__ int64_t rot_row(const AppendArgs& a, int64_t t, int p) {
  if (a.half == 0) return -1;
  const int64_t pos = a.positions ? __ldg(a.positions + t) : p;
  if (pos < 0 || pos >= a.n_pos) {
    raise_error(a.err, ERRBIT_INDEX);
    return -1;
  }
  return pos;
}

// Codes of four values (SMALL: magnitudes below Q + 1/2). int8: adding 1.5 * 2^23 rounds to an integer, which
// the sum's low byte is in two's complement.
template <int FMT, bool SMALL>
__device__ __forceinline__ uint32_t encode4(const float v[4]) {
  if constexpr (FMT == CRVQ_KV_INT8) {
    uint32_t b[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      b[j] = __float_as_uint(__fadd_rn(SMALL ? v[j] : fminf(fmaxf(v[j], -127.f), 127.f), 12582912.f));
    return __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
  } else {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(v[0], v[1]), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(v[2], v[3]), __NV_SATFINITE, __NV_E4M3);
    return lo | hi << 16;
  }
}

template <int FMT>
__device__ __forceinline__ void decode4(uint32_t w, float v[4]) {
  if constexpr (FMT == CRVQ_KV_INT8) {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = (float)(int8_t)(w >> (8 * j));
  } else {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const __half2_raw r = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w >> (16 * j)), __NV_E4M3);
      const float2 f = __half22float2(__half2(r));
      v[2 * j] = f.x;
      v[2 * j + 1] = f.y;
    }
  }
}

// One head's keys or values of a block: this thread's new values x (is_new) or old codes to new codes, with
// the block's scale, from the largest new magnitude (bits) and the old scale.
template <int D, int FMT>
__device__ __forceinline__ void encode_block(float x[16], bool is_new, bool is_old, float s0, uint32_t top,
                                             uint8_t* codes, float* scale, int col) {
  constexpr float kInv = (float)(1.0 / (FMT == CRVQ_KV_INT8 ? 127.0 : 448.0));
  const float s = fmaxf(__fmul_rn(__uint_as_float(top), kInv), s0);
  uint32_t w[4];
  if (is_new) {
    if (plain_divisor(s)) {
      const float inv = __frcp_rn(s);
#pragma unroll
      for (int e = 0; e < 16; ++e) x[e] = quotient(x[e], s, inv);
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = encode4<FMT, true>(x + 4 * e);
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e) x[e] = s > 0.f ? __fdiv_rn(x[e], s) : 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = encode4<FMT, false>(x + 4 * e);
    }
  } else if (is_old && s != s0) {
    const float ratio = s > 0.f ? __fdiv_rn(s0, s) : 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float v[4];
      decode4<FMT>(*reinterpret_cast<const uint32_t*>(codes + channel<D>(col, 4 * e)), v);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = __fmul_rn(v[i], ratio);
      w[e] = encode4<FMT, false>(v);
    }
  }
  if (is_new || (is_old && s != s0)) {
#pragma unroll
    for (int e = 0; e < 4; ++e) *reinterpret_cast<uint32_t*>(codes + channel<D>(col, 4 * e)) = w[e];
  }
  if (threadIdx.x == 0) *scale = s;  // (s0 was read by every thread before the barrier)
}

// The largest magnitude (bits) of 16 values; those that are not finite are set to 0 and reported.
__device__ __forceinline__ uint32_t top_of(float x[16], unsigned* err) {
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 16; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
  if (top < 0x7f800000u) return top;
  raise_error(err, ERRBIT_NUMERIC);
  top = 0;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    if (!finite(x[e])) x[e] = 0.f;
    top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
  }
  return top;
}

// (1536 threads per SM: three fp32 prompts of up to 4091 tokens, 32 heads, are appended and read back in 152 us;
// with the registers left open, 162)
template <int D, int FMT>
__global__ void __launch_bounds__(D, 1536 / D) append_kernel(const __grid_constant__ AppendArgs a) {
  constexpr int kRow = D / 16;  // threads per token
  __shared__ int32_t off_s[kOffShared + 1];
  __shared__ uint32_t top_s[D / 32];
  pdl_trigger();
  pdl_wait();
  const int tid = threadIdx.x;
  const CacheView& c = a.c;
  const int32_t* off = a.rows.off;
  // the sequence of a slot: sequence i's begin at off[i] / 16 + 2 i, n tokens touch at most n / 16 + 2 blocks
  auto sequence = [&](int64_t v) {
    auto key = [&](int i) { return (int64_t)off[i] / kCacheBlock + 2 * i; };
    if (c.n_seq > 32) return last_not_above(c.n_seq, v, key);
    const int lane = tid & 31;  // (whole warps: one look for up to 32 sequences)
    const int64_t mine = lane < c.n_seq ? key(lane) : v + 1;
    return 31 - __clz(max(1u, __ballot_sync(0xffffffffu, mine <= v)));
  };
  if (off && c.n_seq > 32 && c.n_seq <= kOffShared) {
    for (int i = tid; i <= c.n_seq; i += D) off_s[i] = __ldg(a.rows.off + i);
    __syncthreads();
    off = off_s;
  }
  // the same for rows that differ within a warp
  auto sequence_of = [&](int64_t t) {
    if (c.n_seq > 32) return last_not_above(c.n_seq, t, [&](int i) { return (int64_t)off[i]; });
    const int lane = tid & 31;
    const int mine = lane < c.n_seq ? off[lane] : INT32_MAX;
    int b = 0;
#pragma unroll
    for (int step = 16; step; step >>= 1) {
      const int at = __shfl_sync(0xffffffffu, mine, b + step);
      if (at <= t) b += step;
    }
    return b;
  };
  const int col = tid % kRow, r = tid / kRow;
  const int id = blockIdx.x;
  if (id >= a.n_append) {  // queries: 16 (token, head) rows
    const unsigned row = (unsigned)(id - a.n_append) * 16 + r;
    bool live = row < (unsigned)a.n_rows;
    const int at = live ? (int)row : 0, t = a.by_heads.div(at), h = at - t * a.q.heads;
    float x[16];
    if (live) load_row<D>(a.q, a.vec_q, t, h, col, x);
    int p = 0;
    if (a.half && !a.positions) {
      const int b = off ? sequence_of(t) : live ? a.by_per.div(t) : 0;
      if (live) {
        int64_t first;
        int n;
        seq_rows(a.rows, b, &first, &n, a.err);
        live = t >= first && t < first + n;  // (rows outside every sequence stay unwritten)
        p = seq_len(c, b, a.err) - n + (int)(t - first);
      }
    }
    if (live) rotate_row<D>(a, a.q, t, h, col, rot_row(a, t, p), x);
    __syncwarp();  // in place: a warp's rows are read whole before they are written
    if (live) {
      const int64_t out = t * a.qo.ld_tok + h * a.qo.ld_head;
#pragma unroll
      for (int k = 0; k < 4; ++k) store4(a.qo.data, out + channel<D>(col, 4 * k), a.qo.type, a.vec_qo, x + 4 * k);
    }
    return;
  }
  // which block: sequence b, its j-th touched one; which head
  const bool is_key = !(id & 1);
  const int slot = a.by_kv.div(id >> 1), h = (id >> 1) - slot * c.n_kv;
  int b, j;
  if (off) {
    b = sequence(slot);
    j = slot - off[b] / kCacheBlock - 2 * b;
  } else {
    b = a.by_slots.div(slot);
    j = slot - b * a.per_seq;
  }
  int64_t first;
  int n;
  seq_rows(a.rows, b, &first, &n, a.err);
  const int len = seq_len(c, b, a.err);
  if (n == 0 || j < 0) return;
  const int held = len - n;
  if (held < 0) {
    raise_error(a.err, ERRBIT_INDEX);
    return;
  }
  const int64_t first_at = ((int64_t)held / kCacheBlock + j) * kCacheBlock;
  if (first_at >= len) return;
  const int p0 = (int)first_at, in_table = a.by_page.div(p0), in_page = p0 - in_table * c.page;
  // the page's number is on its way while the new rows are loaded and turned
  const int32_t page_id = __ldg(c.pages + b * c.ld_pages + in_table);
  const int p = p0 + r;
  const bool is_old = p < held, is_new = !is_old && p < len;
  float x[16];
  uint32_t top = 0;
  if (is_new) {
    const int64_t t = first + (p - held);
    if (is_key) {
      load_row<D>(a.k, a.vec_k, t, h, col, x);
      rotate_row<D>(a, a.k, t, h, col, rot_row(a, t, p), x);
    } else {
      load_row<D>(a.v, a.vec_v, t, h, col, x);
    }
    top = top_of(x, a.err);
  }
  if (page_id < 0 || page_id >= c.n_pages) {  // (the same for the whole block)
    raise_error(a.err, ERRBIT_INDEX);
    return;
  }
  const int64_t page = page_id;
  const int64_t at = page * c.page_stride + ((int64_t)h * c.page + in_page + r) * D;
  const int64_t at_s = (page * c.n_kv + h) * ((unsigned)c.page / kCacheBlock) + in_page / kCacheBlock;
  uint8_t* codes = (is_key ? c.K : c.V) + at;
  float* scale = (is_key ? c.ks : c.vs) + at_s;
  const float s0 = p0 < held ? *scale : 0.f;
  top = __reduce_max_sync(0xffffffffu, top);
  if ((tid & 31) == 0) top_s[tid >> 5] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < D / 32; ++i) top = max(top, top_s[i]);
  encode_block<D, FMT>(x, is_new, is_old, s0, top, codes, scale, col);
}

// A warp takes up to kReadCodes codes of one token's keys and of its values (heads side by side): each lane four
// (fp32) or eight codes at a time to one 16-byte store, the token's place looked up once.
constexpr int kReadCodes = 1024;

template <int FMT, int TYPE>
__global__ void __launch_bounds__(256)
read_kernel(const __grid_constant__ CacheView c, int log_d, Divisor by_parts, Divisor by_page, const int32_t* __restrict__ start,
            const int32_t* __restrict__ off, int64_t n_tok, void* K_out, void* V_out, unsigned* err) {
  constexpr int kVec = TYPE == CRVQ_F32 ? 4 : 8, kStep = 32 * kVec, kBatch = 4;
  pdl_trigger();
  pdl_wait();
  const int lane = threadIdx.x & 31, all = c.n_kv << log_d;
  const int w = (int)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int64_t t = by_parts.div(w);
  if (t >= n_tok) return;
  const int e0 = (w - (int)t * (int)by_parts.d) * kReadCodes, e1 = min(all, e0 + kReadCodes);
  int b;
  if (c.n_seq <= 32) {
    const int64_t mine = lane < c.n_seq ? __ldg(off + lane) : t + 1;
    b = 31 - __clz(max(1u, __ballot_sync(0xffffffffu, mine <= t)));
  } else {
    b = last_not_above(c.n_seq, t, [&](int i) { return (int64_t)__ldg(off + i); });
  }
  const int64_t i = t - __ldg(off + b);
  const int64_t p = (int64_t)__ldg(start + b) + i;
  const int len = seq_len(c, b, err);
  int64_t page = -1;
  if (i < 0 || t >= __ldg(off + b + 1) || p < 0 || p >= len)
    raise_error(err, ERRBIT_INDEX);
  else
    page = seq_page(c, b, by_page.div((int)p), err);
  const int in = page >= 0 ? (int)p - by_page.div((int)p) * c.page : 0, blocks = (unsigned)c.page / kCacheBlock;
  const int64_t at = page * c.page_stride + ((int64_t)in << log_d);
  const int64_t at_s = page * c.n_kv * blocks + (unsigned)in / kCacheBlock;
  for (int x0 = e0 + lane * kVec; x0 < e1; x0 += kStep * kBatch) {
    uint32_t wk[kBatch][kVec / 4], wv[kBatch][kVec / 4];
    float sk[kBatch], sv[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int x = x0 + u * kStep, h = x >> log_d;
      sk[u] = sv[u] = 0.f;
#pragma unroll
      for (int e = 0; e < kVec / 4; ++e) wk[u][e] = wv[u][e] = 0;
      if (x < e1 && page >= 0) {
        const int64_t src = at + ((int64_t)h * c.page << log_d) + (x - (h << log_d));
#pragma unroll
        for (int e = 0; e < kVec / 4; ++e) {
          wk[u][e] = __ldg(reinterpret_cast<const uint32_t*>(c.K + src) + e);
          wv[u][e] = __ldg(reinterpret_cast<const uint32_t*>(c.V + src) + e);
        }
        sk[u] = __ldg(c.ks + at_s + h * blocks);
        sv[u] = __ldg(c.vs + at_s + h * blocks);
      }
    }
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int x = x0 + u * kStep;
      if (x >= e1) break;
      float k[8], v[8];
#pragma unroll
      for (int e = 0; e < kVec / 4; ++e) {
        decode4<FMT>(wk[u][e], k + 4 * e);
        decode4<FMT>(wv[u][e], v + 4 * e);
      }
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        k[e] = page >= 0 ? k[e] * sk[u] : 0.f;
        v[e] = page >= 0 ? v[e] * sv[u] : 0.f;
      }
      const int64_t dst = t * all + x;
      if constexpr (TYPE == CRVQ_F32) {
        *reinterpret_cast<float4*>(static_cast<float*>(K_out) + dst) = make_float4(k[0], k[1], k[2], k[3]);
        *reinterpret_cast<float4*>(static_cast<float*>(V_out) + dst) = make_float4(v[0], v[1], v[2], v[3]);
      } else {
        store8(K_out, dst, TYPE, true, k);
        store8(V_out, dst, TYPE, true, v);
      }
    }
  }
}

bool vec_ok(const HeadsView& h) {
  const int64_t per = 16 / (int64_t)type_bytes(h.type);
  return ((uintptr_t)h.data & 15u) == 0 && h.ld_tok % per == 0 && h.ld_head % per == 0;
}

template <int FMT>
crvq_status launch_append(const AppendArgs& a, int D, int64_t grid, cudaStream_t stream) {
  const dim3 g((unsigned)grid), t((unsigned)D);
  if (D == 64)
    CRVQ_CUDA(launch_pdl(append_kernel<64, FMT>, g, t, 0, stream, a));
  else if (D == 128)
    CRVQ_CUDA(launch_pdl(append_kernel<128, FMT>, g, t, 0, stream, a));
  else
    CRVQ_CUDA(launch_pdl(append_kernel<256, FMT>, g, t, 0, stream, a));
  CRVQ_LAUNCHED();
  return CRVQ_OK;
}

crvq_status append(const crvq_kv_cache* cache, const crvq_heads* k, const crvq_heads* v,
                   int64_t n_tok, const int32_t* new_off, const crvq_rotary* rot,
                   const crvq_heads* q, const crvq_heads* q_out, cudaStream_t stream) {
  AppendArgs a{};
  CRVQ_TRY(make_cache(cache, &a.c));
  const int D = cache->head_dim;
  CRVQ_TRY(make_rows(new_off, n_tok, a.c.n_seq, &a.rows));
  CRVQ_TRY(make_heads(k, "k", D, n_tok, &a.k));
  CRVQ_TRY(make_heads(v, "v", D, n_tok, &a.v));
  CRVQ_CHECK_ARG(a.k.heads == a.c.n_kv && a.v.heads == a.c.n_kv, "k and v must have n_kv = %d heads", a.c.n_kv);
  CRVQ_CHECK_ARG((q == nullptr) == (q_out == nullptr), "q and q_out: give both or neither");
  a.interleaved = rot && rot->interleaved;
  if (rot) {
    CRVQ_CHECK_ARG(rot->cos && rot->sin, "rot: cos or sin is NULL");
    CRVQ_CHECK_ARG(rot->half >= 1 && rot->half <= D / 2, "rot: half must be in [1, head_dim / 2]");
    CRVQ_CHECK_ARG(rot->n_pos >= 1 && rot->ld >= rot->half, "rot: need n_pos >= 1 and ld >= half");
    CRVQ_TRY(check_dev({{rot->cos, "rot: cos"}, {rot->sin, "rot: sin"}, {rot->positions, "rot: positions"}}));
    a.cos = rot->cos;
    a.sin = rot->sin;
    a.positions = rot->positions;
    a.n_pos = rot->n_pos;
    a.ld_rot = rot->ld;
    a.half = rot->half;
    a.vec_rot = (((uintptr_t)rot->cos | (uintptr_t)rot->sin) & 15u) == 0 && rot->ld % 4 == 0;
  }
  a.pair_regs = a.interleaved || a.half == 0 || 2 * a.half == D;  // (else a partner is another thread's)
  int64_t n_rows = 0;
  if (q) {
    CRVQ_TRY(make_heads(q, "q", D, n_tok, &a.q));
    CRVQ_TRY(make_heads(q_out, "q_out", D, n_tok, &a.qo));
    CRVQ_CHECK_ARG(a.q.heads == a.qo.heads && a.q.type == a.qo.type, "q and q_out differ in heads or type");
    a.vec_q = vec_ok(a.q);
    a.vec_qo = vec_ok(a.qo);
    n_rows = n_tok * a.q.heads;
    a.by_heads = Divisor(a.q.heads);
  }
  a.vec_k = vec_ok(a.k);
  a.vec_v = vec_ok(a.v);
  if (n_tok == 0) return CRVQ_OK;
  // blocks that n tokens can touch: ceil((n - 1) / 16) + 1
  a.per_seq = (a.rows.per + 14) / kCacheBlock + 1;
  a.slots = new_off ? n_tok / kCacheBlock + 2 * (int64_t)a.c.n_seq : (int64_t)a.c.n_seq * a.per_seq;
  const int64_t n_append = a.slots * a.c.n_kv * 2, grid = n_append + ceil_div(n_rows, 16);
  if (grid >= (int64_t)1 << 31 || n_rows >= (int64_t)1 << 31)
    return fail(CRVQ_ERR_UNSUPPORTED, "too many new tokens in one call");
  a.n_append = (int)n_append;
  a.n_rows = (int)n_rows;
  a.by_kv = Divisor(a.c.n_kv);
  a.by_page = Divisor(a.c.page);
  if (!new_off) {
    a.by_per = Divisor(a.rows.per);
    a.by_slots = Divisor(a.per_seq);
  }
  CRVQ_TRY(device_error_word(&a.err));
  ProfScope ps("cache_append", stream, (double)n_tok * D * (2.0 * a.c.n_kv + (q ? a.q.heads : 0)));
  return cache->format == CRVQ_KV_INT8 ? launch_append<CRVQ_KV_INT8>(a, D, grid, stream)
                                       : launch_append<CRVQ_KV_E4M3>(a, D, grid, stream);
}

template <int FMT>
crvq_status launch_read(const CacheView& c, int D, const int32_t* start, const int32_t* off, int64_t n_tok,
                        int type, void* K_out, void* V_out, cudaStream_t stream) {
  unsigned* err = nullptr;
  CRVQ_TRY(device_error_word(&err));
  const int64_t parts = ceil_div((int64_t)c.n_kv * D, kReadCodes), grid = ceil_div(n_tok * parts, 8);
  if (8 * grid >= (int64_t)1 << 31) return fail(CRVQ_ERR_UNSUPPORTED, "too many tokens in one call");
  ProfScope ps("cache_read", stream, (double)n_tok * c.n_kv * D * 2 * (1 + type_bytes(type)));
  const dim3 g((unsigned)grid), t(256);
  const Divisor by_parts(parts), by_page(c.page);
  const int log_d = D == 64 ? 6 : D == 128 ? 7 : 8;
  if (type == CRVQ_F32)
    CRVQ_CUDA(launch_pdl(read_kernel<FMT, CRVQ_F32>, g, t, 0, stream, c, log_d, by_parts, by_page, start, off, n_tok, K_out, V_out, err));
  else if (type == CRVQ_BF16)
    CRVQ_CUDA(launch_pdl(read_kernel<FMT, CRVQ_BF16>, g, t, 0, stream, c, log_d, by_parts, by_page, start, off, n_tok, K_out, V_out, err));
  else
    CRVQ_CUDA(launch_pdl(read_kernel<FMT, CRVQ_F16>, g, t, 0, stream, c, log_d, by_parts, by_page, start, off, n_tok, K_out, V_out, err));
  CRVQ_LAUNCHED();
  return CRVQ_OK;
}

crvq_status read(const crvq_kv_cache* cache, const int32_t* start, const int32_t* off, int64_t n_tok,
                 int32_t type, void* K_out, void* V_out, cudaStream_t stream) {
  CacheView c;
  CRVQ_TRY(make_cache(cache, &c));
  CRVQ_CHECK_ARG(n_tok >= 0 && n_tok < (int64_t)1 << 31, "n_tok must be in [0, 2^31)");
  CRVQ_CHECK_ARG(type >= CRVQ_F32 && type <= CRVQ_F16, "unknown type %d", type);
  if (n_tok == 0) return CRVQ_OK;
  CRVQ_CHECK_ARG(start && off && K_out && V_out, "start, off, K_out and V_out must not be NULL");
  CRVQ_CHECK_ARG((((uintptr_t)K_out | (uintptr_t)V_out) & 15u) == 0, "K_out and V_out must be 16-byte aligned");
  CRVQ_TRY(check_dev({{start, "start"}, {off, "off"}, {K_out, "K_out"}, {V_out, "V_out"}}));
  const int D = cache->head_dim;
  return cache->format == CRVQ_KV_INT8
             ? launch_read<CRVQ_KV_INT8>(c, D, start, off, n_tok, type, K_out, V_out, stream)
             : launch_read<CRVQ_KV_E4M3>(c, D, start, off, n_tok, type, K_out, V_out, stream);
}

}  // namespace

crvq_status make_cache(const crvq_kv_cache* c, CacheView* out) {
  CRVQ_CHECK_ARG(c != nullptr, "cache is NULL");
  CRVQ_CHECK_ARG(c->K && c->V && c->k_scale && c->v_scale && c->pages && c->lens, "cache: an array is NULL");
  CRVQ_CHECK_ARG(c->n_seq >= 1 && c->max_pages >= 1 && c->n_pages >= 1 && c->n_kv >= 1,
                 "cache: need n_seq, max_pages, n_pages, n_kv >= 1");
  CRVQ_CHECK_ARG(c->page >= kCacheBlock && c->page % kCacheBlock == 0, "cache: page must be a multiple of 16");
  CRVQ_CHECK_ARG(c->format == CRVQ_KV_INT8 || c->format == CRVQ_KV_E4M3, "cache: unknown format %d", c->format);
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256)
    return fail(CRVQ_ERR_UNSUPPORTED, "head_dim %d: 64, 128 and 256 are implemented", c->head_dim);
  CRVQ_CHECK_ARG((((uintptr_t)c->K | (uintptr_t)c->V) & 15u) == 0, "cache: K and V must be 16-byte aligned");
  CRVQ_CHECK_ARG(c->page_stride % 16 == 0 &&
                     c->page_stride >= (int64_t)c->n_kv * c->page * c->head_dim,
                 "cache: page_stride must be a multiple of 16 and hold n_kv * page * head_dim codes");
  CRVQ_CHECK_ARG(c->ld_pages >= c->max_pages, "cache: ld_pages < max_pages");
  CRVQ_CHECK_ARG((int64_t)c->max_pages * c->page < (int64_t)1 << 31, "cache: max_pages * page must be below 2^31");
  CRVQ_TRY(check_dev({{c->K, "cache: K"}, {c->V, "cache: V"}, {c->k_scale, "cache: k_scale"},
                      {c->v_scale, "cache: v_scale"}, {c->pages, "cache: pages"}, {c->lens, "cache: lens"}}));
  *out = CacheView{static_cast<uint8_t*>(c->K), static_cast<uint8_t*>(c->V), c->k_scale, c->v_scale,
                   c->pages, c->lens, c->n_pages, c->page_stride, c->ld_pages, c->n_seq, c->max_pages,
                   c->page, c->n_kv};
  return CRVQ_OK;
}

crvq_status make_heads(const crvq_heads* h, const char* name, int head_dim, int64_t n_tok, HeadsView* out) {
  CRVQ_CHECK_ARG(h != nullptr && (h->data != nullptr || n_tok == 0), "%s is NULL", name);
  CRVQ_CHECK_ARG(h->heads >= 1, "%s: heads must be >= 1", name);
  CRVQ_CHECK_ARG(h->type >= CRVQ_F32 && h->type <= CRVQ_F16, "%s: unknown type %d", name, h->type);
  CRVQ_CHECK_ARG(((uintptr_t)h->data % type_bytes(h->type)) == 0, "%s is not aligned to its type", name);
  if (n_tok > 0) CRVQ_TRY(check_dev({{h->data, name}}));
  *out = HeadsView{h->data, h->ld_tok, h->ld_head, h->heads, h->type};
  return CRVQ_OK;
}

crvq_status make_rows(const int32_t* off, int64_t n_tok, int n_seq, RowsView* out) {
  CRVQ_CHECK_ARG(n_tok >= 0 && n_tok < (int64_t)1 << 31, "n_tok must be in [0, 2^31)");
  CRVQ_CHECK_ARG(off != nullptr || n_tok % n_seq == 0,
                 "without row offsets n_tok (%lld) must be a multiple of n_seq (%d)", (long long)n_tok, n_seq);
  CRVQ_TRY(check_dev({{off, "row offsets"}}));
  *out = RowsView{off, n_tok, off ? 0 : (int)(n_tok / n_seq)};
  return CRVQ_OK;
}

}  // namespace crvq

extern "C" {

using namespace crvq;

crvq_status crvq_cache_append(const crvq_kv_cache* cache, const crvq_heads* k, const crvq_heads* v,
                              int64_t n_tok, const int32_t* new_off, const crvq_rotary* rot,
                              const crvq_heads* q, const crvq_heads* q_out, crvq_stream_t stream) {
  CRVQ_ENTRY({ return append(cache, k, v, n_tok, new_off, rot, q, q_out, (cudaStream_t)stream); })
}

crvq_status crvq_cache_read(const crvq_kv_cache* cache, const int32_t* start, const int32_t* off,
                            int64_t n_tok, int32_t type, void* K_out, void* V_out,
                            crvq_stream_t stream) {
  CRVQ_ENTRY({ return read(cache, start, off, n_tok, type, K_out, V_out, (cudaStream_t)stream); })
}

}  // extern "C"
