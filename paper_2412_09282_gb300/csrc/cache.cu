// The paged 8-bit key/value cache: appending rotated keys and values, and reading ranges back.
//
// Append. Per touched block (16 tokens of one kv head, keys or values) with old tokens c_i at scale
// s0 and new values x_i:
//   s = max(max_i |x_i| * (1 / Q), s0 if there are old tokens),  Q = 127 or 448,
//   c_i <- round(c_i * (s0 / s)) for the old,  c_i = round(x_i / s) for the new,
// with x the rotated key (a cos - b sin, b cos + a sin) or the value. One CTA owns one block of one
// head's keys or values, so a scale is found and every code written by the same threads: no atomics,
// no second pass over the inputs. A thread holds 16 channels of one token in registers, eight at i and
// eight at i + D/2 (or 2 x 8 neighbours for interleaved pairs), so a rotation pair is one thread's.
// The grid has a slot for every block that could be touched (the lengths are on the device); the ones
// that are not leave at once. Each product, difference and quotient is rounded to fp32 by itself (no
// fused multiply-add): codes do not depend on how the compiler contracts.
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
  bool pair_regs;    // a rotation pair lies within a thread's 16 channels
  bool vec_k, vec_v, vec_q, vec_qo, vec_rot;
  int64_t slots;     // block slots of all sequences
  int per_seq;       // slots per sequence (rows.off null)
  int64_t n_append;  // CTAs of the append; the rest rotate queries
  unsigned* err;
};

__device__ __forceinline__ bool finite(float x) { return fabsf(x) <= 3.402823466e38f; }

// The 16 channels of a thread, c the thread's index in its row (0 .. D/16 - 1): channel of element e.
template <int D>
__device__ __forceinline__ int channel(int c, int e, bool split) {
  return split ? (e < 8 ? 8 * c + e : D / 2 + 8 * c + e - 8) : 16 * c + e;
}

__device__ __forceinline__ void turn(float& u, float& w, float c, float s) {
  const float x = u;
  u = __fsub_rn(__fmul_rn(u, c), __fmul_rn(w, s));
  w = __fadd_rn(__fmul_rn(w, c), __fmul_rn(x, s));
}

// x: this thread's 16 channels of (token row t, head h), rotated by the angle row `pos` (-1: not).
template <int D>
__device__ __forceinline__ void load_rotated(const AppendArgs& a, const HeadsView& src, bool vec,
                                             int64_t t, int h, int c, bool split, int64_t pos,
                                             float x[16]) {
  const int64_t row = t * src.ld_tok + h * src.ld_head;
  load8(src.data, row + channel<D>(c, 0, split), src.type, vec, x);
  load8(src.data, row + channel<D>(c, 8, split), src.type, vec, x + 8);
  if (pos < 0) return;
  const float* cs = a.cos + pos * a.ld_rot;
  const float* sn = a.sin + pos * a.ld_rot;
  if (a.pair_regs) {
    float cv[8], sv[8];
    const int i0 = 8 * c;  // both forms: the thread's eight pairs are 8c .. 8c + 7
    if (a.vec_rot && i0 + 8 <= a.half) {
      load8(cs, i0, CRVQ_F32, true, cv);
      load8(sn, i0, CRVQ_F32, true, sv);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const bool in = i0 + j < a.half;
        cv[j] = in ? __ldg(cs + i0 + j) : 1.f;
        sv[j] = in ? __ldg(sn + i0 + j) : 0.f;
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (i0 + j >= a.half) continue;  // (an unrotated channel keeps its bits, infinities too)
      if (split)
        turn(x[j], x[j + 8], cv[j], sv[j]);
      else
        turn(x[2 * j], x[2 * j + 1], cv[j], sv[j]);
    }
  } else {
    // pairs (i, i + half) with half < D/2: the partner is another thread's, read again
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int ch = channel<D>(c, e, split);
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

template <int FMT>
__device__ __forceinline__ uint32_t encode4(const float v[4]) {
  if constexpr (FMT == CRVQ_KV_INT8) {
    uint32_t w = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int q = (int)rintf(fminf(fmaxf(v[j], -127.f), 127.f));
      w |= (uint32_t)(q & 255) << (8 * j);
    }
    return w;
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

template <int D, int FMT>
__global__ void __launch_bounds__(D) append_kernel(const __grid_constant__ AppendArgs a) {
  constexpr int kRow = D / 16;  // threads per token
  __shared__ int32_t off_s[kOffShared + 1];
  __shared__ uint32_t top_s[D / 32];
  pdl_trigger();
  pdl_wait();
  const int tid = threadIdx.x;
  const int32_t* off = a.rows.off;
  const CacheView& c = a.c;
  if (off && c.n_seq <= kOffShared) {
    for (int i = tid; i <= c.n_seq; i += D) off_s[i] = __ldg(a.rows.off + i);
    __syncthreads();
    off = off_s;
  }
  const int col = tid % kRow, r = tid / kRow;
  const bool split = !a.interleaved;
  int64_t id = blockIdx.x;
  if (id >= a.n_append) {  // queries: 16 (token, head) rows per CTA
    const int64_t at = (id - a.n_append) * 16 + r;
    bool live = at < a.rows.n_tok * a.q.heads;
    const int64_t t = at / a.q.heads;
    const int h = (int)(at - t * a.q.heads);
    int p = 0;
    if (live && a.half && !a.positions) {
      const int b = off ? last_not_above(c.n_seq, t, [&](int i) { return (int64_t)off[i]; })
                        : (int)(t / a.rows.per);
      int64_t first;
      int n;
      seq_rows(a.rows, b, &first, &n, a.err);
      live = t >= first && t < first + n;  // (rows outside every sequence stay unwritten)
      p = seq_len(c, b, a.err) - n + (int)(t - first);
    }
    float x[16];
    if (live) load_rotated<D>(a, a.q, a.vec_q, t, h, col, split, rot_row(a, t, p), x);
    const int64_t row = t * a.qo.ld_tok + h * a.qo.ld_head;
    __syncwarp();  // in place: a warp's rows are read whole before they are written
    if (live) {
      store8(a.qo.data, row + channel<D>(col, 0, split), a.qo.type, a.vec_qo, x);
      store8(a.qo.data, row + channel<D>(col, 8, split), a.qo.type, a.vec_qo, x + 8);
    }
    return;
  }
  // which block: sequence b, its j-th touched one; which head, keys or values
  const bool values = id & 1;
  id >>= 1;
  const int h = (int)(id % c.n_kv);
  const int64_t slot = id / c.n_kv;
  int b, j;
  if (off) {
    // sequence i's slots begin at off[i] / 16 + 2 i: n tokens touch at most n / 16 + 2 blocks
    b = last_not_above(c.n_seq, slot, [&](int i) { return (int64_t)off[i] / kCacheBlock + 2 * i; });
    j = (int)(slot - off[b] / kCacheBlock - 2 * b);
  } else {
    b = (int)(slot / a.per_seq);
    j = (int)(slot - (int64_t)b * a.per_seq);
  }
  int64_t first;
  int n;
  seq_rows(a.rows, b, &first, &n, a.err);
  if (n == 0 || j < 0) return;
  const int len = seq_len(c, b, a.err);
  const int held = len - n;
  if (held < 0) {
    raise_error(a.err, ERRBIT_INDEX);
    return;
  }
  const int64_t p0 = ((int64_t)held / kCacheBlock + j) * kCacheBlock;
  if (p0 >= len) return;
  const int64_t page = seq_page(c, b, (int)(p0 / c.page), a.err);
  if (page < 0) return;
  const int in_page = (int)(p0 % c.page);
  uint8_t* codes = (values ? c.V : c.K) + page * c.page_stride + ((int64_t)h * c.page + in_page + r) * D;
  float* scale = (values ? c.vs : c.ks) + (page * c.n_kv + h) * (c.page / kCacheBlock) + in_page / kCacheBlock;
  const int p = (int)p0 + r;
  const bool is_old = p < held, is_new = !is_old && p < len;
  const float s0 = p0 < held ? *scale : 0.f;
  uint32_t w[4] = {0, 0, 0, 0};
  if (is_old) {
    const uint2 u0 = *reinterpret_cast<const uint2*>(codes + channel<D>(col, 0, split));
    const uint2 u1 = *reinterpret_cast<const uint2*>(codes + channel<D>(col, 8, split));
    w[0] = u0.x; w[1] = u0.y; w[2] = u1.x; w[3] = u1.y;
  }
  float x[16];
  uint32_t top = 0;
  if (is_new) {
    const int64_t t = first + (p - held);
    if (values)
      load_rotated<D>(a, a.v, a.vec_v, t, h, col, split, -1, x);
    else
      load_rotated<D>(a, a.k, a.vec_k, t, h, col, split, rot_row(a, t, p), x);
    bool bad = false;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      if (!finite(x[e])) {
        x[e] = 0.f;
        bad = true;
      }
      top = max(top, __float_as_uint(fabsf(x[e])));
    }
    if (bad) raise_error(a.err, ERRBIT_NUMERIC);
  }
  top = __reduce_max_sync(0xffffffffu, top);
  if ((tid & 31) == 0) top_s[tid >> 5] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < D / 32; ++i) top = max(top, top_s[i]);
  constexpr float kInv = (float)(1.0 / (FMT == CRVQ_KV_INT8 ? 127.0 : 448.0));
  const float s = fmaxf(__fmul_rn(__uint_as_float(top), kInv), s0);
  const float ratio = s > 0.f ? __fdiv_rn(s0, s) : 0.f;
  if (is_new) {
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = s > 0.f ? __fdiv_rn(x[e], s) : 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = encode4<FMT>(x + 4 * e);
  } else if (is_old && ratio != 1.f) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float v[4];
      decode4<FMT>(w[e], v);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = __fmul_rn(v[i], ratio);
      w[e] = encode4<FMT>(v);
    }
  }
  if (is_new || (is_old && ratio != 1.f)) {
    *reinterpret_cast<uint2*>(codes + channel<D>(col, 0, split)) = make_uint2(w[0], w[1]);
    *reinterpret_cast<uint2*>(codes + channel<D>(col, 8, split)) = make_uint2(w[2], w[3]);
  }
  if (tid == 0) *scale = s;  // (s0 was read by every thread before the barrier)
}

// A thread turns 16 / sizeof(type) codes of K and of V into one 16-byte store each.
template <int FMT, int TYPE>
__global__ void __launch_bounds__(256)
read_kernel(const __grid_constant__ CacheView c, int D, const int32_t* __restrict__ start,
            const int32_t* __restrict__ off_g, int64_t n_tok, void* K_out, void* V_out, unsigned* err) {
  constexpr int kVec = TYPE == CRVQ_F32 ? 4 : 8;
  __shared__ int32_t off_s[kOffShared + 1];
  pdl_trigger();
  pdl_wait();
  const int32_t* off = off_g;
  if (c.n_seq <= kOffShared) {
    for (int i = threadIdx.x; i <= c.n_seq; i += 256) off_s[i] = __ldg(off_g + i);
    __syncthreads();
    off = off_s;
  }
  const int per_head = D / kVec;
  const int64_t per_tok = (int64_t)c.n_kv * per_head;
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= n_tok * per_tok) return;
  const int64_t t = at / per_tok;
  const int rest = (int)(at - t * per_tok), h = rest / per_head, ch = (rest - h * per_head) * kVec;
  const int b = last_not_above(c.n_seq, t, [&](int i) { return (int64_t)off[i]; });
  const int64_t i = t - off[b];
  const int64_t p = (int64_t)__ldg(start + b) + i;
  const int len = seq_len(c, b, err);
  int64_t page = -1;
  if (i < 0 || t >= off[b + 1] || p < 0 || p >= len)
    raise_error(err, ERRBIT_INDEX);
  else
    page = seq_page(c, b, (int)(p / c.page), err);
  float k[8], v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) k[e] = v[e] = 0.f;
  if (page >= 0) {
    const int in = (int)(p % c.page);
    const int64_t at_c = page * c.page_stride + ((int64_t)h * c.page + in) * D + ch;
    const int64_t at_s = (page * c.n_kv + h) * (c.page / kCacheBlock) + in / kCacheBlock;
    const float sk = c.ks[at_s], sv = c.vs[at_s];
#pragma unroll
    for (int e = 0; e < kVec / 4; ++e) {
      decode4<FMT>(reinterpret_cast<const uint32_t*>(c.K + at_c)[e], k + 4 * e);
      decode4<FMT>(reinterpret_cast<const uint32_t*>(c.V + at_c)[e], v + 4 * e);
    }
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      k[e] *= sk;
      v[e] *= sv;
    }
  }
  if constexpr (TYPE == CRVQ_F32) {
    static_cast<float4*>(K_out)[at] = make_float4(k[0], k[1], k[2], k[3]);
    static_cast<float4*>(V_out)[at] = make_float4(v[0], v[1], v[2], v[3]);
  } else {
    store8(K_out, at * 8, TYPE, true, k);
    store8(V_out, at * 8, TYPE, true, v);
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
  a.pair_regs = a.interleaved || a.half == 0 || 2 * a.half == D;
  int64_t n_q = 0;
  if (q) {
    CRVQ_TRY(make_heads(q, "q", D, n_tok, &a.q));
    CRVQ_TRY(make_heads(q_out, "q_out", D, n_tok, &a.qo));
    CRVQ_CHECK_ARG(a.q.heads == a.qo.heads && a.q.type == a.qo.type, "q and q_out differ in heads or type");
    a.vec_q = vec_ok(a.q);
    a.vec_qo = vec_ok(a.qo);
    n_q = ceil_div(n_tok * a.q.heads, 16);
  }
  a.vec_k = vec_ok(a.k);
  a.vec_v = vec_ok(a.v);
  if (n_tok == 0) return CRVQ_OK;
  // blocks that n tokens can touch: ceil((n - 1) / 16) + 1
  a.per_seq = (a.rows.per + 14) / kCacheBlock + 1;
  a.slots = new_off ? n_tok / kCacheBlock + 2 * (int64_t)a.c.n_seq : (int64_t)a.c.n_seq * a.per_seq;
  a.n_append = a.slots * a.c.n_kv * 2;
  const int64_t grid = a.n_append + n_q;
  if (grid >= (int64_t)1 << 31) return fail(CRVQ_ERR_UNSUPPORTED, "too many new tokens in one call");
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
  const int64_t threads = n_tok * c.n_kv * (D / (type == CRVQ_F32 ? 4 : 8));
  const int64_t grid = ceil_div(threads, 256);
  if (grid >= (int64_t)1 << 31) return fail(CRVQ_ERR_UNSUPPORTED, "too many tokens in one call");
  ProfScope ps("cache_read", stream, (double)n_tok * c.n_kv * D * 2 * (1 + type_bytes(type)));
  const dim3 g((unsigned)grid), t(256);
  if (type == CRVQ_F32)
    CRVQ_CUDA(launch_pdl(read_kernel<FMT, CRVQ_F32>, g, t, 0, stream, c, D, start, off, n_tok, K_out, V_out, err));
  else if (type == CRVQ_BF16)
    CRVQ_CUDA(launch_pdl(read_kernel<FMT, CRVQ_BF16>, g, t, 0, stream, c, D, start, off, n_tok, K_out, V_out, err));
  else
    CRVQ_CUDA(launch_pdl(read_kernel<FMT, CRVQ_F16>, g, t, 0, stream, c, D, start, off, n_tok, K_out, V_out, err));
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
