// The paged 8-bit key/value cache as kernels see it, element types, and the sequences of ragged
// token rows (see crvq_kv_cache in crvq.h).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "common.cuh"

namespace crvq {

constexpr int kCacheBlock = 16;  // tokens per scale

struct CacheView {
  uint8_t* K;
  uint8_t* V;
  float* ks;
  float* vs;
  const int32_t* pages;
  const int32_t* lens;
  int64_t n_pages, page_stride, ld_pages;
  int n_seq, max_pages, page, n_kv;
};

struct HeadsView {
  void* data;
  int64_t ld_tok, ld_head;
  int heads, type;
};

// The new token rows of every sequence: off[b] .. off[b + 1), or per each (off null).
struct RowsView {
  const int32_t* off;
  int64_t n_tok;
  int per;
};

// Division of n in [0, 2^31) by a divisor d in [1, 2^31) known before the launch, as a product: with
// l = ceil(log2 d) and mul = ceil(2^(31 + l) / d), floor(n mul / 2^(31 + l)) is exact (Granlund & Montgomery
// 1994, for 31-bit n: mul then fits 32 bits).
struct Divisor {
  uint32_t d = 1, mul = 0, shift = 0;
  Divisor() = default;
  explicit Divisor(int64_t div) : d((uint32_t)div) {
    int l = 0;
    while (((int64_t)1 << l) < div) ++l;
    if (l == 0) return;  // (d = 1: mul would be 2^31 with a shift of -1)
    mul = (uint32_t)((((uint64_t)1 << (31 + l)) + d - 1) / d);
    shift = (uint32_t)(l - 1);
  }
  __device__ __forceinline__ int div(int n) const { return d == 1 ? n : (int)(__umulhi((uint32_t)n, mul) >> shift); }
};

// Checks of the arguments (cache.cu): each sets the last error on refusal.
crvq_status make_cache(const crvq_kv_cache* c, CacheView* out);
crvq_status make_heads(const crvq_heads* h, const char* name, int head_dim, int64_t n_tok,
                       HeadsView* out);
crvq_status make_rows(const int32_t* off, int64_t n_tok, int n_seq, RowsView* out);
// (weights.cu)
crvq_status check_sums(const crvq_token_sums* s, const char* name, int n_seq, int n_kv);
bool sums_overlap(const crvq_token_sums* x, const crvq_token_sums* y, int n_seq, int n_kv);  // from the first to the last element

inline size_t type_bytes(int type) { return type == CRVQ_F32 ? 4 : 2; }

// Rows of sequence b, [first, first + n); n = 0 (reported) for offsets that are not in order.
__device__ __forceinline__ void seq_rows(const RowsView& r, int b, int64_t* first, int* n,
                                         unsigned* err) {
  if (!r.off) {
    *first = (int64_t)b * r.per;
    *n = r.per;
    return;
  }
  const int a = __ldg(r.off + b), e = __ldg(r.off + b + 1);
  *first = a;
  *n = e - a;
  if (a < 0 || e < a || e > r.n_tok) {
    raise_error(err, ERRBIT_INDEX);
    *n = 0;
  }
}

// Tokens of sequence b: its length, 0 (reported) when it is out of range.
__device__ __forceinline__ int seq_len(const CacheView& c, int b, unsigned* err) {
  const int len = __ldg(c.lens + b);
  if (len < 0 || len > (int64_t)c.max_pages * c.page) {
    raise_error(err, ERRBIT_INDEX);
    return 0;
  }
  return len;
}

// Page of table entry i of sequence b (i < max_pages), -1 (reported) when it is out of range.
__device__ __forceinline__ int64_t seq_page(const CacheView& c, int b, int i, unsigned* err) {
  const int32_t p = __ldg(c.pages + b * c.ld_pages + i);
  if (p < 0 || p >= c.n_pages) {
    raise_error(err, ERRBIT_INDEX);
    return -1;
  }
  return p;
}

// The last index b of [0, n) with key(b) <= v, key(0) <= v and key non-decreasing (for other keys some b).
template <class Key>
__device__ __forceinline__ int last_not_above(int n, int64_t v, Key key) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (key(mid) <= v)
      lo = mid;
    else
      hi = mid - 1;
  }
  return lo;
}

// x / s rounded once, for inv = 1 / s rounded once: the first correction brings the product within one unit in the
// last place, and then the remainder is exact and the second one rounds correctly (Markstein 1990). For s
// in (2^-80, 2^80) no step that a code depends on leaves the normal numbers.
__device__ __forceinline__ float quotient(float x, float s, float inv) {
  float q = __fmul_rn(x, inv);
  q = __fmaf_rn(__fmaf_rn(-q, s, x), inv, q);
  return __fmaf_rn(__fmaf_rn(-q, s, x), inv, q);
}
__device__ __forceinline__ bool plain_divisor(float s) { return s > 0x1p-80f && s < 0x1p80f; }

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

__device__ __forceinline__ float load_elem(const void* p, int64_t i, int type) {
  if (type == CRVQ_F32) return static_cast<const float*>(p)[i];
  const uint16_t u = static_cast<const uint16_t*>(p)[i];
  return type == CRVQ_BF16 ? __bfloat162float(__ushort_as_bfloat16(u)) : __half2float(__ushort_as_half(u));
}

__device__ __forceinline__ void store_elem(void* p, int64_t i, int type, float v) {
  if (type == CRVQ_F32)
    static_cast<float*>(p)[i] = v;
  else if (type == CRVQ_BF16)
    static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v);
  else
    static_cast<__half*>(p)[i] = __float2half_rn(v);
}

// Eight consecutive elements (vec: 16-byte aligned, and the type's eight elements contiguous).
__device__ __forceinline__ void load8(const void* p, int64_t i, int type, bool vec, float v[8]) {
  if (!vec) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = load_elem(p, i + j, type);
  } else if (type == CRVQ_F32) {
    const float4* q = reinterpret_cast<const float4*>(static_cast<const float*>(p) + i);
    const float4 a = q[0], b = q[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  } else {
    const uint4 u = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + i);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (type == CRVQ_BF16) {
        v[2 * j] = __uint_as_float(w[j] << 16);
        v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
      } else {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[j]));
        v[2 * j] = f.x;
        v[2 * j + 1] = f.y;
      }
    }
  }
}

__device__ __forceinline__ uint32_t pack2(float a, float b, int type) {
  if (type == CRVQ_BF16) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

__device__ __forceinline__ void store8(void* p, int64_t i, int type, bool vec, const float v[8]) {
  if (!vec) {
#pragma unroll
    for (int j = 0; j < 8; ++j) store_elem(p, i + j, type, v[j]);
  } else if (type == CRVQ_F32) {
    float4* q = reinterpret_cast<float4*>(static_cast<float*>(p) + i);
    q[0] = make_float4(v[0], v[1], v[2], v[3]);
    q[1] = make_float4(v[4], v[5], v[6], v[7]);
  } else {
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p) + i) =
        make_uint4(pack2(v[0], v[1], type), pack2(v[2], v[3], type), pack2(v[4], v[5], type),
                   pack2(v[6], v[7], type));
  }
}

}  // namespace crvq
