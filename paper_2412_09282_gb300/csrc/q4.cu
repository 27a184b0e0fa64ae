// Matrices with 4-bit weights and a scale per group of 32, 64 or 128 inputs: quantizing by rounding,
// and the product with 1 to 32 inputs,
//   y_b[i] = sum_groups s_ig sum_{j in group} (code_ij - zero_ig) x_bj.
//
// Product. code - zero is an integer of at most 15: exact in bf16 and fp16, so the inner sums run on
// mma.sync.m16n8k16 with the weights as A (16 rows) and up to 8 NT inputs as B, in the inputs' own type;
// fp32 inputs are cut into three bf16 pieces of 8 bits each (their sum is the input). A group's sum is
// scaled once, in fp32. The order of the inner index is free: a lane holds 32 (16, 8) consecutive codes
// of a row, one 16- (8-, 4-) byte load, and pairs nibbles e and e + 4 of a word, which three shifts and
// four masks turn into 16-bit floats (1024 + code, or 128 + code, less 1024 + zero or 128 + zero); the
// lane's piece of the inputs is loaded in the same order.
//   A CTA owns 16 RT rows; its eight warps take every eighth 128 inputs, and their sums meet in shared
// memory in a fixed order. One launch, no scratch.
#include "cache.cuh"

#include "kernels.h"

namespace crvq {

namespace {

constexpr int kQWarps = 8;
constexpr int kQThreads = 32 * kQWarps;
constexpr int kStep = 128;  // inputs per warp step
constexpr int kMaxInputs = 32;

struct Q4View {
  uint8_t* codes;
  __nv_bfloat16* scales;
  uint8_t* zeros;
  int64_t M, N, ld_codes, ld_scales;
};

struct MatvecQ4 {
  Q4View m;
  const void* X;
  int64_t ldx;
  void* Y;
  int64_t ldy;
  int b, type;
  bool vec_w, vec_x;
};

template <bool BF16>
__device__ __forceinline__ void mma16(float d[4], const uint32_t a[4], uint32_t b0, uint32_t b1) {
  if constexpr (BF16)
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
        "{%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
        "{%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Codes e and e + 4 of a word, less the zero point (zc: 128 + zero in bf16 or 1024 + zero in fp16, twice).
template <bool BF16>
__device__ __forceinline__ uint32_t codes_pair(uint32_t w, int e, uint32_t zc) {
  const uint32_t u = ((w >> (4 * e)) & 0x000f000fu) | (BF16 ? 0x43004300u : 0x64006400u);
  if constexpr (BF16) {
    const __nv_bfloat162 v = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&u),
                                     *reinterpret_cast<const __nv_bfloat162*>(&zc));
    return *reinterpret_cast<const uint32_t*>(&v);
  } else {
    const __half2 v = __hsub2(*reinterpret_cast<const __half2*>(&u), *reinterpret_cast<const __half2*>(&zc));
    return *reinterpret_cast<const uint32_t*>(&v);
  }
}

// x = p[0] + p[1] + p[2] exactly, each the upper half of an fp32 (8 significant bits).
__device__ __forceinline__ void cut3(float x, uint32_t p[3]) {
  p[0] = __float_as_uint(x);
  const float r = fabsf(x) == INFINITY ? 0.f : x - __uint_as_float(p[0] & 0xffff0000u);
  p[1] = __float_as_uint(r);
  p[2] = __float_as_uint(r - __uint_as_float(p[1] & 0xffff0000u));
}

// The inputs k .. k + 7 of row `row` of X (null: zeros) as B operand pairs (0, 4), (1, 5), (2, 6), (3, 7).
template <int TYPE>
__device__ __forceinline__ void load_x(const MatvecQ4& a, int64_t row, bool live, int64_t k,
                                       uint32_t v[TYPE == CRVQ_F32 ? 3 : 1][4]) {
  if constexpr (TYPE == CRVQ_F32) {
    float x[8];
    const float* p = static_cast<const float*>(a.X) + row * a.ldx;
    if (live && k + 8 <= a.m.N) {
      load8(p, k, CRVQ_F32, a.vec_x, x);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = live && k + j < a.m.N ? p[k + j] : 0.f;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      uint32_t lo[3], hi[3];
      cut3(x[e], lo);
      cut3(x[e + 4], hi);
#pragma unroll
      for (int z = 0; z < 3; ++z) v[z][e] = __byte_perm(lo[z], hi[z], 0x7632);
    }
  } else {
    const uint16_t* p = static_cast<const uint16_t*>(a.X) + row * a.ldx;
    uint32_t w[4];
    if (live && a.vec_x && k + 8 <= a.m.N) {
      const uint4 u = *reinterpret_cast<const uint4*>(p + k);
      w[0] = u.x; w[1] = u.y; w[2] = u.z; w[3] = u.w;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t lo = live && k + 2 * j < a.m.N ? p[k + 2 * j] : 0;
        const uint32_t hi = live && k + 2 * j + 1 < a.m.N ? p[k + 2 * j + 1] : 0;
        w[j] = lo | hi << 16;
      }
    }
    v[0][0] = __byte_perm(w[0], w[2], 0x5410);
    v[0][1] = __byte_perm(w[0], w[2], 0x7632);
    v[0][2] = __byte_perm(w[1], w[3], 0x5410);
    v[0][3] = __byte_perm(w[1], w[3], 0x7632);
  }
}

// WORDS consecutive words of a row's codes from byte `at` on, zeros past the row's end.
template <int WORDS>
__device__ __forceinline__ void load_codes(const MatvecQ4& a, const uint8_t* row, int64_t at, uint32_t w[WORDS]) {
  const int64_t bytes = (a.m.N + 1) / 2;
  if (a.vec_w && at + 4 * WORDS <= bytes) {
    if constexpr (WORDS == 4) {
      const uint4 u = __ldg(reinterpret_cast<const uint4*>(row + at));
      w[0] = u.x; w[1] = u.y; w[2] = u.z; w[3] = u.w;
    } else if constexpr (WORDS == 2) {
      const uint2 u = __ldg(reinterpret_cast<const uint2*>(row + at));
      w[0] = u.x; w[1] = u.y;
    } else {
      w[0] = __ldg(reinterpret_cast<const uint32_t*>(row + at));
    }
  } else {
#pragma unroll
    for (int i = 0; i < WORDS; ++i) {
      w[i] = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (at + 4 * i + j < bytes) w[i] |= (uint32_t)__ldg(row + at + 4 * i + j) << (8 * j);
    }
  }
}

template <int TYPE, int GROUP, int NT, int RT>
__global__ void __launch_bounds__(kQThreads)
q4_matvec_kernel(const __grid_constant__ MatvecQ4 a) {
  constexpr bool BF16 = TYPE != CRVQ_F16;
  constexpr int kPieces = TYPE == CRVQ_F32 ? 3 : 1;
  constexpr int kSubs = kStep / GROUP, WORDS = GROUP / 32;
  constexpr int R = 16 * RT, COLS = 8 * NT;
  extern __shared__ __align__(16) float red[];  // [kQWarps][COLS][R]
  pdl_trigger();
  pdl_wait();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, gid = lane >> 2, tig = lane & 3;
  const int64_t r0 = (int64_t)blockIdx.x * R;
  const Q4View& m = a.m;
  const int64_t steps = (m.N + kStep - 1) / kStep, n_groups = (m.N + GROUP - 1) / GROUP;

  int64_t row[RT][2];
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int i = 0; i < 2; ++i) row[t][i] = min(r0 + 16 * t + gid + 8 * i, m.M - 1);

  float acc[RT][NT][4];
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[t][n][e] = 0.f;

  for (int64_t st = warp; st < steps; st += kQWarps) {
#pragma unroll
    for (int sub = 0; sub < kSubs; ++sub) {
      const int64_t g = min(st * kSubs + sub, n_groups - 1);
      const int64_t k = st * kStep + sub * GROUP + tig * (GROUP / 4);
      uint32_t w[RT][2][WORDS], zc[RT][2];
      float sc[RT][2];
#pragma unroll
      for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          load_codes<WORDS>(a, m.codes + row[t][i] * m.ld_codes, k / 2, w[t][i]);
          sc[t][i] = __bfloat162float(m.scales[row[t][i] * m.ld_scales + g]);
          const uint32_t z = m.zeros ? __ldg(m.zeros + row[t][i] * m.ld_scales + g) & 15u : 8u;
          // 128 + z in bf16, 1024 + z in fp16: the integer's low bits are the mantissa's
          zc[t][i] = ((BF16 ? 0x4300u : 0x6400u) + z) * 0x10001u;
        }
      float part[RT][NT][4];
#pragma unroll
      for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) part[t][n][e] = 0.f;
#pragma unroll
      for (int i = 0; i < WORDS; ++i) {
        uint32_t x[NT][kPieces][4];
#pragma unroll
        for (int n = 0; n < NT; ++n) load_x<TYPE>(a, 8 * n + gid, 8 * n + gid < a.b, k + 8 * i, x[n]);
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
          for (int e = 0; e < 4; e += 2) {
            uint32_t A[4];
            A[0] = codes_pair<BF16>(w[t][0][i], e, zc[t][0]);
            A[1] = codes_pair<BF16>(w[t][1][i], e, zc[t][1]);
            A[2] = codes_pair<BF16>(w[t][0][i], e + 1, zc[t][0]);
            A[3] = codes_pair<BF16>(w[t][1][i], e + 1, zc[t][1]);
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
              for (int z = 0; z < kPieces; ++z) mma16<BF16>(part[t][n], A, x[n][z][e], x[n][z][e + 1]);
          }
      }
#pragma unroll
      for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[t][n][e] = fmaf(sc[t][e >> 1], part[t][n][e], acc[t][n][e]);
    }
  }
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        red[((size_t)warp * COLS + 8 * n + 2 * tig + (e & 1)) * R + 16 * t + gid + 8 * (e >> 1)] = acc[t][n][e];
  __syncthreads();
  for (int e = tid; e < a.b * R; e += kQThreads) {
    const int col = e / R, r = e - col * R;
    if (r0 + r >= m.M) continue;
    float v = 0.f;
#pragma unroll
    for (int i = 0; i < kQWarps; ++i) v += red[((size_t)i * COLS + col) * R + r];
    store_elem(a.Y, col * a.ldy + r0 + r, TYPE, v);
  }
}

// A thread takes eight consecutive weights; the GROUP / 8 threads of a group find its range by shuffles.
struct QuantizeArgs {
  Q4View m;
  const void* W;
  int64_t ldw;
  int type;
  bool vec_w, vec_c, vec_h;
  float* W_hat;
  int64_t threads_row;  // threads per row, whole groups
  unsigned* err;
};

template <int GROUP>
__global__ void __launch_bounds__(256) q4_quantize_kernel(const __grid_constant__ QuantizeArgs a) {
  constexpr int kLanes = GROUP / 8;
  pdl_trigger();
  pdl_wait();
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = at / a.threads_row;
  const int64_t j0 = (at - row * a.threads_row) * 8, g = j0 / GROUP;
  const bool live = row < a.m.M;  // whole groups of lanes
  const int64_t N = a.m.N;
  const int n = live ? (int)max((int64_t)0, min((int64_t)8, N - j0)) : 0;
  float w[8];
  if (n == 8) {
    load8(a.W, row * a.ldw + j0, a.type, a.vec_w, w);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = e < n ? load_elem(a.W, row * a.ldw + j0 + e, a.type) : 0.f;
  }
  float lo = 0.f, hi = 0.f;
  bool bad = false;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if (!(fabsf(w[e]) <= 3.402823466e38f)) {
      w[e] = 0.f;
      bad = true;
    }
    lo = fminf(lo, w[e]);
    hi = fmaxf(hi, w[e]);
  }
  if (bad) raise_error(a.err, ERRBIT_NUMERIC);
#pragma unroll
  for (int d = kLanes / 2; d > 0; d >>= 1) {
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, d));
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, d));
  }
  constexpr float k7 = (float)(1.0 / 7.0), k15 = (float)(1.0 / 15.0);
  const __nv_bfloat16 s16 = __float2bfloat16_rn(a.m.zeros ? __fmul_rn(__fsub_rn(hi, lo), k15)
                                                          : __fmul_rn(fmaxf(hi, -lo), k7));
  const float s = __bfloat162float(s16);
  float z = 8.f;
  if (a.m.zeros) z = s > 0.f ? fminf(fmaxf(rintf(__fdiv_rn(-lo, s)), 0.f), 15.f) : 0.f;
  float v[8];
  uint32_t codes = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float q = s > 0.f ? fminf(fmaxf(rintf(__fdiv_rn(w[e], s)) + z, 0.f), 15.f) : z;
    v[e] = (q - z) * s;
    if (e < n) codes |= (uint32_t)q << (4 * e);
  }
  if (n == 0) return;
  uint8_t* c = a.m.codes + row * a.m.ld_codes + j0 / 2;
  if (a.vec_c && n == 8) {
    *reinterpret_cast<uint32_t*>(c) = codes;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (2 * e < n) c[e] = (uint8_t)(codes >> (8 * e));
  }
  if (j0 % GROUP == 0) {
    a.m.scales[row * a.m.ld_scales + g] = s16;
    if (a.m.zeros) a.m.zeros[row * a.m.ld_scales + g] = (uint8_t)z;
  }
  if (a.W_hat) {
    float* h = a.W_hat + row * N + j0;
    if (n == 8) {
      store8(h, 0, CRVQ_F32, a.vec_h, v);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < n) h[e] = v[e];
    }
  }
}

crvq_status make_q4(const crvq_q4_matrix* m, Q4View* out) {
  CRVQ_CHECK_ARG(m != nullptr && m->codes && m->scales, "the 4-bit matrix, its codes or scales are NULL");
  CRVQ_CHECK_ARG(m->M >= 1 && m->N >= 1, "need M, N >= 1");
  if (m->group != 32 && m->group != 64 && m->group != 128)
    return fail(CRVQ_ERR_UNSUPPORTED, "groups of %d inputs: 32, 64 and 128 are implemented", m->group);
  CRVQ_CHECK_ARG(m->ld_codes >= ceil_div(m->N, 2), "ld_codes < ceil(N / 2)");
  CRVQ_CHECK_ARG(m->ld_scales >= ceil_div(m->N, m->group), "ld_scales < ceil(N / group)");
  CRVQ_CHECK_ARG(((uintptr_t)m->scales & 1u) == 0, "scales are not aligned");
  CRVQ_TRY(check_dev({{m->codes, "codes"}, {m->scales, "scales"}, {m->zeros, "zeros"}}));
  *out = Q4View{m->codes, static_cast<__nv_bfloat16*>(m->scales), m->zeros, m->M, m->N, m->ld_codes, m->ld_scales};
  return CRVQ_OK;
}

template <int TYPE, int GROUP, int NT, int RT>
crvq_status launch_matvec(const MatvecQ4& a, cudaStream_t stream) {
  auto kernel = q4_matvec_kernel<TYPE, GROUP, NT, RT>;
  constexpr size_t smem = (size_t)kQWarps * 8 * NT * 16 * RT * sizeof(float);
  CRVQ_TRY(smem_limit((const void*)kernel, smem));
  const int64_t grid = ceil_div(a.m.M, 16 * RT);
  if (grid >= (int64_t)1 << 31) return fail(CRVQ_ERR_UNSUPPORTED, "too many rows");
  ProfScope ps("q4_matvec", stream, (double)a.m.M * a.m.N * a.b);
  CRVQ_CUDA(launch_pdl(kernel, dim3((unsigned)grid), dim3(kQThreads), smem, stream, a));
  CRVQ_LAUNCHED();
  return CRVQ_OK;
}

template <int TYPE, int GROUP>
crvq_status pick_inputs(const MatvecQ4& a, cudaStream_t stream) {
  if (a.b <= 8) return launch_matvec<TYPE, GROUP, 1, 1>(a, stream);
  if (a.b <= 16) return launch_matvec<TYPE, GROUP, 2, 1>(a, stream);
  return launch_matvec<TYPE, GROUP, 4, 1>(a, stream);
}

template <int TYPE>
crvq_status pick_group(const MatvecQ4& a, int group, cudaStream_t stream) {
  if (group == 32) return pick_inputs<TYPE, 32>(a, stream);
  if (group == 64) return pick_inputs<TYPE, 64>(a, stream);
  return pick_inputs<TYPE, 128>(a, stream);
}

crvq_status matvec(const crvq_q4_matrix* m, const void* X, int64_t ldx, int64_t b, int type, void* Y,
                   int64_t ldy, cudaStream_t stream) {
  MatvecQ4 a{};
  CRVQ_TRY(make_q4(m, &a.m));
  CRVQ_CHECK_ARG(X && Y, "X and Y must not be NULL");
  CRVQ_CHECK_ARG(type >= CRVQ_F32 && type <= CRVQ_F16, "unknown type %d", type);
  CRVQ_CHECK_ARG(b >= 1, "need b >= 1");
  if (b > kMaxInputs) return fail(CRVQ_ERR_UNSUPPORTED, "batches of more than %d inputs are not implemented", kMaxInputs);
  CRVQ_CHECK_ARG(ldx >= m->N && ldy >= m->M, "need ldx >= N, ldy >= M");
  const size_t wide = type_bytes(type);
  CRVQ_CHECK_ARG((uintptr_t)X % wide == 0 && (uintptr_t)Y % wide == 0, "X or Y is not aligned to its type");
  CRVQ_TRY(check_dev({{X, "X"}, {Y, "Y"}}));
  a.X = X;
  a.ldx = ldx;
  a.Y = Y;
  a.ldy = ldy;
  a.b = (int)b;
  a.type = type;
  a.vec_w = ((uintptr_t)m->codes & 15u) == 0 && m->ld_codes % 16 == 0;
  a.vec_x = ((uintptr_t)X & 15u) == 0 && (b == 1 || ldx * (int64_t)wide % 16 == 0);
  if (type == CRVQ_F32) return pick_group<CRVQ_F32>(a, m->group, stream);
  if (type == CRVQ_BF16) return pick_group<CRVQ_BF16>(a, m->group, stream);
  return pick_group<CRVQ_F16>(a, m->group, stream);
}

crvq_status quantize(const void* W, int64_t ldw, int type, const crvq_q4_matrix* m, float* W_hat,
                     cudaStream_t stream) {
  QuantizeArgs a{};
  CRVQ_TRY(make_q4(m, &a.m));
  CRVQ_CHECK_ARG(W != nullptr, "W is NULL");
  CRVQ_CHECK_ARG(type >= CRVQ_F32 && type <= CRVQ_F16, "unknown type %d", type);
  CRVQ_CHECK_ARG(ldw >= m->N, "need ldw >= N");
  const size_t wide = type_bytes(type);
  CRVQ_CHECK_ARG((uintptr_t)W % wide == 0 && ((uintptr_t)W_hat & 3u) == 0, "W or W_hat is not aligned to its type");
  CRVQ_TRY(check_dev({{W, "W"}, {W_hat, "W_hat"}}));
  CRVQ_TRY(device_error_word(&a.err));
  a.W = W;
  a.ldw = ldw;
  a.type = type;
  a.vec_w = ((uintptr_t)W & 15u) == 0 && ldw * (int64_t)wide % 16 == 0;
  a.vec_c = ((uintptr_t)m->codes & 3u) == 0 && m->ld_codes % 4 == 0;
  a.vec_h = ((uintptr_t)W_hat & 15u) == 0 && m->N % 4 == 0;
  a.W_hat = W_hat;
  a.threads_row = ceil_div(m->N, m->group) * (m->group / 8);
  const int64_t grid = ceil_div(m->M * a.threads_row, 256);
  if (grid >= (int64_t)1 << 31) return fail(CRVQ_ERR_UNSUPPORTED, "matrix too large");
  ProfScope ps("q4_quantize", stream, (double)m->M * m->N);
  const dim3 g((unsigned)grid), t(256);
  if (m->group == 32)
    CRVQ_CUDA(launch_pdl(q4_quantize_kernel<32>, g, t, 0, stream, a));
  else if (m->group == 64)
    CRVQ_CUDA(launch_pdl(q4_quantize_kernel<64>, g, t, 0, stream, a));
  else
    CRVQ_CUDA(launch_pdl(q4_quantize_kernel<128>, g, t, 0, stream, a));
  CRVQ_LAUNCHED();
  return CRVQ_OK;
}

}  // namespace

}  // namespace crvq

extern "C" {

crvq_status crvq_q4_quantize(const void* W, int64_t ldw, int32_t type, const crvq_q4_matrix* m, float* W_hat,
                             crvq_stream_t stream) {
  CRVQ_ENTRY({ return crvq::quantize(W, ldw, type, m, W_hat, (cudaStream_t)stream); })
}

crvq_status crvq_q4_matvec(const crvq_q4_matrix* m, const void* X, int64_t ldx, int64_t b, int32_t type,
                           void* Y, int64_t ldy, crvq_stream_t stream) {
  CRVQ_ENTRY({ return crvq::matvec(m, X, ldx, b, type, Y, ldy, (cudaStream_t)stream); })
}

}  // extern "C"
