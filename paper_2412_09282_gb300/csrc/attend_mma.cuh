// Attention over the paged 8-bit cache: o = sum_j p_j V_j / sum_j p_j with p_j = exp(scale q . K_j - max),
// K_j = c_j s^k, V_j = c'_j s^v (one scale per 16 tokens and head).
//
// Form. A warp takes two blocks of 16 tokens at a time (one for 256 channels): S^T (16 tokens x 8 columns) =
// K Q^T on mma.sync.m16n8k16 with the codes as the A operand, O^T += V^T P^T with V^T as A and the weights as
// B. A column is one (query token, query head) pair; a unit is up to 8 NT columns of one kv head, so query
// heads that share a kv head (and a few drafted tokens) share every code that is read: the rows are far too
// few to fill a tcgen05 tile (128), and the products are small beside the codes' way from memory. The
// contraction index of either product may be taken in any order, so each lane's operand pieces are chosen as
// 16 consecutive codes of one token row. Blocks are copied to shared memory by a warp's 32 lanes 512
// consecutive bytes at a time, two steps ahead, and their codes become fp16 by byte permutes (int8:
// 1024 + code + 128, less 1152; exact) or by one conversion per pair (e4m3; exact).
//   The key scale multiplies the block's scores in fp32. The value scale s multiplies the weights, which are
// relative to a power of two of their column, at the largest p s of the tokens that the column sees: a weight is at
// most 2^14, and those below 2^-38 of that vanish. (Relative to the largest scale instead, nothing is left of a column that
// does not see the token with that scale, or gives it no weight.) A weight is two fp16 operands (22 bits: one
// operand's 11 were the largest error of the result), as q is from fp32. Running maxima, rounded up to whole
// numbers in log2 so that rescales are exact, and sums are fp32.
//
// Split, by whether the sequences could be long (their lengths are on the device, the page table's width is not):
//   Line. The work is every (sequence, kv head, column group)'s tiles of 128 tokens (64 for 256 channels) in
// one line, of which each CTA takes an equal share, whatever the lengths are. A unit that lies within a share
// is written at once; the others' parts (maximum, sum, unnormalised output) go to scratch and are joined in
// order by a second kernel, so results do not depend on timing.
//   Clusters. A unit's tiles are dealt out to the 2, 4 or 8 CTAs of a cluster, which join their parts through
// each other's shared memory: no second launch, no scratch.
//
// What bounds it: the bytes of the cache. 64 sequences of up to 4096 tokens, 32 kv heads: 183 us, 6.2 TB/s; 4
// of up to 131072 tokens, 8 kv heads: 162 us, 6.1 TB/s (91 and 89 % of a copy's rate). Short calls: the chain of
// lookups, copies, products and joins of a few tiles. One sequence of 1001 tokens: 8.3 us (12.1 by the line); 16 of up to
// 3001 with up to 5 drafted tokens, fp32: 21 us (25 by the line).
#pragma once

#include "attend.cuh"

namespace crvq {

namespace {

__device__ __forceinline__ void mma_f16(float d[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                        uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
      "{%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

__device__ __forceinline__ int word(const uint4& u, int i) {
  return i == 0 ? u.x : i == 1 ? u.y : i == 2 ? u.z : u.w;
}

// A block's 16 rows of keys or values in shared memory: lines of eight 16-byte units, whose places are
// exchanged within the line (by `turn` of the line) so that both readers are free of bank conflicts: keys
// (eight lanes: two rows, four neighbouring units each) and values (eight lanes: every other row of
// eight, two neighbouring units each; for 64 channels 16 lanes of half units).
template <int D>
struct Tile {
  static constexpr int kBytes = kCacheBlock * D;
  static __device__ __forceinline__ uint32_t turn(int line) {
    if constexpr (D == 64) return 2 * (line & 3);  // two rows in a line
    const int r = D == 128 ? line : line >> 1;
    return (r & 6) ^ ((r & 1) << 2);
  }
  // Byte offset of 16-byte unit c of row r.
  static __device__ __forceinline__ uint32_t at(int r, int c) {
    const int u = r * (D / 16) + c, line = u >> 3;
    return (uint32_t)(line * 8 + ((u & 7) ^ turn(line))) * 16;
  }
};

// Asynchronous copies; PART: of the first n bytes, zeros for the rest.
template <bool PART>
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, int n) {
  if constexpr (PART)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
  else
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
// Starts the copies of a block from src to its tile at dst, a warp's 32 lanes 512 consecutive bytes at a
// time (lanes that copied just the pieces that they read, 8 rows of 64 bytes, got 5.2 TB/s instead of 7.0).
// n: rows that there are (PART); the others are set to 0 (a page holds anything there).
template <int D, bool PART>
__device__ __forceinline__ void start_block(const uint8_t* src, uint32_t dst, int n) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int j = 0; j < Tile<D>::kBytes / 512; ++j) {
    const int u = 32 * j + lane, line = u >> 3;
    const bool in = !PART || u < n * (D / 16);
    copy16<PART>(dst + (line * 8 + ((u & 7) ^ Tile<D>::turn(line))) * 16, src + (in ? u * 16 : 0), in ? 16 : 0);
  }
}

__device__ __forceinline__ float load_remote(const float* p, int rank) {
  uint32_t at;
  float v;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
  return v;
}

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Joins a unit that its cluster's CTAs hold parts of (outputs [COLS][D] at `ring`, maxima, sums): each takes every
// cluster-th column, the parts in the order of the ranks.
template <int D, int COLS>
__device__ __forceinline__ void join_cluster(const AttendArgs& a, const Unit& u, int col0, int n_cols, const char* ring,
                                             const float* m_s, const float* l_s) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, rank = blockIdx.x & (a.cluster - 1);
  const float* o_s = reinterpret_cast<const float*>(ring);
  cluster_sync();
  for (int col = rank + warp * a.cluster; col < n_cols; col += kWarps * a.cluster) {
    const float mine = lane < a.cluster ? load_remote(m_s + col, lane) : -INFINITY;
    const float sum = lane < a.cluster ? load_remote(l_s + col, lane) : 0.f;
    float M = mine;
#pragma unroll
    for (int d = 4; d > 0; d >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, d));
    M = __shfl_sync(0xffffffffu, M, 0);
    const float f = pow2(mine - (M == -INFINITY ? 0.f : M));
    float L = 0.f, o[D / 32];
#pragma unroll
    for (int e = 0; e < D / 32; ++e) o[e] = 0.f;
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      if (r >= a.cluster) break;
      const float fr = __shfl_sync(0xffffffffu, f, r);
      L += __shfl_sync(0xffffffffu, sum, r) * fr;
#pragma unroll
      for (int e = 0; e < D / 32; ++e) o[e] += load_remote(o_s + col * D + lane + 32 * e, r) * fr;
    }
    const int j = (col0 + col) / a.group, h = u.h * a.group + (col0 + col) % a.group;
    const float inv = L > 0.f ? 1.f / L : (L == 0.f ? 0.f : L);
#pragma unroll
    for (int e = 0; e < D / 32; ++e)
      store_elem(a.o.data, (u.s.first + j) * a.o.ld_tok + h * a.o.ld_head + lane + 32 * e, a.o.type, o[e] * inv);
    if (lane == 0 && a.lse)
      a.lse[(u.s.first + j) * a.q.heads + h] = L > 0.f ? (M + log2f(L)) / kLog2e : (L == 0.f ? -INFINITY : L);
  }
  cluster_sync();  // (no CTA leaves while its memory is read)
}

template <int D, int NT, int FMT, bool SPLIT>
struct Shape {
  static constexpr int kCols = 8 * NT;
  static constexpr int kQRow = D + 8;  // halves per query row, padded against bank conflicts
  static constexpr size_t kQ = (size_t)kCols * kQRow * 2 * (SPLIT ? 2 : 1);
  // keys and values on their way and in work; at a unit's end each warp's outputs [kCols][D] lie in its part
  static constexpr int kStages = 2;
  static constexpr int kHalf = Tile<D>::kBytes * kBlocks<D> * kStages;
  static constexpr int kRing = 2 * kHalf;
  static_assert(kRing >= kCols * D * 4, "outputs fit the ring");
  static constexpr size_t kSmem = kQ + (size_t)kWarps * kRing + 3 * kCols * 4 + 3 * kWarps * kCols * 4;
  // CTAs per SM, by registers (128 threads of 128 or 168) and shared memory
  static constexpr int kPerSm = D == 64 ? (NT == 1 ? 4 : 3) : (D == 128 ? 3 : 2);
  static constexpr int kSlot = kCols * (D + 2);  // floats of a part
};

template <int D, int NT, int FMT, bool SPLIT, bool CLUSTER>
__global__ void __launch_bounds__(kThreads, Shape<D, NT, FMT, SPLIT>::kPerSm)
attend_kernel(const __grid_constant__ AttendArgs a) {
  using S = Shape<D, NT, FMT, SPLIT>;
  constexpr int COLS = S::kCols;
  extern __shared__ __align__(16) char sm[];
  __half* q_s = reinterpret_cast<__half*>(sm);                       // [split][COLS][kQRow]
  char* ring = sm + S::kQ;                                           // [kWarps][keys, values][kStages][blocks] tiles
  float* f_s = reinterpret_cast<float*>(ring + kWarps * S::kRing);   // [COLS] score factor
  int* beg_s = reinterpret_cast<int*>(f_s + COLS);                   // [COLS] first and last + 1 key seen
  int* end_s = beg_s + COLS;
  float* m_s = reinterpret_cast<float*>(end_s + COLS);               // [kWarps][COLS]
  float* l_s = m_s + kWarps * COLS;
  float* r_s = l_s + kWarps * COLS;                                  // weights' reference
  pdl_wait();  // (no early trigger: waiting blocks of the next kernels would take this one's places)
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, gid = lane >> 2, tig = lane & 3;
  Line<D, COLS> line;
  int64_t w = 0, w1 = 1;
  if constexpr (!CLUSTER) {
    line = Line<D, COLS>(a);
    const int shares = (int)min((int64_t)a.shares, line.total);
    if ((int)blockIdx.x >= shares) return;
    w = share_begin(line.total, blockIdx.x, shares);
    w1 = share_begin(line.total, blockIdx.x + 1, shares);
  }
  char* mine = ring + warp * S::kRing;
  const uint32_t mine_u = (uint32_t)__cvta_generic_to_shared(mine);
  const uint32_t key_at = Tile<D>::at(gid, tig);
  const uint32_t val_at[2] = {D == 64 ? Tile<D>::at(2 * tig, gid >> 1) + (gid & 1) * 8 : Tile<D>::at(2 * tig, gid),
                              D == 64 ? Tile<D>::at(2 * tig + 1, gid >> 1) + (gid & 1) * 8 : Tile<D>::at(2 * tig + 1, gid)};

  while (w < w1) {
    Unit u;
    int t_end;
    if constexpr (CLUSTER) {
      if (!Line<D, COLS>::unit_only(a, blockIdx.x >> a.log_cluster, &u)) return;  // (with its whole cluster)
      const int64_t rank = blockIdx.x & (a.cluster - 1);
      u.tile = (int)(u.s.tiles * rank >> a.log_cluster);
      t_end = (int)(u.s.tiles * (rank + 1) >> a.log_cluster);
      w = w1;
    } else {
      u = line.locate(a, w);
      const int64_t tile0 = u.begin + kStart, unit_end = tile0 + u.s.tiles;
      t_end = (int)max((int64_t)0, min(unit_end, w1) - tile0);
      w = min(unit_end, w1);
      if (u.tile >= t_end) continue;  // (this share ends before the unit's first tile)
    }
    const int len = u.s.len, group = a.group;
    const int col0 = u.cg * COLS, n_cols = min(COLS, u.s.n * group - col0);
    __syncthreads();  // the previous unit's shared memory has been read

    // A lane looks up the place and the scales of every 32nd of this warp's blocks. Step i takes the warp's
    // blocks NB i .. of the part; while it works on its values and on the next step's keys, the copies of
    // the next values and of the keys after those are on their way.
    const int reach = u.s.len - u.s.n + (col0 + n_cols - 1) / group + 1;  // past the last column's place
    const int some_e = a.causal ? min(len, reach) : len;
    const int some_b = a.window > 0 ? max(0, len - u.s.n + col0 / group - a.window + 1) : 0;
    constexpr int NB = kBlocks<D>;
    constexpr uint32_t kAll = (1u << NB) - 1;
    const int n_tiles = t_end - u.tile;
    int64_t at_l = -1, at_old = -1;
    float sk_l = 0.f, sv_l = 0.f, sk_old = 0.f, sv_old = 0.f;
    uint32_t has = 0, has_old = 0;  // blocks of the present 32 and of the 32 before that some query sees
    int batch = -1;
    auto look_up = [&](int i) {     // before step i's keys are wanted, each i in turn
      if (i >= n_tiles || (i * NB & 31) != 0) return;
      at_old = at_l;
      sk_old = sk_l;
      sv_old = sv_l;
      has_old = has;
      batch = i * NB >> 5;
      const int tl = u.tile + i + lane / NB;
      const int tok = (u.s.lo + tl) * kTile<D> + (warp * NB + lane % NB) * kCacheBlock;
      at_l = -1;
      if (tl < t_end && tok < some_e && tok + kCacheBlock > some_b) {
        const int64_t page = seq_page(a.c, u.b, tok / a.c.page, a.err);
        if (page >= 0) {
          const int in = tok % a.c.page;
          at_l = page * a.c.page_stride + ((int64_t)u.h * a.c.page + in) * D;
          const int64_t at_s = (page * a.c.n_kv + u.h) * (a.c.page / kCacheBlock) + in / kCacheBlock;
          sk_l = __ldg(a.c.ks + at_s);
          sv_l = __ldg(a.c.vs + at_s);
        }
      }
      has = __ballot_sync(0xffffffffu, at_l >= 0);
    };
    auto start_k = [&](int i) {
      if (i >= n_tiles) return;
      const bool old = (i * NB >> 5) != batch;
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const int64_t at = __shfl_sync(0xffffffffu, old ? at_old : at_l, (i * NB + b) & 31);
        if (at >= 0) start_block<D, false>(a.c.K + at, mine_u + ((i & 1) * NB + b) * Tile<D>::kBytes, kCacheBlock);
      }
    };
    auto start_v = [&](int i) {
      if (i >= n_tiles) return;
      const bool old = (i * NB >> 5) != batch;
      const int tok = (u.s.lo + u.tile + i) * kTile<D> + warp * NB * kCacheBlock;
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const int64_t at = __shfl_sync(0xffffffffu, old ? at_old : at_l, (i * NB + b) & 31);
        const uint32_t dst = mine_u + S::kHalf + ((i & 1) * NB + b) * Tile<D>::kBytes;
        const int n = at >= 0 ? len - (tok + b * kCacheBlock) : 0;
        if (n >= kCacheBlock)
          start_block<D, false>(a.c.V + at, dst, n);
        else
          start_block<D, true>(a.c.V + max(at, (int64_t)0), dst, max(n, 0));
      }
    };
    float qx[COLS / kWarps][D / 32];
#pragma unroll
    for (int k = 0; k < COLS / kWarps; ++k) {
      const int col = warp + k * kWarps, j = (col0 + col) / group, h = u.h * group + (col0 + col) % group;
#pragma unroll
      for (int e = 0; e < D / 32; ++e)
        qx[k][e] = col < n_cols ? load_elem(a.q.data, (u.s.first + j) * a.q.ld_tok + h * a.q.ld_head + lane + 32 * e,
                                            a.q.type)
                                : 0.f;
    }
    look_up(0);
    start_k(0);
    asm volatile("cp.async.commit_group;" ::: "memory");
    look_up(1);
    start_k(1);
    start_v(0);
    asm volatile("cp.async.commit_group;" ::: "memory");

    // queries: a warp per column, relative to the power of two at its largest element
#pragma unroll
    for (int k = 0; k < COLS / kWarps; ++k) {
      const int col = warp + k * kWarps, j = (col0 + col) / group;
      float* x = qx[k];
      float top = 0.f;
#pragma unroll
      for (int e = 0; e < D / 32; ++e) top = fmaxf(top, fabsf(x[e]));
      top = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top)));
      // 2^-e for a top in [2^e, 2^(e + 1)); 1 for zeros, subnormals and infinities
      const uint32_t ex = __float_as_uint(top) >> 23;
      const bool plain = ex == 0 || ex == 255;
      const float inv = plain ? 1.f : __uint_as_float(ex == 254 ? 0x00400000u : (254u - ex) << 23);
      const float back = plain ? 1.f : __uint_as_float(ex << 23);
#pragma unroll
      for (int e = 0; e < D / 32; ++e) {
        const float v = x[e] * inv;
        const __half hi = __float2half_rn(v);
        q_s[col * S::kQRow + lane + 32 * e] = hi;
        if constexpr (SPLIT)
          q_s[(COLS + col) * S::kQRow + lane + 32 * e] = __float2half_rn(v - __half2float(hi));
      }
      if (lane == 0) {
        f_s[col] = back * a.scale;
        const int pos = len - u.s.n + j;
        beg_s[col] = a.window > 0 ? max(0, pos - a.window + 1) : 0;
        end_s[col] = a.causal ? min(len, pos + 1) : len;
      }
    }
    __syncthreads();
    float f[NT][2];
    int kb[NT][2], ke[NT][2];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        f[t][e] = f_s[8 * t + 2 * tig + e];
        kb[t][e] = beg_s[8 * t + 2 * tig + e];
        ke[t][e] = end_s[8 * t + 2 * tig + e];
      }
    // keys that every column sees (positions do not fall from column to column)
    const int every_b = beg_s[n_cols - 1], every_e = end_s[0];

    float o[D / 16][NT][4];
    // in log2, whole numbers: m at the largest score or above, and in shared memory (two reads a step, and registers are
    // scarce) the weights' reference at the largest score + log2 s or above
    float m[NT][2], l[NT][2];
    float2* refs = reinterpret_cast<float2*>(r_s + warp * COLS) + tig;  // of this lane's columns: 4 further on for n + 1
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[i][t][e] = 0.f;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        m[t][e] = -INFINITY;
        l[t][e] = 0.f;
      }
#pragma unroll
    for (int t = 0; t < NT; ++t)
      if (gid == 0) refs[4 * t] = make_float2(-INFINITY, -INFINITY);
    __syncwarp();

    // S^T of step i's keys (what lies there is masked later where no key does)
    auto scores = [&](int i, float s[NB][NT][4]) {
      const char* keys = mine + (i & 1) * NB * Tile<D>::kBytes;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[b][n][e] = 0.f;
#pragma unroll
      for (int j = 0; j < D / 64; ++j) {
        uint32_t qv[SPLIT ? 2 : 1][NT][8];
#pragma unroll
        for (int z = 0; z < (SPLIT ? 2 : 1); ++z)
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            const uint4* p = reinterpret_cast<const uint4*>(
                q_s + (z * COLS + 8 * n + gid) * S::kQRow + 64 * j + 16 * tig);
            const uint4 x = p[0], y = p[1];
            qv[z][n][0] = x.x; qv[z][n][1] = x.y; qv[z][n][2] = x.z; qv[z][n][3] = x.w;
            qv[z][n][4] = y.x; qv[z][n][5] = y.y; qv[z][n][6] = y.z; qv[z][n][7] = y.w;
          }
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          // (8 rows on, the same turn; every other 64 channels, the other half of the line)
          const char* k = keys + b * Tile<D>::kBytes + (j >> 1) * 128;
          const uint4 k0 = *reinterpret_cast<const uint4*>(k + (key_at ^ (j & 1) * 64));
          const uint4 k1 = *reinterpret_cast<const uint4*>(k + 8 * D + (key_at ^ (j & 1) * 64));
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const uint32_t x = word(k0, w), y = word(k1, w);
            const uint32_t a0 = codes2<FMT, 0>(x), a2 = codes2<FMT, 1>(x);
            const uint32_t a1 = codes2<FMT, 0>(y), a3 = codes2<FMT, 1>(y);
#pragma unroll
            for (int z = 0; z < (SPLIT ? 2 : 1); ++z)
#pragma unroll
              for (int n = 0; n < NT; ++n) mma_f16(s[b][n], a0, a1, a2, a3, qv[z][n][2 * w], qv[z][n][2 * w + 1]);
          }
        }
      }
    };
    float s[NB][NT][4];
    asm volatile("cp.async.wait_group 1;" ::: "memory");
    __syncwarp();
    scores(0, s);
    for (int i = 0; i < n_tiles; ++i) {
      const bool old = (i * NB >> 5) != batch;
      const uint32_t live = (old ? has_old : has) >> (i * NB & 31);
      float sk[NB], sv[NB];
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        sk[b] = __shfl_sync(0xffffffffu, old ? sk_old : sk_l, (i * NB + b) & 31);
        sv[b] = __shfl_sync(0xffffffffu, old ? sv_old : sv_l, (i * NB + b) & 31);
      }
      __syncwarp();  // every lane has read what these copies overwrite
      start_v(i + 1);
      look_up(i + 2);
      start_k(i + 2);
      asm volatile("cp.async.commit_group;" ::: "memory");
      const int tok = (u.s.lo + u.tile + i) * kTile<D> + warp * NB * kCacheBlock;

      // scores in units of log2, masked (a block that no query sees: all of it); their maxima
      const bool whole = tok >= every_b && tok + NB * kCacheBlock <= every_e && (live & kAll) == kAll;
      float lg[NB];
#pragma unroll
      for (int b = 0; b < NB; ++b) lg[b] = __log2f(sv[b]);
      bool grew = false;  // in this lane's tokens (the lanes' maxima are joined only when one has)
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const float2 r = refs[4 * n];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
          for (int b = 0; b < NB; ++b) {
            const float g = f[n][e] * sk[b];
            s[b][n][e] *= g;
            s[b][n][e + 2] *= g;
            if (!whole) {
              const int t0 = tok + b * kCacheBlock + gid;
              const bool in = live >> b & 1;
              if (!in || t0 < kb[n][e] || t0 >= ke[n][e]) s[b][n][e] = -INFINITY;
              if (!in || t0 + 8 < kb[n][e] || t0 + 8 >= ke[n][e]) s[b][n][e + 2] = -INFINITY;
            }
            const float v = fmaxf(s[b][n][e], s[b][n][e + 2]);
            grew = grew || v > m[n][e] || v + lg[b] > (e ? r.y : r.x);
          }
        }
      }
      if (__any_sync(0xffffffffu, grew)) {
        auto over_lanes = [](float v) {
          v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 4));
          v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 8));
          return fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 16));
        };
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const float2 r2 = refs[4 * n];
          float r[2] = {r2.x, r2.y};
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float v = -INFINITY, t = -INFINITY;
#pragma unroll
            for (int b = 0; b < NB; ++b) v = fmaxf(v, fmaxf(s[b][n][e], s[b][n][e + 2]));
            const float mn = fmaxf(m[n][e], ceilf(over_lanes(v)));
#pragma unroll
            for (int b = 0; b < NB; ++b) {  // (what is 0 as an fp32 weight has no say)
              v = fmaxf(s[b][n][e], s[b][n][e + 2]);
              if (v > mn - 126.f) t = fmaxf(t, v + lg[b]);
            }
            // (not below mn - 112: a weight's factor stays below 2^127)
            const float rn = fmaxf(r[e], fmaxf(ceilf(over_lanes(t)), mn - 112.f));
            const float fac = r[e] == rn ? 1.f : pow2(r[e] - rn);
            if (m[n][e] != mn) l[n][e] *= pow2(m[n][e] - mn);
            m[n][e] = mn;
            r[e] = rn;
#pragma unroll
            for (int d = 0; d < D / 16; ++d) {
              o[d][n][e] *= fac;
              o[d][n][e + 2] *= fac;
            }
          }
          __syncwarp();  // every lane has read it
          if (gid == 0) refs[4 * n] = make_float2(r[0], r[1]);
        }
        __syncwarp();
      }
      uint32_t pb[NB][2][NT][2];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const float m0 = m[n][0] == -INFINITY ? 0.f : m[n][0], m1 = m[n][1] == -INFINITY ? 0.f : m[n][1];
        const float2 r = refs[4 * n];
        const float g0 = pow2(m0 - r.x + kLogWeight), g1 = pow2(m1 - r.y + kLogWeight);
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          // (finite: the largest scale of all may be one that a column does not see)
          const float w0 = live >> b & 1 ? fminf(sv[b] * g0, 0x1p126f) : 0.f, w1 = live >> b & 1 ? fminf(sv[b] * g1, 0x1p126f) : 0.f;
          float p0 = pow2(s[b][n][0] - m0), p1 = pow2(s[b][n][1] - m1);
          float p2 = pow2(s[b][n][2] - m0), p3 = pow2(s[b][n][3] - m1);
          l[n][0] += p0 + p2;
          l[n][1] += p1 + p3;
          p0 *= w0; p1 *= w1; p2 *= w0; p3 *= w1;
          const uint32_t h0 = half2_bits(p0, p1), h1 = half2_bits(p2, p3);
          pb[b][0][n][0] = transpose8(h0);
          pb[b][0][n][1] = transpose8(h1);
          pb[b][1][n][0] = transpose8(half2_rest(p0, p1, h0));
          pb[b][1][n][1] = transpose8(half2_rest(p2, p3, h1));
        }
      }
      asm volatile("cp.async.wait_group 1;" ::: "memory");
      __syncwarp();
      // the next step's scores and this one's outputs: independent, in the same stretch of code
      float next[NB][NT][4];
      scores(i + 1, next);
      const char* values = mine + S::kHalf + (i & 1) * NB * Tile<D>::kBytes;
#pragma unroll
      for (int b = 0; b < NB; ++b) {
#pragma unroll
        for (int j = 0; j < (D == 64 ? 1 : D / 128); ++j) {
          uint4 v[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const char* p = values + b * Tile<D>::kBytes + j * 128 + (k >> 1) * 8 * D + val_at[k & 1];
            if constexpr (D == 64) {
              const uint2 x = *reinterpret_cast<const uint2*>(p);
              v[k] = make_uint4(x.x, x.y, 0, 0);
            } else {
              v[k] = *reinterpret_cast<const uint4*>(p);
            }
          }
#pragma unroll
          for (int w = 0; w < (D == 64 ? 2 : 4); ++w) {
            // tokens 2 tig, 2 tig + 1 side by side, channel by channel; then + 8, + 9
            const uint32_t x0 = word(v[0], w), x1 = word(v[1], w);
            const uint32_t y0 = word(v[2], w), y1 = word(v[3], w);
            const uint32_t xl = __byte_perm(x0, x1, 0x5140), xh = __byte_perm(x0, x1, 0x7362);
            const uint32_t yl = __byte_perm(y0, y1, 0x5140), yh = __byte_perm(y0, y1, 0x7362);
            const uint32_t a0 = codes2<FMT, 0>(xl), a1 = codes2<FMT, 1>(xl);
            const uint32_t a2 = codes2<FMT, 0>(yl), a3 = codes2<FMT, 1>(yl);
            const uint32_t c0 = codes2<FMT, 0>(xh), c1 = codes2<FMT, 1>(xh);
            const uint32_t c2 = codes2<FMT, 0>(yh), c3 = codes2<FMT, 1>(yh);
            const int mt = 8 * j + 2 * w;
#pragma unroll
            for (int z = 0; z < 2; ++z)
#pragma unroll
              for (int n = 0; n < NT; ++n) {
                mma_f16(o[mt][n], a0, a1, a2, a3, pb[b][z][n][0], pb[b][z][n][1]);
                mma_f16(o[mt + 1][n], c0, c1, c2, c3, pb[b][z][n][0], pb[b][z][n][1]);
              }
          }
        }
      }
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[b][n][e] = next[b][n][e];
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncwarp();  // every lane has read its pieces: the ring takes the outputs
    float* o_s = reinterpret_cast<float*>(mine);

    // join the warps
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float v = l[n][e];
        v += __shfl_xor_sync(0xffffffffu, v, 4);
        v += __shfl_xor_sync(0xffffffffu, v, 8);
        v += __shfl_xor_sync(0xffffffffu, v, 16);
        const int col = 8 * n + 2 * tig + e;
        if (gid == 0) {
          m_s[warp * COLS + col] = m[n][e];
          l_s[warp * COLS + col] = v;
        }
        float* row = o_s + col * D;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
          // m-tile i: channels 2 i and 2 i + 1 of the lane's piece
          const int d = D == 64 ? 8 * gid + 2 * i : 128 * (i / 8) + 16 * gid + 2 * (i % 8);
          *reinterpret_cast<float2*>(row + d) = make_float2(o[i][n][e], o[i][n][e + 2]);
        }
      }
    __syncthreads();
    const bool complete = !CLUSTER && u.tile == 0 && t_end == u.s.tiles;
    float* part = a.part + (int64_t)(2 * blockIdx.x + (u.tile == 0 ? 1 : 0)) * S::kSlot;
    for (int col = warp; col < n_cols; col += kWarps) {
      float M = -INFINITY, L = 0.f;
#pragma unroll
      for (int i = 0; i < kWarps; ++i) M = fmaxf(M, m_s[i * COLS + col]);
      const float mm = M == -INFINITY ? 0.f : M;
      float fac[kWarps];
#pragma unroll
      for (int i = 0; i < kWarps; ++i) {
        L += l_s[i * COLS + col] * pow2(m_s[i * COLS + col] - mm);
        fac[i] = pow2(r_s[i * COLS + col] - mm - kLogWeight);
      }
      const int j = (col0 + col) / group, h = u.h * group + (col0 + col) % group;
      const float inv = L > 0.f ? 1.f / L : (L == 0.f ? 0.f : L);
#pragma unroll
      for (int e = 0; e < D / 32; ++e) {
        const int d = lane + 32 * e;
        float v = 0.f;
#pragma unroll
        for (int i = 0; i < kWarps; ++i) v += reinterpret_cast<const float*>(ring + i * S::kRing)[col * D + d] * fac[i];
        if (complete)
          store_elem(a.o.data, (u.s.first + j) * a.o.ld_tok + h * a.o.ld_head + d, a.o.type, v * inv);
        else if (CLUSTER)  // (over warp 0's outputs, of which this lane alone reads this one)
          reinterpret_cast<float*>(ring)[col * D + d] = v;
        else
          part[col * D + d] = v;
      }
      __syncwarp();
      if (lane == 0) {
        if (CLUSTER) {
          m_s[col] = M;
          l_s[col] = L;
        } else if (!complete) {
          part[COLS * D + col] = M;
          part[COLS * D + COLS + col] = L;
        } else if (a.lse) {
          a.lse[(u.s.first + j) * a.q.heads + h] = L > 0.f ? (M + log2f(L)) / kLog2e : (L == 0.f ? -INFINITY : L);
        }
      }
    }
    if constexpr (CLUSTER) join_cluster<D, COLS>(a, u, col0, n_cols, ring, m_s, l_s);
  }
}

}  // namespace

}  // namespace crvq
