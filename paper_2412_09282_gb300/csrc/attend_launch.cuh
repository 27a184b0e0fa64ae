// Attention over the paged 8-bit cache: the choice among the forms (attend_mma.cuh by shares of a line or, in
// attend_cluster.cuh, by clusters; attend_tc.cuh), and the line's launches.
#pragma once

#include "attend_mma.cuh"

namespace crvq {

namespace {

// Clusters where a CTA then has no more than this many tiles, whatever the lengths are: by the page table's width, so a
// table for long contexts takes the line for short sequences, too. Line against clusters, us, for (units, tiles per
// CTA): (8, 1) 12.3, 8.4; (8, 4) 16.4, 11.6; (32, 2) 14.2, 9.2; (96, 1) 15.5, 8.3; (96, 5) 18.6, 14.0; (130, 8, of 64
// channels) 25.3, 21.4; (32, 8) 20.2, 15.5; (8, 16) 24.2, 24.0; (96, 12) 24.9, 25.5; (8, 32) 28.5, 39.6.
constexpr int kClusterTiles = 8;

template <int D, int NT, int FMT, bool SPLIT, bool TREE>
crvq_status launch_attend(AttendArgs& a, cudaStream_t stream) {
  using S = Shape<D, NT, FMT, SPLIT>;
  constexpr int COLS = S::kCols;
  auto kernel = attend_kernel<D, NT, FMT, SPLIT, false, TREE>;
  a.shares = sm_count() * S::kPerSm;
  // the most tokens that a unit's columns see, in tiles
  const int64_t held = (int64_t)a.c.max_pages * a.c.page, seen = a.window > 0 ? min(held, a.window + a.rows.n_tok) : held;
  const int64_t units = most_units<COLS>(a), most = seen / kTile<D>;
  for (int size = 8; size >= 2; size /= 2) {
    if (units * size > a.shares) continue;
    if (most > kClusterTiles * size) break;
    return TREE ? launch_tree_clusters(a, D, NT, FMT, units, size, stream)
                : launch_attend_clusters(a, D, NT, FMT, units, size, stream);
  }
  CRVQ_TRY(smem_limit((const void*)kernel, S::kSmem));
  ProfScope ps("cache_attention", stream, (double)a.rows.n_tok * a.q.heads * D);
  Scratch mem;
  CRVQ_TRY(mem.alloc((size_t)2 * a.shares * S::kSlot * sizeof(float), stream));
  a.part = mem.as<float>();
  CRVQ_CUDA(launch_pdl(kernel, dim3((unsigned)a.shares), dim3(kThreads), S::kSmem, stream, a));
  CRVQ_LAUNCHED();
  return launch_join<D, S::kCols>(a, stream);
}

// Columns per sequence, on average, from which tiles of 128 rows (attend_tc.cu) are taken. This form against that, us,
// for (sequences of up to 4096 tokens x kv heads, columns): (64 x 32, 32) 691, 853; (16 x 8, 32) 61, 68; (16 x 8, 48)
// 83, 69; (8 x 8, 64) 62, 44; (1 x 8, 64) 19, 28; (64 x 32, 64) 1359, 855; (1 x 8, 128) 27, 32; (1 x 8, 256) 52, 41.
constexpr int64_t kManyColumns = 64;

template <int D, int FMT, bool SPLIT, bool TREE>
crvq_status pick_columns(AttendArgs& a, cudaStream_t stream) {
  // 16 columns where a sequence has more than 8 (by the average: the rows' offsets are on the device)
  const bool wide = a.rows.n_tok * a.group > 8 * (int64_t)a.c.n_seq;
  if constexpr (D == 256)
    return launch_attend<D, 1, FMT, SPLIT, TREE>(a, stream);
  else
    return wide ? launch_attend<D, 2, FMT, SPLIT, TREE>(a, stream) : launch_attend<D, 1, FMT, SPLIT, TREE>(a, stream);
}

template <int D, bool TREE>
crvq_status pick_format(AttendArgs& a, int format, cudaStream_t stream) {
  const bool split = a.q.type == CRVQ_F32;
  if (format == CRVQ_KV_INT8)
    return split ? pick_columns<D, CRVQ_KV_INT8, true, TREE>(a, stream) : pick_columns<D, CRVQ_KV_INT8, false, TREE>(a, stream);
  return split ? pick_columns<D, CRVQ_KV_E4M3, true, TREE>(a, stream) : pick_columns<D, CRVQ_KV_E4M3, false, TREE>(a, stream);
}

// Trees with that many columns over short sequences: units of 16 columns, at two CTAs each or more, up to this many tiles of
// 128 tokens in all; by clusters up to 64 tiles a unit, else by shares of the line. This form against tiles of 128 rows, us, for
// (sequences x kv heads, columns, tokens): (1 x 1, 512, 4000) 25, 52; (1 x 8, 64, 4000) 25, 37; (1 x 8, 128, 1000) 21, 32; (1 x
// 8, 256, 2000) 35, 44; (4 x 8, 64, 1000) 25, 36; (4 x 8, 64, 2000) 35, 38; (1 x 8, 256, 4000) 67, 50; (4 x 8, 128, 1000) 52, 38;
// (1 x 8, 512, 1000) 52, 42; in a graph (32 x 1, 64, 1500) 24, 29. By the line, in a graph: (1 x 1, 64, 20000) 37, 61; (1 x 1, 64,
// 50000) 44, 64; (1 x 1, 64, 4000 of a table for 50000) 20, 26; (1 x 2, 64, 10000) 30, 43; (1 x 2, 64, 20000) 34, 45; (4 x 1, 64,
// 12000) 36, 36. (Attention without trees keeps its rule, and with it its results.)
constexpr int64_t kFewTiles = 2048;
inline bool few_tiles(const AttendArgs& a) {
  const int64_t units = most_units<16>(a), tiles = ceil_div((int64_t)a.c.max_pages * a.c.page, 128);
  return 2 * units <= 3 * (int64_t)sm_count() && units * tiles <= kFewTiles;
}

template <bool TREE>
crvq_status launch_form(AttendArgs& a, int D, int format, cudaStream_t stream) {
  if (D != 256 && a.q.type != CRVQ_F32 && a.rows.n_tok * a.group >= kManyColumns * (int64_t)a.c.n_seq && !(TREE && few_tiles(a)))
    return TREE ? launch_tree_many(a, D, format, stream) : launch_attend_many(a, D, format, stream);
  if (D == 64) return pick_format<64, TREE>(a, format, stream);
  if (D == 128) return pick_format<128, TREE>(a, format, stream);
  return pick_format<256, TREE>(a, format, stream);
}

}  // namespace

}  // namespace crvq
