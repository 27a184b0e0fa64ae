// Attention for few queries over short sequences: launches of the kernel of attend_mma.cuh with a unit's tiles dealt
// out to the CTAs of a cluster.
#pragma once

#include "attend_mma.cuh"

namespace crvq {

namespace {

inline crvq_status launch_clusters(void (*kernel)(AttendArgs), dim3 grid, int size, size_t smem, cudaStream_t stream,
                            const AttendArgs& a) {
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = size;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  CRVQ_CUDA(cudaLaunchKernelEx(&cfg, kernel, a));
  CRVQ_LAUNCHED();
  return CRVQ_OK;
}

template <int D, int NT, int FMT, bool SPLIT, bool TREE>
crvq_status launch(AttendArgs& a, int64_t units, int size, cudaStream_t stream) {
  using S = Shape<D, NT, FMT, SPLIT>;
  auto kernel = attend_kernel<D, NT, FMT, SPLIT, true, TREE>;
  CRVQ_TRY(smem_limit((const void*)kernel, S::kSmem));
  ProfScope ps("cache_attention", stream, (double)a.rows.n_tok * a.q.heads * D);
  a.cluster = size;
  a.log_cluster = size == 8 ? 3 : size == 4 ? 2 : 1;
  return launch_clusters(kernel, dim3((unsigned)(units * size)), size, S::kSmem, stream, a);
}

template <int D, int NT, bool TREE>
crvq_status pick(AttendArgs& a, int format, int64_t units, int size, cudaStream_t stream) {
  const bool split = a.q.type == CRVQ_F32;
  if (format == CRVQ_KV_INT8)
    return split ? launch<D, NT, CRVQ_KV_INT8, true, TREE>(a, units, size, stream)
                 : launch<D, NT, CRVQ_KV_INT8, false, TREE>(a, units, size, stream);
  return split ? launch<D, NT, CRVQ_KV_E4M3, true, TREE>(a, units, size, stream)
               : launch<D, NT, CRVQ_KV_E4M3, false, TREE>(a, units, size, stream);
}

template <bool TREE>
crvq_status pick_clusters(AttendArgs& a, int D, int NT, int format, int64_t units, int size, cudaStream_t stream) {
  if (D == 256) return pick<256, 1, TREE>(a, format, units, size, stream);
  if (D == 128)
    return NT == 1 ? pick<128, 1, TREE>(a, format, units, size, stream) : pick<128, 2, TREE>(a, format, units, size, stream);
  return NT == 1 ? pick<64, 1, TREE>(a, format, units, size, stream) : pick<64, 2, TREE>(a, format, units, size, stream);
}

}  // namespace

}  // namespace crvq
