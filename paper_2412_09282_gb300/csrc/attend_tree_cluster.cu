// Attention of drafted trees over short sequences (attend_cluster.cuh).
#include "attend_cluster.cuh"

namespace crvq {

crvq_status launch_tree_clusters(AttendArgs& a, int D, int NT, int format, int64_t units, int size,
                                 cudaStream_t stream) {
  return pick_clusters<true>(a, D, NT, format, units, size, stream);
}

}  // namespace crvq
