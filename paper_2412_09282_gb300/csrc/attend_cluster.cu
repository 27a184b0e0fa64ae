// Attention for few queries over short sequences (attend_cluster.cuh).
#include "attend_cluster.cuh"

namespace crvq {

crvq_status launch_attend_clusters(AttendArgs& a, int D, int NT, int format, int64_t units, int size,
                                   cudaStream_t stream) {
  return pick_clusters<false>(a, D, NT, format, units, size, stream);
}

}  // namespace crvq
