// Attention of drafted trees with many (query token, head) pairs per sequence (attend_tc.cuh).
#include "attend_tc.cuh"

namespace crvq {

crvq_status launch_tree_many(AttendArgs& a, int D, int format, cudaStream_t stream) {
  return D == 64 ? pick_tc<64, true>(a, format, stream) : pick_tc<128, true>(a, format, stream);
}

}  // namespace crvq
