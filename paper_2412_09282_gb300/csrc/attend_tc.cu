// Attention for many queries per sequence (attend_tc.cuh).
#include "attend_tc.cuh"

namespace crvq {

crvq_status launch_attend_many(AttendArgs& a, int D, int format, cudaStream_t stream) {
  return D == 64 ? pick_tc<64, false>(a, format, stream) : pick_tc<128, false>(a, format, stream);
}

}  // namespace crvq
