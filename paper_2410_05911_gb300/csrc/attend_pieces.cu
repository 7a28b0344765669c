// attend_pieces.cu -- the kernels of attend.cuh for codes, with float and half queries: two pieces
#include "attend.cuh"

namespace aecct {

cudaError_t run_attend_pieces(int dim, int group, const AttendArgs *a, AttendPlan *plan, cudaStream_t st) {
  return run_width<int8_t, 2>(dim, group, a, plan, st);
}

}  // namespace aecct
