// attend_half.cu -- the kernels of attend.cuh for a cache in half
#include "attend.cuh"

namespace aecct {

cudaError_t run_attend_half(int dim, int group, const AttendArgs *a, AttendPlan *plan, cudaStream_t st) {
  return run_width<__half, 2>(dim, group, a, plan, st);
}

}  // namespace aecct
