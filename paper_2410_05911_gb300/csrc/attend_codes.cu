// attend_codes.cu -- the kernels of attend.cuh for codes, with bfloat16 queries: weights in one half
#include "attend.cuh"

namespace aecct {

cudaError_t run_attend_codes(int dim, int group, const AttendArgs *a, AttendPlan *plan, cudaStream_t st) {
  return run_width<int8_t, 1>(dim, group, a, plan, st);
}

}  // namespace aecct
