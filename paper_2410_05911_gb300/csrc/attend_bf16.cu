// attend_bf16.cu -- the kernels of attend.cuh for a cache in bfloat16
#include "attend.cuh"

namespace aecct {

cudaError_t run_attend_bf16(int dim, int group, const AttendArgs *a, AttendPlan *plan, cudaStream_t st) {
  return run_width<__nv_bfloat16, 2>(dim, group, a, plan, st);
}

}  // namespace aecct
