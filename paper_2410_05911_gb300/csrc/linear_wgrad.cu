// linear_wgrad.cu -- the gradient of the AAP linear layer's weights, dW = sum over tokens of dy scale codes
// (linear.cu has the formulas).  dy scale is no 16-bit number: it goes through the tensor cores in as many
// bfloat16 pieces as the gradient's own type has room for (1: bfloat16, 2: half, 3: float, exact).  One
// piece rounds each term to 8 bits, which many tokens average out; the few terms of up to kFewTokens are
// taken in two pieces, where the product is bound by writing dW and the second one costs nothing.
#include <cuda_runtime.h>

#include <cstdint>

#include "linear_gemm.cuh"

namespace aecct {

namespace {

constexpr int64_t kFewTokens = 64;

int pieces_of(int64_t M, int wdtype) { return wdtype == 0 ? 3 : wdtype == 1 || M <= kFewTokens ? 2 : 1; }

template <typename T, int P>
cudaError_t weight_grad(const AapLinearGradCall &c, float *work, cudaStream_t st) {
  const CodesT a = {c.codes, c.K, c.ldc, codes_unit(c.codes, c.ldc, c.K)};
  const OutW out = {c.dw, c.wdtype, c.K};
  return with_tile<P == 1 ? 256 : 128>(c.K, c.N, [&](auto tb, auto cg) {
    constexpr int TB = decltype(tb)::value, CG = decltype(cg)::value;
    using B = GradT<T, TB / CG, P>;
    const B b = {static_cast<const T *>(c.dy), c.N, c.lddy, c.scale, grads_vec<T>(c.dy, c.lddy, c.N)};
    return launch_gemm<CodesT, B, OutW, TB, CG>(c.K, c.N, c.M, a, b, out, work, sm_count(), linear_status(), st);
  });
}

template <int P>
int64_t workspace_of(int64_t M, int64_t K, int64_t N) {
  return with_tile<P == 1 ? 256 : 128>(K, N, [&](auto tb, auto cg) {
    constexpr int TB = decltype(tb)::value, CG = decltype(cg)::value;
    const GemmPlan p = gemm_plan<CodesT, GradT<float, TB / CG, P>, TB, CG>(K, N, M, sm_count());
    return p.splits > 1 ? p.splits * K * N : int64_t(0);
  });
}

template <typename T>
cudaError_t weight_grad(const AapLinearGradCall &c, float *work, cudaStream_t st) {
  const int p = pieces_of(c.M, c.wdtype);
  return p == 3 ? weight_grad<T, 3>(c, work, st) : p == 2 ? weight_grad<T, 2>(c, work, st) : weight_grad<T, 1>(c, work, st);
}

}  // namespace

int64_t weight_grad_workspace(int64_t M, int64_t K, int64_t N, int wdtype) {
  const int p = pieces_of(M, wdtype);
  return p == 3 ? workspace_of<3>(M, K, N) : p == 2 ? workspace_of<2>(M, K, N) : workspace_of<1>(M, K, N);
}

cudaError_t launch_weight_grad(const AapLinearGradCall &c, float *work, cudaStream_t st) {
  return c.dtype == 0 ? weight_grad<float>(c, work, st) : c.dtype == 1 ? weight_grad<__half>(c, work, st) : weight_grad<__nv_bfloat16>(c, work, st);
}

}  // namespace aecct
