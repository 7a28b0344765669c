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
  auto run = [&](auto tb) {
    constexpr int TB = decltype(tb)::value;
    const GradT<T, TB, P> b = {static_cast<const T *>(c.dy), c.N, c.lddy, c.scale, grads_vec<T>(c.dy, c.lddy, c.N)};
    return launch_gemm<CodesT, GradT<T, TB, P>, OutW, TB>(c.K, c.N, c.M, a, b, out, work, sm_count(), linear_status(), st);
  };
  if (c.N <= 64) return run(std::integral_constant<int, 64>());
  return run(std::integral_constant<int, P == 1 ? 256 : 128>());
}

template <typename T>
cudaError_t weight_grad(const AapLinearGradCall &c, float *work, cudaStream_t st) {
  const int p = pieces_of(c.M, c.wdtype);
  return p == 3 ? weight_grad<T, 3>(c, work, st) : p == 2 ? weight_grad<T, 2>(c, work, st) : weight_grad<T, 1>(c, work, st);
}

}  // namespace

int64_t weight_grad_workspace(int64_t M, int64_t K, int64_t N, int wdtype) {
  const int sms = sm_count();
  const int pieces = pieces_of(M, wdtype);
  const GemmPlan p = pieces == 3   ? (N <= 64 ? gemm_plan<64, 3>(K, N, M, sms) : gemm_plan<128, 3>(K, N, M, sms))
                     : pieces == 2 ? (N <= 64 ? gemm_plan<64, 2>(K, N, M, sms) : gemm_plan<128, 2>(K, N, M, sms))
                                   : (N <= 64 ? gemm_plan<64, 1>(K, N, M, sms) : gemm_plan<256, 1>(K, N, M, sms));
  return p.splits > 1 ? p.splits * K * N : 0;
}

cudaError_t launch_weight_grad(const AapLinearGradCall &c, float *work, cudaStream_t st) {
  return c.dtype == 0 ? weight_grad<float>(c, work, st) : c.dtype == 1 ? weight_grad<__half>(c, work, st) : weight_grad<__nv_bfloat16>(c, work, st);
}

}  // namespace aecct
