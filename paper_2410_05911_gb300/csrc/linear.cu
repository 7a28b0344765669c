// linear.cu -- the AAP linear layer of eq. AAPLinear (Sec. 4.1) on int8 codes and 2-bit weights, any
// shape, and its gradients.
//
//   y[m, n]  = scale_m w_scale sum_k q[m, k] T[n, k] + b_n
//   dx[m, k] = w_scale sum_n dy[m, n] T[n, k]
//   dW[n, k] = sum_m dy[m, n] scale_m q[m, k]      (straight through Ternary)
//   db[n]    = sum_m dy[m, n]
//
// The three products run on the tensor cores (linear_gemm.cuh).  The forward sum is one of integers up to
// 127 * 65536 < 2^23: exact in 32 bits, and the same however it is split.
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>
#include <mutex>

#include "linear_gemm.cuh"

namespace aecct {

namespace {

// the tile: few tokens take a narrow one, whose rest would be converted zeros
template <class F>
auto with_forward_tile(int64_t M, int64_t N, const F &f) {
  if (M <= 16) return f(std::integral_constant<int, 16>(), std::integral_constant<int, 1>());
  if (M > 64 && M <= 128) return f(std::integral_constant<int, 128>(), std::integral_constant<int, 1>());
  return with_tile<256>(N, M, f);
}

}  // namespace

int64_t aap_linear_workspace(int64_t M, int64_t K, int64_t N) {
  const int sms = sm_count();
  return with_forward_tile(M, N, [&](auto tb, auto cg) {
    constexpr int TB = decltype(tb)::value, CG = decltype(cg)::value;
    const GemmPlan p = gemm_plan<WeightsK, CodesK<TB / CG>, TB, CG>(N, M, K, sms);
    return p.splits > 1 ? p.splits * M * N * static_cast<int64_t>(sizeof(float)) : int64_t(0);
  });
}

cudaError_t launch_aap_linear(const AapLinearCall &c, cudaStream_t st) {
  const WeightsK a = {c.packed, c.N, c.K, weights_unit(c.packed, c.K)};
  const OutY out = {c.y, c.dtype, c.N, c.scale, c.w_scale, c.bias};
  return with_forward_tile(c.M, c.N, [&](auto tb, auto cg) {
    constexpr int TB = decltype(tb)::value, CG = decltype(cg)::value;
    using B = CodesK<TB / CG>;
    const B b = {c.codes, c.M, c.ldc, codes_unit(c.codes, c.ldc, c.K)};
    return launch_gemm<WeightsK, B, OutY, TB, CG>(c.N, c.M, c.K, a, b, out, static_cast<float *>(c.workspace), sm_count(),
                                                  linear_status(), st);
  });
}

// The word that a wait without an end would set, in host memory that every device sees: read before the
// next call, so that no call queues a copy behind its kernel.
int *linear_status() {
  static std::mutex lock;
  static int *word = nullptr;
  std::lock_guard<std::mutex> held(lock);
  if (!word) {
    cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;  // (a first call under capture may allocate)
    cudaThreadExchangeStreamCaptureMode(&mode);
    if (cudaHostAlloc(reinterpret_cast<void **>(&word), sizeof(int), cudaHostAllocPortable | cudaHostAllocMapped) == cudaSuccess)
      *word = 0;
    else word = nullptr;
    cudaThreadExchangeStreamCaptureMode(&mode);
  }
  return word;
}

}  // namespace aecct
