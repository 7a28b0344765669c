// linear.cu -- the AAP linear layer of eq. AAPLinear (Sec. 4.1) on int8 codes and 2-bit weights, any
// shape, and its gradients.
//
//   y[m, n]  = scale_m w_scale sum_k q[m, k] T[n, k] + b_n
//   dx[m, k] = w_scale sum_n dy[m, n] T[n, k]
//   dW[n, k] = sum_m dy[m, n] scale_m q[m, k]      (straight through Ternary)
//   db[n]    = sum_m dy[m, n]
//
// The three products run on the tensor cores (linear_gemm.cuh), a few tokens' forward product in integers
// (linear_few.cu).  The forward sum is one of integers up to
// 128 * 65536 = 2^23: exact in 32 bits, and the same however it is split.
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>
#include <mutex>

#include "linear_gemm.cuh"

namespace aecct {

namespace {

using Staged = Tiled<128, false, false, 1, WeightsK::kSpan>;

// Whether a pair's product reads staged codes: staging costs its bytes, and saves each tile of 256 along N the conversion
// (8,192 x 4,096 codes, with 512 weights 38.7 us converted, 39.4 us with 15 us of staging, with 768 67 and 58 us, with 4,096
// 226 and 169).
bool stages_codes(int64_t N) { return N > 512; }

// The products of so few tokens that reading the weights is the work (linear_few.cu): 1 token 3.7 us, 8.4 us on the
// tensor cores, 4 tokens 5.4 and 8.5 us at 4,096 x 4,096, 13.6 and 18.6 us at 16,384 x 4,096; a token more costs 1.5 us there,
// and next to nothing on the tensor cores.
constexpr int64_t kIntegerTokens = 4;

// the other tiles: 16 tokens where there are no more
template <class F>
auto with_forward_tile(int64_t M, const F &f) {
  if (M <= 16) return f(std::integral_constant<int, 16>());
  return with_single_tile<1>(M, f);
}

constexpr int64_t kFloat = sizeof(float);

}  // namespace

// the staged codes, and the splits' sums (of integers, so that they hang on no type)
int64_t aap_linear_workspace(int64_t M, int64_t K, int64_t N) {
  const int sms = sm_count();
  if (M <= kIntegerTokens) return 0;
  if (pair_tiles(N, M, sms)) {
    if (stages_codes(N)) return partial_floats<WeightsK, Staged, 256, 2>(N, M, K, sms, 0) * kFloat + 2 * M * staged_k(K);
    return partial_floats<WeightsK, CodesK<128>, 256, 2>(N, M, K, sms, 0) * kFloat;
  }
  return with_forward_tile(M, [&](auto tb) {
    constexpr int TB = decltype(tb)::value;
    return partial_floats<WeightsK, CodesK<TB>, TB, 1>(N, M, K, sms, 0) * kFloat;
  });
}

cudaError_t launch_aap_linear(const AapLinearCall &c, cudaStream_t st) {
  if (c.M <= kIntegerTokens) return launch_aap_linear_few(c, st);
  const WeightsK a = {c.packed, c.N, c.K, weights_unit(c.packed, c.K)};
  const OutY out = {c.y, c.dtype, c.N, c.scale, c.w_scale, c.bias};
  const int sms = sm_count();
  if (pair_tiles(c.N, c.M, sms)) {
    if (!stages_codes(c.N)) {
      const CodesK<128> b = {c.codes, c.M, c.K, c.ldc, codes_unit(c.codes, c.ldc, c.K)};
      return launch_gemm<WeightsK, CodesK<128>, OutY, 256, 2>(c.N, c.M, c.K, a, b, out, static_cast<float *>(c.workspace), sms,
                                                             wait_status(), Order::kFirst, st);
    }
    cudaError_t e = launch_stage_codes(c.codes, c.ldc, c.M, c.K, c.workspace, st);
    if (e != cudaSuccess) return e;
    Staged b;
    if ((e = tensor_map(&b.map, c.workspace, false, staged_k(c.K), c.M, staged_k(c.K), 1, Staged::X)) != cudaSuccess) return e;
    float *partial = reinterpret_cast<float *>(static_cast<uint8_t *>(c.workspace) + 2 * c.M * staged_k(c.K));
    return launch_gemm<WeightsK, Staged, OutY, 256, 2>(c.N, c.M, c.K, a, b, out, partial, sms, wait_status(), Order::kAfter, st);
  }
  return with_forward_tile(c.M, [&](auto tb) {
    constexpr int TB = decltype(tb)::value;
    const CodesK<TB> b = {c.codes, c.M, c.K, c.ldc, codes_unit(c.codes, c.ldc, c.K)};
    return launch_gemm<WeightsK, CodesK<TB>, OutY, TB, 1>(c.N, c.M, c.K, a, b, out, static_cast<float *>(c.workspace), sms,
                                                         wait_status(), Order::kFirst, st);
  });
}

// The word that a wait without an end would set, in host memory that every device sees: read before the
// next call, so that no call queues a copy behind its kernel.
int *wait_status() {
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
