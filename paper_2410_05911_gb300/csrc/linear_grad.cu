// linear_grad.cu -- the gradient of the AAP linear layer's input, and of its bias (linear.cu has the formulas).
#include <cuda_runtime.h>

#include <cstdint>

#include "linear_gemm.cuh"

namespace aecct {

namespace {

constexpr int kSumThreads = 256;

// sums of dy over every gridDim.y-th group of 8 rows: 32 columns a CTA
template <typename T>
__global__ void __launch_bounds__(kSumThreads) bias_grad_kernel(const T *dy, int64_t ld, int64_t M, int64_t N, float *partial) {
  __shared__ float s[8][32];
  const int64_t n = static_cast<int64_t>(blockIdx.x) * 32 + (threadIdx.x & 31);
  const int k = threadIdx.x >> 5;
  float v = 0.0f;
  if (n < N)
    for (int64_t m = static_cast<int64_t>(blockIdx.y) * 8 + k; m < M; m += 8 * static_cast<int64_t>(gridDim.y)) v += to_f32(dy[m * ld + n]);
  s[k][threadIdx.x & 31] = v;
  __syncthreads();
  if (k == 0 && n < N) {
    for (int i = 1; i < 8; ++i) v += s[i][threadIdx.x];
    partial[blockIdx.y * N + n] = v;
  }
}
__global__ void __launch_bounds__(kSumThreads) bias_join_kernel(const float *partial, int parts, int64_t N, float *db) {
  const int64_t n = static_cast<int64_t>(blockIdx.x) * kSumThreads + threadIdx.x;
  if (n >= N) return;
  float v = 0.0f;
  for (int k = 0; k < parts; ++k) v += partial[k * N + n];
  db[n] = v;
}

int bias_parts(int64_t M, int64_t N) {
  const int64_t groups = (M + 63) / 64, columns = (N + 31) / 32, most = (8 * static_cast<int64_t>(sm_count()) + columns - 1) / columns;
  const int64_t p = groups < most ? groups : most;
  return static_cast<int>(p < 1 ? 1 : p > 65535 ? 65535 : p);
}

// j of a single CTA's tile: three pieces of 256 rows would leave room for one stage
template <typename T>
constexpr int kSingle = sizeof(T) == 4 ? 128 : 256;

template <typename T>
cudaError_t input_grad(const AapLinearGradCall &c, float *work, cudaStream_t st) {
  using A = WeightsT<GradK<T, 64>::kBf>;
  const A a = {c.packed, c.N, c.K, weights_unit(c.packed, c.K)};
  const OutX out = {c.dx, c.dtype, c.K, c.w_scale};
  return with_tile<kSingle<T>>(c.K, c.M, [&](auto tb, auto cg) {
    constexpr int TB = decltype(tb)::value, CG = decltype(cg)::value;
    using B = GradK<T, TB / CG>;
    const B b = {static_cast<const T *>(c.dy), c.M, c.lddy, grads_vec<T>(c.dy, c.lddy, c.N)};
    return launch_gemm<A, B, OutX, TB, CG>(c.K, c.M, c.N, a, b, out, work, sm_count(), linear_status(), st);
  });
}

template <typename T>
int64_t input_grad_workspace(int64_t M, int64_t K, int64_t N) {
  return with_tile<kSingle<T>>(K, M, [&](auto tb, auto cg) {
    constexpr int TB = decltype(tb)::value, CG = decltype(cg)::value;
    using B = GradK<T, TB / CG>;
    const GemmPlan p = gemm_plan<WeightsT<B::kBf>, B, TB, CG>(K, M, N, sm_count());
    return p.splits > 1 ? p.splits * M * K : int64_t(0);
  });
}

template <typename T>
cudaError_t bias_grad(const AapLinearGradCall &c, float *work, cudaStream_t st) {
  const int parts = bias_parts(c.M, c.N);
  bias_grad_kernel<T><<<dim3(static_cast<unsigned>((c.N + 31) / 32), parts), kSumThreads, 0, st>>>(static_cast<const T *>(c.dy), c.lddy, c.M, c.N, work);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  bias_join_kernel<<<static_cast<unsigned>((c.N + kSumThreads - 1) / kSumThreads), kSumThreads, 0, st>>>(work, parts, c.N, c.db);
  return cudaGetLastError();
}

}  // namespace

// the three products run one after the other and share the workspace
int64_t aap_linear_grad_workspace(int64_t M, int64_t K, int64_t N, int dtype, int wdtype) {
  const int64_t x = dtype == 0 ? input_grad_workspace<float>(M, K, N) : input_grad_workspace<__half>(M, K, N);
  const int64_t w = weight_grad_workspace(M, K, N, wdtype), b = static_cast<int64_t>(bias_parts(M, N)) * N;
  const int64_t most = x > w ? (x > b ? x : b) : (w > b ? w : b);
  return most * static_cast<int64_t>(sizeof(float));
}

cudaError_t launch_aap_linear_grad(const AapLinearGradCall &c, cudaStream_t st) {
  float *work = static_cast<float *>(c.workspace);
  cudaError_t e = cudaSuccess;
  if (c.dx) e = c.dtype == 0 ? input_grad<float>(c, work, st) : c.dtype == 1 ? input_grad<__half>(c, work, st) : input_grad<__nv_bfloat16>(c, work, st);
  if (e == cudaSuccess && c.dw) e = launch_weight_grad(c, work, st);
  if (e == cudaSuccess && c.db)
    e = c.dtype == 0 ? bias_grad<float>(c, work, st) : c.dtype == 1 ? bias_grad<__half>(c, work, st) : bias_grad<__nv_bfloat16>(c, work, st);
  return e;
}

}  // namespace aecct
