// linear.cu -- the AAP linear layer of eq. AAPLinear (Sec. 4.1) on int8 codes and 2-bit weights, any
// shape, and its gradients.
//
//   y[m, n]  = scale_m w_scale sum_k q[m, k] T[n, k] + b_n
//   dx[m, k] = w_scale sum_n dy[m, n] T[n, k]
//   dW[n, k] = sum_m dy[m, n] scale_m q[m, k]      (straight through Ternary)
//   db[n]    = sum_m dy[m, n]
#include <cuda_runtime.h>

#include <cstdint>

#include "aecct_internal.h"
#include "rowtypes.cuh"

namespace aecct {

namespace {

constexpr int kTile = 64, kStep = 16;

__device__ __forceinline__ float ternary(const uint8_t *packed, int64_t i) {
  const uint32_t f = (packed[i >> 2] >> (2 * (i & 3))) & 3u;
  return f == 1u ? 1.0f : f == 3u ? -1.0f : 0.0f;
}

// out(i, j) = sum over r of a(i, r) b(j, r), for i < I, j < J, r < R
template <class A, class B, class Out>
__global__ void __launch_bounds__(256) product_kernel(const int64_t I, const int64_t J, const int64_t R, const A a, const B b,
                                                      const Out out) {
  __shared__ float sa[kStep][kTile + 1], sb[kStep][kTile + 1];
  const int64_t i0 = static_cast<int64_t>(blockIdx.x) * kTile, j0 = static_cast<int64_t>(blockIdx.y) * kTile;
  const int ti = threadIdx.x & 15, tj = threadIdx.x >> 4;
  float acc[4][4] = {};
  for (int64_t r0 = 0; r0 < R; r0 += kStep) {
    for (int e = threadIdx.x; e < kTile * kStep; e += 256) {
      const int x = e / kStep, r = e % kStep;
      sa[r][x] = i0 + x < I && r0 + r < R ? a(i0 + x, r0 + r) : 0.0f;
      sb[r][x] = j0 + x < J && r0 + r < R ? b(j0 + x, r0 + r) : 0.0f;
    }
    __syncthreads();
    for (int r = 0; r < kStep; ++r)
      for (int x = 0; x < 4; ++x)
        for (int y = 0; y < 4; ++y) acc[x][y] = fmaf(sa[r][ti + 16 * x], sb[r][tj + 16 * y], acc[x][y]);
    __syncthreads();
  }
  for (int x = 0; x < 4; ++x)
    for (int y = 0; y < 4; ++y)
      if (i0 + ti + 16 * x < I && j0 + tj + 16 * y < J) out(i0 + ti + 16 * x, j0 + tj + 16 * y, acc[x][y]);
}

template <class A, class B, class Out>
cudaError_t product(int64_t I, int64_t J, int64_t R, const A &a, const B &b, const Out &out, cudaStream_t st) {
  if (I == 0 || J == 0) return cudaSuccess;
  const dim3 grid(static_cast<unsigned>((I + kTile - 1) / kTile), static_cast<unsigned>((J + kTile - 1) / kTile));
  product_kernel<<<grid, 256, 0, st>>>(I, J, R, a, b, out);
  return cudaGetLastError();
}

struct Codes {  // (row, k)
  const int8_t *q;
  int64_t ld;
  __device__ float operator()(int64_t m, int64_t k) const { return static_cast<float>(q[m * ld + k]); }
};
struct CodesT {  // (k, row)
  const int8_t *q;
  int64_t ld;
  __device__ float operator()(int64_t k, int64_t m) const { return static_cast<float>(q[m * ld + k]); }
};
struct Weights {  // (n, k)
  const uint8_t *p;
  int64_t K;
  __device__ float operator()(int64_t n, int64_t k) const { return ternary(p, n * K + k); }
};
struct WeightsT {  // (k, n)
  const uint8_t *p;
  int64_t K;
  __device__ float operator()(int64_t k, int64_t n) const { return ternary(p, n * K + k); }
};
template <typename T>
struct Grad {  // (m, n)
  const T *dy;
  int64_t ld;
  __device__ float operator()(int64_t m, int64_t n) const { return to_f32(dy[m * ld + n]); }
};
template <typename T>
struct GradT {  // (n, m), scaled
  const T *dy;
  int64_t ld;
  const float *scale;
  __device__ float operator()(int64_t n, int64_t m) const { return to_f32(dy[m * ld + n]) * scale[m]; }
};
template <typename T>
struct PutY {
  T *y;
  int64_t N;
  const float *scale, *w_scale, *bias;
  __device__ void operator()(int64_t n, int64_t m, float v) const {
    const float s = v * (scale[m] * *w_scale);
    y[m * N + n] = from_f32<T>(bias ? s + bias[n] : s);
  }
};
template <typename T>
struct Put {  // (column, row)
  T *o;
  int64_t ld;
  const float *by;
  __device__ void operator()(int64_t c, int64_t r, float v) const { o[r * ld + c] = from_f32<T>(by ? v * *by : v); }
};

template <typename T>
__global__ void bias_grad_kernel(const T *dy, int64_t ld, int64_t M, int64_t N, float *db) {
  const int64_t n = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
  if (n >= N) return;
  float s = 0.0f;
  for (int64_t m = 0; m < M; ++m) s += to_f32(dy[m * ld + n]);
  db[n] = s;
}

template <typename T>
cudaError_t linear_of(const AapLinearCall &c, cudaStream_t st) {
  return product(c.N, c.M, c.K, Weights{c.packed, c.K}, Codes{c.codes, c.ldc},
                 PutY<T>{static_cast<T *>(c.y), c.N, c.scale, c.w_scale, c.bias}, st);
}

template <typename T, typename W>
cudaError_t grad_of(const AapLinearGradCall &c, cudaStream_t st) {
  const T *dy = static_cast<const T *>(c.dy);
  cudaError_t e = cudaSuccess;
  if (c.dx) e = product(c.K, c.M, c.N, WeightsT{c.packed, c.K}, Grad<T>{dy, c.lddy}, Put<T>{static_cast<T *>(c.dx), c.K, c.w_scale}, st);
  if (e == cudaSuccess && c.dw)
    e = product(c.K, c.N, c.M, CodesT{c.codes, c.ldc}, GradT<T>{dy, c.lddy, c.scale}, Put<W>{static_cast<W *>(c.dw), c.K, nullptr}, st);
  if (e == cudaSuccess && c.db) {
    bias_grad_kernel<T><<<static_cast<unsigned>((c.N + 63) / 64), 64, 0, st>>>(dy, c.lddy, c.M, c.N, c.db);
    e = cudaGetLastError();
  }
  return e;
}

template <typename T>
cudaError_t grad_of(const AapLinearGradCall &c, cudaStream_t st) {
  return c.wdtype == 0 ? grad_of<T, float>(c, st) : c.wdtype == 1 ? grad_of<T, __half>(c, st) : grad_of<T, __nv_bfloat16>(c, st);
}

}  // namespace

int64_t aap_linear_workspace(int64_t, int64_t, int64_t) { return 0; }
int64_t aap_linear_grad_workspace(int64_t, int64_t, int64_t, int, int) { return 0; }

cudaError_t launch_aap_linear(const AapLinearCall &c, cudaStream_t st) {
  return c.dtype == 0 ? linear_of<float>(c, st) : c.dtype == 1 ? linear_of<__half>(c, st) : linear_of<__nv_bfloat16>(c, st);
}

cudaError_t launch_aap_linear_grad(const AapLinearGradCall &c, cudaStream_t st) {
  return c.dtype == 0 ? grad_of<float>(c, st) : c.dtype == 1 ? grad_of<__half>(c, st) : grad_of<__nv_bfloat16>(c, st);
}

}  // namespace aecct
