// linear_grad.cu -- the gradients of the AAP linear layer (linear.cu has the formulas): its input's, here, and
// the bias's, on the way of staging or alone; the weights' is in linear_wgrad.cu.
#include <cuda_runtime.h>

#include <cstdint>

#include "linear_gemm.cuh"

namespace aecct {

namespace {

template <typename T>
constexpr int kPieces = sizeof(T) == 4 ? 3 : 1;
template <typename T>
using Staged = Tiled<kPairTile<kPieces<T>> / 2, false, !std::is_same_v<T, __half>, kPieces<T>, 1>;
template <typename T>
using Weights = WeightsT<!std::is_same_v<T, __half>>;

int64_t padded(int64_t n) { return (n + 7) / 8 * 8; }

// 16-bit gradients that TMA reads where they are
template <typename T>
bool in_place(const void *dy, int64_t ld) {
  return sizeof(T) == 2 && (reinterpret_cast<uintptr_t>(dy) & 15u) == 0 && ld % 8 == 0;
}

// Whether 16-bit rows that are not whole 16-byte pieces are laid out as such first: with more than one tile of k each
// tile would put the pieces together again (277 x 1,972 x 3,561: 53 us, staged 38 us; 2,000 x 132 x 1,001: 23 and 22 us).
template <typename T>
bool stages_rows(int64_t K) {
  return sizeof(T) == 2 && K > kTileI;
}

constexpr int64_t kFloat = sizeof(float);

template <typename T>
cudaError_t input_grad(const AapLinearGradCall &c, uint8_t *work, cudaStream_t st) {
  const Weights<T> a = {c.packed, c.N, c.K, weights_unit(c.packed, c.K)};
  const OutX out = {c.dx, c.dtype, c.K, c.w_scale};
  const int sms = sm_count();
  if (grad_pairs<kPieces<T>>(c.K, c.M, c.N, sms)) {
    Staged<T> b;
    const void *rows = c.dy;
    int64_t ld = c.lddy;
    const bool staged = !in_place<T>(c.dy, c.lddy);
    cudaError_t e = cudaSuccess;
    if (staged) {
      rows = work, ld = padded(c.N);
      const StageGrads s = {c.dy, c.lddy, c.M, c.N, c.dtype, nullptr, sizeof(T) == 4 ? 3 : 0, work, nullptr, nullptr, Order::kFirst};
      if ((e = launch_stage_grads(s, st)) != cudaSuccess) return e;
    }
    if ((e = tensor_map(&b.map, rows, Staged<T>::kBf, c.N, c.M, ld, kPieces<T>, Staged<T>::X)) != cudaSuccess) return e;
    float *partial = reinterpret_cast<float *>(work + 2 * kPieces<T> * c.M * padded(c.N));
    return launch_gemm<Weights<T>, Staged<T>, OutX, kPairTile<kPieces<T>>, 2>(c.K, c.M, c.N, a, b, out, partial, sms, wait_status(), staged ? Order::kAfter : Order::kFirst, st);
  }
  const void *dy = c.dy;
  int64_t ld = c.lddy, width = c.N;
  const bool staged = stages_rows<T>(c.K) && !grads_vec<T>(dy, ld, width);
  if (staged) {
    const StageGrads s = {dy, ld, c.M, c.N, c.dtype, nullptr, 0, work, nullptr, nullptr, Order::kFirst};
    const cudaError_t e = launch_stage_grads(s, st);
    if (e != cudaSuccess) return e;
    dy = work, ld = width = padded(c.N), work += up16(2 * c.M * ld);
  }
  return with_single_tile<kPieces<T>>(c.M, [&](auto tb) {
    constexpr int TB = decltype(tb)::value;
    using B = GradK<T, TB>;
    const B b = {static_cast<const T *>(dy), c.M, width, ld, grads_vec<T>(dy, ld, width)};
    return launch_gemm<Weights<T>, B, OutX, TB, 1>(c.K, c.M, c.N, a, b, out, reinterpret_cast<float *>(work), sms, wait_status(), staged ? Order::kAfter : Order::kFirst, st);
  });
}

template <typename T>
int64_t input_grad_workspace(int64_t M, int64_t K, int64_t N, int dtype) {
  const int sms = sm_count();
  if (grad_pairs<kPieces<T>>(K, M, N, sms)) return partial_floats<Weights<T>, Staged<T>, kPairTile<kPieces<T>>, 2>(K, M, N, sms, dtype) * kFloat + 2 * kPieces<T> * M * padded(N);
  return with_single_tile<kPieces<T>>(M, [&](auto tb) {
    constexpr int TB = decltype(tb)::value;
    return partial_floats<Weights<T>, GradK<T, TB>, TB, 1>(K, M, N, sms, dtype) * kFloat + (stages_rows<T>(K) ? up16(2 * M * padded(N)) : 0);
  });
}

int64_t input_part(int64_t M, int64_t K, int64_t N, int dtype) {
  return up16(dtype == 0 ? input_grad_workspace<float>(M, K, N, dtype) : input_grad_workspace<__half>(M, K, N, dtype));
}

}  // namespace

// dX's part, and that of dW and db beside it
int64_t aap_linear_grad_workspace(int64_t M, int64_t K, int64_t N, int dtype, int wdtype) {
  return input_part(M, K, N, dtype) + weight_grad_workspace(M, K, N, wdtype);
}

cudaError_t launch_aap_linear_grad(const AapLinearGradCall &c, cudaStream_t st) {
  uint8_t *work = static_cast<uint8_t *>(c.workspace);
  cudaError_t e = cudaSuccess;
  if (c.dx) e = c.dtype == 0 ? input_grad<float>(c, work, st) : c.dtype == 1 ? input_grad<__half>(c, work, st) : input_grad<__nv_bfloat16>(c, work, st);
  if (e == cudaSuccess && (c.dw || c.db)) e = launch_weight_grad(c, work + input_part(c.M, c.K, c.N, c.dtype), c.dx != nullptr, st);
  return e;
}

}  // namespace aecct
