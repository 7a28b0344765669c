// linear_wgrad.cu -- the gradient of the AAP linear layer's weights, dW = sum over tokens of dy scale codes, and
// of its bias (linear.cu has the formulas).  dy scale is no 16-bit number: it goes through the tensor cores in
// bfloat16 pieces, two (16 bits) for a gradient of 16 bits, three (exact) for one of 32.  Two, so that what is cut off
// a term stays under the rounding of the gradient itself, to 8 bits in bfloat16 and 11 in half.  With one piece
// for bfloat16 each term would lose as much as the result: the error of 8,192 x 4,096 x 4,096 in the 2-norm was 2.3e-3 of
// it, where the rounding of the result alone is 1.7e-3, and terms alike kept all of their own 2^-8.  (dW then took 188 us,
// and takes 326 us: the second piece is as much work again.)
#include <cuda_runtime.h>

#include <cstdint>

#include "linear_gemm.cuh"

namespace aecct {

namespace {

int pieces_of(int wdtype) { return wdtype == 0 ? 3 : 2; }

int64_t padded(int64_t n) { return (n + 7) / 8 * 8; }

constexpr int64_t kFloat = sizeof(float);

int64_t sums_bytes(int64_t M, int64_t N) { return up16(static_cast<int64_t>(stage_parts(M, N)) * N * sizeof(float)); }

template <int P>
using Staged = Tiled<kPairTile<P> / 2, true, true, P, 1>;

template <int P>
cudaError_t staged_grad(const AapLinearGradCall &c, uint8_t *work, cudaStream_t st) {
  Staged<P> b;
  const cudaError_t e = tensor_map(&b.map, work, true, c.N, c.M, padded(c.N), P, kStep);
  if (e != cudaSuccess) return e;
  const CodesT a = {c.codes, c.M, c.K, c.ldc, codes_unit(c.codes, c.ldc, c.K)};
  const OutW out = {c.dw, c.wdtype, c.K};
  float *partial = reinterpret_cast<float *>(work + 2 * P * c.M * padded(c.N));
  return launch_gemm<CodesT, Staged<P>, OutW, kPairTile<P>, 2>(c.K, c.N, c.M, a, b, out, partial, sm_count(), wait_status(), Order::kAfter, st);
}

template <typename T, int P>
cudaError_t weight_grad(const AapLinearGradCall &c, uint8_t *work, Order order, cudaStream_t st) {
  const CodesT a = {c.codes, c.M, c.K, c.ldc, codes_unit(c.codes, c.ldc, c.K)};
  const OutW out = {c.dw, c.wdtype, c.K};
  return with_single_tile<P>(c.N, [&](auto tb) {
    constexpr int TB = decltype(tb)::value;
    using B = GradT<T, TB, P>;
    const B b = {static_cast<const T *>(c.dy), c.M, c.N, c.lddy, c.scale, grads_vec<T>(c.dy, c.lddy, c.N)};
    return launch_gemm<CodesT, B, OutW, TB, 1>(c.K, c.N, c.M, a, b, out, reinterpret_cast<float *>(work), sm_count(), wait_status(), order, st);
  });
}

template <typename T>
cudaError_t weight_grad(const AapLinearGradCall &c, uint8_t *work, Order order, cudaStream_t st) {
  return pieces_of(c.wdtype) == 3 ? weight_grad<T, 3>(c, work, order, st) : weight_grad<T, 2>(c, work, order, st);
}

template <int P>
int64_t workspace_of(int64_t M, int64_t K, int64_t N, int wdtype) {
  const int sms = sm_count();
  if (grad_pairs<P>(K, N, M, sms)) return partial_floats<CodesT, Staged<P>, kPairTile<P>, 2>(K, N, M, sms, wdtype) * kFloat + 2 * P * M * padded(N);
  return with_single_tile<P>(N, [&](auto tb) {
    constexpr int TB = decltype(tb)::value;
    return partial_floats<CodesT, GradT<float, TB, P>, TB, 1>(K, N, M, sms, wdtype) * kFloat;
  });
}

}  // namespace

// the column sums, and after them the staged pieces and the splits' sums
int64_t weight_grad_workspace(int64_t M, int64_t K, int64_t N, int wdtype) {
  return sums_bytes(M, N) + (pieces_of(wdtype) == 3 ? workspace_of<3>(M, K, N, wdtype) : workspace_of<2>(M, K, N, wdtype));
}

cudaError_t launch_weight_grad(const AapLinearGradCall &c, uint8_t *work, bool beside, cudaStream_t st) {
  Order order = beside ? Order::kBeside : Order::kFirst;
  const int p = pieces_of(c.wdtype);
  uint8_t *rest = work + sums_bytes(c.M, c.N);
  const int sms = sm_count();
  const bool staged = c.dw && (p == 3 ? grad_pairs<3>(c.K, c.N, c.M, sms) : grad_pairs<2>(c.K, c.N, c.M, sms));
  if (staged || c.db) {
    const StageGrads s = {c.dy, c.lddy, c.M, c.N, c.dtype, c.scale, staged ? p : 0, staged ? rest : nullptr, c.db,
                          reinterpret_cast<float *>(work), order};
    const cudaError_t e = launch_stage_grads(s, st);
    if (e != cudaSuccess) return e;
    order = Order::kBeside;
  }
  if (!c.dw) return cudaSuccess;
  if (staged) return p == 3 ? staged_grad<3>(c, rest, st) : staged_grad<2>(c, rest, st);
  return c.dtype == 0   ? weight_grad<float>(c, rest, order, st)
         : c.dtype == 1 ? weight_grad<__half>(c, rest, order, st)
                        : weight_grad<__nv_bfloat16>(c, rest, order, st);
}

}  // namespace aecct
