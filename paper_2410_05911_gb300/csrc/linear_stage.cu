// linear_stage.cu -- 16-bit rows for the tensor-core products that copy an operand by TMA (linear_gemm.cuh):
// int8 codes as halves in the order of the unpacked weights, gradients in bfloat16 pieces, times their row's
// scale where the weights' gradient wants it, and, on the way, the sums of the gradients' columns (the bias's
// gradient).  One pass over the operand, bound by its bytes; the tiles of a product then read it many times.
#include <cuda_runtime.h>

#include <cstdint>

#include "linear_gemm.cuh"

namespace aecct {

namespace {

constexpr int kStageThreads = 256;

// codes [M][ld] to halves [M][Kp], Kp a multiple of 128: 64 k of a block's first step, then those of its second
__global__ void __launch_bounds__(kStageThreads) stage_codes_kernel(const int8_t *codes, int64_t ld, int unit, int64_t M, int K, int Kp,
                                                                    __half *out) {
  grid_trigger();
  const int pieces = Kp / 16;  // of 16 codes, 8 to a block
  const int64_t all = M * pieces;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * kStageThreads + threadIdx.x; i < all; i += static_cast<int64_t>(gridDim.x) * kStageThreads) {
    const int64_t m = i / pieces;
    const int c = static_cast<int>(i - m * pieces), left = K - 16 * c;
    uint32_t w[4], o[4];
    load_codes(codes + m * ld + 16 * c, left, unit, codes, codes + (M - 1) * ld + K, w);
    __half *to = out + m * Kp + (c >> 3) * 128 + (c & 7) * 8;
    codes8_half(w[0], w[2], o);
    *reinterpret_cast<uint4 *>(to) = make_uint4(o[0], o[1], o[2], o[3]);
    codes8_half(w[1], w[3], o);
    *reinterpret_cast<uint4 *>(to + 64) = make_uint4(o[0], o[1], o[2], o[3]);
  }
}

// dy [M][ld] to P pieces [P][M][Np] (Np a multiple of 8): dy times scale (NULL: 1) in bfloat16, or 16-bit dy as it is
// (P = 0); and the sums of dy's columns over the CTA's rows to partial[blockIdx.y][N] (NULL: none).  out NULL: the
// sums alone.  A CTA takes 256 columns, 8 a thread, of every gridDim.y-th group of 8 rows.
template <typename T, int P>
__global__ void __launch_bounds__(kStageThreads) stage_grads_kernel(const T *dy, int64_t ld, bool vec, int64_t M, int64_t N, int64_t Np,
                                                                    const float *scale, uint16_t *out, float *partial, Order order) {
  __shared__ float sums[8][256];
  grid_trigger();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t n = static_cast<int64_t>(blockIdx.x) * 256 + 8 * lane;
  const int left = static_cast<int>(N - n < 8 ? N - n : 8);
  float sum[8] = {};
#pragma unroll 4
  for (int64_t m = static_cast<int64_t>(blockIdx.y) * 8 + warp; m < M; m += 8 * static_cast<int64_t>(gridDim.y)) {
    uint32_t w[kWords8<T>];
    float v[8];
    load_grad8<T>(dy + m * ld + n, left, vec, dy, dy + (M - 1) * ld + N, w);
    grad8_f32<T>(w, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] += v[e];
    if (out && n < Np) {
      uint16_t *to = out + m * Np + n;
      if constexpr (P == 0) {
        *reinterpret_cast<uint4 *>(to) = make_uint4(w[0], w[1], w[2], w[3]);
      } else {
        if (scale) {
          const float s = __ldg(scale + m);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] *= s;
        }
        split8<P>(v, [&](int p, const uint32_t (&o)[4]) { *reinterpret_cast<uint4 *>(to + p * M * Np) = make_uint4(o[0], o[1], o[2], o[3]); });
      }
    }
  }
  if (partial) {
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[warp][8 * lane + e] = sum[e];
    __syncthreads();
    const int64_t c = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (c < N) {
      float s = 0.0f;
      for (int k = 0; k < 8; ++k) s += sums[k][threadIdx.x];
      partial[blockIdx.y * N + c] = s;
    }
  }
  if (order == Order::kBeside) grid_wait();
}

template <typename T, int P>
cudaError_t stage_of(const StageGrads &c, cudaStream_t st) {
  const dim3 grid(static_cast<unsigned>((c.N + 255) / 256), static_cast<unsigned>(stage_parts(c.M, c.N)));
  const bool vec = grads_vec<T>(c.dy, c.ld, c.N);
  const int64_t Np = (c.N + 7) / 8 * 8;
  float *partial = !c.db ? nullptr : grid.y == 1 ? c.db : c.partial;
  cudaError_t e;
  if (c.order != Order::kFirst) {
    e = launch_dependent(stage_grads_kernel<T, P>, grid, kStageThreads, 0, st, static_cast<const T *>(c.dy), c.ld, vec, c.M, c.N, Np,
                         c.scale, static_cast<uint16_t *>(c.out), partial, c.order);
  } else {
    stage_grads_kernel<T, P><<<grid, kStageThreads, 0, st>>>(static_cast<const T *>(c.dy), c.ld, vec, c.M, c.N, Np, c.scale,
                                                             static_cast<uint16_t *>(c.out), partial, c.order);
    e = cudaGetLastError();
  }
  if (e != cudaSuccess || !c.db || grid.y == 1) return e;  // (one part is the sum)
  return launch_join_columns(c.partial, static_cast<int>(grid.y), c.N, c.db, st);
}

template <typename T>
cudaError_t stage_of(const StageGrads &c, cudaStream_t st) {
  return c.pieces == 3 ? stage_of<T, 3>(c, st) : c.pieces == 2 ? stage_of<T, 2>(c, st) : stage_of<T, 0>(c, st);
}

}  // namespace

// row groups of a CTA column: eight CTAs an SM, no more than there are rows for
int stage_parts(int64_t M, int64_t N) {
  const int64_t groups = (M + 63) / 64, columns = (N + 255) / 256, most = (8 * static_cast<int64_t>(sm_count()) + columns - 1) / columns;
  const int64_t p = groups < most ? groups : most;
  return static_cast<int>(p < 1 ? 1 : p);
}

cudaError_t launch_stage_codes(const int8_t *codes, int64_t ld, int64_t M, int64_t K, void *out, cudaStream_t st) {
  const int Kp = static_cast<int>(staged_k(K));
  const int64_t blocks = (M * (Kp / 16) + kStageThreads - 1) / kStageThreads, most = static_cast<int64_t>(sm_count()) * 32;
  stage_codes_kernel<<<static_cast<unsigned>(blocks < most ? blocks : most), kStageThreads, 0, st>>>(
      codes, ld, codes_unit(codes, ld, K), M, static_cast<int>(K), Kp, static_cast<__half *>(out));
  return cudaGetLastError();
}

cudaError_t launch_stage_grads(const StageGrads &c, cudaStream_t st) {
  return c.dtype == 0 ? stage_of<float>(c, st) : c.dtype == 1 ? stage_of<__half>(c, st) : stage_of<__nv_bfloat16>(c, st);
}

cudaError_t tensor_map(CUtensorMap *map, const void *base, bool bf, int64_t width, int64_t rows, int64_t ld, int pieces, int box_rows) {
  using Encode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                              const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                              CUtensorMapFloatOOBfill);
  static const Encode encode = [] {
    void *f = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess)
      f = nullptr;
    return reinterpret_cast<Encode>(f);
  }();
  if (!encode) return cudaErrorNotSupported;
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(width), static_cast<cuuint64_t>(rows), static_cast<cuuint64_t>(pieces)};
  const cuuint64_t strides[2] = {static_cast<cuuint64_t>(ld) * 2, static_cast<cuuint64_t>(ld) * 2 * static_cast<cuuint64_t>(rows)};
  const cuuint32_t box[3] = {64, static_cast<cuuint32_t>(box_rows), 1}, step[3] = {1, 1, 1};
  const CUresult r = encode(map, bf ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void *>(base), dims,
                            strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

}  // namespace aecct
