// clip.cu -- the global norm over every gradient of a model, and the gradients scaled down to it.
//
//   norm = sqrt(sum over all tensors and elements of g^2),  c = min(1, max_norm / (norm + eps)),  out = g c
//
// Two kernels over a table of the tensors, cut into pieces of kPiece elements that the CTAs take in turn.
// The first leaves a sum of squares per CTA: a thread's own in 32 bits over one piece (64 squares), pieces
// and threads joined in 64 bits in a fixed order, so that a norm is the same bits on every run.  The second
// adds those up again in each CTA (a few thousand numbers in L2), so that no third kernel and no copy to the
// host stands between, and scales.
#include <cuda_runtime.h>

#include <cmath>
#include <cstdint>

#include "aecct_internal.h"
#include "rowtypes.cuh"
#include "sm103_ptx.cuh"

namespace aecct {

namespace {

constexpr int kThreads1 = 256;
constexpr int kPer = 64;  // elements of a piece that a thread takes
constexpr int kPiece = kThreads1 * kPer;

template <int N>
struct ClipTable {
  const void *g[N];
  void *out[N];
  int64_t len[N];
  int64_t first[N + 1];  // first piece of tensor j; first[n] = pieces
  uint8_t dtype[N];
  int n;
};

// sum of v over the CTA, in every thread, in a fixed order
__device__ __forceinline__ double cta_sum(double v, double *buf) {
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
  __syncthreads();
  double s = 0.0;
  for (int i = 0; i < kThreads1 / 32; ++i) s += buf[i];
  return s;
}

template <int N>
__device__ __forceinline__ int tensor_of(const ClipTable<N> &t, int64_t piece) {
  int lo = 0, hi = t.n - 1;  // the last tensor whose first piece is at most `piece`
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.first[mid] <= piece) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// sum of squares of a thread's share of elements [0, n) of a piece at p
template <typename T>
__device__ __forceinline__ float square_sum(const T *p, int n) {
  constexpr int V = kVec<T>;
  float s = 0.0f;
  if (n == kPiece && (reinterpret_cast<uintptr_t>(p) & 15u) == 0) {
    constexpr int kStep = 4;  // loads in flight
#pragma unroll 1
    for (int j = 0; j < kPer / V; j += kStep) {
      float v[kStep][V];
#pragma unroll
      for (int u = 0; u < kStep; ++u) load_v<T, V>(p + ((j + u) * kThreads1 + threadIdx.x) * V, v[u]);
#pragma unroll
      for (int u = 0; u < kStep; ++u)
#pragma unroll
        for (int e = 0; e < V; ++e) s = fmaf(v[u][e], v[u][e], s);
    }
  } else {
#pragma unroll 4
    for (int i = threadIdx.x; i < n; i += kThreads1) {
      const float v = to_f32(p[i]);
      s = fmaf(v, v, s);
    }
  }
  return s;
}

template <typename T>
__device__ __forceinline__ void scale_piece(const T *p, T *o, int n, float c) {
  constexpr int V = kVec<T>;
  if (n == kPiece && ((reinterpret_cast<uintptr_t>(p) | reinterpret_cast<uintptr_t>(o)) & 15u) == 0) {
    constexpr int kStep = 4;
#pragma unroll 1
    for (int j = 0; j < kPer / V; j += kStep) {
      float v[kStep][V];
#pragma unroll
      for (int u = 0; u < kStep; ++u) load_v<T, V>(p + ((j + u) * kThreads1 + threadIdx.x) * V, v[u]);
#pragma unroll
      for (int u = 0; u < kStep; ++u) {
#pragma unroll
        for (int e = 0; e < V; ++e) v[u][e] *= c;
        store_v<T, V>(o + ((j + u) * kThreads1 + threadIdx.x) * V, v[u]);
      }
    }
  } else {
#pragma unroll 4
    for (int i = threadIdx.x; i < n; i += kThreads1) o[i] = from_f32<T>(to_f32(p[i]) * c);
  }
}

template <int N>
__global__ void __launch_bounds__(kThreads1) clip_norm_kernel(const __grid_constant__ ClipTable<N> t, double *partial) {
  __shared__ double buf[kThreads1 / 32];
  grid_trigger();
  double sum = 0.0;
  for (int64_t piece = blockIdx.x; piece < t.first[t.n]; piece += gridDim.x) {
    const int j = tensor_of(t, piece);
    const int64_t at = (piece - t.first[j]) * kPiece, left = t.len[j] - at;
    const int n = static_cast<int>(left < kPiece ? left : kPiece);
    if (t.dtype[j] == 0) sum += square_sum(static_cast<const float *>(t.g[j]) + at, n);
    else if (t.dtype[j] == 1) sum += square_sum(static_cast<const __half *>(t.g[j]) + at, n);
    else sum += square_sum(static_cast<const __nv_bfloat16 *>(t.g[j]) + at, n);
  }
  const double s = cta_sum(sum, buf);
  if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

// pieces from the last to the first: what the norm's kernel read last is still in L2
template <int N>
__global__ void __launch_bounds__(kThreads1) clip_scale_kernel(const __grid_constant__ ClipTable<N> t, const double *partial,
                                                               int parts, float max_norm, float eps, float *norm) {
  __shared__ double buf[kThreads1 / 32];
  grid_wait();
  double v = 0.0;
  for (int i = threadIdx.x; i < parts; i += kThreads1) v += partial[i];
  const float nm = static_cast<float>(sqrt(cta_sum(v, buf)));
  const float by = __fdiv_rn(max_norm, nm + eps);
  const float c = by > 1.0f ? 1.0f : by;  // (a norm that is not a number makes every gradient one)
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = nm;
  for (int64_t piece = t.first[t.n] - 1 - blockIdx.x; piece >= 0; piece -= gridDim.x) {
    const int j = tensor_of(t, piece);
    if (c == 1.0f && t.g[j] == t.out[j]) continue;  // in place, and nothing to scale
    const int64_t at = (piece - t.first[j]) * kPiece, left = t.len[j] - at;
    const int n = static_cast<int>(left < kPiece ? left : kPiece);
    if (t.dtype[j] == 0) scale_piece(static_cast<const float *>(t.g[j]) + at, static_cast<float *>(t.out[j]) + at, n, c);
    else if (t.dtype[j] == 1) scale_piece(static_cast<const __half *>(t.g[j]) + at, static_cast<__half *>(t.out[j]) + at, n, c);
    else
      scale_piece(static_cast<const __nv_bfloat16 *>(t.g[j]) + at, static_cast<__nv_bfloat16 *>(t.out[j]) + at, n, c);
  }
}

template <int N>
int fill(ClipTable<N> &t, int j0, int count, const void *const *g, const int64_t *len, const int32_t *dtype, void *const *out) {
  int64_t pieces = 0;
  for (int j = 0; j < count; ++j) {
    t.g[j] = g[j0 + j], t.out[j] = out[j0 + j], t.len[j] = len[j0 + j], t.dtype[j] = static_cast<uint8_t>(dtype[j0 + j]);
    t.first[j] = pieces;
    pieces += (len[j0 + j] + kPiece - 1) / kPiece;
  }
  t.first[count] = pieces;
  t.n = count;
  return static_cast<int>(pieces < kClipMaxBlocks ? (pieces > 0 ? pieces : 1) : kClipMaxBlocks);
}

template <int N>
cudaError_t run_clip(int n, const void *const *g, const int64_t *len, const int32_t *dtype, void *const *out, float max_norm,
                     float eps, float *norm, double *partial, cudaStream_t st) {
  ClipTable<N> t;
  int parts = 0;
  for (int pass = 0; pass < 2; ++pass)
    for (int j0 = 0; j0 < n || (j0 == 0 && n == 0); j0 += N) {
      const int blocks = fill(t, j0, n - j0 < N ? n - j0 : N, g, len, dtype, out);
      cudaError_t e;
      if (pass == 0) {
        clip_norm_kernel<N><<<blocks, kThreads1, 0, st>>>(t, partial + parts);
        e = cudaGetLastError();
        parts += blocks;
      } else {
        e = launch_dependent(clip_scale_kernel<N>, dim3(blocks), kThreads1, 0, st, t, partial, parts, max_norm, eps,
                             j0 == 0 ? norm : static_cast<float *>(nullptr));
      }
      if (e != cudaSuccess) return e;
    }
  return cudaSuccess;
}

}  // namespace

int64_t clip_partials(int n) {
  return static_cast<int64_t>(kClipMaxBlocks) * (n > kClipMaxTensors ? (n + kClipMaxTensors - 1) / kClipMaxTensors : 1);
}

cudaError_t launch_clip_gradients(int n, const void *const *g, const int64_t *len, const int32_t *dtype, void *const *out,
                                  float max_norm, float eps, float *norm, double *partial, cudaStream_t st) {
  if (n <= 64) return run_clip<64>(n, g, len, dtype, out, max_norm, eps, norm, partial, st);
  return run_clip<kClipMaxTensors>(n, g, len, dtype, out, max_norm, eps, norm, partial, st);
}

}  // namespace aecct
