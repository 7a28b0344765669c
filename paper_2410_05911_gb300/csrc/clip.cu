// clip.cu -- the global norm over every gradient of a model, and the gradients scaled down to it.
//
//   norm = sqrt(sum over all tensors and elements of g^2),  c = min(1, max_norm / (norm + eps)),  out = g c
//
// Two kernels over a table of the tensors, cut into pieces that the CTAs take in turn: of 64 elements a thread, of
// 16 where those leave SMs idle (160 tensors of 2 M elements: a piece's four rounds of loads, one after the other, were most
// of 12 us).  The first leaves a sum of squares per CTA: a thread's own in 32 bits over one piece (64 squares at
// most), pieces and threads joined in pairs of them in a fixed order, so that a norm is the same bits on every run.  The second
// adds those up again in each CTA (a few thousand numbers in L2), so that no third kernel and no copy to the
// host stands between, and scales.
//
// Bound by memory.  What the chip's L2 does not hold is read twice: the floor is two reads and a write of it, one and one
// of the rest.  302 M elements, most of them in bfloat16, take 270 us (1.2 GB read and written, and 0.5 GB of it read again);
// the 160 tensors of a ten-layer decoder, 2 M elements in float32, 7.2 us: two launches and their trips to memory.
#include <cuda_runtime.h>

#include <climits>
#include <cmath>
#include <cstdint>

#include "aecct_internal.h"
#include "rowtypes.cuh"
#include "sm103_ptx.cuh"

namespace aecct {

namespace {

constexpr int kThreads1 = 256;
constexpr int64_t kKeepBytes = 80 << 20;  // of the last pieces, in L2 (129 MB) until the second kernel reads them
constexpr int kLong = 64, kShort = 16;  // elements of a piece that a thread takes

constexpr int kMapped = 1024;

// A kernel's parameters are read through the constant cache, cold in every SM: the tensor of a piece from a map is one
// miss, a search over `first` is a chain of eight.
template <int N>
struct ClipTable {
  const void *g[N];
  void *out[N];
  int64_t len[N];
  int32_t first[N + 1];  // first piece of tensor j; first[n] = pieces
  uint8_t dtype[N];
  uint16_t of[kMapped];  // tensor of a piece, where there are no more than kMapped
  int n, kept;           // kept: the first piece that is to stay in L2
};

// Sums go from 32 to 64 bits as pairs of floats (a sum and the rounding error of it, Knuth's two-sum): operations in 64 bits
// run at a sixty-fourth of the rate here, and a CTA's worth of them took longer than its loads.
struct Pair {
  float hi, lo;
};
__device__ __forceinline__ Pair add(Pair a, Pair b) {
  const float s = a.hi + b.hi, t = s - a.hi;
  const float e = ((a.hi - (s - t)) + (b.hi - t)) + (a.lo + b.lo);
  return {s, fabsf(s) < INFINITY ? e : 0.0f};  // (an infinity stays one)
}
__device__ __forceinline__ Pair warp_sum(Pair v) {
  for (int o = 16; o > 0; o >>= 1) {
    const Pair w = {__shfl_xor_sync(0xffffffffu, v.hi, o), __shfl_xor_sync(0xffffffffu, v.lo, o)};
    v = add(v, w);
  }
  return v;
}
// sum of v over the CTA, in thread 0, in a fixed order
__device__ __forceinline__ Pair cta_sum(Pair v, Pair *buf) {
  v = warp_sum(v);
  if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
  __syncthreads();
  Pair s = {0.0f, 0.0f};
  if (threadIdx.x < 32) s = warp_sum(threadIdx.x < kThreads1 / 32 ? buf[threadIdx.x] : s);
  return s;
}

template <int N>
__device__ __forceinline__ int tensor_of(const ClipTable<N> &t, int piece) {
  if (t.first[t.n] <= kMapped) return t.of[piece];
  int lo = 0, hi = t.n - 1;  // the last tensor whose first piece is at most `piece`
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.first[mid] <= piece) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// L2's policy for what the second kernel will read next, and for what passes through
__device__ __forceinline__ uint64_t keep_policy() {
  uint64_t p;
  asm("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(p));
  return p;
}
__device__ __forceinline__ uint64_t pass_policy() {
  uint64_t p;
  asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(p));
  return p;
}
template <typename T>
__device__ __forceinline__ void load_hint(const T *p, uint64_t policy, float *v) {
  uint32_t w[4];
  asm volatile("ld.global.L1::no_allocate.L2::cache_hint.v4.b32 {%0, %1, %2, %3}, [%4], %5;"
               : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
               : "l"(p), "l"(policy));
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(w[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) unpack2<T>(w[i], v[2 * i], v[2 * i + 1]);
  }
}

// sum of squares of a thread's share of elements [0, n) of a piece at p
template <typename T, int kPer>
__device__ __forceinline__ float square_sum(const T *p, int n, uint64_t policy) {
  constexpr int V = kVec<T>;
  float s = 0.0f;
  if (n == kPer * kThreads1 && (reinterpret_cast<uintptr_t>(p) & 15u) == 0) {
    constexpr int kStep = kPer / V < 4 ? kPer / V : 4;  // loads in flight
#pragma unroll 1
    for (int j = 0; j < kPer / V; j += kStep) {
      float v[kStep][V];
#pragma unroll
      for (int u = 0; u < kStep; ++u) load_hint<T>(p + ((j + u) * kThreads1 + threadIdx.x) * V, policy, v[u]);
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

template <typename T, int kPer>
__device__ __forceinline__ void scale_piece(const T *p, T *o, int n, float c, uint64_t policy) {
  constexpr int V = kVec<T>;
  if (n == kPer * kThreads1 && ((reinterpret_cast<uintptr_t>(p) | reinterpret_cast<uintptr_t>(o)) & 15u) == 0) {
    constexpr int kStep = kPer / V < 4 ? kPer / V : 4;
#pragma unroll 1
    for (int j = 0; j < kPer / V; j += kStep) {
      float v[kStep][V];
#pragma unroll
      for (int u = 0; u < kStep; ++u) load_hint<T>(p + ((j + u) * kThreads1 + threadIdx.x) * V, policy, v[u]);
#pragma unroll
      for (int u = 0; u < kStep; ++u) {
#pragma unroll
        for (int e = 0; e < V; ++e) v[u][e] *= c;
        store_stream<T>(o + ((j + u) * kThreads1 + threadIdx.x) * V, v[u]);
      }
    }
  } else {
#pragma unroll 4
    for (int i = threadIdx.x; i < n; i += kThreads1) o[i] = from_f32<T>(to_f32(p[i]) * c);
  }
}

template <int N, int PER>
__global__ void __launch_bounds__(kThreads1) clip_norm_kernel(const __grid_constant__ ClipTable<N> t, float2 *partial) {
  constexpr int kPiece = PER * kThreads1;
  __shared__ Pair buf[kThreads1 / 32];
  grid_trigger();
  Pair sum = {0.0f, 0.0f};
  const uint64_t keep = keep_policy(), pass = pass_policy();
  for (int piece = blockIdx.x; piece < t.first[t.n]; piece += gridDim.x) {
    const int j = tensor_of(t, piece);
    const int64_t at = static_cast<int64_t>(piece - t.first[j]) * kPiece, left = t.len[j] - at;
    const int n = static_cast<int>(left < kPiece ? left : kPiece);
    float q;
    if (t.dtype[j] == 0) q = square_sum<float, PER>(static_cast<const float *>(t.g[j]) + at, n, piece >= t.kept ? keep : pass);
    else if (t.dtype[j] == 1) q = square_sum<__half, PER>(static_cast<const __half *>(t.g[j]) + at, n, piece >= t.kept ? keep : pass);
    else q = square_sum<__nv_bfloat16, PER>(static_cast<const __nv_bfloat16 *>(t.g[j]) + at, n, piece >= t.kept ? keep : pass);
    sum = add(sum, {q, 0.0f});
  }
  const Pair s = cta_sum(sum, buf);
  if (threadIdx.x == 0) partial[blockIdx.x] = make_float2(s.hi, s.lo);
}

// pieces from the last to the first: what the norm's kernel read last is still in L2
template <int N, int PER>
__global__ void __launch_bounds__(kThreads1) clip_scale_kernel(const __grid_constant__ ClipTable<N> t, const float2 *partial,
                                                               int parts, float max_norm, float eps, float *norm) {
  constexpr int kPiece = PER * kThreads1;
  __shared__ Pair buf[kThreads1 / 32];
  __shared__ float factor;
  grid_wait();
  Pair v = {0.0f, 0.0f};
  for (int i = threadIdx.x; i < parts; i += kThreads1) v = add(v, {partial[i].x, partial[i].y});
  v = cta_sum(v, buf);
  if (threadIdx.x == 0) {
    const float nm = __fsqrt_rn(v.hi + v.lo), by = __fdiv_rn(max_norm, nm + eps);
    factor = by > 1.0f ? 1.0f : by;  // (a norm that is not a number makes every gradient one)
    if (norm && blockIdx.x == 0) *norm = nm;
  }
  __syncthreads();
  const float c = factor;
  const uint64_t pass = pass_policy();
  for (int piece = t.first[t.n] - 1 - static_cast<int>(blockIdx.x); piece >= 0; piece -= gridDim.x) {
    const int j = tensor_of(t, piece);
    if (c == 1.0f && t.g[j] == t.out[j]) continue;  // in place, and nothing to scale
    const int64_t at = static_cast<int64_t>(piece - t.first[j]) * kPiece, left = t.len[j] - at;
    const int n = static_cast<int>(left < kPiece ? left : kPiece);
    if (t.dtype[j] == 0) scale_piece<float, PER>(static_cast<const float *>(t.g[j]) + at, static_cast<float *>(t.out[j]) + at, n, c, pass);
    else if (t.dtype[j] == 1) scale_piece<__half, PER>(static_cast<const __half *>(t.g[j]) + at, static_cast<__half *>(t.out[j]) + at, n, c, pass);
    else
      scale_piece<__nv_bfloat16, PER>(static_cast<const __nv_bfloat16 *>(t.g[j]) + at, static_cast<__nv_bfloat16 *>(t.out[j]) + at, n, c, pass);
  }
}

// tensors j0 .. j0 + count - 1 of a call; returns the CTAs of a launch over them, 0 for more pieces than a launch numbers
template <int N>
int fill(ClipTable<N> &t, int j0, int count, int piece, const void *const *g, const int64_t *len, const int32_t *dtype, void *const *out) {
  int64_t pieces = 0;
  for (int j = 0; j < count; ++j) {
    t.g[j] = g[j0 + j], t.out[j] = out[j0 + j], t.len[j] = len[j0 + j], t.dtype[j] = static_cast<uint8_t>(dtype[j0 + j]);
    t.first[j] = static_cast<int32_t>(pieces);
    pieces += (len[j0 + j] + piece - 1) / piece;
    if (pieces > INT32_MAX / 2) return 0;
  }
  t.first[count] = static_cast<int32_t>(pieces);
  t.n = count;
  t.kept = 0;
  int64_t room = kKeepBytes;
  for (int j = count - 1; j >= 0 && t.kept == 0; --j) {
    const int64_t each = static_cast<int64_t>(piece) * (t.dtype[j] == 0 ? 4 : 2), mine = t.first[j + 1] - t.first[j];
    if (mine * each > room) t.kept = t.first[j + 1] - static_cast<int32_t>(room / each);
    room -= mine * each;
  }
  if (pieces <= kMapped)
    for (int j = 0; j < count; ++j)
      for (int k = t.first[j]; k < t.first[j + 1]; ++k) t.of[k] = static_cast<uint16_t>(j);
  return static_cast<int>(pieces < kClipMaxBlocks ? (pieces > 0 ? pieces : 1) : kClipMaxBlocks);
}

template <int N, int PER>
cudaError_t run_clip(int n, const void *const *g, const int64_t *len, const int32_t *dtype, void *const *out, float max_norm,
                     float eps, float *norm, float2 *partial, cudaStream_t st) {
  ClipTable<N> t;
  int parts = 0, blocks = 0;
  for (int pass = 0; pass < 2; ++pass)
    for (int j0 = 0; j0 < n || (j0 == 0 && n == 0); j0 += N) {
      if (pass == 0 || n > N) blocks = fill(t, j0, n - j0 < N ? n - j0 : N, PER * kThreads1, g, len, dtype, out);
      if (blocks == 0) return cudaErrorInvalidValue;
      cudaError_t e;
      if (pass == 0) {
        clip_norm_kernel<N, PER><<<blocks, kThreads1, 0, st>>>(t, partial + parts);
        e = cudaGetLastError();
        parts += blocks;
      } else {
        e = launch_dependent(clip_scale_kernel<N, PER>, dim3(blocks), kThreads1, 0, st, t, partial, parts, max_norm, eps,
                             j0 == 0 ? norm : static_cast<float *>(nullptr));
      }
      if (e != cudaSuccess) return e;
    }
  return cudaSuccess;
}

template <int PER>
cudaError_t clip_of(int n, const void *const *g, const int64_t *len, const int32_t *dtype, void *const *out, float max_norm, float eps,
                    float *norm, float2 *partial, cudaStream_t st) {
  // (a launch carries its table: 4 KB for 64 tensors, 8 KB for 192, 17 KB for 512)
  if (n <= 64) return run_clip<64, PER>(n, g, len, dtype, out, max_norm, eps, norm, partial, st);
  if (n <= 192) return run_clip<192, PER>(n, g, len, dtype, out, max_norm, eps, norm, partial, st);
  return run_clip<kClipMaxTensors, PER>(n, g, len, dtype, out, max_norm, eps, norm, partial, st);
}

}  // namespace

int64_t clip_partials(int n) {
  return static_cast<int64_t>(kClipMaxBlocks) * (n > kClipMaxTensors ? (n + kClipMaxTensors - 1) / kClipMaxTensors : 1);
}

cudaError_t launch_clip_gradients(int n, const void *const *g, const int64_t *len, const int32_t *dtype, void *const *out,
                                  float max_norm, float eps, float *norm, float2 *partial, cudaStream_t st) {
  int64_t all = 0;
  for (int j = 0; j < n; ++j) all += len[j];
  if (all < static_cast<int64_t>(kLong) * kThreads1 * 4 * sm_count())
    return clip_of<kShort>(n, g, len, dtype, out, max_norm, eps, norm, partial, st);
  return clip_of<kLong>(n, g, len, dtype, out, max_norm, eps, norm, partial, st);
}

}  // namespace aecct
