// attend.cu -- one new token of each sequence over its keys and values in a paged cache.
//
//   s_j = scale sum_i q_i k_ji,  out = sum_j exp(s_j - m) v_j / l,  m = max_j s_j,  l = sum_j exp(s_j - m)
//
// One pass over the keys with the running maximum and sum: where a new maximum m' comes, what was summed is multiplied by
// exp(m - m').
#include <cuda_runtime.h>

#include <cmath>
#include <cstdint>

#include "aecct_internal.h"
#include "kv_pages.cuh"
#include "rowtypes.cuh"

namespace aecct {

namespace {

template <typename C>
__device__ __forceinline__ float element_of(const C *p) {
  if constexpr (sizeof(C) == 1) return static_cast<float>(*p);
  else return to_f32(*p);
}

// a warp to a query head
template <typename T, typename C>
__global__ void attend_kernel(AttendCall c) {
  constexpr int E = kCacheMaxDim / 32;
  const int lane = threadIdx.x & 31, dim = c.cache.dim;
  const int64_t i = blockIdx.x * int64_t(blockDim.x / 32) + threadIdx.x / 32;
  if (i >= static_cast<int64_t>(c.seqs.batch) * c.q_heads) return;
  const int b = static_cast<int>(i / c.q_heads), head = static_cast<int>(i % c.q_heads), h = head / (c.q_heads / c.cache.heads);
  float q[E], acc[E], m = -INFINITY, l = 0.0f;
  for (int e = 0; e < E; ++e) {
    const int at = e * 32 + lane;
    q[e] = at < dim ? to_f32((static_cast<const T *>(c.q) + b * c.ld_row + head * c.ld_head)[at]) : 0.0f, acc[e] = 0.0f;
  }
  const int n = sequence_length(c.seqs, b, c.cache.page_size);
  for (int p = c.first && c.first[b] > 0 ? c.first[b] : 0; p < n; ++p) {
    const int64_t place = token_place(c.cache, c.seqs, b, p);
    if (place < 0) continue;
    const int64_t row = cache_row(c.cache, place, h);
    const C *k = static_cast<const C *>(c.cache.k) + row * c.cache.ld, *v = static_cast<const C *>(c.cache.v) + row * c.cache.ld;
    float s = 0.0f;
    for (int e = 0; e < E; ++e)
      if (e * 32 + lane < dim) s = fmaf(q[e], element_of(k + e * 32 + lane), s);
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    float vs = 1.0f;
    if constexpr (sizeof(C) == 1) s *= c.cache.k_scale[row], vs = c.cache.v_scale[row];
    s *= c.scale;
    const float top = fmaxf(m, s), old = top == -INFINITY ? 1.0f : expf(m - top), w = top == -INFINITY ? 0.0f : expf(s - top);
    m = top, l = fmaf(l, old, w);
    for (int e = 0; e < E; ++e)
      if (e * 32 + lane < dim) acc[e] = fmaf(acc[e], old, w * vs * element_of(v + e * 32 + lane));
  }
  T *out = static_cast<T *>(c.out) + i * dim;
  for (int e = 0; e < E; ++e)
    if (e * 32 + lane < dim) out[e * 32 + lane] = from_f32<T>(l == 0.0f ? 0.0f : __fdiv_rn(acc[e], l));
  if (c.lse && lane == 0) c.lse[i] = m + logf(l);
}

template <typename T, typename C>
cudaError_t launch(const AttendCall &c, cudaStream_t st) {
  attend_kernel<T, C><<<static_cast<unsigned>((static_cast<int64_t>(c.seqs.batch) * c.q_heads + 3) / 4), 128, 0, st>>>(c);
  return cudaGetLastError();
}

}  // namespace

int64_t attend_workspace(int, int, int, int, int, int) { return 0; }

cudaError_t launch_attend(const AttendCall &c, cudaStream_t st) {
  if (c.cache_dtype == 1) return launch<__half, __half>(c, st);
  if (c.cache_dtype == 2) return launch<__nv_bfloat16, __nv_bfloat16>(c, st);
  if (c.dtype == 0) return launch<float, int8_t>(c, st);
  if (c.dtype == 1) return launch<__half, int8_t>(c, st);
  return launch<__nv_bfloat16, int8_t>(c, st);
}

}  // namespace aecct
