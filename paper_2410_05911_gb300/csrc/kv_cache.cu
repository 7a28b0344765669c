// kv_cache.cu -- keys and values of new tokens into a paged cache, quantised by eq. Quant as they are written, and
// back.
//
//   alpha = max(max_i |x_i|, 2^-100),  code_i = rint(x_i (127 / alpha)),  scale = alpha / 127    (a row of one token and head)
//   value_i = code_i scale
#include <cuda_runtime.h>

#include <cstdint>

#include "aecct_internal.h"
#include "kv_pages.cuh"
#include "rowtypes.cuh"

namespace aecct {

namespace {

constexpr float kAlphaMin = 0x1p-100f;

__device__ __forceinline__ float warp_max(float v) {
  for (int o = 16; o > 0; o >>= 1) {
    const float w = __shfl_xor_sync(0xffffffffu, v, o);
    v = (w > v || w != w) ? w : v;  // (a NaN stays)
  }
  return v;
}

// a warp to a row (of one token, one head, keys or values)
template <typename T, typename C>
__global__ void append_kernel(KvRowsCall c) {
  const int lane = threadIdx.x & 31;
  const int64_t n = c.total * c.cache.heads * 2;
  for (int64_t i = blockIdx.x * int64_t(blockDim.x / 32) + threadIdx.x / 32; i < n; i += int64_t(gridDim.x) * (blockDim.x / 32)) {
    const int which = static_cast<int>(i & 1), h = static_cast<int>((i >> 1) % c.cache.heads);
    const int64_t r = (i >> 1) / c.cache.heads, place = row_place(c.cache, c.seqs, static_cast<int>(r));
    if (place < 0) continue;
    const T *x = static_cast<const T *>(which ? c.v : c.k) + (which ? r * c.v_row + h * c.v_head : r * c.k_row + h * c.k_head);
    const int64_t row = cache_row(c.cache, place, h);
    C *out = static_cast<C *>(which ? c.cache.v : c.cache.k) + row * c.cache.ld;
    if constexpr (sizeof(C) == 1) {
      float m = 0.0f;
      for (int e = lane; e < c.cache.dim; e += 32) {
        const float v = fabsf(to_f32(x[e]));
        m = (v > m || v != v) ? v : m;
      }
      m = warp_max(m);
      const float alpha = m < kAlphaMin ? kAlphaMin : m, by = __fdiv_rn(127.0f, alpha);
      for (int e = lane; e < c.cache.dim; e += 32) out[e] = static_cast<int8_t>(__float2int_rn(__fmul_rn(to_f32(x[e]), by)));
      if (lane == 0) (which ? c.cache.v_scale : c.cache.k_scale)[row] = __fdiv_rn(alpha, 127.0f);
    } else {
      for (int e = lane; e < c.cache.dim; e += 32) out[e] = from_f32<C>(to_f32(x[e]));
    }
  }
}

template <typename C, typename T>
__global__ void read_kernel(KvRowsCall c) {
  const int lane = threadIdx.x & 31;
  const int64_t n = c.total * c.cache.heads * 2;
  for (int64_t i = blockIdx.x * int64_t(blockDim.x / 32) + threadIdx.x / 32; i < n; i += int64_t(gridDim.x) * (blockDim.x / 32)) {
    const int which = static_cast<int>(i & 1), h = static_cast<int>((i >> 1) % c.cache.heads);
    const int64_t r = (i >> 1) / c.cache.heads, place = row_place(c.cache, c.seqs, static_cast<int>(r));
    T *out = static_cast<T *>(which ? c.v_out : c.k_out) + (r * c.cache.heads + h) * c.cache.dim;
    const int64_t row = place < 0 ? 0 : cache_row(c.cache, place, h);
    const C *x = static_cast<const C *>(which ? c.cache.v : c.cache.k) + row * c.cache.ld;
    float scale = 1.0f;
    if constexpr (sizeof(C) == 1) scale = place < 0 ? 0.0f : (which ? c.cache.v_scale : c.cache.k_scale)[row];
    for (int e = lane; e < c.cache.dim; e += 32) {
      float v = 0.0f;
      if (place >= 0) {
        if constexpr (sizeof(C) == 1) v = __fmul_rn(static_cast<float>(x[e]), scale);
        else v = to_f32(x[e]);
      }
      out[e] = from_f32<T>(v);
    }
  }
}

int grid_of(const KvRowsCall &c) {
  const int64_t n = (c.total * c.cache.heads * 2 + 7) / 8, most = 16 * static_cast<int64_t>(sm_count());
  return static_cast<int>(n < most ? n : most);
}

}  // namespace

cudaError_t launch_kv_append(const KvRowsCall &c, cudaStream_t st) {
  const int g = grid_of(c);
  if (c.cache_dtype != 3) {
    if (c.dtype == 1) append_kernel<__half, __half><<<g, 256, 0, st>>>(c);
    else append_kernel<__nv_bfloat16, __nv_bfloat16><<<g, 256, 0, st>>>(c);
  } else if (c.dtype == 0) {
    append_kernel<float, int8_t><<<g, 256, 0, st>>>(c);
  } else if (c.dtype == 1) {
    append_kernel<__half, int8_t><<<g, 256, 0, st>>>(c);
  } else {
    append_kernel<__nv_bfloat16, int8_t><<<g, 256, 0, st>>>(c);
  }
  return cudaGetLastError();
}

namespace {
template <typename C>
void read_as(const KvRowsCall &c, int g, cudaStream_t st) {
  if (c.dtype == 0) read_kernel<C, float><<<g, 256, 0, st>>>(c);
  else if (c.dtype == 1) read_kernel<C, __half><<<g, 256, 0, st>>>(c);
  else read_kernel<C, __nv_bfloat16><<<g, 256, 0, st>>>(c);
}
}  // namespace

cudaError_t launch_kv_read(const KvRowsCall &c, cudaStream_t st) {
  const int g = grid_of(c);
  if (c.cache_dtype == 3) read_as<int8_t>(c, g, st);
  else if (c.cache_dtype == 1) read_as<__half>(c, g, st);
  else read_as<__nv_bfloat16>(c, g, st);
  return cudaGetLastError();
}

}  // namespace aecct
