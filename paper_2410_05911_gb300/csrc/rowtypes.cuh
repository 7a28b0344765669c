// rowtypes.cuh -- the three element types of activations and gradients (float, half, bfloat16) as
// 32-bit values: loads and stores of 16 bytes, or of one element where rows do not start on one.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cstdint>
#include <type_traits>

namespace aecct {

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T>
__device__ __forceinline__ T from_f32(float v) {
  if constexpr (sizeof(T) == 4) return v;
  else if constexpr (std::is_same_v<T, __half>) return __float2half_rn(v);
  else return __float2bfloat16_rn(v);
}
// two values in one 32-bit word, the first in the low half
template <typename T>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  if constexpr (std::is_same_v<T, __half>) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
  } else {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
  }
}
template <typename T>
__device__ __forceinline__ void unpack2(uint32_t w, float &a, float &b) {
  if constexpr (std::is_same_v<T, __half>) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w));
    a = f.x, b = f.y;
  } else {
    a = __uint_as_float(w << 16), b = __uint_as_float(w & 0xFFFF0000u);
  }
}
// pairs of 32-bit values, two operations an instruction
using f32x2 = uint64_t;
__device__ __forceinline__ f32x2 pair(float lo, float hi) {
  f32x2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void unpair(f32x2 v, float &lo, float &hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
// elements in 16 bytes
template <typename T>
constexpr int kVec = 16 / static_cast<int>(sizeof(T));

// V elements at p: one 16-byte load (V = kVec<T>, p on 16 bytes), or a single element (V = 1)
template <typename T, int V>
__device__ __forceinline__ void load_v(const T *p, float *v) {
  if constexpr (V == 1) {
    v[0] = to_f32(*p);
  } else if constexpr (sizeof(T) == 4) {
    const float4 f = *reinterpret_cast<const float4 *>(p);
    v[0] = f.x, v[1] = f.y, v[2] = f.z, v[3] = f.w;
  } else {
    const uint4 u = *reinterpret_cast<const uint4 *>(p);
    unpack2<T>(u.x, v[0], v[1]), unpack2<T>(u.y, v[2], v[3]);
    unpack2<T>(u.z, v[4], v[5]), unpack2<T>(u.w, v[6], v[7]);
  }
}
template <typename T, int V>
__device__ __forceinline__ void store_v(T *p, const float *v) {
  if constexpr (V == 1) *p = from_f32<T>(v[0]);
  else if constexpr (sizeof(T) == 4) *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
  else
    *reinterpret_cast<uint4 *>(p) = make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]),
                                               pack2<T>(v[6], v[7]));
}
// the 16-byte store of values that nothing reads soon
template <typename T>
__device__ __forceinline__ void store_stream(T *p, const float *v) {
  if constexpr (sizeof(T) == 4) __stcs(reinterpret_cast<float4 *>(p), make_float4(v[0], v[1], v[2], v[3]));
  else
    __stcs(reinterpret_cast<uint4 *>(p), make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7])));
}

}  // namespace aecct
