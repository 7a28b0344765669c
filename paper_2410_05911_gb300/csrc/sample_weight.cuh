// sample_weight.cuh -- the weight of a logit in sample.cu, for the device and for a host compiler.
#pragma once
#include <cmath>
#include <cstdint>
#include <cstring>

#ifdef __CUDACC__
#define AECCT_BOTH __host__ __device__ __forceinline__
#else
#define AECCT_BOTH inline
#endif

namespace aecct {

constexpr int kSteps = 128;  // of the table of powers of two

// 2^-(j / kSteps) as a whole number of 2^-30.  From square roots of 1/2, by Newton's iteration, and their products.
struct PowerTable {
  uint32_t e[kSteps];
  constexpr PowerTable() : e{} {
    double root[7] = {};
    double r = 0.5;
    for (int i = 6; i >= 0; --i) {
      double s = r;
      for (int k = 0; k < 60; ++k) s = 0.5 * (s + r / s);
      root[i] = r = s;  // 2^-(2^i / 128)
    }
    for (int j = 0; j < kSteps; ++j) {
      double v = 1.0;
      for (int i = 0; i < 7; ++i)
        if (j >> i & 1) v *= root[i];
      e[j] = static_cast<uint32_t>(v * 0x1p30 + 0.5);
    }
  }
};

AECCT_BOTH uint32_t float_bits(float v) {
#ifdef __CUDA_ARCH__
  return __float_as_uint(v);
#else
  uint32_t b;
  std::memcpy(&b, &v, 4);
  return b;
#endif
}
AECCT_BOTH float bits_float(uint32_t b) {
#ifdef __CUDA_ARCH__
  return __uint_as_float(b);
#else
  float v;
  std::memcpy(&v, &b, 4);
  return v;
#endif
}

// 2^-(c (top - v)) as a whole number of 2^-44, c in two floats, power(j) the table's j-th entry.  most_off: where weights end.
// Off by less than 2^-28 of itself and a unit.
template <class F>
AECCT_BOTH uint64_t weight_of(float v, float top, float c, float c_low, float most_off, F &&power) {
  // y = c (top - v) in two floats, up to 45 (where the weight ends).  The difference of floats is one as a sum of two (Knuth), for logits of 16 bits
  // too: without what its rounding leaves out, those of 1e-7 under one of 8 would be off by 2^-22.
  const float off = top - v, d = fminf(fmaxf(off, 0.0f), most_off);  // (of infinity under itself, no number: 0, and nothing left out)
  const float y = d * c, t = d - top;
  const float y_low = fmaf(off < most_off ? (top - (d - t)) - (v + t) : 0.0f, c, fmaf(d, c_low, fmaf(d, c, -y)));
  const float j = fmaf(y, static_cast<float>(kSteps), 12582912.0f);  // (1.5 2^23: rounded to a whole number)
  const uint32_t n = float_bits(j);
  const float r = fmaf(j - 12582912.0f, -1.0f / kSteps, y) + y_low;  // |r| < 2^-8 and a little
  // e (2^-r - 1) by the series (to 2^-39), in units of 2^-30, rounded to a whole number; e as a float from its upper 24 bits
  constexpr float kC1 = -0.6931471805599453f * 0x1p30f, kC2 = 0.2402265069591007f * 0x1p30f, kC3 = -0.0555041086648216f * 0x1p30f;
  const uint32_t e = power(n % kSteps);
  const float q = r * fmaf(r, fmaf(r, kC3, kC2), kC1);
  const uint32_t m = e + float_bits(fmaf(bits_float((e >> 6) + (125u << 23)), q, 12582912.0f)) - 0x4b400000u;
  return (static_cast<uint64_t>(m) << 32) >> ((n / kSteps & 63) + 18);  // (n / kSteps <= 45)
}

}  // namespace aecct
