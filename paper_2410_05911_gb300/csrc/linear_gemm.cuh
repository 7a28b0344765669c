// linear_gemm.cuh -- the tensor-core product behind the AAP linear layer and its gradients:
//
//   out(j, i) = sum over r of A(i, r) B(j, r),   i < I, j < J, r < R
//
// with 16-bit operands that no memory holds: int8 codes, 2-bit weights and scaled gradients become half or
// bfloat16 core matrices on their way from global to shared memory, in the registers of producer warps, and
// tcgen05.mma multiplies them there (32-bit accumulators in tensor memory).  Reading 1 byte a code and
// a quarter of one a weight keeps L2 traffic under what 16-bit operands would need, and no pass over memory
// lays operands out before the product.
//
// One CTA makes a tile of 128 i by TB j.  Eight producer warps load kStep = 64 of r a step ahead, convert and
// store; a ninth warp issues the MMAs.  Lanes hold consecutive i in tensor memory, so that the epilogue's
// stores of one j are 32 neighbouring elements.  Two CTAs share an SM where their operands fit, one's
// epilogue behind the other's products.
//
// Operand tiles are 8 x 16-byte core matrices without swizzle: element (x, r) of a K-major tile (16 bytes
// along r) at (x / 8) 1024 + (r / 8) 128 + (x % 8) 16 + (r % 8) 2, of an MN-major tile (16 bytes along x) at
// (x / 8) 1024 + (r / 8) 128 + (r % 8) 16 + (x % 8) 2.  In both, core matrices along r are 128 bytes
// apart and those along x 1024, and eight lanes that hold eight consecutive rows of the source store
// 128 consecutive bytes.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

#include "aecct_internal.h"
#include "rowtypes.cuh"
#include "sm103_ptx.cuh"

namespace aecct {

constexpr int kStep = 64;           // r per stage
constexpr int kTileI = 128;         // i per CTA: the lanes of tensor memory
constexpr int kProducerWarps = 8;
constexpr int kProducers = kProducerWarps * 32;
constexpr int kGemmThreads = kProducers + 32;
constexpr uint32_t kTileABytes = kTileI * kStep * 2;
constexpr long long kGemmWaitCycles = 1ll << 32;  // a wait that takes longer (about 2 s) has lost its arrival

// instruction descriptor of kind::f16: 32-bit accumulators; BF: bfloat16 operands, else half; MN: both
// operands' 16-byte rows run along i and j
__host__ __device__ constexpr uint32_t gemm_idesc(bool bf, bool mn_a, bool mn_b, uint32_t n) {
  return (1u << 4) | (bf ? (1u << 7) | (1u << 10) : 0u) | (mn_a ? 1u << 15 : 0u) | (mn_b ? 1u << 16 : 0u) | ((n >> 3) << 17) |
         ((128u >> 4) << 24);
}

__device__ __forceinline__ void st_shared16(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

// ----------------------------------------------------------------------------- conversions
// 16 weights of 2 bits (00 = 0, 01 = +1, 11 = -1) as 16-bit floats of twice their value, 0 and +-2: their
// low bytes are zero in half and in bfloat16 alike, so that one byte permutation makes two of them, with
// the codes as selectors into a table of high bytes.  Position 4 p + b of the 16 holds weight 4 b + p
// (field p of byte b); mix16 is that order.
__host__ __device__ constexpr int mix16(int pos) { return ((pos & 3) << 2) | (pos >> 2); }
__device__ __forceinline__ void weights16(uint32_t w, uint32_t (&o)[8]) {
  constexpr uint32_t table = 0xC0004000u;
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    const uint32_t s = (p < 2 ? w << (4 - 2 * p) : w >> (2 * p - 4)) & 0x30303030u;
    o[2 * p] = __byte_perm(table, 0, s & 0xFFFFu);
    o[2 * p + 1] = __byte_perm(table, 0, s >> 16);
  }
}
// 16 int8 codes as halves in the order of mix16: (code + 128) in the low byte of 1024, less 1152
__device__ __forceinline__ void codes16_half_mixed(const uint32_t (&b)[4], uint32_t (&o)[8]) {
#pragma unroll
  for (int p = 0; p < 4; ++p)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t t = __byte_perm(b[2 * h], b[2 * h + 1], 0x0400u + 0x0101u * p);
      const uint32_t u = (t & 0x00FF00FFu) ^ 0x64806480u;
      const __half2 v = __hsub2(*reinterpret_cast<const __half2 *>(&u), __half2{__ushort_as_half(0x6480), __ushort_as_half(0x6480)});
      o[2 * p + h] = *reinterpret_cast<const uint32_t *>(&v);
    }
}
// 4 int8 codes as bfloat16, in order: the low 7 bits in the mantissa of 128, less 128, or 256 for a negative one
__device__ __forceinline__ void codes4_bf16(uint32_t b, uint32_t &o0, uint32_t &o1) {
  const uint32_t t0 = __byte_perm(b, 0x43434343u, 0x4140), t1 = __byte_perm(b, 0x43434343u, 0x4342);
  auto sub = [](uint32_t t) {
    const uint32_t v = t & 0xFF7FFF7Fu, c = t & 0xFF80FF80u;
    const __nv_bfloat162 d = __hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&v), *reinterpret_cast<const __nv_bfloat162 *>(&c));
    return *reinterpret_cast<const uint32_t *>(&d);
  };
  o0 = sub(t0), o1 = sub(t1);
}
// 8 values in 32 bits as P bfloat16 pieces each, the largest first: rounded where there is one; else each piece
// cuts off 8 bits and the next takes what is left, so that three hold a 32-bit value exactly.  An infinity
// stays one in its first piece, and its others are zero.
template <int P>
__device__ __forceinline__ void split8(const float (&v)[8], uint32_t addr, uint32_t piece_bytes) {
  if constexpr (P == 1) {
    st_shared16(addr, pack2<__nv_bfloat16>(v[0], v[1]), pack2<__nv_bfloat16>(v[2], v[3]), pack2<__nv_bfloat16>(v[4], v[5]),
                pack2<__nv_bfloat16>(v[6], v[7]));
  } else {
    uint32_t x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = v[e] == v[e] ? __float_as_uint(v[e]) : 0x7FC00000u;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      st_shared16(addr + p * piece_bytes, __byte_perm(x[0], x[1], 0x7632), __byte_perm(x[2], x[3], 0x7632),
                  __byte_perm(x[4], x[5], 0x7632), __byte_perm(x[6], x[7], 0x7632));
      if (p + 1 < P) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float top = __uint_as_float(x[e] & 0xFFFF0000u);
          x[e] = fabsf(top) < INFINITY ? __float_as_uint(__uint_as_float(x[e]) - top) : 0u;
        }
      }
    }
  }
}

// ----------------------------------------------------------------------------- operands
// Each has kMN (16-byte rows run along x), kRegs (a thread's registers of one step), init(x0, tid),
// load(r0, r1, regs) for r0 .. r0 + 63, zeros from r1 on, and store(regs, tile); a B also kBf (bfloat16 or
// half) and P (pieces of an element).

// A(i = n, r = k): 2-bit weights, K-major, mixed order along k.  A thread holds 32 weights of one row.
struct WeightsK {
  static constexpr bool kMN = false;
  static constexpr int kRegs = 2;
  const uint8_t *packed;
  int64_t N, K;
  bool vec;  // rows are whole 8-byte words
  struct Thread {
    const uint8_t *p;
    uint32_t off;
    int k;
    bool live;
  };
  __device__ __forceinline__ Thread init(int64_t x0, int tid) const {
    const int lane = tid & 31, row = (tid >> 5) * 16 + ((lane >> 4) << 3) + (lane & 7), half = (lane >> 3) & 1;
    const int64_t n = x0 + row;
    return {packed + (n * K >> 2) + half * 8, (row >> 3) * 1024u + half * 512u + (row & 7) * 16u, half * 32, n < N};
  }
  __device__ __forceinline__ void load(const Thread &t, int64_t r0, int64_t r1, uint32_t (&w)[kRegs]) const {
    const uint8_t *p = t.p + (r0 >> 2);
    const int64_t left = r1 - r0 - t.k;  // weights of this thread's row that are left
    w[0] = w[1] = 0;
    if (!t.live || left <= 0) return;
    if (vec) {
      const uint2 v = __ldg(reinterpret_cast<const uint2 *>(p));
      w[0] = v.x, w[1] = v.y;
    } else {
#pragma unroll
      for (int b = 0; b < 8; ++b)
        if (4 * b < left) w[b >> 2] |= static_cast<uint32_t>(__ldg(p + b)) << (8 * (b & 3));
    }
  }
  __device__ __forceinline__ void store(const Thread &t, const uint32_t (&w)[kRegs], uint32_t tile) const {
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      uint32_t o[8];
      weights16(w[g], o);
      st_shared16(tile + t.off + g * 256u, o[0], o[1], o[2], o[3]);
      st_shared16(tile + t.off + g * 256u + 128u, o[4], o[5], o[6], o[7]);
    }
  }
};

// A(i = k, r = n): the same weights, MN-major; row i of the tile is k = i with its low 4 bits mixed.
// A thread holds 32 k of one n.
struct WeightsT {
  static constexpr bool kMN = true;
  static constexpr int kRegs = 2;
  const uint8_t *packed;
  int64_t N, K;
  bool vec;
  struct Thread {
    const uint8_t *p;
    uint32_t off;
    int n, left;
  };
  __device__ __forceinline__ Thread init(int64_t x0, int tid) const {
    const int lane = tid & 31, n = (tid >> 5) * 8 + (lane & 7), q = lane >> 3;
    const int64_t k = x0 + 32 * q, left = K - k;
    return {packed + (k >> 2), q * 4096u + (n >> 3) * 128u + (n & 7) * 16u, n, static_cast<int>(left < 32 ? left : 32)};
  }
  __device__ __forceinline__ void load(const Thread &t, int64_t r0, int64_t r1, uint32_t (&w)[kRegs]) const {
    w[0] = w[1] = 0;
    if (r0 + t.n >= r1 || t.left <= 0) return;
    const uint8_t *p = t.p + ((r0 + t.n) * K >> 2);
    if (vec) {
      const uint2 v = __ldg(reinterpret_cast<const uint2 *>(p));
      w[0] = v.x, w[1] = v.y;
    } else {
#pragma unroll
      for (int b = 0; b < 8; ++b)
        if (4 * b < t.left) w[b >> 2] |= static_cast<uint32_t>(__ldg(p + b)) << (8 * (b & 3));
    }
  }
  __device__ __forceinline__ void store(const Thread &t, const uint32_t (&w)[kRegs], uint32_t tile) const {
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      uint32_t o[8];
      weights16(w[g], o);
      st_shared16(tile + t.off + g * 2048u, o[0], o[1], o[2], o[3]);
      st_shared16(tile + t.off + g * 2048u + 1024u, o[4], o[5], o[6], o[7]);
    }
  }
};

// 16 codes at p, `left` of them in range (1 .. 16).  unit: 16 or 4 bytes that every row is a multiple of, or 1
__device__ __forceinline__ void load_codes(const int8_t *p, int left, int unit, uint32_t *w) {
  if (unit == 16) {
    const uint4 v = __ldg(reinterpret_cast<const uint4 *>(p));
    w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
  } else if (unit == 4) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = 4 * i < left ? __ldg(reinterpret_cast<const uint32_t *>(p) + i) : 0u;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (i < left) w[i >> 2] |= (static_cast<uint32_t>(__ldg(p + i)) & 0xFFu) << (8 * (i & 3));
  }
}

// B(j = m, r = k): int8 codes as halves, K-major, mixed order along k.  A thread holds 16 codes of each of
// TB / 64 rows.
template <int TB>
struct CodesK {
  static constexpr bool kMN = false, kBf = false;
  static constexpr int P = 1;
  static constexpr int kUnits = TB >= 64 ? TB / 64 : 1;
  static constexpr int kRegs = 4 * kUnits;
  const int8_t *codes;
  int64_t M, ld;
  int unit;
  struct Thread {
    const int8_t *p;
    uint32_t off;
    int k;
    int64_t left;  // rows from this thread's first on
  };
  __device__ __forceinline__ Thread init(int64_t x0, int tid) const {
    const int lane = tid & 31, row = (tid >> 5) * 8 + (lane & 7), q = lane >> 3;
    const int64_t m = x0 + row;
    return {codes + m * ld + 16 * q, (row >> 3) * 1024u + q * 256u + (row & 7) * 16u, 16 * q, row < TB ? M - m : 0};
  }
  __device__ __forceinline__ void load(const Thread &t, int64_t r0, int64_t r1, uint32_t (&w)[kRegs]) const {
    const int64_t left = r1 - r0 - t.k;
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      w[4 * u] = w[4 * u + 1] = w[4 * u + 2] = w[4 * u + 3] = 0;
      if (left > 0 && t.left > 64 * u)
        load_codes(t.p + r0 + 64 * u * ld, static_cast<int>(left < 16 ? left : 16), unit, w + 4 * u);
    }
  }
  __device__ __forceinline__ void store(const Thread &t, const uint32_t (&w)[kRegs], uint32_t tile) const {
    if (TB < 64 && t.off >= TB * 128u) return;
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const uint32_t b[4] = {w[4 * u], w[4 * u + 1], w[4 * u + 2], w[4 * u + 3]};
      uint32_t o[8];
      codes16_half_mixed(b, o);
      st_shared16(tile + t.off + u * 8192u, o[0], o[1], o[2], o[3]);
      st_shared16(tile + t.off + u * 8192u + 128u, o[4], o[5], o[6], o[7]);
    }
  }
};

// A(i = k, r = m): int8 codes as bfloat16, MN-major.  A thread holds 2 x 16 codes of one m.
struct CodesT {
  static constexpr bool kMN = true;
  static constexpr int kRegs = 8;
  const int8_t *codes;
  int64_t K, ld;
  int unit;
  struct Thread {
    const int8_t *p;
    uint32_t off;
    int m;
    int64_t left;
  };
  __device__ __forceinline__ Thread init(int64_t x0, int tid) const {
    const int lane = tid & 31, m = (tid >> 5) * 8 + (lane & 7), q = lane >> 3;
    return {codes + x0 + 16 * q, q * 2048u + (m >> 3) * 128u + (m & 7) * 16u, m, K - x0 - 16 * q};
  }
  __device__ __forceinline__ void load(const Thread &t, int64_t r0, int64_t r1, uint32_t (&w)[kRegs]) const {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      w[4 * u] = w[4 * u + 1] = w[4 * u + 2] = w[4 * u + 3] = 0;
      const int64_t left = t.left - 64 * u;
      if (r0 + t.m < r1 && left > 0)
        load_codes(t.p + (r0 + t.m) * ld + 64 * u, static_cast<int>(left < 16 ? left : 16), unit, w + 4 * u);
    }
  }
  __device__ __forceinline__ void store(const Thread &t, const uint32_t (&w)[kRegs], uint32_t tile) const {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      uint32_t o[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) codes4_bf16(w[4 * u + i], o[2 * i], o[2 * i + 1]);
      st_shared16(tile + t.off + u * 8192u, o[0], o[1], o[2], o[3]);
      st_shared16(tile + t.off + u * 8192u + 1024u, o[4], o[5], o[6], o[7]);
    }
  }
};

// 8 elements at p as loaded words (4 of two 16-bit elements, or 8 of one), `left` of them in range (1 .. 8)
template <typename T>
constexpr int kWords8 = sizeof(T) == 4 ? 8 : 4;
template <typename T>
__device__ __forceinline__ void load_grad8(const T *p, int left, bool vec, uint32_t *w) {
  if (vec) {
    const uint4 v = __ldg(reinterpret_cast<const uint4 *>(p));
    w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
    if constexpr (sizeof(T) == 4) {
      const uint4 u = __ldg(reinterpret_cast<const uint4 *>(p) + 1);
      w[4] = u.x, w[5] = u.y, w[6] = u.z, w[7] = u.w;
    }
  } else if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = i < left ? __ldg(reinterpret_cast<const uint32_t *>(p) + i) : 0u;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint16_t *h = reinterpret_cast<const uint16_t *>(p) + 2 * i;
      w[i] = (2 * i < left ? static_cast<uint32_t>(__ldg(h)) : 0u) | (2 * i + 1 < left ? static_cast<uint32_t>(__ldg(h + 1)) << 16 : 0u);
    }
  }
}
template <typename T>
__device__ __forceinline__ void grad8_f32(const uint32_t *w, float (&v)[8]) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) unpack2<T>(w[i], v[2 * i], v[2 * i + 1]);
  }
}

// B(j = m, r = n): gradients, K-major: 16-bit ones as they are, 32-bit ones in three pieces.  A thread holds
// 8 elements of each of TB / 32 places: 4 groups of 8 columns, 2 of them a thread, of TB / 64 rows.
template <typename T, int TB>
struct GradK {
  static constexpr bool kMN = false, kBf = !std::is_same_v<T, __half>;
  static constexpr int P = sizeof(T) == 4 ? 3 : 1;
  static constexpr int kRows = TB >= 64 ? TB / 64 : 1, kUnits = 2 * kRows;
  static constexpr int kRegs = kWords8<T> * kUnits;
  const T *dy;
  int64_t M, ld;
  bool vec;
  struct Thread {
    const T *p;
    uint32_t off;
    int n;
    int64_t left;
  };
  __device__ __forceinline__ Thread init(int64_t x0, int tid) const {
    const int lane = tid & 31, row = (tid >> 5) * 8 + (lane & 7), q = lane >> 3;
    const int64_t m = x0 + row;
    return {dy + m * ld + 8 * q, (row >> 3) * 1024u + q * 128u + (row & 7) * 16u, 8 * q, row < TB ? M - m : 0};
  }
  __device__ __forceinline__ void load(const Thread &t, int64_t r0, int64_t r1, uint32_t (&w)[kRegs]) const {
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      uint32_t *o = w + kWords8<T> * u;
#pragma unroll
      for (int i = 0; i < kWords8<T>; ++i) o[i] = 0;
      const int64_t left = r1 - r0 - t.n - 32 * (u & 1);
      if (left > 0 && t.left > 64 * (u >> 1))
        load_grad8<T>(t.p + r0 + 32 * (u & 1) + 64 * (u >> 1) * ld, static_cast<int>(left < 8 ? left : 8), vec, o);
    }
  }
  __device__ __forceinline__ void store(const Thread &t, const uint32_t (&w)[kRegs], uint32_t tile) const {
    if (TB < 64 && t.off >= TB * 128u) return;
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const uint32_t at = tile + t.off + (u & 1) * 512u + (u >> 1) * 8192u;
      const uint32_t *o = w + kWords8<T> * u;
      if constexpr (P == 1) {
        st_shared16(at, o[0], o[1], o[2], o[3]);
      } else {
        float v[8];
        grad8_f32<T>(o, v);
        split8<P>(v, at, TB * kStep * 2);
      }
    }
  }
};

// B(j = n, r = m): gradients times their row's scale, in P bfloat16 pieces, MN-major.  A thread holds TB / 32
// groups of 8 columns of one m, and its scale.
template <typename T, int TB, int P_>
struct GradT {
  static constexpr bool kMN = true, kBf = true;
  static constexpr int P = P_;
  static constexpr int kUnits = TB / 32;
  static constexpr int kRegs = kWords8<T> * kUnits + 1;
  const T *dy;
  int64_t N, ld;
  const float *scale;
  bool vec;
  struct Thread {
    const T *p;
    uint32_t off;
    int m;
    int64_t left;
  };
  __device__ __forceinline__ Thread init(int64_t x0, int tid) const {
    const int lane = tid & 31, m = (tid >> 5) * 8 + (lane & 7), q = lane >> 3;
    return {dy + x0 + 8 * q, q * 1024u + (m >> 3) * 128u + (m & 7) * 16u, m, N - x0 - 8 * q};
  }
  __device__ __forceinline__ void load(const Thread &t, int64_t r0, int64_t r1, uint32_t (&w)[kRegs]) const {
    const bool live = r0 + t.m < r1;
    w[kRegs - 1] = live ? __float_as_uint(__ldg(scale + r0 + t.m)) : 0u;
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      uint32_t *o = w + kWords8<T> * u;
#pragma unroll
      for (int i = 0; i < kWords8<T>; ++i) o[i] = 0;
      const int64_t left = t.left - 32 * u;
      if (live && left > 0) load_grad8<T>(t.p + (r0 + t.m) * ld + 32 * u, static_cast<int>(left < 8 ? left : 8), vec, o);
    }
  }
  __device__ __forceinline__ void store(const Thread &t, const uint32_t (&w)[kRegs], uint32_t tile) const {
    const float s = __uint_as_float(w[kRegs - 1]);
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      float v[8];
      grad8_f32<T>(w + kWords8<T> * u, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] *= s;
      split8<P>(v, tile + t.off + u * 4096u, TB * kStep * 2);
    }
  }
};

// ----------------------------------------------------------------------------- epilogues
// put(j, i, v): one element of the product; consecutive lanes hold consecutive i (in mixed order for
// weights that run along i: `i` is the true one).
struct OutY {  // y[m][n] = v / 2 scale_m w_scale + b_n
  void *y;
  int dtype;
  int64_t ld;
  const float *scale, *w_scale, *bias;
  __device__ __forceinline__ float factor(int64_t j) const { return __ldg(scale + j) * __ldg(w_scale) * 0.5f; }
  __device__ __forceinline__ float add(int64_t i) const { return bias ? __ldg(bias + i) : 0.0f; }
};
struct OutX {  // dx[m][k] = v / 2 w_scale
  void *y;
  int dtype;
  int64_t ld;
  const float *w_scale;
  __device__ __forceinline__ float factor(int64_t) const { return __ldg(w_scale) * 0.5f; }
  __device__ __forceinline__ float add(int64_t) const { return 0.0f; }
};
struct OutW {  // dW[n][k] = v
  void *y;
  int dtype;
  int64_t ld;
  __device__ __forceinline__ float factor(int64_t) const { return 1.0f; }
  __device__ __forceinline__ float add(int64_t) const { return 0.0f; }
};
__device__ __forceinline__ void put_element(void *y, int dtype, int64_t at, float v) {
  if (dtype == 0) static_cast<float *>(y)[at] = v;
  else if (dtype == 1) static_cast<__half *>(y)[at] = __float2half_rn(v);
  else static_cast<__nv_bfloat16 *>(y)[at] = __float2bfloat16_rn(v);
}

// ----------------------------------------------------------------------------- the kernel
template <class A, class B, class Out>
struct GemmArgs {
  int64_t I, J, R;
  A a;
  B b;
  Out out;
  int tiles_i, steps;  // tiles along i; steps of a split
  float *partial;      // [splits][J][I] where there are several, else NULL
  int *err;            // set to 1 by a wait that gave up
};

template <int TB, int P>
struct GemmShape {
  static constexpr uint32_t kPieceBytes = TB * kStep * 2;
  static constexpr uint32_t kStageBytes = kTileABytes + P * kPieceBytes;
  static constexpr int kStages = P == 3 ? 3 : TB >= 128 ? 2 : 4;
  static constexpr uint32_t kSmem = kStages * kStageBytes + 256;
  static constexpr int kCtasPerSm = kSmem * 2 <= kSmemPerSm - 2048 ? 2 : 1;
  static constexpr uint32_t kTmemCols = TB < 32 ? 32 : TB;
};

template <class A, class B, class Out, int TB>
__global__ void __launch_bounds__(kGemmThreads, GemmShape<TB, B::P>::kCtasPerSm)
    gemm_kernel(const __grid_constant__ GemmArgs<A, B, Out> g) {
  constexpr int P = B::P;
  using S = GemmShape<TB, P>;
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t base = smem_u32(smem);
  const uint32_t bars = base + S::kStages * S::kStageBytes;  // full[stages], empty[stages], done; then 2 words
  const uint32_t full = bars, empty = bars + 8 * S::kStages, done = bars + 16 * S::kStages;
  volatile uint32_t *word = reinterpret_cast<volatile uint32_t *>(smem + S::kStages * S::kStageBytes + 16 * S::kStages + 8);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int64_t i0 = static_cast<int64_t>(blockIdx.x % g.tiles_i) * kTileI, j0 = static_cast<int64_t>(blockIdx.x / g.tiles_i) * TB;
  const int64_t first = static_cast<int64_t>(blockIdx.y) * g.steps * kStep;
  const int64_t end = first + static_cast<int64_t>(g.steps) * kStep < g.R ? first + static_cast<int64_t>(g.steps) * kStep : g.R;
  const int steps = static_cast<int>((end - first + kStep - 1) / kStep);

  if (tid == 0) {
    for (int s = 0; s < S::kStages; ++s) mbar_init(full + 8 * s, kProducerWarps), mbar_init(empty + 8 * s, 1);
    mbar_init(done, 1);
    fence_mbar_init_cluster();
    word[1] = 0;
  }
  if (warp == kProducerWarps) {
    tmem_alloc(smem_u32(const_cast<uint32_t *>(word)), S::kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = word[0];
  // a wait with an end: one that gives up stops the CTA's others too
  auto wait = [&](uint32_t bar, uint32_t parity) -> bool {
    if (mbar_try_wait(bar, parity)) return true;
    const long long t0 = clock64();
    while (!mbar_try_wait(bar, parity)) {
      if (word[1]) return false;
      if (clock64() - t0 > kGemmWaitCycles) {
        word[1] = 1;
        *g.err = 1;
        return false;
      }
    }
    return true;
  };

  if (warp < kProducerWarps) {
    const typename A::Thread ta = g.a.init(i0, tid);
    const typename B::Thread tb = g.b.init(j0, tid);
    uint32_t ra[A::kRegs], rb[B::kRegs];
    g.a.load(ta, first, end, ra);
    g.b.load(tb, first, end, rb);
    for (int it = 0; it < steps; ++it) {
      const int s = it % S::kStages;
      const bool free = it < S::kStages || wait(empty + 8 * s, (it / S::kStages - 1) & 1);
      if (!__all_sync(0xffffffffu, free)) break;
      const uint32_t stage = base + s * S::kStageBytes;
      g.a.store(ta, ra, stage);
      g.b.store(tb, rb, stage + kTileABytes);
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(full + 8 * s);
      if (it + 1 < steps) {  // the next step's, in flight while the tensor cores work through the stages
        g.a.load(ta, first + static_cast<int64_t>(it + 1) * kStep, end, ra);
        g.b.load(tb, first + static_cast<int64_t>(it + 1) * kStep, end, rb);
      }
    }
  } else {
    constexpr uint32_t idesc = gemm_idesc(B::kBf, A::kMN, B::kMN, TB);
    for (int it = 0; it < steps; ++it) {
      const int s = it % S::kStages;
      if (!__all_sync(0xffffffffu, wait(full + 8 * s, (it / S::kStages) & 1))) break;
      tc_fence_after();
      const uint32_t at = base + s * S::kStageBytes, bt = at + kTileABytes;
#pragma unroll
      for (int p = 0; p < P; ++p)
#pragma unroll
        for (int ks = 0; ks < kStep / 16; ++ks)
          mma_bf16_warp(tmem, make_sdesc(at + ks * 256, 128, 1024), make_sdesc(bt + p * S::kPieceBytes + ks * 256, 128, 1024), idesc,
                        it > 0 || p > 0 || ks > 0 ? 1u : 0u);
      mma_commit_warp(empty + 8 * s);
    }
    mma_commit_warp(done);
  }
  __syncwarp();
  const bool ready = __all_sync(0xffffffffu, wait(done, 0) && !word[1]);
  tc_fence_after();
  if (warp < kProducerWarps) {
    const int64_t row = 32 * (warp & 3) + lane;  // of the tile, and the lane of tensor memory
    const int64_t i = i0 + (std::is_same_v<A, WeightsT> ? (row & ~15) | mix16(row & 15) : row);
    const uint32_t tl = tmem + (static_cast<uint32_t>(32 * (warp & 3)) << 16);
    constexpr int kHalf = TB / 2;  // columns of each of the two warps of a lane quadrant
    constexpr int kGroup = kHalf < 16 ? 8 : 16;
    const int c0 = (warp >> 2) * kHalf;
    const float add = !g.partial && i < g.I ? g.out.add(i) : 0.0f;
    if (ready) {
#pragma unroll 1
      for (int c = c0; c < c0 + kHalf; c += kGroup) {
        if (j0 + c >= g.J) break;
        float v[kGroup];
        tmem_ld<kGroup>(tl + c, v);
        tmem_wait_ld();
        if (i < g.I) {
          if (g.partial) {
            float *o = g.partial + (static_cast<int64_t>(blockIdx.y) * g.J + j0 + c) * g.I + i;
#pragma unroll
            for (int e = 0; e < kGroup; ++e)
              if (j0 + c + e < g.J) o[e * g.I] = v[e];
          } else {
#pragma unroll
            for (int e = 0; e < kGroup; ++e)
              if (j0 + c + e < g.J) put_element(g.out.y, g.out.dtype, (j0 + c + e) * g.out.ld + i, v[e] * g.out.factor(j0 + c + e) + add);
          }
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kProducerWarps) {
    tc_fence_after();
    tmem_dealloc(tmem, S::kTmemCols);
  }
}

// the splits' sums, added in order, and the epilogue
template <class Out>
__global__ void __launch_bounds__(256) gemm_join_kernel(const float *partial, int splits, int64_t I, int64_t J, const Out out) {
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, j = blockIdx.y;
  for (int64_t jj = j; jj < J; jj += gridDim.y) {
    if (i >= I) return;
    float v = 0.0f;
    for (int s = 0; s < splits; ++s) v += partial[(s * J + jj) * I + i];
    put_element(out.y, out.dtype, jj * out.ld + i, v * out.factor(jj) + out.add(i));
  }
}

// what every row of codes is a multiple of and starts on, for load_codes; and whether rows of gradients are
// whole 16-byte pieces
inline int codes_unit(const int8_t *codes, int64_t ld, int64_t K) {
  const uintptr_t all = reinterpret_cast<uintptr_t>(codes) | static_cast<uintptr_t>(ld) | static_cast<uintptr_t>(K);
  return (all & 15u) == 0 ? 16 : (all & 3u) == 0 ? 4 : 1;
}
template <typename T>
bool grads_vec(const void *dy, int64_t ld, int64_t N) {
  return (reinterpret_cast<uintptr_t>(dy) & 15u) == 0 && ld * static_cast<int64_t>(sizeof(T)) % 16 == 0 && N % 8 == 0;
}

// How the sum over R is split: into as many parts as leave every SM a tile, of at least kMinSteps steps each.
struct GemmPlan {
  int64_t tiles_i, tiles_j;
  int splits, steps;
};
constexpr int kMinSteps = 4;
template <int TB, int P>
GemmPlan gemm_plan(int64_t I, int64_t J, int64_t R, int sms) {
  GemmPlan p;
  p.tiles_i = (I + kTileI - 1) / kTileI, p.tiles_j = (J + TB - 1) / TB;
  const int64_t all = (R + kStep - 1) / kStep, room = static_cast<int64_t>(sms) * GemmShape<TB, P>::kCtasPerSm;
  int64_t splits = room / (p.tiles_i * p.tiles_j);
  if (splits > all / kMinSteps) splits = all / kMinSteps;
  if (splits < 1) splits = 1;
  p.steps = static_cast<int>((all + splits - 1) / splits);
  p.splits = p.steps > 0 ? static_cast<int>((all + p.steps - 1) / p.steps) : 1;
  if (p.splits < 1) p.splits = 1;
  return p;
}

template <class A, class B, class Out, int TB>
cudaError_t launch_gemm(int64_t I, int64_t J, int64_t R, const A &a, const B &b, const Out &out, float *partial, int sms, int *err,
                        cudaStream_t st) {
  constexpr int P = B::P;
  using S = GemmShape<TB, P>;
  const GemmPlan p = gemm_plan<TB, P>(I, J, R, sms);
  const GemmArgs<A, B, Out> g = {I, J, R, a, b, out, static_cast<int>(p.tiles_i), p.steps, p.splits > 1 ? partial : nullptr, err};
  auto *kernel = gemm_kernel<A, B, Out, TB>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem);
  if (e != cudaSuccess) return e;
  kernel<<<dim3(static_cast<unsigned>(p.tiles_i * p.tiles_j), p.splits), kGemmThreads, S::kSmem, st>>>(g);
  if ((e = cudaGetLastError()) != cudaSuccess || p.splits == 1) return e;
  gemm_join_kernel<Out><<<dim3(static_cast<unsigned>((I + 255) / 256), static_cast<unsigned>(J < 65535 ? J : 65535)), 256, 0, st>>>(
      partial, p.splits, I, J, out);
  return cudaGetLastError();
}

}  // namespace aecct
