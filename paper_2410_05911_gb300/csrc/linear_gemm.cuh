// linear_gemm.cuh -- the tensor-core product behind the AAP linear layer and its gradients:
//
//   out(j, i) = sum over r of A(i, r) B(j, r),   i < I, j < J, r < R
//
// with 16-bit operands.  A (2-bit weights, or int8 codes) is in no memory as such: it becomes half or bfloat16 core
// matrices on its way from global to shared memory, in the registers of producer warps, and tcgen05.mma multiplies them
// there (32-bit accumulators in tensor memory).  Reading 1 byte a code and a quarter of one a weight keeps L2 traffic
// under what 16-bit operands would need.  B (codes, or gradients) goes the same way in a single CTA's product, and in a
// pair's that few tiles read; where many do, it is copied by TMA from 16-bit rows, as they lie or as a pass over memory has
// laid them out first (linear_stage.cu).
//
// A CTA makes a tile of 128 i by TB j; from 256 of both on, a cluster of two makes 256 by 256 (cta_group::2),
// each CTA with its own 128 rows of A and half of B in shared memory, so that a B is converted and stored by one
// of two SMs.  Two groups of eight producer warps take the spans of r in turn (a warp's waits and its
// arrivals cost it some 700 cycles a stage, whatever it stores in between): each loads its next span while the
// other stores, converts and stores; another warp (of the first CTA) issues the MMAs.  Lanes hold consecutive i in
// tensor memory, so that the epilogue's stores of one j are 32 neighbouring elements.  Two CTAs share an SM where their
// operands fit, one's epilogue behind the other's products.
//
// What it reaches, and what bounds it: 8,192 x 4,096 x 4,096 (tokens, K, N) the forward product 154 us after 15 us of
// staging, dX 156 us, dW 298 us (two products' work) after 31 us: 1.78, 1.76 and 1.85 PFLOP/s, the tensor cores 73 to 78% busy,
// the rest the filling of a tile's first stages and the last wave of tiles.  37 x 4,096 x 16,384 (few tokens: 128 single tiles) 20 us: the
// shared memory of an SM, which takes the weights as halves, twice their loads' wavefronts, and gives them to the tensor cores
// (its pipe 88% busy on the SMs at work).  32-bit gradients, 23,040 x 128 x 512: dX 22 us, dW 23 us, 3 products each, bound
// by the conversion to three pieces.
//
// Operand tiles are 8 x 16-byte core matrices without swizzle.  Element (x, r) of a K-major tile (16 bytes
// along r) is at (x / 8) 1152 + (r / 8) 144 + (x % 8) 16 + (r % 8) 2, of an MN-major tile (16 bytes along x)
// at (x / 8) 1040 + (r / 8) 128 + (r % 8) 16 + (x % 8) 2.  The 16 bytes of padding between core matrices along
// the source's contiguous dimension let eight lanes read one 128-byte line of a row and store their eight
// pieces to eight different bank groups.  (Eight lanes on eight rows store without padding, but their loads take
// a wavefront per row: 1,330 a step of 256 rows, where the tensor cores need 512 cycles.)
#pragma once
#include <cuda_runtime.h>

#include <atomic>
#include <climits>
#include <cstdint>

#include <cuda.h>

#include "aecct_internal.h"
#include "rowtypes.cuh"
#include "sm103_ptx.cuh"

namespace aecct {

constexpr int kStep = 64;           // r per stage
constexpr int kTileI = 128;         // i per CTA: the lanes of tensor memory
constexpr int kGroups = 2;          // of producers, which take the spans of r in turn
constexpr int kGroupWarps = 8;
constexpr int kProducerWarps = kGroups * kGroupWarps;
constexpr int kProducers = kProducerWarps * 32;
constexpr int kGemmThreads = kProducers + 64;  // and the warps of the MMAs and of the copies
constexpr int kPass = kGroupWarps * 4;  // rows of 8 lanes that a group holds at a time
// a tile of x rows, and its descriptor's strides
__host__ __device__ constexpr uint32_t tile_bytes(bool mn, int x) { return x / 8 * (mn ? 1040u : 1152u); }
__host__ __device__ constexpr uint32_t tile_lbo(bool mn) { return mn ? 128u : 144u; }
__host__ __device__ constexpr uint32_t tile_sbo(bool mn) { return mn ? 1040u : 1152u; }
constexpr int kGemmWaitTries = 1 << 24;  // a wait that has looked so often (seconds) has lost its arrival

// instruction descriptor of kind::f16: 32-bit accumulators; BF: bfloat16 operands, else half; MN: both
// operands' 16-byte rows run along i and j
__host__ __device__ constexpr uint32_t gemm_idesc(bool bf, bool mn_a, bool mn_b, uint32_t m, uint32_t n) {
  return (1u << 4) | (bf ? (1u << 7) | (1u << 10) : 0u) | (mn_a ? 1u << 15 : 0u) | (mn_b ? 1u << 16 : 0u) | ((n >> 3) << 17) |
         ((m >> 4) << 24);
}

__device__ __forceinline__ void st_shared16(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

// ----------------------------------------------------------------------------- conversions
// 16 2-bit weights (00 = 0, 01 = +1, 11 = -1, 10 = 0) of a word as 16-bit floats, two at a time: fields f and f + 8
// sit at the same place of the word's halves, in the low bits of a mantissa where the exponent makes them
// integers (1024 + x: 10 bits of a half; 128 + x: 7 bits of a bfloat16), so that one logical operation takes both
// fields, with their high bit turned over (0, 1, -1 become 2, 3, 1), and one multiply-add brings them down by
// 4^f and subtracts 2.  No shift until the mantissa's bits run out.  o[p] holds
// weights f and f + 8 for f = p, or f = 4 + p where `high`; mix16 is the order of both in a row.
__host__ __device__ constexpr int mix16(int pos) { return ((pos & 1) << 3) | ((pos >> 3) << 2) | ((pos >> 1) & 3); }
template <bool BF>
__device__ __forceinline__ void weights4(uint32_t w, bool high, uint32_t (&o)[4]) {
  w &= 0x55555555u | (w + w);  // 10 is 00
  constexpr int kFields = BF ? 3 : 5;
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    const int f = (high ? 4 : 0) + p, g = f % kFields;
    const uint32_t x = w >> (2 * (f - g));
    const uint32_t u = (x & (0x00030003u << (2 * g))) ^ ((BF ? 0x43004300u : 0x64006400u) | (0x00020002u << (2 * g)));
    const float by = 1.0f / static_cast<float>(1 << (2 * g)), less = -((BF ? 128.0f : 1024.0f) * by + 2.0f);
    if constexpr (BF) {
      const __nv_bfloat162 v = __hfma2(*reinterpret_cast<const __nv_bfloat162 *>(&u), __float2bfloat162_rn(by), __float2bfloat162_rn(less));
      o[p] = *reinterpret_cast<const uint32_t *>(&v);
    } else {
      const __half2 v = __hfma2(*reinterpret_cast<const __half2 *>(&u), __float2half2_rn(by), __float2half2_rn(less));
      o[p] = *reinterpret_cast<const uint32_t *>(&v);
    }
  }
}
// 4 + 4 int8 codes of two words as halves, codes p of both in o[p]: (code + 128) in the low byte of 1024, less 1152
__device__ __forceinline__ void codes8_half(uint32_t b0, uint32_t b1, uint32_t (&o)[4]) {
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    const uint32_t t = __byte_perm(b0, b1, 0x0400u + 0x0101u * p);
    const uint32_t u = (t & 0x00FF00FFu) ^ 0x64806480u;
    const __half2 v = __hsub2(*reinterpret_cast<const __half2 *>(&u), __half2{__ushort_as_half(0x6480), __ushort_as_half(0x6480)});
    o[p] = *reinterpret_cast<const uint32_t *>(&v);
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
// 8 values in 32 bits as P bfloat16 pieces each, the largest first: each piece cuts off 8 bits and the next takes what is
// left, so that two hold 16 bits and three a 32-bit value exactly.  An infinity stays one in its first piece, and its others
// are zero.  put(p, words) takes a piece at a time.
template <int P, class Put>
__device__ __forceinline__ void split8(const float (&v)[8], const Put &put) {
  uint32_t o[4], x[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = v[e] == v[e] ? __float_as_uint(v[e]) : 0x7FC00000u;
#pragma unroll
  for (int p = 0; p < P; ++p) {
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = __byte_perm(x[2 * i], x[2 * i + 1], 0x7632);
    put(p, o);
    if (p + 1 < P) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float top = __uint_as_float(x[e] & 0xFFFF0000u);
        x[e] = fabsf(top) < INFINITY ? __float_as_uint(__uint_as_float(x[e]) - top) : 0u;
      }
    }
  }
}
template <int P>
__device__ __forceinline__ void store_split8(const float (&v)[8], uint32_t addr, uint32_t piece_bytes) {
  split8<P>(v, [&](int p, const uint32_t (&o)[4]) { st_shared16(addr + p * piece_bytes, o[0], o[1], o[2], o[3]); });
}

// ----------------------------------------------------------------------------- operands
// Each has kMN (16-byte rows run along x), kSpan (steps that one load feeds), kRegs (a thread's registers
// of them), init(x0, r0, tid), full(thread, regs): the next span, every r in range and every row whole 16-byte
// (weights: 8-byte) pieces, in plain loads; load(thread, left, regs): the same where only `left` r are in range,
// or rows are not such, zeros beyond; aligned(): rows are; and store(thread, regs, step of the span, tile).
// A row or column of the tile past the operand's last one reads that one again: its products are dropped.
// A B also has kBf (bfloat16 or half) and P (pieces of an element), an A kMixed (its rows are in the order of
// mix16) and kExact (its sums are integers that 32 bits hold).  The forward product's operands span two steps: the first takes k = 0 .. 3 and 8 .. 11 of every 16 k, the
// second the others, so that a load is 16 bytes of codes and a row's 128 bytes are one line.

// 4 W bytes at any p, of which the first `left` are in range, the others zeros: aligned words that hold any of them, shifted.
// An array lies in [base, limit): a word that reaches out of it (at its very ends) is read byte by byte.
template <int W>
__device__ __forceinline__ void load_bytes(const void *at, int left, const void *base, const void *limit, uint32_t *w) {
#pragma unroll
  for (int i = 0; i < W; ++i) w[i] = 0;
  if (left <= 0) return;
  const uint8_t *p = static_cast<const uint8_t *>(at);
  const int n = left < 4 * W ? left : 4 * W, off = static_cast<int>(reinterpret_cast<uintptr_t>(p) & 3);
  const uint8_t *a = p - off;
  if (a >= static_cast<const uint8_t *>(base) && a + ((off + n + 3) & ~3) <= static_cast<const uint8_t *>(limit)) {
    uint32_t v[W + 1];
#pragma unroll
    for (int i = 0; i <= W; ++i) v[i] = 4 * i < off + n ? __ldg(reinterpret_cast<const uint32_t *>(a) + i) : 0u;
#pragma unroll
    for (int i = 0; i < W; ++i) {
      w[i] = __funnelshift_r(v[i], v[i + 1], 8 * off);
      if (4 * i + 4 > n) w[i] = 4 * i < n ? w[i] & (0xFFFFFFFFu >> (8 * (4 * i + 4 - n))) : 0u;
    }
  } else {
#pragma unroll
    for (int b = 0; b < 4 * W; ++b)
      if (b < n) w[b >> 2] |= static_cast<uint32_t>(__ldg(p + b)) << (8 * (b & 3));
  }
}

// 2-bit weights at p, 4 W bytes, `left` weights in range (a multiple of 4).  unit: 16, 8 or 4 bytes that every
// row is a multiple of, or 1
template <int W>
__device__ __forceinline__ void load_weights(const uint8_t *p, int left, int unit, const uint8_t *base, const uint8_t *limit,
                                             uint32_t (&w)[W]) {
  if (unit >= 4) {
#pragma unroll
    for (int i = 0; i < W; ++i) w[i] = 16 * i < left ? __ldg(reinterpret_cast<const uint32_t *>(p) + i) : 0u;
  } else {
    load_bytes<W>(p, left / 4, base, limit, w);
  }
}

// A(i = n, r = k): 2-bit weights, K-major, mixed order along k.  A thread holds 64 weights of one row.
struct WeightsK {
  static constexpr bool kMN = false, kMixed = false, kExact = true;
  static constexpr int kSpan = 2, kRegs = 4;
  const uint8_t *packed;
  int64_t N, K;
  int unit;
  struct Thread {
    const uint8_t *p;
    uint32_t off;
    int k;
  };
  bool aligned() const { return unit == 16; }
  __device__ __forceinline__ Thread init(int64_t x0, int64_t r0, int tid) const {
    const int lane = tid & 31, row = (tid >> 5) * 16 + ((lane >> 4) << 3) + (lane & 7), half = (lane >> 3) & 1;
    const int64_t n = x0 + row < N ? x0 + row : N - 1;
    return {packed + ((n * K + r0) >> 2) + half * 16, (row >> 3) * 1152u + half * 576u + (row & 7) * 16u, half * 64};
  }
  __device__ __forceinline__ void full(Thread &t, uint32_t (&w)[kRegs]) const {
    const uint4 v = __ldg(reinterpret_cast<const uint4 *>(t.p));
    w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
    t.p += kGroups * kSpan * kStep / 4;
  }
  __device__ __forceinline__ void load(Thread &t, int left, uint32_t (&w)[kRegs]) const {
    load_weights<4>(t.p, left - t.k, unit, packed, packed + (N * K >> 2), w);
    t.p += kGroups * kSpan * kStep / 4;
  }
  __device__ __forceinline__ void store(const Thread &t, const uint32_t (&w)[kRegs], bool second, uint32_t tile) const {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      uint32_t o[4];
      weights4<false>(w[g], second, o);
      st_shared16(tile + t.off + g * 144u, o[0], o[1], o[2], o[3]);
    }
  }
};

// A(i = k, r = n): the same weights as bfloat16 or half, MN-major; row i of the tile is k = i with its low 4
// bits mixed.  A thread holds 32 k of one n.
template <bool BF>
struct WeightsT {
  static constexpr bool kMN = true, kMixed = true, kExact = false;
  static constexpr int kSpan = 1, kRegs = 2;
  const uint8_t *packed;
  int64_t N, K;
  int unit;
  struct Thread {
    const uint8_t *p;
    uint32_t off;
    int n, k;  // k: how many of the 32 are in range
  };
  bool aligned() const { return unit >= 8; }
  __device__ __forceinline__ Thread init(int64_t x0, int64_t r0, int tid) const {
    const int lane = tid & 31, n = (tid >> 5) * 8 + (lane & 7), q = lane >> 3;
    const int64_t left = K - x0 - 32 * q, k = left > 0 ? x0 + 32 * q : K - (K < 32 ? K : 32);
    return {packed + (((r0 + n) * K + k) >> 2), q * 4160u + (n >> 3) * 128u + (n & 7) * 16u, n,
            static_cast<int>(left < 32 ? left : 32)};
  }
  __device__ __forceinline__ void full(Thread &t, uint32_t (&w)[kRegs]) const {
    const uint2 v = __ldg(reinterpret_cast<const uint2 *>(t.p));
    w[0] = v.x, w[1] = v.y;
    t.p += kGroups * kStep / 4 * K;
  }
  __device__ __forceinline__ void load(Thread &t, int left, uint32_t (&w)[kRegs]) const {
    load_weights<2>(t.p, t.n < left ? t.k : 0, unit, packed, packed + (N * K >> 2), w);
    t.p += kGroups * kStep / 4 * K;
  }
  __device__ __forceinline__ void store(const Thread &t, const uint32_t (&w)[kRegs], bool, uint32_t tile) const {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      uint32_t o[4];
      weights4<BF>(w[g >> 1], g & 1, o);
      st_shared16(tile + t.off + g * 1040u, o[0], o[1], o[2], o[3]);
    }
  }
};

// 16 codes at p, `left` of them in range.  unit: 16 or 4 bytes that every row is a multiple of, or 1; the rows lie in
// [base, limit)
__device__ __forceinline__ void load_codes(const int8_t *p, int left, int unit, const int8_t *base, const int8_t *limit, uint32_t *w) {
  if (unit >= 4) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = 4 * i < left ? __ldg(reinterpret_cast<const uint32_t *>(p) + i) : 0u;
  } else {
    load_bytes<4>(p, left, base, limit, w);
  }
}

// rows of `have` from the first one on that x rows of a tile may read, as an int
__device__ __forceinline__ int rows_left(int64_t have) {
  return static_cast<int>(have < 0 ? 0 : have < 1024 ? have : 1024);
}

// B(j = m, r = k): int8 codes as halves, K-major, mixed order along k.  A thread holds 16 codes of each of
// X / kPass rows.
template <int X>
struct CodesK {
  static constexpr bool kTma = false, kMN = false, kBf = false;
  static constexpr int P = 1;
  static constexpr int kUnits = X >= kPass ? X / kPass : 1;
  static constexpr int kSpan = 2, kRegs = 4 * kUnits;
  const int8_t *codes;
  int64_t M, K, ld;
  int unit;
  struct Thread {
    const int8_t *p[kUnits];
    uint32_t off;
    int k;
  };
  bool aligned() const { return unit == 16; }
  __device__ __forceinline__ Thread init(int64_t x0, int64_t r0, int tid) const {
    const int lane = tid & 31, row = (tid >> 5) * 4 + (lane >> 3), q = lane & 7;
    Thread t = {{}, (row >> 3) * 1152u + q * 144u + (row & 7) * 16u, 16 * q};
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const int64_t m = x0 + row + u * kPass;
      t.p[u] = codes + (m < M ? m : M - 1) * ld + r0 + 16 * q;
    }
    return t;
  }
  __device__ __forceinline__ void full(Thread &t, uint32_t (&w)[kRegs]) const {
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const uint4 v = __ldg(reinterpret_cast<const uint4 *>(t.p[u]));
      w[4 * u] = v.x, w[4 * u + 1] = v.y, w[4 * u + 2] = v.z, w[4 * u + 3] = v.w;
      t.p[u] += kGroups * kSpan * kStep;
    }
  }
  __device__ __forceinline__ void load(Thread &t, int left, uint32_t (&w)[kRegs]) const {
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      load_codes(t.p[u], left - t.k, unit, codes, codes + (M - 1) * ld + K, w + 4 * u);
      t.p[u] += kGroups * kSpan * kStep;
    }
  }
  __device__ __forceinline__ void store(const Thread &t, const uint32_t (&w)[kRegs], bool second, uint32_t tile) const {
    if (X < kPass && t.off >= tile_bytes(false, X)) return;
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      uint32_t o[4];
      codes8_half(second ? w[4 * u + 1] : w[4 * u], second ? w[4 * u + 3] : w[4 * u + 2], o);
      st_shared16(tile + t.off + u * (kPass / 8 * 1152u), o[0], o[1], o[2], o[3]);
    }
  }
};

// A(i = k, r = m): int8 codes as bfloat16, MN-major.  A thread holds 16 codes of each of 2 m, and stores their
// two pieces in an order that gives eight lanes eight bank groups.
struct CodesT {
  static constexpr bool kMN = true, kMixed = false, kExact = false;
  static constexpr int kSpan = 1, kRegs = 8;
  static_assert(2 * kPass == kStep, "two passes are a step's tokens");
  const int8_t *codes;
  int64_t M, K, ld;
  int unit;
  struct Thread {
    const int8_t *p;
    uint32_t off, turn;
    int m, k;  // k: how many of the 16 are in range
  };
  bool aligned() const { return unit == 16; }
  __device__ __forceinline__ Thread init(int64_t x0, int64_t r0, int tid) const {
    const int lane = tid & 31, m = (tid >> 5) * 4 + (lane >> 3), q = lane & 7;
    const int64_t left = K - x0 - 16 * q, k = left > 0 ? x0 + 16 * q : K - (K < 16 ? K : 16);
    return {codes + (r0 + m) * ld + k, q * 2080u + (m >> 3) * 128u + (m & 7) * 16u, static_cast<uint32_t>(q >> 2), m,
            static_cast<int>(left < 16 ? left : 16)};
  }
  __device__ __forceinline__ void full(Thread &t, uint32_t (&w)[kRegs]) const {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const uint4 v = __ldg(reinterpret_cast<const uint4 *>(t.p + u * kPass * ld));
      w[4 * u] = v.x, w[4 * u + 1] = v.y, w[4 * u + 2] = v.z, w[4 * u + 3] = v.w;
    }
    t.p += kGroups * kStep * ld;
  }
  __device__ __forceinline__ void load(Thread &t, int left, uint32_t (&w)[kRegs]) const {
#pragma unroll
    for (int u = 0; u < 2; ++u)
      load_codes(t.p + u * kPass * ld, t.m + u * kPass < left ? t.k : 0, unit, codes, codes + (M - 1) * ld + K, w + 4 * u);
    t.p += kGroups * kStep * ld;
  }
  __device__ __forceinline__ void store(const Thread &t, const uint32_t (&w)[kRegs], bool, uint32_t tile) const {
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const bool high = (h ^ t.turn) != 0;
        uint32_t o[4];
        codes4_bf16(high ? w[4 * u + 2] : w[4 * u], o[0], o[1]);
        codes4_bf16(high ? w[4 * u + 3] : w[4 * u + 1], o[2], o[3]);
        st_shared16(tile + t.off + (high ? 1040u : 0u) + u * (kPass / 8 * 128u), o[0], o[1], o[2], o[3]);
      }
  }
};

// 8 elements at p as loaded words (4 of two 16-bit elements, or 8 of one), `left` of them in range
template <typename T>
constexpr int kWords8 = sizeof(T) == 4 ? 8 : 4;
template <typename T>
__device__ __forceinline__ void load_grad8(const T *p, int left, bool vec, const T *base, const T *limit, uint32_t *w) {
  if (vec) {
#pragma unroll
    for (int i = 0; i < kWords8<T>; ++i) w[i] = 0;
    if (left <= 0) return;
#pragma unroll
    for (int i = 0; i < kWords8<T> / 4; ++i) {
      const uint4 v = __ldg(reinterpret_cast<const uint4 *>(p) + i);
      w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
    }
  } else if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = i < left ? __ldg(reinterpret_cast<const uint32_t *>(p) + i) : 0u;
  } else {
    load_bytes<4>(p, left < 8 ? 2 * left : 16, base, limit, w);
  }
}
template <typename T>
__device__ __forceinline__ void full_grad8(const T *p, uint32_t *w) {
#pragma unroll
  for (int i = 0; i < kWords8<T> / 4; ++i) {
    const uint4 v = __ldg(reinterpret_cast<const uint4 *>(p) + i);
    w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
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
// 8 elements of each of X / kPass rows.
template <typename T, int X>
struct GradK {
  static constexpr bool kTma = false, kMN = false, kBf = !std::is_same_v<T, __half>;
  static constexpr int P = sizeof(T) == 4 ? 3 : 1;
  static constexpr int kUnits = X / kPass;
  static constexpr int kSpan = 1, kRegs = kWords8<T> * kUnits;
  const T *dy;
  int64_t M, N, ld;
  bool vec;
  struct Thread {
    const T *p[kUnits];
    uint32_t off;
    int n;
  };
  bool aligned() const { return vec; }
  __device__ __forceinline__ Thread init(int64_t x0, int64_t r0, int tid) const {
    const int lane = tid & 31, row = (tid >> 5) * 4 + (lane >> 3), q = lane & 7;
    Thread t = {{}, (row >> 3) * 1152u + q * 144u + (row & 7) * 16u, 8 * q};
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const int64_t m = x0 + row + u * kPass;
      t.p[u] = dy + (m < M ? m : M - 1) * ld + r0 + 8 * q;
    }
    return t;
  }
  __device__ __forceinline__ void full(Thread &t, uint32_t (&w)[kRegs]) const {
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      full_grad8<T>(t.p[u], w + kWords8<T> * u);
      t.p[u] += kGroups * kStep;
    }
  }
  __device__ __forceinline__ void load(Thread &t, int left, uint32_t (&w)[kRegs]) const {
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      load_grad8<T>(t.p[u], left - t.n, vec, dy, dy + (M - 1) * ld + N, w + kWords8<T> * u);
      t.p[u] += kGroups * kStep;
    }
  }
  __device__ __forceinline__ void store(const Thread &t, const uint32_t (&w)[kRegs], bool, uint32_t tile) const {
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const uint32_t *o = w + kWords8<T> * u, at = tile + t.off + u * (kPass / 8 * 1152u);
      if constexpr (P == 1) {
        st_shared16(at, o[0], o[1], o[2], o[3]);
      } else {
        float v[8];
        grad8_f32<T>(o, v);
        store_split8<P>(v, at, tile_bytes(false, X));
      }
    }
  }
};

// B(j = n, r = m): gradients times their row's scale, in P bfloat16 pieces, MN-major.  A thread holds X / 64
// pieces of 8 columns of each of 2 m, and their scales.
template <typename T, int X, int P_>
struct GradT {
  static constexpr bool kTma = false, kMN = true, kBf = true;
  static constexpr int P = P_;
  static constexpr int kPieces = X / 64;
  static constexpr int kSpan = 1, kRegs = 2 * kWords8<T> * kPieces + 2;
  const T *dy;
  int64_t M, N, ld;
  const float *scale;
  bool vec;
  struct Thread {
    const T *p;
    const float *s;
    uint32_t off;
    int m, columns, last;  // last: the furthest piece that starts in range
  };
  bool aligned() const { return vec; }
  __device__ __forceinline__ Thread init(int64_t x0, int64_t r0, int tid) const {
    const int lane = tid & 31, m = (tid >> 5) * 4 + (lane >> 3), q = lane & 7;
    const int columns = rows_left(N - x0 - 8 * q);  // (none: back to the last 8)
    return {dy + (r0 + m) * ld + x0 + 8 * q, scale + r0 + m, q * 1040u + (m >> 3) * 128u + (m & 7) * 16u, m, columns,
            columns > 0 ? (columns - 1) / 64 * 64 : static_cast<int>(N - x0 - 8 * q) - 8};
  }
  __device__ __forceinline__ void full(Thread &t, uint32_t (&w)[kRegs]) const {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      w[kRegs - 2 + h] = __float_as_uint(__ldg(t.s + h * kPass));
#pragma unroll
      for (int u = 0; u < kPieces; ++u)
        full_grad8<T>(t.p + h * kPass * ld + (64 * u < t.last ? 64 * u : t.last), w + kWords8<T> * (h * kPieces + u));
    }
    t.p += kGroups * kStep * ld, t.s += kGroups * kStep;
  }
  __device__ __forceinline__ void load(Thread &t, int left, uint32_t (&w)[kRegs]) const {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const bool live = t.m + h * kPass < left;
      w[kRegs - 2 + h] = live ? __float_as_uint(__ldg(t.s + h * kPass)) : 0u;
#pragma unroll
      for (int u = 0; u < kPieces; ++u)
        load_grad8<T>(t.p + h * kPass * ld + 64 * u, live ? t.columns - 64 * u : 0, vec, dy, dy + (M - 1) * ld + N,
                      w + kWords8<T> * (h * kPieces + u));
    }
    t.p += kGroups * kStep * ld, t.s += kGroups * kStep;
  }
  __device__ __forceinline__ void store(const Thread &t, const uint32_t (&w)[kRegs], bool, uint32_t tile) const {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int u = 0; u < kPieces; ++u) {
        float v[8];
        grad8_f32<T>(w + kWords8<T> * (h * kPieces + u), v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= __uint_as_float(w[kRegs - 2 + h]);
        store_split8<P>(v, tile + t.off + u * 8320u + h * (kPass / 8 * 128u), tile_bytes(true, X));
      }
  }
};

// B from 16-bit rows in memory, copied by TMA with a 128-byte swizzle: `map` has the dimensions (contiguous,
// rows, pieces); elements out of range are zeros.  MN: the contiguous dimension runs along j, and a step is 64 of
// its rows; else it runs along r.
template <int X_, bool MN, bool BF, int P_, int SPAN>
struct Tiled {
  static constexpr bool kTma = true, kMN = MN, kBf = BF;
  static constexpr int P = P_, X = X_, kSpan = SPAN;
  CUtensorMap map;
  bool aligned() const { return true; }
  // the copies of one step into `tile` (P pieces of X rows of 64): j from x0, r from r0
  __device__ __forceinline__ void copy(int64_t x0, int64_t r0, uint32_t tile, uint32_t bar) const {
#pragma unroll
    for (int p = 0; p < P; ++p) {
      if constexpr (MN) {
#pragma unroll
        for (int b = 0; b < X / 64; ++b)
          tensor_g2s(tile + p * X * 128 + b * 8192, &map, static_cast<int>(x0) + 64 * b, static_cast<int>(r0), p, bar);
      } else {
        tensor_g2s(tile + p * X * 128, &map, static_cast<int>(r0), static_cast<int>(x0), p, bar);
      }
    }
  }
};

// ----------------------------------------------------------------------------- epilogues
// out(j, i) = product factor(j) + add(i)
struct OutY {  // y[m][n] = v scale_m w_scale + b_n
  void *y;
  int dtype;
  int64_t ld;
  const float *scale, *w_scale, *bias;
  __device__ __forceinline__ float factor(int64_t j) const { return __ldg(scale + j) * __ldg(w_scale); }
  __device__ __forceinline__ float add(int64_t i) const { return bias ? __ldg(bias + i) : 0.0f; }
};
struct OutX {  // dx[m][k] = v w_scale
  void *y;
  int dtype;
  int64_t ld;
  const float *w_scale;
  __device__ __forceinline__ float factor(int64_t) const { return __ldg(w_scale); }
  __device__ __forceinline__ float add(int64_t) const { return 0.0f; }
};
struct OutW {  // dW[n][k] = v
  void *y;
  int dtype;
  int64_t ld;
  __device__ __forceinline__ float factor(int64_t) const { return 1.0f; }
  __device__ __forceinline__ float add(int64_t) const { return 0.0f; }
};
// The CTA's sums (get(c, v): columns c .. of a lane), 32 lanes of i by kColumns of j a warp: to y (rows of j, `ld`
// apart), times the column's factor, plus the lane's `add`
template <typename T, int kColumns, bool REGISTERS, class Get>
__device__ __forceinline__ void put_tile(T *y, int64_t ld, int columns, bool live, const Get &get, const float *factor, float add) {
  constexpr int kGroup = kColumns < 16 ? kColumns : 16;
  static_assert(kColumns % kGroup == 0 && kGroup >= 4, "columns of a warp");
#pragma unroll(REGISTERS ? kColumns : 1)
  for (int c = 0; c < kColumns; c += kGroup) {
    if (c >= columns) break;
    float v[kGroup];
    get(c, v);
    if (!live) continue;
#pragma unroll
    for (int e = 0; e < kGroup; ++e) {
      if (c + e < columns) *y = from_f32<T>(fmaf(v[e], factor[c + e], add));
      y += ld;
    }
  }
}
__device__ __forceinline__ void put_element(void *y, int dtype, int64_t at, float v) {
  if (dtype == 0) static_cast<float *>(y)[at] = v;
  else if (dtype == 1) static_cast<__half *>(y)[at] = __float2half_rn(v);
  else static_cast<__nv_bfloat16 *>(y)[at] = __float2bfloat16_rn(v);
}

// ----------------------------------------------------------------------------- the kernel
// A kernel's order to the one before it on the stream.  kFirst: the first of a call, which begins when all before is over.
// kAfter: it reads what the kernel before it writes, and waits for that one's end at its start.  kBeside: it neither reads nor
// writes what the call's kernels before it write, as the gradients of one call in workspaces of their own, and waits for
// the one before it at its own end, so that what follows on the stream follows both.  (All that the call reads was there when its
// first kernel began.)
enum class Order { kFirst, kAfter, kBeside };
template <class A, class B, class Out>
struct GemmArgs {
  int64_t I, J, R;
  A a;
  B b;
  Out out;
  int tiles_i, steps;  // tiles along i (whole clusters); steps of a split
  int full;            // r that are left for a span to be loaded by full(), more than there are without alignment
  int stages;
  Order order;         // to the kernel before it on the stream
  int parts;           // splits that are one cluster and join in shared memory, else 1
  bool joins;          // the splits' sums join in a second kernel
  float *partial;      // [splits][J][I] where they do, or where a part of R is in chunks (kCarry)
  int *err;            // set to 1 by a wait that gave up
};

// CG CTAs on a tile of 128 CG i by TB j; a B operand of X = TB / CG rows each.  A stage is B's pieces, then A
// (on 1024 bytes where B is swizzled)
template <class A, class B, int TB, int CG>
struct GemmShape {
  static constexpr uint32_t kABytes = tile_bytes(A::kMN, kTileI);
  static constexpr uint32_t kPieceBytes = B::kTma ? TB / CG * 128u : tile_bytes(B::kMN, TB / CG);
  static constexpr uint32_t kOperands = kABytes + B::P * kPieceBytes;
  static constexpr uint32_t kStepBytes = B::kTma ? (kOperands + 1023u) & ~1023u : kOperands;
  // steps of a stage: a single CTA's product has its barriers once a span (they cost the issuing warp more than
  // the MMAs of its narrower step)
  static constexpr int kSteps = CG == 1 ? A::kSpan : 1;
  static constexpr uint32_t kStageBytes = kSteps * kStepBytes;
  // Three pieces carry 32-bit operands, and the tensor cores' 32-bit additions cut off what does not fit: each one
  // loses up to 2^-23 of the sum (4e-6 in all over 96 of them, measured).  So such sums are kept in parts: the lower
  // pieces' in one (2^-8 of the size), the first pieces' in kSets - 1 in turn, each over kChunk steps at most, then
  // added in registers: 28 additions to a part at most.
  static constexpr int kSets = B::P == 3 ? 4 : 1;
  static constexpr int kChunk = 20;  // a multiple of the producers' groups
  // Results of 16 bits have one sum, of so many additions at most (four a step and piece) that it loses a quarter of what
  // rounding it to its type does: 1,024 in half, 2^-13, and 8,192 in bfloat16, 2^-10.  Longer ones are split (gemm_plan: dW of
  // 20,000 x 4,096 x 4,096 in half 895 us in three parts, in bfloat16 785 us whole).
  static constexpr int most_steps(int dtype) { return (dtype == 2 ? 2048 : 256) / B::P; }
  // (Pairs wait for each other's tensor memory, so no mix of these products, of any streams, may run short of it: one of
  // more than half has an SM's shared memory to itself, and of the others a third CTA does not fit that.)
  static constexpr uint32_t kTmemCols = TB * kSets < 32 ? 32 : TB * kSets;
  static constexpr uint32_t kBars = 256 + TB * 4;  // barriers and two words; the columns' factors
  static constexpr int kMaxStages = 8;
  static constexpr int fit(uint32_t room) { return static_cast<int>((room - kBars) / kStageBytes); }
  static constexpr uint32_t kHalfSm = kSmemPerSm / 2 - 1024;
  static constexpr int kCtasPerSm = fit(kHalfSm) >= 2 && 2 * kTmemCols <= 512 ? 2 : 1;
  // stages of a CTA that has half of an SM, or all of one
  static constexpr int stages(bool half) {
    const int n = half ? fit(kHalfSm) : fit(kMaxDynSmem);
    return n < kMaxStages ? n : kMaxStages;
  }
  static constexpr uint32_t smem(int stages) { return stages * kStageBytes + kBars; }
  static_assert(stages(kCtasPerSm == 2) >= 2 && kStageBytes % 16 == 0 && kCtasPerSm * kTmemCols <= 512, "stages and accumulators");
  static_assert(stages(kCtasPerSm == 2) * kStageBytes > kSmemPerSm / 3, "at most two CTAs on an SM");
  static_assert(kTmemCols <= 256 || stages(false) * kStageBytes > kSmemPerSm * 2 / 3, "one CTA on an SM");
  static constexpr bool kClusters = CG == 1 && TB == 16;  // parts of R may join in a cluster (gemm_plan)
  static_assert(!kClusters || stages(kCtasPerSm == 2) * kStageBytes >= kTileI * TB * 4, "a cluster joins its tile in the stages");
  static_assert(A::kSpan == B::kSpan, "operands load together");
};

template <class A, class B, class Out, int TB, int CG>
__global__ void __launch_bounds__(kGemmThreads, GemmShape<A, B, TB, CG>::kCtasPerSm)
    gemm_kernel(const __grid_constant__ GemmArgs<A, B, Out> g) {
  constexpr int P = B::P, kSpan = A::kSpan;
  using S = GemmShape<A, B, TB, CG>;
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t base = smem_u32(smem);
  // full[stages]: this CTA's producers, its copies, and in a pair's first CTA the other's stage, in one barrier (each
  // wait costs the issuing warp some 200 cycles); empty[stages], done; 2 words
  constexpr uint32_t kB = 8 * S::kMaxStages;
  uint8_t *tail = smem + g.stages * S::kStageBytes;
  const uint32_t full = smem_u32(tail), empty = full + kB, done = empty + kB, drained = done + 8;
  volatile uint32_t *word = reinterpret_cast<volatile uint32_t *>(tail + 2 * kB + 16);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = CG == 2 ? cluster_ctarank() : 0;
  // this CTA's tile and part of R.  (In shared memory, and read where they are used: the main loop has no registers
  // to spare for them.)
  volatile int64_t *place = reinterpret_cast<volatile int64_t *>(tail + 2 * kB + 24);
  const auto i0_of = [&]() -> int64_t { return place[0]; };
  const auto j0_of = [&]() -> int64_t { return place[1]; };
  const auto first_of = [&]() -> int64_t { return place[2]; };
  const auto end_of = [&]() -> int64_t { return place[3]; };
  const auto steps_of = [&] { return static_cast<int>(place[4]); };

  if (tid == 0) {
    for (int s = 0; s < g.stages; ++s) {
      mbar_init(full + 8 * s, kGroupWarps + (B::kTma ? 1 : 0) + (CG == 2 && rank == 0 ? 1 : 0));
      mbar_init(empty + 8 * s, 1);
    }
    mbar_init(done, 1);
    mbar_init(drained, CG * kProducerWarps);
    fence_mbar_init_cluster();
    word[1] = 0;
    const int64_t first = static_cast<int64_t>(blockIdx.y) * g.steps * kStep, whole = static_cast<int64_t>(g.steps) * kStep;
    const int64_t end = first + whole < g.R ? first + whole : g.R;
    place[0] = static_cast<int64_t>(blockIdx.x % g.tiles_i) * kTileI, place[1] = static_cast<int64_t>(blockIdx.x / g.tiles_i) * TB;
    place[2] = first, place[3] = end;
    place[4] = kSpan * ((end - first + kSpan * kStep - 1) / (kSpan * kStep));
  }
  grid_trigger();
  // (before the allocation: a pair that held tensor memory while it waited could keep it from a pair that it waits for)
  if (g.order == Order::kAfter) grid_wait();
  if (warp == kProducerWarps) {
    tmem_alloc_cg<CG>(smem_u32(const_cast<uint32_t *>(word)), S::kTmemCols);
    tmem_relinquish_cg<CG>();
  }
  tc_fence_before();
  if constexpr (CG == 2) cluster_sync_all();  // (the other CTA's barriers too)
  else __syncthreads();
  tc_fence_after();
  const uint32_t tmem = word[0];
  // a wait with an end: one that gives up stops the CTA's others too
  auto wait = [&](uint32_t bar, uint32_t parity) -> bool {
    for (int tries = 0; !mbar_try_wait(bar, parity); ++tries) {
      if (word[1]) return false;
      if (tries > kGemmWaitTries) {
        word[1] = 1;
        *g.err = 1;
        return false;
      }
    }
    return true;
  };

  constexpr int kColumns = TB / (kProducerWarps / 4);  // of each of the warps of a lane quadrant
  // this thread's place in the tile: its row (lane of tensor memory), its warp's first column, i, the columns'
  // address.  (Computed where it is used: the main loop has no registers to spare for it.)
  const auto row_of = [] { return static_cast<int>(threadIdx.x & 127); };
  const auto column_of = [] { return static_cast<int>((threadIdx.x >> 7) & 3) * kColumns; };
  const auto i_of = [&] {
    const int r = row_of();
    return i0_of() + (A::kMixed ? (r & ~15) | mix16(r & 15) : r);
  };
  const auto tmem_of = [&] { return tmem + (static_cast<uint32_t>(threadIdx.x & 96) << 16) + column_of(); };
  const auto carry_of = [&](int c) {
    return g.partial + (static_cast<int64_t>(blockIdx.y) * g.J + j0_of() + column_of() + c) * g.I + i_of();
  };
  // Three pieces: the sums over the chunks that are over stay in this thread's registers (a pair's CTA, alone on its
  // SM), or in the part's place of `partial` (half of an SM's registers are too few).
  constexpr bool kKeep = P == 3 && CG == 2, kCarry = P == 3 && CG == 1;
  float acc[kKeep ? kColumns : 1];
  const auto chunks_of = [&] { return P == 3 ? (steps_of() + S::kChunk - 1) / S::kChunk : 1; };
  bool ready = true;
  // the n columns from c on of this warp's: the parts of the chunk in tensor memory
  const auto parts_of = [&](int chunk, int c, auto &v) {
    constexpr int n = sizeof(v) / sizeof(float);
    const uint32_t tl = tmem_of();
    const int left = P == 3 ? steps_of() - chunk * S::kChunk : 0;
    tmem_ld<n>(tl + c, v);
    tmem_wait_ld();
#pragma unroll
    for (int set = 1; set < S::kSets; ++set) {
      float u[n];
      tmem_ld<n>(tl + set * TB + c, u);
      tmem_wait_ld();
      // (a chunk of fewer steps than parts has not written them all)
      const bool used = set == S::kSets - 1 || left > set;
#pragma unroll
      for (int e = 0; e < n; ++e) v[e] += used ? u[e] : 0.0f;
    }
  };
  const auto drain = [&](int chunk) {  // (a whole warp)
    ready = __all_sync(0xffffffffu, wait(done, chunk & 1) && !word[1]);
    if (!ready) return;
    tc_fence_after();
    constexpr int kGroup = kColumns < 16 ? kColumns : 16;
#pragma unroll(kKeep ? kColumns : 1)
    for (int c = 0; c < kColumns; c += kGroup) {
      float v[kGroup];
      parts_of(chunk, c, v);
#pragma unroll
      for (int e = 0; e < kGroup; ++e) {
        if constexpr (kKeep) {
          acc[c + e] = chunk == 0 ? v[e] : acc[c + e] + v[e];
        } else if (i_of() < g.I && j0_of() + column_of() + c + e < g.J) {
          float *o = carry_of(c + e);
          *o = chunk == 0 ? v[e] : *o + v[e];
        }
      }
    }
    tc_fence_before();
    __syncwarp();
    if (lane == 0) {
      if constexpr (CG == 2) mbar_arrive_peer(mapa_cluster(drained, 0));
      else mbar_arrive(drained);
    }
  };
  float *factor = reinterpret_cast<float *>(tail + 256);
  for (int c = tid; c < TB; c += kGemmThreads) factor[c] = g.joins ? 1.0f : j0_of() + c < g.J ? g.out.factor(j0_of() + c) : 0.0f;
  if (warp < kProducerWarps) {
    const int group = warp / kGroupWarps, at = tid - group * kGroupWarps * 32;
    constexpr int kSpanR = kSpan * kStep;
    const auto skip = [&](int &s, uint32_t &parity, int by) {
      s += by;
      if (s >= g.stages) s -= g.stages, parity ^= 1;
    };
    int s = 0;
    uint32_t parity = 1;  // (a stage's first wait is for the phase before its first, and over at once)
    skip(s, parity, group * (kSpan / S::kSteps));
    int chunk = 0;
    // the group's spans among `steps` from `first` on: `load` the next one's, `store` the step's
    const auto produce = [&](int64_t first, int64_t end, int steps) {
      typename A::Thread ta = g.a.init(i0_of(), first + group * kSpanR, at);
      uint32_t ra[A::kRegs];
      int left = static_cast<int>(end - first) - group * kSpanR;
      const auto spans = [&](const auto &load_b, const auto &store_b) {
        const auto load = [&] {
          if (left >= g.full) g.a.full(ta, ra);
          else g.a.load(ta, left, ra);
          load_b(left);
          left -= kGroups * kSpanR;
        };
        load();
        for (int it = group * kSpan; it < steps; it += kGroups * kSpan) {
          if (kKeep && it >= (chunk + 1) * S::kChunk) {
            drain(chunk++);
            if (!ready) return;
          }
#pragma unroll
          for (int h = 0; h < kSpan; ++h) {
            const bool opens = h % S::kSteps == 0, closes = h % S::kSteps == S::kSteps - 1;
            if (opens && !__all_sync(0xffffffffu, wait(empty + 8 * s, parity))) return;
            const uint32_t tile = base + s * S::kStageBytes + h % S::kSteps * S::kStepBytes;
            g.a.store(ta, ra, h == 1, tile + B::P * S::kPieceBytes);
            store_b(h == 1, tile);
            if (closes) {
              __syncwarp();
              if (lane == 0) mbar_arrive(full + 8 * s);
              skip(s, parity, 1);
            }
          }
          load();
          skip(s, parity, (kGroups - 1) * (kSpan / S::kSteps));
        }
      };
      if constexpr (B::kTma) {
        spans([](int) {}, [](bool, uint32_t) {});
      } else {
        typename B::Thread tb = g.b.init(j0_of() + rank * (TB / CG), first + group * kSpanR, at);
        uint32_t rb[B::kRegs];
        spans([&](int left) {
          if (left >= g.full) g.b.full(tb, rb);
          else g.b.load(tb, left, rb);
        }, [&](bool second, uint32_t tile) { g.b.store(tb, rb, second, tile); });
      }
    };
    if constexpr (kCarry) {
      // a chunk at a time, from its own first loads on: the other CTA of the SM has the meantime
      for (;; drain(chunk++)) {
        if (!ready) break;
        const int64_t from = first_of() + static_cast<int64_t>(chunk) * (S::kChunk * kStep), to = from + S::kChunk * kStep;
        const int64_t end = end_of();
        const int steps = steps_of() - chunk * S::kChunk;
        produce(from, to < end ? to : end, steps < S::kChunk ? steps : S::kChunk);
        if (chunk + 1 >= chunks_of()) break;
      }
    } else {
      produce(first_of(), end_of(), steps_of());
    }
    if constexpr (kKeep) {
      // (a group's last step may lie in an earlier chunk than the other's)
      while (ready && chunk < chunks_of()) drain(chunk++);
    }
    named_bar_sync(1, kProducers);  // (the factors)
  } else if (warp == kProducerWarps) {
    // A stage that the producers have written becomes the tensor cores' with one fence between the proxies, here,
    // on the way from their writes to the MMA, and not one in every producer, where it would also wait for
    // the loads in flight.  In the second CTA that is all; it tells the first.
    constexpr uint32_t idesc = gemm_idesc(B::kBf, A::kMN, B::kMN, 128 * CG, TB);
    constexpr uint32_t la = tile_lbo(A::kMN), lb = tile_lbo(B::kMN);
    constexpr uint32_t ka = 2 * la / 16, kb = (!B::kTma ? 2 * lb : B::kMN ? 2048u : 32u) / 16;  // 16 of r on, in 16-byte units
    const uint64_t a0 = make_sdesc(base + P * S::kPieceBytes, la, tile_sbo(A::kMN));
    const uint64_t b0 = !B::kTma ? make_sdesc(base, lb, tile_sbo(B::kMN)) : make_sdesc_sw128(base, B::kMN ? 8192 : 16, 1024);
    const uint32_t full0 = CG == 2 ? mapa_cluster(full, 0) : full;
    int s = 0;
    uint32_t parity = 0;
    const int steps = steps_of();
    for (int it = 0, in = 0, chunk = 0; it < steps; it += S::kSteps, ++in) {  // in: steps of the chunk
      if (P == 3 && in == S::kChunk) {
        in = 0;
        if (rank == 0) {
          mma_commit_cg_warp<CG>(done);
          if (!__all_sync(0xffffffffu, wait(drained, chunk & 1))) break;
          tc_fence_after();
        }
        ++chunk;
      }
      if (!__all_sync(0xffffffffu, wait(full + 8 * s, parity))) break;
      fence_proxy_async_smem();
      if (rank == 0) {
        tc_fence_after();
        // descriptors of stage 0 moved on: an address is in 16-byte units in a descriptor's low word
#pragma unroll
        for (int u = 0; u < S::kSteps; ++u) {
          const uint32_t off = (s * S::kStageBytes + u * S::kStepBytes) >> 4;
#pragma unroll
          for (int p = 0; p < P; ++p) {
            const uint32_t set = P != 3 ? 0u : p > 0 ? S::kSets - 1u : static_cast<uint32_t>(in) % (S::kSets - 1u);
            const bool first = P != 3 ? it == 0 && u == 0 && p == 0 : p == 1 ? in == 0 : p == 0 && in < S::kSets - 1;
            mma_f16_x4_warp<CG, ka, kb>(tmem + set * TB, static_cast<uint32_t>(a0) + off, static_cast<uint32_t>(a0 >> 32),
                                        static_cast<uint32_t>(b0) + off + (p * S::kPieceBytes >> 4), static_cast<uint32_t>(b0 >> 32), idesc,
                                        first ? 0u : 1u);
          }
        }
        mma_commit_cg_warp<CG>(empty + 8 * s);
      } else {
        __syncwarp();
        if (lane == 0) mbar_arrive_peer(full0 + 8 * s);
      }
      if (++s == g.stages) s = 0, parity ^= 1;
    }
    if (rank == 0) mma_commit_cg_warp<CG>(done);
  } else if constexpr (B::kTma) {
    const int64_t x0 = j0_of() + rank * (TB / CG), first = first_of();
    const int steps = steps_of();
    int s = 0, it = 0;
    uint32_t parity = 1;
    for (; it < steps; ++it) {
      if (!__all_sync(0xffffffffu, wait(empty + 8 * s, parity))) break;
      if (lane == 0) {
        mbar_arrive_expect_tx(full + 8 * s, P * S::kPieceBytes);
        g.b.copy(x0, first + static_cast<int64_t>(it) * kStep, base + s * S::kStageBytes, full + 8 * s);
      }
      __syncwarp();
      if (++s == g.stages) s = 0, parity ^= 1;
    }
    // a CTA that gives up still waits for the copies it has begun: until they are over, or with an end
    if (it < steps)
      for (int k = it < g.stages ? 0 : it - g.stages; k < it; ++k)
        for (int tries = 0; !mbar_try_wait(full + 8 * (k % g.stages), (k / g.stages) & 1) && tries < kGemmWaitTries; ++tries) {}
  }
  __syncwarp();
  if constexpr (!kKeep) ready = __all_sync(0xffffffffu, ready && wait(done, (chunks_of() - 1) & 1) && !word[1]);
  tc_fence_after();
  const int64_t i = i_of(), j0 = j0_of();
  const int row = row_of(), c0 = column_of(), chunks = chunks_of();
  // columns c .. of this warp's, whole
  const auto columns_of = [&](int c, auto &v) {
    constexpr int n = sizeof(v) / sizeof(float);
    if constexpr (kKeep) {
#pragma unroll
      for (int e = 0; e < n; ++e) v[e] = acc[c + e];
    } else {
      parts_of(chunks - 1, c, v);
      if (kCarry && chunks > 1 && i < g.I) {
#pragma unroll
        for (int e = 0; e < n; ++e)
          if (j0 + c0 + c + e < g.J) v[e] += *carry_of(c + e);
      }
    }
  };
  if (S::kClusters && g.parts > 1) {
    // A cluster's CTAs hold sums over parts of R.  Each joins TB / parts of the columns: the others send theirs to
    // its shared memory (the stages, once every CTA is done with its own), and it adds them in the parts' order.
    const int part = blockIdx.y, mine = TB / g.parts;
    const bool any = steps_of() > 0;
    cluster_sync_all();
    if (warp < kProducerWarps && ready) {
      constexpr int kGroup = kColumns < 16 ? kColumns : 16;
#pragma unroll(kKeep ? kColumns : 1)
      for (int c = 0; c < kColumns; c += kGroup) {
        float v[kGroup];
        columns_of(c, v);
#pragma unroll
        for (int e = 0; e < kGroup; ++e) {
          const int to = (c0 + c + e) / mine, at = part * mine + (c0 + c + e) - to * mine;
          st_cluster_f32(mapa_cluster(base + 4u * (at * kTileI + row), to), any ? v[e] : 0.0f);
        }
      }
    }
    cluster_sync_all();
    if (warp < kProducerWarps && ready && i < g.I) {
      const float *sums = reinterpret_cast<const float *>(smem);
      const float add = g.out.add(i);
      for (int c = warp >> 2; c < mine; c += kProducerWarps / 4) {
        const int64_t jj = j0 + part * mine + c;
        if (jj >= g.J) break;
        float v = 0.0f;
        for (int k = 0; k < g.parts; ++k) v += sums[(k * mine + c) * kTileI + row];
        put_element(g.out.y, g.out.dtype, jj * g.out.ld + i, fmaf(v, factor[part * mine + c], add));
      }
    }
  } else if (warp < kProducerWarps && ready) {
    const int columns = rows_left(g.J - j0 - c0);
    const bool live = i < g.I;
    const float add = !g.joins && live ? g.out.add(i) : 0.0f;
    const int64_t at = (j0 + c0) * g.out.ld + i;
    if (g.joins)
      put_tile<float, kColumns, kKeep>(carry_of(0), g.I, columns, live, columns_of, factor + c0, 0.0f);
    else if (g.out.dtype == 0)
      put_tile<float, kColumns, kKeep>(static_cast<float *>(g.out.y) + at, g.out.ld, columns, live, columns_of, factor + c0, add);
    else if (g.out.dtype == 1)
      put_tile<__half, kColumns, kKeep>(static_cast<__half *>(g.out.y) + at, g.out.ld, columns, live, columns_of, factor + c0, add);
    else
      put_tile<__nv_bfloat16, kColumns, kKeep>(static_cast<__nv_bfloat16 *>(g.out.y) + at, g.out.ld, columns, live, columns_of,
                                               factor + c0, add);
  }
  tc_fence_before();
  if constexpr (CG == 2) cluster_sync_all();
  else __syncthreads();
  if (warp == kProducerWarps) {
    tc_fence_after();
    tmem_dealloc_cg<CG>(tmem, S::kTmemCols);
  }
  if (g.order == Order::kBeside) grid_wait();
}

// the splits' sums, added in order, and the epilogue: an element a thread
template <class Out>
__global__ void __launch_bounds__(256) gemm_join_kernel(const float *partial, int splits, int64_t I, int64_t J, const Out out) {
  grid_trigger();
  grid_wait();
  const int64_t all = I * J;
  for (int64_t at = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; at < all; at += static_cast<int64_t>(gridDim.x) * 256) {
    const int64_t j = at / I, i = at - j * I;
    float v = 0.0f;
#pragma unroll 8
    for (int s = 0; s < splits; ++s) v += partial[s * all + at];
    put_element(out.y, out.dtype, j * out.ld + i, fmaf(v, out.factor(j), out.add(i)));
  }
}

// the bytes that every row of codes or weights is a multiple of and starts on (load_codes, load_weights), and
// whether rows of gradients are whole 16-byte pieces
inline int codes_unit(const int8_t *codes, int64_t ld, int64_t K) {
  const uintptr_t all = reinterpret_cast<uintptr_t>(codes) | static_cast<uintptr_t>(ld) | static_cast<uintptr_t>(K);
  return (all & 15u) == 0 ? 16 : (all & 3u) == 0 ? 4 : 1;
}
inline int weights_unit(const uint8_t *packed, int64_t K) {
  const uintptr_t p = reinterpret_cast<uintptr_t>(packed);
  return K % 64 == 0 && (p & 15u) == 0 ? 16 : K % 32 == 0 && (p & 7u) == 0 ? 8 : K % 16 == 0 && (p & 3u) == 0 ? 4 : 1;
}
template <typename T>
bool grads_vec(const void *dy, int64_t ld, int64_t N) {
  return (reinterpret_cast<uintptr_t>(dy) & 15u) == 0 && ld * static_cast<int64_t>(sizeof(T)) % 16 == 0 && N % 8 == 0;
}

// How the sum over R is split where there are fewer tiles than SMs: into as many parts as SMs are left for, of at least
// kMinSteps steps each (a pair's, with four times the sums of a single tile: twice as many; dX of 2,048 x 1,024 x 1,024
// whole 11.1 us, in two parts of 8 steps 18.3 us), whose sums a second kernel joins.  Two CTAs to an SM for the parts'
// sake lose more in the joining than they gain (8,192 x 4,096 x 512 39 us whole, 59 us in two parts; 37 x 4,096 x 16,384
// 20 and 25 us), but not where parts of 32-bit sums are longer than a chunk and stop at its end (dX of 2,048 x 512 x
// 16,384 in single tiles: 249 and 219 us; shorter parts, dW of 23,040 x 128 x 512: 23 us in 19, 27 us in 38).
//
// Up to 4 parts of a tile of 16 j are a cluster, which joins them itself: there the second kernel would be an eighth of the time
// (16 x 4,096 x 4,096: 8.6 and 9.7 us).  Wider tiles are slower so (64 x 4,096 x 4,096: 11.7 us in clusters, 11.1 us without;
// 300 x 2,048 x 2,048: 17.7 and 13.2 us), and so are clusters of 8, which wait for 8 SMs of one kind
// (16 x 16,384 x 2,048: 21.9 and 13.0 us).
//
// Sums that are not exact are split too where one accumulator would take more additions than it should (most_steps).
struct GemmPlan {
  int64_t tiles_i, tiles_j;
  int splits, steps;
  bool cluster;
};
constexpr int kMinSteps = 8;
constexpr int64_t kMaxSplits = 65535;  // of a grid (2^29 tokens, or outputs, and more have longer sums)
template <class A, class B, int TB, int CG>
GemmPlan gemm_plan(int64_t I, int64_t J, int64_t R, int sms, int dtype) {
  GemmPlan p;
  p.tiles_i = (I + CG * kTileI - 1) / (CG * kTileI) * CG, p.tiles_j = (J + TB - 1) / TB;
  const int64_t all = (R + kStep - 1) / kStep;
  using S = GemmShape<A, B, TB, CG>;
  const int64_t tiles = p.tiles_i * p.tiles_j;
  int64_t splits = sms / tiles;
  if (B::P == 3 && CG == 1 && all > S::kChunk * (splits < 1 ? 1 : splits)) splits = S::kCtasPerSm * static_cast<int64_t>(sms) / tiles;
  if (splits > all / (CG * kMinSteps)) splits = all / (CG * kMinSteps);
  if (splits < 1) splits = 1;
  if (!A::kExact && B::P < 3) {
    const int64_t least = (all + S::most_steps(dtype) - 1) / S::most_steps(dtype);
    if (splits < least) splits = least < kMaxSplits ? least : kMaxSplits;
  }
  p.cluster = S::kClusters && splits > 1 && splits < 8;
  if (p.cluster) splits = splits >= 4 ? 4 : 2;  // (a power of two, as it divides the tile's columns)
  const int64_t steps = (all + splits - 1) / splits;
  p.steps = static_cast<int>((steps + A::kSpan - 1) / A::kSpan * A::kSpan);
  // (a cluster keeps its parts, the last ones empty where R runs out)
  p.splits = p.cluster ? static_cast<int>(splits) : static_cast<int>((all + p.steps - 1) / p.steps);
  return p;
}
// floats of workspace that the splits' sums take, or those of their chunks
template <class A, class B, int TB, int CG>
int64_t partial_floats(int64_t I, int64_t J, int64_t R, int sms, int dtype) {
  const GemmPlan p = gemm_plan<A, B, TB, CG>(I, J, R, sms, dtype);
  const bool carries = B::P == 3 && CG == 1 && p.steps > GemmShape<A, B, TB, CG>::kChunk;
  return (p.splits > 1 && !p.cluster) || carries ? p.splits * I * J : 0;
}

// (A pair is never kBeside: two kernels of pairs at a time could each hold the tensor memory that the other's pairs lack.)
template <class A, class B, class Out, int TB, int CG>
cudaError_t launch_gemm(int64_t I, int64_t J, int64_t R, const A &a, const B &b, const Out &out, float *partial, int sms, int *err,
                        Order order, cudaStream_t st) {
  using S = GemmShape<A, B, TB, CG>;
  const GemmPlan p = gemm_plan<A, B, TB, CG>(I, J, R, sms, out.dtype);
  const int64_t ctas = p.tiles_i * p.tiles_j * p.splits;
  const int stages = S::stages(S::kCtasPerSm == 2 && ctas > sms);
  const GemmArgs<A, B, Out> g = {I, J, R, a, b, out, static_cast<int>(p.tiles_i), p.steps,
                                   a.aligned() && b.aligned() ? A::kSpan * kStep : INT_MAX, stages, order, p.cluster ? p.splits : 1,
                                   p.splits > 1 && !p.cluster, partial, err};
  auto *kernel = gemm_kernel<A, B, Out, TB, CG>;
  static std::atomic<uint64_t> allowed{0};  // devices on which the kernel may use its shared memory
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = uint64_t(1) << (dev & 63);
  if (dev >= 64 || !(allowed.load(std::memory_order_relaxed) & bit)) {
    if ((e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxDynSmem)) != cudaSuccess) return e;
    if (dev < 64) allowed.fetch_or(bit, std::memory_order_relaxed);
  }
  cudaLaunchAttribute attr[2];
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = CG, attr[0].val.clusterDim.y = p.cluster ? p.splits : 1, attr[0].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(p.tiles_i * p.tiles_j), p.splits);
  cfg.blockDim = dim3(kGemmThreads);
  cfg.dynamicSmemBytes = S::smem(stages);
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = order == Order::kFirst ? 1 : 2;
  if ((e = cudaLaunchKernelEx(&cfg, kernel, g)) != cudaSuccess || !g.joins) return e;
  const int64_t blocks = (I * J + 255) / 256, most = static_cast<int64_t>(sms) * 32;
  return launch_dependent(gemm_join_kernel<Out>, dim3(static_cast<unsigned>(blocks < most ? blocks : most)), 256, 0, st,
                          static_cast<const float *>(partial), p.splits, I, J, out);
}

// The tile of a product.  A pair's 256 x 256 where those fill half of the SMs at least (2,048 x 1,024 x 1,024: 64 CTAs in
// pairs 14.6 us, 128 single ones 9.8 us; 1,024 x 4,096 x 4,096: 128 in pairs 28 us, 256 single ones 50 us), else a
// single CTA's, of 64 j at most where there are no more (the rest of a tile would be converted zeros) or three pieces of
// more would leave an SM one CTA, of 128.
template <int P>
constexpr int kPairTile = P == 3 ? 128 : 256;  // j of a pair's tile: three pieces' sums take four parts of tensor memory
inline bool pair_tiles(int64_t I, int64_t J, int sms) {
  return I > kTileI && J > kTileI && 2 * ((I + 255) / 256 * 2) * ((J + 255) / 256) >= sms;
}
// The gradients' products, of any R, also where single tiles would take each SM through many steps: they convert dy for
// every 128 k, a pair's once for 256, from rows that lie there or are laid out once (long_steps single steps an SM: dW of
// 20,000 x 1,088 x 784 (tokens, K, N) 130 steps, 151 us in single tiles, 88 us in pairs, in 32 bits 291 and 142 us; dX of
// 1,500 x 1,088 x 784 9 steps, 12.7 and 9.9 us.  Of dW's two pieces there is the most to lay out for the least to convert: 3,000 x
// 768 x 1,024 15 steps, 25.2 and 29.9 us; 6,000 x 512 x 1,024 20 steps, 31.7 and 29.4 us).  With up to 256 k dy is
// not read often enough to be laid out (dW of 20,000 x 256 x 1,024: 40 us in single tiles, 47 us in pairs).
template <int P>
constexpr int64_t long_steps = P == 2 ? 16 : 9;
template <int P>
bool grad_pairs(int64_t I, int64_t J, int64_t R, int sms) {
  const int64_t steps = ((I + kTileI - 1) / kTileI) * ((J + 127) / 128) * ((R + kStep - 1) / kStep);
  return pair_tiles(I, J, sms) || (I > 2 * kTileI && J > kTileI && steps >= long_steps<P> * sms);
}
template <int P, class F>
auto with_single_tile(int64_t J, const F &f) {
  return J <= 64 || P == 3 ? f(std::integral_constant<int, 64>()) : f(std::integral_constant<int, 128>());
}

// linear_stage.cu
constexpr int64_t staged_k(int64_t K) { return (K + 127) / 128 * 128; }
struct StageGrads {
  const void *dy;  // [M][N], ld apart
  int64_t ld, M, N;
  int dtype;
  const float *scale;  // [M] or NULL
  int pieces;          // bfloat16 pieces; 0: 16-bit gradients as they are, or the sums alone
  void *out;           // [pieces][M][N up to a multiple of 8] 16-bit, or NULL
  float *db;           // [N] column sums, or NULL
  float *partial;      // [stage_parts(M, N)][N] with db
  Order order;         // kFirst or kBeside: it reads nothing that a call writes
};
int stage_parts(int64_t M, int64_t N);
cudaError_t launch_stage_codes(const int8_t *codes, int64_t ld, int64_t M, int64_t K, void *out, cudaStream_t st);
cudaError_t launch_stage_grads(const StageGrads &c, cudaStream_t st);
// the map of 16-bit rows [pieces][rows][width], ld apart, in boxes of 64 by box_rows
cudaError_t tensor_map(CUtensorMap *map, const void *base, bool bf, int64_t width, int64_t rows, int64_t ld, int pieces, int box_rows);
constexpr int64_t up16(int64_t bytes) { return (bytes + 15) / 16 * 16; }

}  // namespace aecct
