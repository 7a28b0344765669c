// attend.cuh -- the kernel of attend.cu: one new token's query heads over the paged keys and values of its sequence.
//
//   s_j = scale q . k_j,  out = sum_j 2^(x_j - m) v_j / l,  x_j = s_j log2 e,  m = max_j x_j,  l = sum_j 2^(x_j - m)
//
// Work.  The G query heads of a cache head read the same keys and values, so they are one operand of a matrix product: S^T = K q^T
// and O^T = V^T P^T on the tensor cores, 16 keys (and 16 elements of a head) by 8 columns.  A column is a query head, or for P = 2
// half of one: its numbers in two pieces of 16 bits (the number rounded, and what the rounding left), whose products are added up.
// A warp has 8 columns, or 16 where heads are up to 128 wide.  Query heads that do not fit (more than 16 / P, or 8 / P of wider heads) are a piece
// of heads of their own, whose tiles read the same keys and values again: 64 contexts of up to 8,000 tokens, 8 heads of 128 in bfloat16, 193 us for
// 8 query heads to each and 353 for 16; of 256 388 for 4, 710 for 8 and 1,436 for 16.
// The positions of all sequences and cache heads are one list of tiles of TK keys, cut evenly over CTAs and
// over their warps, whatever the lengths are: a warp takes several short sequences, or a part of a long one.  A warp needs no other
// one while it works: it has a ring of stages in shared memory, filled by asynchronous copies that also put zeros where no
// token is, and writes whole sequences out itself.  Parts are joined in shared memory, and those that pass a CTA's
// border by the kernel in attend.cu.
//
// Operands.  The order of the contracted index is free, and so is that of the output's rows.  A lane's share of an
// operand is therefore what it can read from shared memory in 16 bytes: of K, for key g of 8 (g = lane / 4), elements that follow one another
// (the queries are loaded in the same order); of V, for four keys of 16 (2 t, 2 t + 1, 2 t + 8, 2 t + 9; t = lane % 4), elements that
// follow one another, paired by key with byte permutes.  No transposed copy of V is made.  Codes become halves exactly:
// 0x6400 + (code + 128) is the half 1152 + code.
//
// The forms with 16 columns over codes spill: attend_kernel 70 bytes of its 128 registers at 64 wide, 28 of its 255 at 128 (64 contexts as above
// 116 us for 8 query heads in 8 columns, 167 for 16 in 16); attend_whole_kernel 36 and 20, attend_lone_kernel 4 at 64; the others 4 at most.
//
// Bound by memory where sequences are long: a million tokens of 8 cache heads of 128, 8 query heads to each, take 346 us, 6.1 TB/s (a copy of the
// same bytes 313).  Where they are short, by a piece's start and end and by what a warp alone waits for: 512 sequences of up to 180 tokens, 8 heads
// of 16, 16 us.
//
// 32 bits: sums of products, maxima, exponents and sums (exponentials and the scales' logarithms by the hardware's, to 2^-22).  What is rounded: the
// weights, as the tensor cores' operand, to 11 bits in one half for bfloat16 results over codes, else to two pieces (22 bits in halves, 16 in
// bfloat16); float queries over codes, to 22.  A float result is 2.4 times as far from 64 bits as the plain form (5.1e-7 and 2.1e-7), a result in 16
// bits as far.  With codes the scale of a value row belongs to the
// weight: 2^(x_j - m) vs_j = 2^(y_j), y_j = x_j - m + log2 vs_j, has a running maximum of its own, so that the weights that
// count use the whole range of a half.  Queries times codes are exact products: a bfloat16 or half query is scaled by a power of two to fit a half, a float one is cut in two.
#pragma once
#include <cuda_runtime.h>

#include <atomic>
#include <cmath>
#include <cstdint>

#include "aecct_internal.h"
#include "kv_pages.cuh"
#include "rowtypes.cuh"
#include "sm103_ptx.cuh"

namespace aecct {

// a piece of a sequence's attention that passes a CTA's border
struct AttendPiece {
  int b, j;  // the sequence (-1: none), and the piece of its heads
  int ends;  // the last tile is in it
  int last;  // (within a CTA) the warp that it ends in
};
struct AttendArgs {
  KvPages cache;
  KvSequences seqs;
  const int32_t *first;
  const void *q;
  int64_t ld_row, ld_head;
  int group, q_heads, dtype;
  int parts;    // pieces of at most kHeads query heads that the group is cut into
  float scale;  // times log2 e
  void *out;
  float *lse;
  float *partial;      // [CTAs][2][kPart]
  AttendPiece *piece;  // [CTAs][2]
  int ctas;            // of a cluster that takes one piece of heads of one sequence; 0: tiles are dealt out; -1: a warp to each piece
};

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float log2_fast(float x) {
  float r;
  asm("lg2.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, int bytes) {  // the rest of the 16 become zeros
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t dst, const void *src, int bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
template <bool BF16>
__device__ __forceinline__ void mma_16816(float *c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if constexpr (BF16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// the same on nothing
template <bool BF16>
__device__ __forceinline__ void mma_16816_first(float *c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if constexpr (BF16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
}
// an 8 x 8 matrix of 16-bit elements, transposed over the warp
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
// bytes 0 and 1 (or 2 and 3) of codes + 128 as two halves
__device__ __forceinline__ uint32_t halves_of(uint32_t codes, uint32_t select) {
  const uint32_t w = __byte_perm(codes, 0x64646464u, select);
  uint32_t r;
  asm("sub.f16x2 %0, %1, %2;" : "=r"(r) : "r"(w), "r"(0x64806480u));
  return r;
}
constexpr uint32_t kLow = 0x4140u, kHigh = 0x4342u;

// The shapes of a kernel.  C: the cache's type; DP: the head's width, padded; NB: blocks of 8 columns; P: pieces of a number.
// A tile's work that does not grow with its keys is a third of it at 32: tiles of 16 took 492 us for the million tokens, 412 with 12 warps; tiles
// of 32 with 6 warps 459, with 12 (168 registers) 367.  Longer rows have tiles of 16, so that a ring has two stages at least.
template <typename C_, int DP_, int NB_, int P_>
struct AttendShape {
  using C = C_;
  static constexpr int DP = DP_, NB = NB_, P = P_;
  static constexpr int kSize = sizeof(C), kRow = DP * kSize;
  static constexpr int kHeads = 8 * NB / P;
  static constexpr int TK = kRow <= 128 ? 32 : 16;
  static constexpr int kWarps = kRow <= 256 ? 8 : 4;
  static constexpr int kCtas = kRow <= 64 ? 2 : 1;  // to an SM
  static constexpr int kStage = 2 * TK * kRow + 2 * TK * 4 + 16;
  static constexpr int kPart = kHeads * (DP + 2);  // floats of a piece: maxima, sums, rows
  static constexpr int kFixed = 16 * kWarps + 8 * 32 * kWarps + (3 * kWarps + 1) * 16 + (kWarps + kWarps + 1) * 2 * kHeads * 4 + kWarps * kPart * 4;
  static constexpr int kRoom = (227 * 1024 / kCtas - 1024 * (kCtas - 1) - kFixed) / (kWarps * kStage);
  static constexpr int kStages = kRoom > 4 ? 4 : kRoom;
  static constexpr int kSmem = kFixed + kWarps * kStages * kStage;
  static_assert(kStages >= 2 && kStages * kStage >= kPart * 4, "a ring holds a piece");
  static_assert(kStage % 16 == 0 && kFixed % 16 == 0, "copies of 16 bytes");
};

template <class S>
struct AttendWarp {
  using C = typename S::C;
  static constexpr bool kCodes = sizeof(C) == 1;
  static constexpr bool kBf16 = std::is_same_v<C, __nv_bfloat16>;
  static constexpr int DP = S::DP, NB = S::NB, P = S::P, TK = S::TK, M = TK / 16, UPR = S::kRow / 16;
  static constexpr int HC = NB * (3 - P);  // heads of a lane's columns
  static constexpr float kOffset = kBf16 ? 0.0f : 15.0f;  // weights up to 2^15, so that halves reach down to 2^-39 of the largest

  // where in the list of tiles
  struct Cursor {
    int b, j, tile, tiles, t0, lo, hi;
  };

  const AttendArgs &a;
  const uint32_t ring;  // shared memory
  const int lane, g, t;
  const int all;    // pieces of heads of a sequence
  const bool even;  // a tile lies in one page, and its rows follow one another without a gap

  uint32_t qf[DP / 16][NB][2];
  float o[DP / 16][NB][4], top[HC], vtop[HC], l[HC], qs[HC];

  __device__ AttendWarp(const AttendArgs &args, uint32_t ring_)
      : a(args), ring(ring_), lane(threadIdx.x & 31), g((threadIdx.x & 31) >> 2), t(threadIdx.x & 3), all(args.cache.heads * args.parts), even(args.cache.page_size % TK == 0 && args.cache.ld == DP && args.cache.dim == DP) {}

  static __device__ int tiles_of(const AttendArgs &a, int b, int &lo, int &hi) {
    hi = sequence_length(a.seqs, b, a.cache.page_size);
    lo = a.first ? a.first[b] : 0;
    lo = lo < 0 ? 0 : lo;
    return lo < hi ? (hi - 1) / TK - lo / TK + 1 : 0;
  }
  __device__ void sequence(Cursor &c) const {
    c.tiles = tiles_of(a, c.b, c.lo, c.hi);
    c.t0 = c.lo / TK;
  }
  // the next tile; the caller knows that there is one
  __device__ void advance(Cursor &c) const {
    if (++c.tile < c.tiles) return;
    c.tile = 0;
    if (++c.j < all) return;
    c.j = 0;
    do {
      ++c.b;
      sequence(c);
    } while (c.tiles == 0);
  }

  // this lane's row of a tile: its page and place in it, -1 for none
  __device__ void find(const Cursor &c, int &page, int &place) const {
    const int p0 = (c.t0 + c.tile) * TK, p = p0 + lane;
    page = -1, place = 0;
    if (lane < TK && p >= c.lo && p < c.hi) {
      const int of = even ? p0 : p, column = of / a.cache.page_size;  // (a tile in one page: the same for all)
      place = p - column * a.cache.page_size;
      page = a.seqs.table[static_cast<int64_t>(c.b) * a.seqs.ldt + column];
    }
  }
  // the 16-byte unit of a row that a row's unit u is kept in, so that the 8 lanes of a read lie in 8 groups of banks
  static __device__ __forceinline__ uint32_t k_unit(uint32_t row, uint32_t u) { return UPR >= 8 ? u ^ ((row & 1) << 2) : u; }
  static __device__ __forceinline__ uint32_t v_unit(uint32_t row, uint32_t u) {
    return UPR >= 8 ? u ^ (((row >> 1) & 3) << 1) : UPR == 4 ? u ^ (((row >> 1) & 1) << 1) : u;
  }
  // the copies of a tile into a stage; rows without a token and what is past a row's end become zeros
  __device__ void fill(int stage, const Cursor &c, int page, int place) const {
    const uint32_t at = ring + stage * S::kStage;
    const bool fine = page >= 0 && page < a.cache.pages;
    const int64_t row = fine ? (static_cast<int64_t>(page) * a.cache.heads + c.j / a.parts) * a.cache.page_size + place : 0;
    const uint32_t mask = __ballot_sync(0xffffffffu, fine);
    const int64_t from = row * (static_cast<int64_t>(a.cache.ld) * S::kSize);
    constexpr uint32_t kWhole = TK == 32 ? 0xffffffffu : (1u << TK) - 1;
    constexpr int kRows = 32 / UPR > 0 ? 32 / UPR : 1;  // of 32 units
    if (even && mask == kWhole) {  // rows that follow one another, all of them: a copy is one instruction
      const int64_t first = __shfl_sync(0xffffffffu, from, 0) + lane * 16;
      const char *k = static_cast<const char *>(a.cache.k) + first, *v = static_cast<const char *>(a.cache.v) + first;
      const uint32_t r0 = lane / UPR, u = lane % UPR, ku = at + r0 * S::kRow, vu = ku + TK * S::kRow;
#pragma unroll
      for (int i = 0; i < TK * UPR / 32; ++i) {  // (a row is r0 and i kRows in disjoint bits, and so are their parts of a unit's number)
        copy16(ku + i * kRows * S::kRow + (k_unit(r0, u) ^ k_unit(i * kRows, 0)) * 16, k + i * 512, 16);
        copy16(vu + i * kRows * S::kRow + (v_unit(r0, u) ^ v_unit(i * kRows, 0)) * 16, v + i * 512, 16);
      }
    } else {
      const int width = a.cache.dim * S::kSize;
#pragma unroll
      for (int i = 0; i < TK * UPR / 32; ++i) {
        const int r = (i * 32 + lane) / UPR, u = (i * 32 + lane) % UPR;
        const int64_t off = __shfl_sync(0xffffffffu, from, r) + u * 16;
        int bytes = width - u * 16;
        bytes = (mask >> r) & 1 ? (bytes < 0 ? 0 : bytes < 16 ? bytes : 16) : 0;
        const int64_t src = bytes > 0 ? off : 0;
        copy16(at + r * S::kRow + k_unit(r, u) * 16, static_cast<const char *>(a.cache.k) + src, bytes);
        copy16(at + TK * S::kRow + r * S::kRow + v_unit(r, u) * 16, static_cast<const char *>(a.cache.v) + src, bytes);
      }
    }
    if constexpr (kCodes) {
      if (lane < TK) {
        copy4(at + 2 * TK * S::kRow + lane * 4, a.cache.k_scale + row, fine ? 4 : 0);
        copy4(at + 2 * TK * S::kRow + TK * 4 + lane * 4, a.cache.v_scale + row, fine ? 4 : 0);
      }
    }
    if (lane == 0) asm volatile("st.shared.u32 [%0], %1;" ::"r"(at + 2 * TK * S::kRow + 2 * TK * 4), "r"(mask) : "memory");
  }

  static __device__ __forceinline__ float lds(uint32_t p) {
    float v;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(p));
    return v;
  }
  template <int N>
  static __device__ __forceinline__ void lds_words(uint32_t p, uint32_t *w) {
    if constexpr (N == 4) asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(p));
    else if constexpr (N == 2) asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(p));
    else asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[0]) : "r"(p));
  }

  // query head of a column of this piece (its number in the group's piece), and which piece of the number
  static __device__ __forceinline__ int head_of(int column) { return column / P; }
  // EL elements of a row of queries from e on, zeros past its end
  template <typename T, int EL>
  __device__ __forceinline__ void queries(const T *row, int e, bool vectors, float *v) const {
    constexpr int V = kVec<T> < EL ? kVec<T> : EL;
    if (V == kVec<T> && vectors) {
#pragma unroll
      for (int i = 0; i < EL; i += V) {
        if (e + i < a.cache.dim) {
          load_v<T, V>(row + e + i, v + i);
        } else {
#pragma unroll
          for (int k = 0; k < V; ++k) v[i + k] = 0.0f;
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < EL; ++i) v[i] = e + i < a.cache.dim ? to_f32(row[e + i]) : 0.0f;
    }
  }
  template <typename T, int EL>
  __device__ __forceinline__ void query_row(int64_t at, bool on, float (&v)[DP / 4]) const {
    const T *row = static_cast<const T *>(a.q) + at;
    // rows that all start on 16 bytes, and end on them
    const bool vectors = ((reinterpret_cast<uintptr_t>(a.q) | (a.ld_row * sizeof(T)) | (a.ld_head * sizeof(T)) | (a.cache.dim * sizeof(T))) & 15u) == 0;
#pragma unroll
    for (int i = 0; i < DP / 4; ++i) v[i] = 0.0f;
    if (on) {
#pragma unroll
      for (int i = 0; i < DP / 4; i += EL) queries<T, EL>(row, 4 * i + EL * t, vectors, v + i);
    }
  }
  // a sequence's or a head's first tile: the queries in the order of the keys' elements, and nothing summed yet
  __device__ void begin(const Cursor &c) {
    constexpr int EL = DP / 4 < 16 / S::kSize ? DP / 4 : 16 / S::kSize;  // elements of a lane's piece of a key
    const int part = c.j % a.parts, heads = min(S::kHeads, a.group - part * S::kHeads), head0 = c.j / a.parts * a.group + part * S::kHeads;
    float by_column[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const int column = nb * 8 + g, head = head_of(column), which = column % P;
      const bool on = head < heads;
      const int64_t from = c.b * a.ld_row + (head0 + (on ? head : 0)) * a.ld_head;
      float v[DP / 4], most = 0.0f;
      if constexpr (kBf16 || (kCodes && P == 1)) query_row<__nv_bfloat16, EL>(from, on, v);
      else if (kCodes && a.dtype == 0) query_row<float, EL>(from, on, v);
      else query_row<__half, EL>(from, on, v);
#pragma unroll
      for (int i = 0; i < DP / 4; ++i) most = fmaxf(most, fabsf(v[i]));
      float by = 1.0f;
      if constexpr (kCodes) {  // to 2^14 at most
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
        const int e = (__float_as_uint(most) >> 23) - 127;  // (of a denormal: -127)
        const int up = most > 0.0f && most < INFINITY ? 13 - e : 0;  // -114 .. 140, in two factors
        const float f0 = __uint_as_float((127u + up / 2) << 23), f1 = __uint_as_float((127u + up - up / 2) << 23);
#pragma unroll
        for (int i = 0; i < DP / 4; ++i) v[i] = v[i] * f0 * f1;
        by = __uint_as_float((127u - up / 2) << 23) * __uint_as_float((127u - (up - up / 2)) << 23);
      }
      by_column[nb] = by;
#pragma unroll
      for (int i = 0; i < DP / 4; i += 2) {
        uint32_t w = 0;
        if constexpr (kBf16) {
          w = pack2<__nv_bfloat16>(v[i], v[i + 1]);
          if (P == 2 && which == 1) w = 0;  // (a bfloat16 query has one piece)
        } else {
          w = pack2<__half>(v[i], v[i + 1]);
          if (P == 2 && which == 1) {
            float x, y;
            unpack2<__half>(w, x, y);
            w = pack2<__half>(v[i] - x, v[i + 1] - y);
          }
        }
        qf[i / 4][nb][(i / 2) & 1] = w;
      }
    }
#pragma unroll
    for (int hc = 0; hc < HC; ++hc) {
      const int nb = hc / (3 - P), column = P == 2 ? 2 * t : 2 * t + hc % 2;  // (within the block)
      qs[hc] = a.scale;
      if constexpr (kCodes) qs[hc] *= __shfl_sync(0xffffffffu, by_column[nb], column * 4);
      top[hc] = vtop[hc] = -INFINITY, l[hc] = 0.0f;
    }
#pragma unroll
    for (int m = 0; m < DP / 16; ++m)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[m][nb][i] = 0.0f;
  }

  __device__ __forceinline__ static float over_keys_max(float v) {
    v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 4));
    v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 8));
    return fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 16));
  }

  // a tile in a stage
  __device__ void tile(int stage) {
    const uint32_t at = ring + stage * S::kStage, vat = at + TK * S::kRow, scales = vat + TK * S::kRow;
    const uint32_t mask = __float_as_uint(lds(scales + 2 * TK * 4));
    float s[M][NB][4];
    // S^T = K q^T
    constexpr int KB = S::kRow / 4, KW = KB < 16 ? KB / 4 : 4, KP = KB < 16 ? 1 : KB / 16;  // a lane's bytes of a key, words of a piece, pieces
#pragma unroll
    for (int pc = 0; pc < KP; ++pc) {
#pragma unroll
      for (int mt = 0; mt < M; ++mt) {
        uint32_t w[2][KW];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32_t r = mt * 16 + i * 8 + g;
          lds_words<KW>(KB < 16 ? at + r * S::kRow + t * KB : at + r * S::kRow + k_unit(r, pc * 4 + t) * 16, w[i]);
        }
        if constexpr (kCodes) {
#pragma unroll
          for (int i = 0; i < KW; ++i) {
            const uint32_t x = w[0][i] ^ 0x80808080u, y = w[1][i] ^ 0x80808080u;
            const uint32_t a0 = halves_of(x, kLow), a1 = halves_of(y, kLow), a2 = halves_of(x, kHigh), a3 = halves_of(y, kHigh);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
              const uint32_t *b = qf[pc * KW + i][nb];
              if (pc == 0 && i == 0) mma_16816_first<false>(s[mt][nb], a0, a1, a2, a3, b[0], b[1]);
              else mma_16816<false>(s[mt][nb], a0, a1, a2, a3, b[0], b[1]);
            }
          }
        } else {
#pragma unroll
          for (int i = 0; i < KW / 2; ++i)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
              const uint32_t *b = qf[pc * (KW / 2) + i][nb];
              if (pc == 0 && i == 0) mma_16816_first<kBf16>(s[mt][nb], w[0][2 * i], w[1][2 * i], w[0][2 * i + 1], w[1][2 * i + 1], b[0], b[1]);
              else mma_16816<kBf16>(s[mt][nb], w[0][2 * i], w[1][2 * i], w[0][2 * i + 1], w[1][2 * i + 1], b[0], b[1]);
            }
        }
      }
    }
    // scores in powers of two, maxima, weights
    float x[M][2][HC], vs[M][2];
    float most[HC], vmost[HC];
#pragma unroll
    for (int hc = 0; hc < HC; ++hc) most[hc] = top[hc], vmost[hc] = vtop[hc];
#pragma unroll
    for (int mt = 0; mt < M; ++mt)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t r = mt * 16 + i * 8 + g;
        const bool on = (mask >> r) & 1;
        float ks = 1.0f;
        if constexpr (kCodes) ks = lds(scales + r * 4), vs[mt][i] = log2_fast(lds(scales + TK * 4 + r * 4));
#pragma unroll
        for (int hc = 0; hc < HC; ++hc) {
          const int nb = hc / (3 - P);
          float v = P == 2 ? s[mt][nb][2 * i] + s[mt][nb][2 * i + 1] : s[mt][nb][2 * i + hc % 2];
          v = on ? v * (kCodes ? ks * qs[hc] : qs[hc]) : -INFINITY;  // (the factors first: queries and scales may be far from one)
          x[mt][i][hc] = v;
          most[hc] = fmaxf(most[hc], v);
          if constexpr (kCodes) vmost[hc] = fmaxf(vmost[hc], v + vs[mt][i]);
        }
      }
    // (most tiles of a long sequence have no new maximum: one vote instead of its 6 shuffles a head)
    float keep[HC];
    bool higher = false;
#pragma unroll
    for (int hc = 0; hc < HC; ++hc) higher |= most[hc] > top[hc] || (kCodes && vmost[hc] > vtop[hc]), keep[hc] = 1.0f;
    if (__any_sync(0xffffffffu, higher)) {
#pragma unroll
      for (int hc = 0; hc < HC; ++hc) {
        most[hc] = over_keys_max(most[hc]);
        keep[hc] = exp2_fast(top[hc] - (most[hc] == -INFINITY ? 0.0f : most[hc]));
        top[hc] = most[hc], l[hc] *= keep[hc];
        if constexpr (kCodes) {
          vmost[hc] = over_keys_max(vmost[hc]);
          keep[hc] = exp2_fast(vtop[hc] - (vmost[hc] == -INFINITY ? 0.0f : vmost[hc]));
          vtop[hc] = vmost[hc];
        }
      }
    }
#pragma unroll
    for (int hc = 0; hc < HC; ++hc) {  // (0 where no key has been)
      most[hc] = (top[hc] == -INFINITY ? 0.0f : top[hc]) - (kCodes ? 0.0f : kOffset);
      vmost[hc] = (vtop[hc] == -INFINITY ? 0.0f : vtop[hc]) - kOffset;
    }
    uint32_t pf[M][NB][2];
#pragma unroll
    for (int mt = 0; mt < M; ++mt)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float w[HC];
#pragma unroll
        for (int hc = 0; hc < HC; ++hc) {
          const float p = exp2_fast(x[mt][i][hc] - most[hc]);
          l[hc] += p;
          w[hc] = kCodes ? exp2_fast(x[mt][i][hc] + vs[mt][i] - vmost[hc]) : p;
        }
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          using E = std::conditional_t<kBf16, __nv_bfloat16, __half>;
          if constexpr (P == 2) pf[mt][nb][i] = transpose_8x8(pack2<E>(w[nb], w[nb] - to_f32(from_f32<E>(w[nb]))));
          else pf[mt][nb][i] = transpose_8x8(pack2<E>(w[2 * nb], w[2 * nb + 1]));
        }
      }
    // O^T += V^T P^T: the tile's part by itself, added to what there is in one rounded operation
    constexpr int VB = S::kRow / 8, VW = VB < 16 ? VB / 4 : 4, VP = VB < 16 ? 1 : VB / 16;
#pragma unroll
    for (int pc = 0; pc < VP; ++pc) {
      uint32_t w[M][4][VW];
#pragma unroll
      for (int mt = 0; mt < M; ++mt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t r = mt * 16 + 2 * t + (i & 1) + (i >> 1) * 8;
          const uint32_t u = VB >= 16 ? pc * 8 + g : g * VB / 16;
          lds_words<VW>(vat + r * S::kRow + v_unit(r, u) * 16 + (VB >= 16 ? 0 : g * VB % 16), w[mt][i]);
        }
#pragma unroll
      for (int i = 0; i < VW; ++i) {
        constexpr int kPairs = kCodes ? 2 : 1;  // pairs of elements in a word
        float c[kPairs][NB][4];
#pragma unroll
        for (int mt = 0; mt < M; ++mt) {
          if constexpr (kCodes) {
            const uint32_t x0 = w[mt][0][i] ^ 0x80808080u, x1 = w[mt][1][i] ^ 0x80808080u, x2 = w[mt][2][i] ^ 0x80808080u, x3 = w[mt][3][i] ^ 0x80808080u;
#pragma unroll
            for (int h = 0; h < 2; ++h) {  // elements 2 h and 2 h + 1 of the word, each of two keys
              const uint32_t y = __byte_perm(x0, x1, h == 0 ? 0x5140u : 0x7362u), z = __byte_perm(x2, x3, h == 0 ? 0x5140u : 0x7362u);
              const uint32_t a0 = halves_of(y, kLow), a1 = halves_of(y, kHigh), a2 = halves_of(z, kLow), a3 = halves_of(z, kHigh);
#pragma unroll
              for (int nb = 0; nb < NB; ++nb) {
                if (mt == 0) mma_16816_first<false>(c[h][nb], a0, a1, a2, a3, pf[mt][nb][0], pf[mt][nb][1]);
                else mma_16816<false>(c[h][nb], a0, a1, a2, a3, pf[mt][nb][0], pf[mt][nb][1]);
              }
            }
          } else {
            const uint32_t a0 = __byte_perm(w[mt][0][i], w[mt][1][i], 0x5410u), a1 = __byte_perm(w[mt][0][i], w[mt][1][i], 0x7632u);
            const uint32_t a2 = __byte_perm(w[mt][2][i], w[mt][3][i], 0x5410u), a3 = __byte_perm(w[mt][2][i], w[mt][3][i], 0x7632u);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
              if (mt == 0) mma_16816_first<kBf16>(c[0][nb], a0, a1, a2, a3, pf[mt][nb][0], pf[mt][nb][1]);
              else mma_16816<kBf16>(c[0][nb], a0, a1, a2, a3, pf[mt][nb][0], pf[mt][nb][1]);
            }
          }
        }
#pragma unroll
        for (int h = 0; h < kPairs; ++h)
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              float &v = o[(pc * VW + i) * kPairs + h][nb][e];
              v = fmaf(v, keep[P == 2 ? nb : 2 * nb + (e & 1)], c[h][nb][e]);
            }
      }
    }
  }

  static constexpr int EL = DP / 8 < 16 / S::kSize ? DP / 8 : 16 / S::kSize;  // elements that a lane has of a row side by side
  // The last tile of a piece: maxima, sums over the keys and rows that belong to them (in units of 2^top).  f(head, number of the lane's head,
  // element, EL values from there on) takes the rows, s(head, number, top, l) the rest; l is the whole sum in every lane.
  template <class F, class G>
  __device__ void end(F &&f, G &&s) {
    float by[HC];
#pragma unroll
    for (int hc = 0; hc < HC; ++hc) {
      l[hc] += __shfl_xor_sync(0xffffffffu, l[hc], 4);
      l[hc] += __shfl_xor_sync(0xffffffffu, l[hc], 8);
      l[hc] += __shfl_xor_sync(0xffffffffu, l[hc], 16);
      if constexpr (kCodes) by[hc] = vtop[hc] == -INFINITY ? 0.0f : exp2_fast(vtop[hc] - top[hc] - kOffset);
      else by[hc] = exp2_fast(-kOffset), l[hc] *= by[hc];
      const int head = P == 2 ? hc * 4 + t : hc / 2 * 8 + 2 * t + hc % 2;
      s(head, hc, top[hc], l[hc]);
    }
#pragma unroll
    for (int hc = 0; hc < HC; ++hc) {
      const int head = P == 2 ? hc * 4 + t : hc / 2 * 8 + 2 * t + hc % 2;
#pragma unroll
      for (int m0 = 0; m0 < DP / 16; m0 += EL / 2) {
        float row[EL];
#pragma unroll
        for (int i = 0; i < EL / 2; ++i) {
          const float *v = o[m0 + i][hc / (3 - P)];
          row[2 * i] = (P == 2 ? v[0] + v[1] : v[hc % 2]) * by[hc];
          row[2 * i + 1] = (P == 2 ? v[2] + v[3] : v[2 + hc % 2]) * by[hc];
        }
        f(head, hc, 16 * m0 + EL * g, row);
      }
    }
  }
};

__device__ __forceinline__ void store_out(const AttendArgs &a, int64_t at, float v) {
  if (a.dtype == 0) static_cast<float *>(a.out)[at] = v;
  else if (a.dtype == 1) static_cast<__half *>(a.out)[at] = from_f32<__half>(v);
  else static_cast<__nv_bfloat16 *>(a.out)[at] = from_f32<__nv_bfloat16>(v);
}
// N results side by side, in pieces of 16 bytes where rows of the output lie on them (single stores of 32 lanes' results, none of them next to each other,
// were most of the time of short sequences)
template <int N>
__device__ __forceinline__ void store_outs(const AttendArgs &a, int64_t row, int e, const float (&v)[N]) {
  const int64_t at = row * a.cache.dim + e;
  const auto pieces = [&](auto *p) {
    using T = std::remove_reference_t<decltype(*p)>;
    if constexpr (N % kVec<T> == 0) {
      if (((reinterpret_cast<uintptr_t>(p) | a.cache.dim * sizeof(T)) & 15u) == 0 && e + N <= a.cache.dim) {
#pragma unroll
        for (int i = 0; i < N; i += kVec<T>) store_v<T, kVec<T>>(p + at + i, v + i);
        return;
      }
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (e + i < a.cache.dim) p[at + i] = from_f32<T>(v[i]);
  };
  if (a.dtype == 0) pieces(static_cast<float *>(a.out));
  else if (a.dtype == 1) pieces(static_cast<__half *>(a.out));
  else pieces(static_cast<__nv_bfloat16 *>(a.out));
}
// a row's share, of what its keys' weights add up to: nothing where no key was there
__device__ __forceinline__ float share(float v, float l) { return l == 0.0f ? 0.0f : __fdiv_rn(v, l); }
__device__ __forceinline__ float lse_of(float top, float l) { return l == 0.0f ? -INFINITY : fmaf(top, kLn2, logf(l)); }

template <class S>
__global__ void __launch_bounds__(S::kWarps * 32, S::kCtas) attend_kernel(const __grid_constant__ AttendArgs a) {
  constexpr int NT = S::kWarps * 32, W = S::kWarps, TK = S::TK, DP = S::DP, H = S::kHeads;
  using Warp = AttendWarp<S>;
  extern __shared__ __align__(16) unsigned char smem[];
  long long *sums = reinterpret_cast<long long *>(smem);  // [2 W]
  long long *before = sums + 2 * W;                       // [NT]
  AttendPiece *pieces = reinterpret_cast<AttendPiece *>(before + NT);    // [W][2]: what a warp leaves
  AttendPiece *chains = pieces + 2 * W;                                  // [W + 1]: what belongs together
  float *factors = reinterpret_cast<float *>(chains + W + 1);            // [W][2][H]
  float *totals = factors + 2 * W * H;                                   // [W + 1][2][H]: maxima and sums of the chains
  float *heads_of_parts = totals + 2 * (W + 1) * H;                      // [W][kPart]
  unsigned char *rings = smem + S::kFixed;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  grid_trigger();

  // the list of tiles: sequences one after the other, in each its pieces of heads, in each its tiles.  Lane i of every warp adds up the i-th of 32
  // runs of sequences (each warp for itself: no barrier, and the lengths are in L2 or nearer); where there are many, thread i the i-th of NT.
  const int all = a.cache.heads * a.parts;
  const bool wide = a.seqs.batch > 32 * 32;
  const int runs = wide ? NT : 32, run = (a.seqs.batch + runs - 1) / runs, mine_run = wide ? tid : lane;
  const auto lanes_before = [&](long long v) {
    long long s = v;
    for (int d = 1; d < 32; d <<= 1) {
      const long long o = __shfl_up_sync(0xffffffffu, s, d);
      if (lane >= d) s += o;
    }
    return s - v;
  };
  const auto tiles_in = [&](int b) {
    int lo, hi;
    return b < a.seqs.batch ? static_cast<long long>(Warp::tiles_of(a, b, lo, hi)) : 0ll;
  };
  long long sum = 0;
#pragma unroll 4
  for (int i = 0; i < run; ++i) sum += tiles_in(mine_run * run + i);
  long long earlier = lanes_before(sum), total = __shfl_sync(0xffffffffu, earlier + sum, 31);
  if (wide) {
    if (lane == 0) sums[warp] = total;
    __syncthreads();
    total = 0;
    for (int v = 0; v < W; ++v) {
      if (v < warp) earlier += sums[v];
      total += sums[v];
    }
    before[tid] = earlier;
    __syncthreads();
  }
  const long long tiles = total * all, per_cta = max((tiles + gridDim.x - 1) / gridDim.x, static_cast<long long>(W));
  const long long from = min(tiles, blockIdx.x * per_cta), count = min(tiles, from + per_cta) - from;
  const long long per = (count + W - 1) / W;
  const long long mine = from + min(count, warp * per);
  const int n = static_cast<int>(min(per, from + count - mine));  // this warp's tiles
  typename Warp::Cursor at = {};
  if (n > 0) {
    // the last run, and in it the last sequence, with no more than `want` tiles before it
    const long long want = mine / all;
    int i = -1;
    if (wide) {
      for (int k = 0; k < W; ++k) i += __popc(__ballot_sync(0xffffffffu, before[k * 32 + lane] <= want));
      earlier = before[i];
    } else {
      i += __popc(__ballot_sync(0xffffffffu, earlier <= want));
      earlier = __shfl_sync(0xffffffffu, earlier, i);
    }
    long long passed = earlier;
    for (int b = i * run;; b += 32) {
      const long long here = b + lane < (i + 1) * run ? tiles_in(b + lane) : 0, first = passed + lanes_before(here);
      const uint32_t who = __ballot_sync(0xffffffffu, here > 0 && first <= want);
      const int k = 31 - __clz(who);
      const long long end = __shfl_sync(0xffffffffu, first + here, 31);
      if (want < end || b + 32 >= (i + 1) * run) {
        at.b = b + k;
        const long long into = mine - __shfl_sync(0xffffffffu, first, k) * all, len = __shfl_sync(0xffffffffu, here, k);
        at.j = static_cast<int>(into / len), at.tile = static_cast<int>(into % len);
        break;
      }
      passed = end;
    }
  }

  Warp w(a, smem_u32(rings + warp * (S::kStages * S::kStage)));
  if (lane < 2) pieces[warp * 2 + lane] = {-1, 0, 0, 0};
  __syncwarp();
  if (n > 0) {
    w.sequence(at);
    typename Warp::Cursor next = at;
    int page, place, filled = 0;
    w.find(next, page, place);
    const auto fill = [&]() {
      if (filled < n) {
        w.fill(filled % S::kStages, next, page, place);
        if (++filled < n) {
          w.advance(next);
          w.find(next, page, place);
        }
      }
      copies_commit();
    };
    for (int i = 0; i < S::kStages - 1; ++i) fill();
    bool starts = at.tile == 0, fresh = true;
#pragma unroll 1
    for (int i = 0; i < n; ++i) {
      if (fresh) w.begin(at);  // (its loads, while the first copies are under way)
      copies_wait<S::kStages - 2>();
      __syncwarp();
      fill();
      w.tile(i % S::kStages);
      fresh = at.tile == at.tiles - 1;
      if (fresh || i == n - 1) {
        const int part = at.j % a.parts, heads = min(H, a.group - part * H);
        if (starts && fresh) {  // all of it
          const int64_t head0 = static_cast<int64_t>(at.b) * a.q_heads + at.j / a.parts * a.group + part * H;
          float inv[Warp::HC];
          w.end(
              [&](int head, int hc, int e, float (&v)[Warp::EL]) {
#pragma unroll
                for (int k = 0; k < Warp::EL; ++k) v[k] *= inv[hc];
                if (head < heads) store_outs(a, head0 + head, e, v);
              },
              [&](int head, int hc, float top, float l) {
                inv[hc] = l == 0.0f ? 0.0f : __fdiv_rn(1.0f, l);
                if (a.lse && head < heads && w.g == 0) a.lse[head0 + head] = lse_of(top, l);
              });
        } else {
          __syncwarp();
          // (a piece that begins here lasts to the end of this warp's tiles: its place is the ring, where nothing is left to come)
          float *to = starts ? reinterpret_cast<float *>(rings + warp * (S::kStages * S::kStage)) : heads_of_parts + warp * S::kPart;
          w.end(
              [&](int head, int, int e, const float (&v)[Warp::EL]) {
#pragma unroll
                for (int k = 0; k < Warp::EL; k += 4) *reinterpret_cast<float4 *>(to + 2 * H + head * DP + e + k) = make_float4(v[k], v[k + 1], v[k + 2], v[k + 3]);
              },
                [&](int head, int, float top, float l) {
                  if (w.g == 0) to[head] = top, to[H + head] = l;
                });
          if (lane == 0) pieces[warp * 2 + starts] = {at.b, at.j, fresh, 0};
        }
        starts = true;
      }
      if (i < n - 1) w.advance(at);
    }
  }
  __syncthreads();

  // The parts of a sequence's piece in this CTA, joined.  A chain of them begins in slot 0 of warp 0 (it goes on from the CTA before), or in
  // slot 1 of a warp, and goes on in slot 0 of the warps after it.
  const auto part_of = [&](int v, int slot) -> const float * {
    return slot == 1 ? reinterpret_cast<const float *>(rings + v * (S::kStages * S::kStage)) : heads_of_parts + v * S::kPart;
  };
  const int most_heads = min(H, a.group);
  for (int c = warp; c <= W; c += W) {
    const int w0 = c == 0 ? 0 : c - 1, slot = c == 0 ? 0 : 1;
    AttendPiece p = pieces[w0 * 2 + slot];
    p.last = w0;
    if (p.b >= 0) {
      while (!p.ends && p.last + 1 < W && pieces[(p.last + 1) * 2].b >= 0) p.ends = pieces[++p.last * 2].ends;
      // W lanes to a head, one to each part
      const int v = w0 + lane % W;
      const bool in = v <= p.last;
      const float *from_part = part_of(in ? v : w0, v == w0 ? slot : 0);
      for (int h = lane / W; h < most_heads + lane / W; h += 32 / W) {  // (all lanes take part in each round)
        const bool on = in && h < H;
        const float mine = on ? from_part[h] : -INFINITY;
        float top = mine;
        for (int o = W / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        const float by = on ? exp2_fast(mine - (top == -INFINITY ? 0.0f : top)) : 0.0f;
        float l = on ? from_part[H + h] * by : 0.0f;
        for (int o = W / 2; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
        if (on) factors[(v * 2 + (v == w0 ? slot : 0)) * H + h] = by;
        if (on && v == w0) totals[c * 2 * H + h] = top, totals[(c * 2 + 1) * H + h] = l;
      }
    }
    if (lane == 0) chains[c] = p;
  }
  __syncthreads();
  // the chains that there are, and four elements of a head of one of them to a thread
  int chain_of[W + 1], count_of_chains = 0;
  bool noted[2] = {false, false};
#pragma unroll
  for (int c = 0; c <= W; ++c) {
    chain_of[c] = 0;
    const AttendPiece p = chains[c];
    if (p.b < 0) continue;
    const int slot = c == 0 ? 0 : 1;
#pragma unroll
    for (int i = 0; i <= c; ++i)
      if (i == count_of_chains) chain_of[i] = c;
    ++count_of_chains;
    if (slot == 0 || !p.ends) {  // out with a note
      noted[slot] = true;
      if (tid == 0) a.piece[blockIdx.x * 2 + slot] = {p.b, p.j, p.ends, 0};
    }
  }
  for (int i = tid; i < count_of_chains * most_heads * (DP / 4); i += NT) {
    const int n = i / (most_heads * (DP / 4)), head = i / (DP / 4) % most_heads, e = i % (DP / 4) * 4;
    int c = chain_of[0];
#pragma unroll
    for (int k = 1; k <= W; ++k) c = k == n ? chain_of[k] : c;
    const AttendPiece p = chains[c];
    const int w0 = c == 0 ? 0 : c - 1, slot = c == 0 ? 0 : 1, part = p.j % a.parts;
    if (head >= a.group - part * H) continue;
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (int k = w0; k <= p.last; ++k) {
      const int s = k == w0 ? slot : 0;
      const float by = factors[(k * 2 + s) * H + head];
      const float4 x = *reinterpret_cast<const float4 *>(part_of(k, s) + 2 * H + head * DP + e);
      v[0] = fmaf(x.x, by, v[0]), v[1] = fmaf(x.y, by, v[1]), v[2] = fmaf(x.z, by, v[2]), v[3] = fmaf(x.w, by, v[3]);
    }
    const float top = totals[c * 2 * H + head], l = totals[(c * 2 + 1) * H + head];
    if (slot == 1 && p.ends) {
      const int64_t at = static_cast<int64_t>(p.b) * a.q_heads + p.j / a.parts * a.group + part * H + head;
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = share(v[k], l);
      store_outs(a, at, e, v);
      if (e == 0 && a.lse) a.lse[at] = lse_of(top, l);
    } else {
      float *to = a.partial + (blockIdx.x * 2 + slot) * static_cast<int64_t>(S::kPart);
      *reinterpret_cast<float4 *>(to + 2 * H + head * DP + e) = make_float4(v[0], v[1], v[2], v[3]);
      if (e == 0) to[head] = top, to[H + head] = l;
    }
  }
  if (tid < 2 && !noted[tid]) a.piece[blockIdx.x * 2 + tid] = {-1, 0, 0, 0};
}

// Few and short sequences: a cluster of CTAs to each piece of heads of each of them, whose parts are joined through distributed shared memory.  No list, no
// second kernel: one request of 500 tokens 7.2 us instead of 11.3.
template <class S>
__global__ void __launch_bounds__(S::kWarps * 32, S::kCtas) attend_whole_kernel(const __grid_constant__ AttendArgs a) {
  constexpr int NT = S::kWarps * 32, W = S::kWarps, DP = S::DP, H = S::kHeads;
  using Warp = AttendWarp<S>;
  extern __shared__ __align__(16) unsigned char smem[];
  float *factors = reinterpret_cast<float *>(smem);  // [W][H]
  float *sum = factors + W * H;                      // [kPart]: maxima, sums and rows of this CTA's parts together
  unsigned char *rings = smem + S::kFixed;
  static_assert((W * H + S::kPart) * 4 <= S::kFixed, "room before the rings");
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int ctas = a.ctas, rank = ctas > 1 ? static_cast<int>(cluster_ctarank()) : 0, all = a.cache.heads * a.parts;
  typename Warp::Cursor at = {};
  at.b = blockIdx.x / ctas / all, at.j = blockIdx.x / ctas % all;
  Warp w(a, smem_u32(rings + warp * (S::kStages * S::kStage)));
  w.sequence(at);
  const int per_cta = (at.tiles + ctas - 1) / ctas, from = min(at.tiles, rank * per_cta), count = min(at.tiles, from + per_cta) - from;
  const int per = (count + W - 1) / W, used = per > 0 ? (count + per - 1) / per : 0;  // tiles of a warp, and warps that have some
  const int n = warp < used ? min(per, count - warp * per) : 0;
  at.tile = from + warp * per;
  const int part = at.j % a.parts, heads = min(H, a.group - part * H);
  const int64_t head0 = static_cast<int64_t>(at.b) * a.q_heads + at.j / a.parts * a.group + part * H;
  if (n > 0) {
    typename Warp::Cursor next = at;
    int page, place, filled = 0;
    w.find(next, page, place);
    const auto fill = [&]() {
      if (filled < n) {
        w.fill(filled % S::kStages, next, page, place);
        if (++filled < n) ++next.tile, w.find(next, page, place);
      }
      copies_commit();
    };
    for (int i = 0; i < S::kStages - 1; ++i) fill();
    w.begin(at);
#pragma unroll 1
    for (int i = 0; i < n; ++i) {
      copies_wait<S::kStages - 2>();
      __syncwarp();
      fill();
      w.tile(i % S::kStages);
    }
    __syncwarp();
    float *to = reinterpret_cast<float *>(rings + warp * (S::kStages * S::kStage));  // (nothing is left to come there)
    w.end(
        [&](int head, int, int e, const float (&v)[Warp::EL]) {
#pragma unroll
          for (int k = 0; k < Warp::EL; k += 4) *reinterpret_cast<float4 *>(to + 2 * H + head * DP + e + k) = make_float4(v[k], v[k + 1], v[k + 2], v[k + 3]);
        },
        [&](int head, int, float top, float l) {
          if (w.g == 0) to[head] = top, to[H + head] = l;
        });
  }
  __syncthreads();
  const auto part_of = [&](int v) { return reinterpret_cast<const float *>(rings + v * (S::kStages * S::kStage)); };
  for (int h0 = warp * (32 / W); h0 < heads; h0 += 32) {  // W lanes to a head, one to each part
    const int h = h0 + lane / W, v = lane % W;
    const bool on = v < used && h < H;
    const float mine = on ? part_of(v)[h] : -INFINITY;
    float top = mine;
    for (int o = W / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const float by = on ? exp2_fast(mine - (top == -INFINITY ? 0.0f : top)) : 0.0f;
    float l = on ? part_of(v)[H + h] * by : 0.0f;
    for (int o = W / 2; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
    if (h < H) factors[v * H + h] = by;
    if (h < H && v == 0) sum[h] = top, sum[H + h] = l;
  }
  __syncthreads();
  const auto out = [&](int head, int e, float (&v)[4], float top, float l) {
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = share(v[k], l);
    store_outs(a, head0 + head, e, v);
    if (e == 0 && a.lse) a.lse[head0 + head] = lse_of(top, l);
  };
  for (int i = tid; i < heads * (DP / 4); i += NT) {
    const int head = i / (DP / 4), e = i % (DP / 4) * 4;
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (int k = 0; k < used; ++k) {
      const float by = factors[k * H + head];
      const float4 x = *reinterpret_cast<const float4 *>(part_of(k) + 2 * H + head * DP + e);
      v[0] = fmaf(x.x, by, v[0]), v[1] = fmaf(x.y, by, v[1]), v[2] = fmaf(x.z, by, v[2]), v[3] = fmaf(x.w, by, v[3]);
    }
    if (ctas == 1) out(head, e, v, sum[head], sum[H + head]);
    else *reinterpret_cast<float4 *>(sum + 2 * H + head * DP + e) = make_float4(v[0], v[1], v[2], v[3]);
  }
  if (ctas == 1) return;
  cluster_sync_all();
  const uint32_t sums = smem_u32(sum);
  for (int i = rank * NT + tid; i < heads * (DP / 4); i += ctas * NT) {
    const int head = i / (DP / 4), e = i % (DP / 4) * 4;
    float top = -INFINITY, l = 0.0f, v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int r = 0; r < ctas; ++r) top = fmaxf(top, ld_cluster_f32(mapa_cluster(sums + head * 4, r)));
    const float base = top == -INFINITY ? 0.0f : top;
    for (int r = 0; r < ctas; ++r) {
      const float by = exp2_fast(ld_cluster_f32(mapa_cluster(sums + head * 4, r)) - base);
      const float4 x = ld_cluster_f32x4(mapa_cluster(sums + (2 * H + head * DP + e) * 4, r));
      l = fmaf(ld_cluster_f32(mapa_cluster(sums + (H + head) * 4, r)), by, l);
      v[0] = fmaf(x.x, by, v[0]), v[1] = fmaf(x.y, by, v[1]), v[2] = fmaf(x.z, by, v[2]), v[3] = fmaf(x.w, by, v[3]);
    }
    out(head, e, v, top, l);
  }
  cluster_sync_all();  // (no CTA ends while another one reads its sums)
}

// Many short sequences: a warp to each piece of heads of each of them, and nothing to join (512 of up to 180 tokens, 8 heads of 16, 16 us, 25 dealt
// out).
template <class S>
__global__ void __launch_bounds__(S::kWarps * 32, S::kCtas) attend_lone_kernel(const __grid_constant__ AttendArgs a, int pieces) {
  constexpr int H = S::kHeads;
  using Warp = AttendWarp<S>;
  extern __shared__ __align__(16) unsigned char smem[];
  const int warp = threadIdx.x >> 5, all = a.cache.heads * a.parts, piece = blockIdx.x * S::kWarps + warp;
  if (piece >= pieces) return;
  typename Warp::Cursor at = {};
  at.b = piece / all, at.j = piece % all;
  Warp w(a, smem_u32(smem + warp * (S::kStages * S::kStage)));
  w.sequence(at);
  typename Warp::Cursor next = at;
  const int n = at.tiles;
  int page = -1, place = 0, filled = 0;
  if (n > 0) w.find(next, page, place);
  const auto fill = [&]() {
    if (filled < n) {
      w.fill(filled % S::kStages, next, page, place);
      if (++filled < n) ++next.tile, w.find(next, page, place);
    }
    copies_commit();
  };
  for (int i = 0; i < S::kStages - 1; ++i) fill();
  w.begin(at);
#pragma unroll 1
  for (int i = 0; i < n; ++i) {
    copies_wait<S::kStages - 2>();
    __syncwarp();
    fill();
    w.tile(i % S::kStages);
  }
  const int part = at.j % a.parts, heads = min(H, a.group - part * H);
  const int64_t head0 = static_cast<int64_t>(at.b) * a.q_heads + at.j / a.parts * a.group + part * H;
  float inv[Warp::HC];
  w.end(
      [&](int head, int hc, int e, float (&v)[Warp::EL]) {
#pragma unroll
        for (int k = 0; k < Warp::EL; ++k) v[k] *= inv[hc];
        if (head < heads) store_outs(a, head0 + head, e, v);
      },
      [&](int head, int hc, float top, float l) {
        inv[hc] = l == 0.0f ? 0.0f : __fdiv_rn(1.0f, l);
        if (a.lse && head < heads && w.g == 0) a.lse[head0 + head] = lse_of(top, l);
      });
}

// a launch of the kernel: the grid that fills the GPU
struct AttendPlan {
  int ctas, heads, width, part;  // CTAs, query heads of a piece, DP, floats of a piece
  int tile, warps;               // keys of a tile, warps of a CTA
  int at_once[4];                // clusters of 1, 2, 4 and 8 CTAs that the GPU holds
};
template <class S>
cudaError_t launch_whole(const AttendArgs &a, int pieces, cudaStream_t st, int *at_once = nullptr) {
  const cudaError_t e = cudaFuncSetAttribute(attend_whole_kernel<S>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem);
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = static_cast<unsigned>(a.ctas), attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(pieces * a.ctas));
  cfg.blockDim = dim3(S::kWarps * 32);
  cfg.dynamicSmemBytes = S::kSmem;
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (at_once) return cudaOccupancyMaxActiveClusters(at_once, attend_whole_kernel<S>, &cfg);
  return cudaLaunchKernelEx(&cfg, attend_whole_kernel<S>, a);
}
template <class S>
cudaError_t run_attend(const AttendArgs *a, AttendPlan *plan, cudaStream_t st) {
  if (!a) {
    static std::atomic<int> known[64][4];  // by device
    *plan = {sm_count() * S::kCtas, S::kHeads, S::DP, S::kPart, S::TK, S::kWarps, {}};
    int device = 0;
    if (cudaGetDevice(&device) != cudaSuccess || device < 0 || device >= 64) return cudaSuccess;
    for (int i = 0; i < 4; ++i) {
      int n = known[device][i].load(std::memory_order_relaxed);
      if (n == 0) {
        AttendArgs one = {};
        one.ctas = 1 << i;
        if (launch_whole<S>(one, 1, nullptr, &n) != cudaSuccess) n = 0;
        known[device][i].store(n, std::memory_order_relaxed);
      }
      plan->at_once[i] = n;
    }
    return cudaSuccess;
  }
  const int64_t pieces = static_cast<int64_t>(a->seqs.batch) * a->cache.heads * a->parts;
  if (a->ctas > 0) return launch_whole<S>(*a, static_cast<int>(pieces), st);
  if (a->ctas < 0) {
    constexpr int kSmem = S::kWarps * S::kStages * S::kStage;
    const cudaError_t e = cudaFuncSetAttribute(attend_lone_kernel<S>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
    if (e != cudaSuccess) return e;
    attend_lone_kernel<S><<<static_cast<unsigned>((pieces + S::kWarps - 1) / S::kWarps), S::kWarps * 32, kSmem, st>>>(*a, static_cast<int>(pieces));
    return cudaGetLastError();
  }
  const cudaError_t e = cudaFuncSetAttribute(attend_kernel<S>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem);
  if (e != cudaSuccess) return e;
  attend_kernel<S><<<plan->ctas, S::kWarps * 32, S::kSmem, st>>>(*a);
  return cudaGetLastError();
}
// two blocks of columns where one does not hold the group; 256 wide, their queries and rows would not fit the registers
template <typename C, int DP, int P>
cudaError_t run_columns(int group, const AttendArgs *a, AttendPlan *plan, cudaStream_t st) {
  if constexpr (DP <= 128) {
    if (group * P > 8) return run_attend<AttendShape<C, DP, 2, P>>(a, plan, st);
  }
  return run_attend<AttendShape<C, DP, 1, P>>(a, plan, st);
}
template <typename C, int P>
cudaError_t run_width(int dim, int group, const AttendArgs *a, AttendPlan *plan, cudaStream_t st) {
  if (dim <= 32) return run_columns<C, 32, P>(group, a, plan, st);
  if (dim <= 64) return run_columns<C, 64, P>(group, a, plan, st);
  if (dim <= 128) return run_columns<C, 128, P>(group, a, plan, st);
  return run_columns<C, 256, P>(group, a, plan, st);
}

// by the cache's type (attend_codes.cu, attend_pieces.cu, attend_half.cu, attend_bf16.cu); a: NULL for the plan alone
cudaError_t run_attend_codes(int dim, int group, const AttendArgs *a, AttendPlan *plan, cudaStream_t st);   // one piece
cudaError_t run_attend_pieces(int dim, int group, const AttendArgs *a, AttendPlan *plan, cudaStream_t st);  // two
cudaError_t run_attend_half(int dim, int group, const AttendArgs *a, AttendPlan *plan, cudaStream_t st);
cudaError_t run_attend_bf16(int dim, int group, const AttendArgs *a, AttendPlan *plan, cudaStream_t st);

}  // namespace aecct
