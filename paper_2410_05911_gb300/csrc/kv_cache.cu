// kv_cache.cu -- keys and values of new tokens into a paged cache, quantised by eq. Quant as they are written, and
// back.
//
//   alpha = max(max_i |x_i|, 2^-100),  code_i = rint(x_i (127 / alpha)),  scale = alpha / 127    (a row of one token and head)
//   value_i = code_i scale
//
// A row is read and written once.  It has some lanes of a warp (a power of two, 16 elements each), which take its maximum by shuffles; a thread has kAhead
// rows on their way at once.  Reading back is bound by memory (67,700 tokens of 8 heads of 128 into bfloat16 74 us, 5.7 TB/s), writing by its
// instructions too, some 60 for a row of 128 in each of its 8 lanes' warps (19,400 tokens 24 us, 5.0 TB/s; into a 16-bit cache 31.5 us, 5.0 TB/s).  A row
// takes the lanes and the time of the next power of two: 12,300 tokens of 12 float heads of 100 33 to 34 us, of 128 34.
#include <cuda_runtime.h>

#include <cstdint>

#include "aecct_internal.h"
#include "kv_pages.cuh"
#include "rowtypes.cuh"

namespace aecct {

namespace {

constexpr float kAlphaMin = 0x1p-100f;
constexpr int kRowsThreads = 256, kCtas = 4;  // of a CTA; CTAs to an SM
constexpr int E = 16;  // elements of a row to a lane
constexpr int kSearched = 1024, kMaxTokens = 512;  // of a CTA
constexpr int kAhead = 2;  // rows that a lane group has on their way at once, where it has several (4 new ones of 16 bits)

struct RowsPlan {
  int lanes, tokens;  // lanes to a row; tokens of a CTA at most
};

// A lane's E elements of a row of dim (those past its end are 0) as they lie there, so that rows on their way take few registers, and as numbers.
// WIDE: rows of 16-byte pieces.  Else by whole words, two 16-bit elements each, shifted into place where the first is the second of its word (single
// elements, a warp to a row: 65 us for 19,400 tokens of 8 heads of 77).  Elements side by side, but wide rows of floats, of which a lane takes every
// lanes-th piece: with 64 bytes to a lane, lanes read a quarter of a line each (12,300 tokens of 12 heads of 100 35 us, 33 so).
template <typename T, bool WIDE>
struct NewRow {
  static constexpr int kWords = E * sizeof(T) / 4 + (!WIDE && sizeof(T) == 2);
  static constexpr bool kApart = WIDE && sizeof(T) == 4;
  uint32_t w[kWords];
  bool odd;
  // the first of the i-th four elements
  static __device__ __forceinline__ int four(int i, int lane, int lanes) { return kApart ? (i * lanes + lane) * 4 : lane * E + i * 4; }
  __device__ __forceinline__ void load(const T *row, int lane, int lanes, int dim) {
    odd = false;
    if constexpr (WIDE) {
      constexpr int V = kVec<T>;
#pragma unroll
      for (int i = 0; i < E / V; ++i) {
        const int e = four(i * V / 4, lane, lanes);
        uint4 q = make_uint4(0, 0, 0, 0);
        if (e + V <= dim) {
          q = *reinterpret_cast<const uint4 *>(row + e);
        } else if (e < dim) {  // (a row's last elements)
          uint32_t part[4] = {0, 0, 0, 0};
#pragma unroll
          for (int k = 0; k < V; ++k) {
            uint32_t bits = 0;
            if (e + k < dim) {
              if constexpr (sizeof(T) == 4) bits = reinterpret_cast<const uint32_t *>(row)[e + k];
              else bits = reinterpret_cast<const uint16_t *>(row)[e + k];
            }
            part[k * sizeof(T) / 4] |= bits << (k * sizeof(T) % 4 * 8);
          }
          q = make_uint4(part[0], part[1], part[2], part[3]);
        }
        w[4 * i] = q.x, w[4 * i + 1] = q.y, w[4 * i + 2] = q.z, w[4 * i + 3] = q.w;
      }
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < E; ++i) w[i] = lane * E + i < dim ? reinterpret_cast<const uint32_t *>(row)[lane * E + i] : 0;
    } else {
      const T *x = row + lane * E;
      const int n = dim - lane * E;
      odd = reinterpret_cast<uintptr_t>(x) >> 1 & 1;
      const uint32_t *from = reinterpret_cast<const uint32_t *>(reinterpret_cast<uintptr_t>(x) & ~uintptr_t(3));
#pragma unroll
      for (int i = 0; i < kWords; ++i) w[i] = reads_new_word(n, i, odd, E) ? from[i] : 0;
    }
  }
  __device__ __forceinline__ void numbers(int n, float (&v)[E]) const {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < E; ++i) v[i] = __uint_as_float(w[i]);
    } else if constexpr (WIDE) {
#pragma unroll
      for (int i = 0; i < E / 2; ++i) unpack2<T>(w[i], v[2 * i], v[2 * i + 1]);
    } else {
#pragma unroll
      for (int i = 0; i < E / 2; ++i) {
        float a, b;
        unpack2<T>(__funnelshift_r(w[i], w[i + 1], odd * 16), a, b);
        v[2 * i] = 2 * i < n ? a : 0.0f, v[2 * i + 1] = 2 * i + 1 < n ? b : 0.0f;
      }
    }
  }
};
template <typename T>
__device__ __forceinline__ void store_piece(T *x, int e, int dim, const float *v) {
  if (e + kVec<T> <= dim) {
    store_v<T, kVec<T>>(x + e, v);
  } else {
#pragma unroll
    for (int k = 0; k < kVec<T>; ++k)
      if (e + k < dim) x[e + k] = from_f32<T>(v[k]);
  }
}
// Four numbers of up to 127 as codes, each rounded to a whole number by adding 1.5 2^23, whose last byte it then is.
__device__ __forceinline__ uint32_t codes_of(const float *v) {
  const auto b = [&](int i) { return __float_as_uint(v[i] + 12582912.0f); };
  return __byte_perm(__byte_perm(b(0), b(1), 0x0040u), __byte_perm(b(2), b(3), 0x0040u), 0x5410u);
}
// and back: 2^23 + 128 + code, less 2^23 + 128
__device__ __forceinline__ float code_value(uint32_t biased, int i) {
  return __uint_as_float(__byte_perm(biased, 0x4b000000u, 0x7440u | static_cast<uint32_t>(i))) - 8388736.0f;
}

// alpha / 127: the product with 1 / 127 and Markstein's correction by what it leaves of alpha (checked for every mantissa to be the rounded quotient)
__device__ __forceinline__ float scale_of(float alpha) {
  const float by = 1.0f / 127.0f, q = __fmul_rn(alpha, by);
  return fmaf(fmaf(-q, 127.0f, alpha), by, q);
}

// four codes of a row of dim, from element e on; and V (4 or 8) of them back
__device__ __forceinline__ void store_codes(int8_t *row, int e, int dim, uint32_t w) {
  if (e + 4 <= dim) {
    *reinterpret_cast<uint32_t *>(row + e) = w;
  } else {
#pragma unroll
    for (int k = 0; k < 3; ++k)
      if (e + k < dim) row[e + k] = static_cast<int8_t>(w >> (k * 8));
  }
}
template <int V>
__device__ __forceinline__ uint2 load_codes(const int8_t *row, int e, int dim) {
  uint32_t w[2] = {0, 0};
  if (e + V <= dim) {
    if constexpr (V == 8) return *reinterpret_cast<const uint2 *>(row + e);
    else w[0] = *reinterpret_cast<const uint32_t *>(row + e);
  } else {
#pragma unroll
    for (int k = 0; k < V; ++k)
      if (e + k < dim) w[k / 4] |= static_cast<uint32_t>(static_cast<uint8_t>(row[e + k])) << (k % 4 * 8);
  }
  return make_uint2(w[0], w[1]);
}

// the rows of a CTA that a lane group takes: every step-th, as a token and one of its `per` rows
struct RowsWalk {
  int token, at, per, tokens_on, on;
  __device__ RowsWalk(int first, int step, int per_) : token(first / per_), at(first - first / per_ * per_), per(per_), tokens_on(step / per_), on(step - step / per_ * per_) {}
  __device__ __forceinline__ void next() {
    token += tokens_on, at += on;
    if (at >= per) at -= per, ++token;
  }
};

// the places of a CTA's tokens; the search over the sequences in shared memory where they fit (a step in L2 takes 0.3 us)
__device__ __forceinline__ void find_places(const KvRowsCall &c, int64_t token0, int tokens, int64_t *place) {
  __shared__ int32_t rows[kSearched + 1];
  const bool near = c.seqs.rows && c.seqs.batch <= kSearched;
  if (near) {
    for (int i = threadIdx.x; i <= c.seqs.batch; i += kRowsThreads) rows[i] = c.seqs.rows[i];
    __syncthreads();
  }
  for (int i = threadIdx.x; i < tokens; i += kRowsThreads) place[i] = token_row(c.cache, c.seqs, near ? rows : c.seqs.rows, static_cast<int>(token0) + i);
  __syncthreads();
}

// A CTA takes `tokens` tokens, all heads, keys and values.
template <typename T, typename C, int AHEAD, bool WIDE>
__global__ void __launch_bounds__(kRowsThreads, kCtas) append_kernel(const __grid_constant__ KvRowsCall c, RowsPlan p) {
  extern __shared__ int64_t place[];
  const int64_t token0 = static_cast<int64_t>(blockIdx.x) * p.tokens;
  const int lane = threadIdx.x % p.lanes, step = kRowsThreads / p.lanes, dim = c.cache.dim;
  const int tokens = static_cast<int>(min(static_cast<int64_t>(p.tokens), c.total - token0)), rows = tokens * 2 * c.cache.heads;
  RowsWalk w(threadIdx.x / p.lanes, step, 2 * c.cache.heads);
  for (int i = 0; i < rows; i += AHEAD * step) {
    NewRow<T, WIDE> x[AHEAD];
    int token[AHEAD], at[AHEAD];
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
      token[a] = w.token, at[a] = w.at;
      w.next();
      const bool values = at[a] >= c.cache.heads;
      const int64_t r = token0 + token[a];
      const T *from = values ? static_cast<const T *>(c.v) + (r * c.v_row + (at[a] - c.cache.heads) * c.v_head) : static_cast<const T *>(c.k) + (r * c.k_row + at[a] * c.k_head);
      x[a].load(from, lane, p.lanes, token[a] < tokens ? dim : 0);
    }
    if (i == 0) find_places(c, token0, tokens, place);  // (beside the first rows' loads)
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
      const bool values = at[a] >= c.cache.heads;
      const int head = values ? at[a] - c.cache.heads : at[a];
      const int64_t first = token[a] < tokens ? place[token[a]] : -1, row = first + static_cast<int64_t>(head) * c.cache.page_size;
      C *out = static_cast<C *>(values ? c.cache.v : c.cache.k) + row * c.cache.ld;
      float v[E];
      x[a].numbers(dim - lane * E, v);
      if constexpr (sizeof(C) == 1) {
        uint32_t m = 0;  // (as whole numbers, magnitudes keep their order, and a NaN is the largest)
#pragma unroll
        for (int k = 0; k < E; ++k) m = max(m, __float_as_uint(v[k]) & 0x7fffffffu);
        for (int o = p.lanes / 2; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
        const float alpha = __uint_as_float(max(m, __float_as_uint(kAlphaMin))), by = __fdiv_rn(127.0f, alpha);
        if (first < 0) continue;
#pragma unroll
        for (int k = 0; k < E; ++k) v[k] = __fmul_rn(v[k], by);
        const uint4 w4 = make_uint4(codes_of(v), codes_of(v + 4), codes_of(v + 8), codes_of(v + 12));
        const int e = lane * E;
        if (!NewRow<T, WIDE>::kApart && e + E <= dim) {
          *reinterpret_cast<uint4 *>(out + e) = w4;  // (rows start on 16 bytes)
        } else {
          const uint32_t words[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
          for (int k = 0; k < 4; ++k) store_codes(out, NewRow<T, WIDE>::four(k, lane, p.lanes), dim, words[k]);
        }
        if (lane == 0) (values ? c.cache.v_scale : c.cache.k_scale)[row] = scale_of(alpha);
      } else {
        if (first < 0) continue;
#pragma unroll
        for (int k = 0; k < E; k += kVec<C>) store_piece<C>(out, lane * E + k, dim, v + k);
      }
    }
  }
}

// E elements of a cached row (`have` of them, 0 for the others) as they lie there, and as numbers
template <typename C>
struct CachedRow {
  uint4 raw[sizeof(C)];
  float scale;
  __device__ __forceinline__ void load(const C *x, int have, const float *scales) {
    scale = sizeof(C) == 1 && have > 0 ? *scales : 0.0f;
#pragma unroll
    for (int k = 0; k < static_cast<int>(sizeof(C)); ++k) {  // (16 bytes each; a row's last ones element by element)
      constexpr int V = 16 / sizeof(C);
      raw[k] = make_uint4(0, 0, 0, 0);
      if (have >= (k + 1) * V) {
        raw[k] = reinterpret_cast<const uint4 *>(x)[k];
      } else if (have > k * V) {
        uint32_t words[4] = {0, 0, 0, 0};
#pragma unroll
        for (int h = 0; h < V; ++h) {
          uint32_t bits = 0;
          if (k * V + h < have) {
            if constexpr (sizeof(C) == 1) bits = reinterpret_cast<const uint8_t *>(x)[k * V + h];
            else bits = reinterpret_cast<const uint16_t *>(x)[k * V + h];
          }
          words[h * sizeof(C) / 4] |= bits << (h * sizeof(C) % 4 * 8);
        }
        raw[k] = make_uint4(words[0], words[1], words[2], words[3]);
      }
    }
  }
  __device__ __forceinline__ void numbers(float (&v)[E]) const {
    if constexpr (sizeof(C) == 1) {
      const uint32_t words[4] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w};
#pragma unroll
      for (int k = 0; k < E; ++k) v[k] = __fmul_rn(code_value(words[k / 4] ^ 0x80808080u, k % 4), scale);
    } else {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint32_t words[4] = {raw[k].x, raw[k].y, raw[k].z, raw[k].w};
#pragma unroll
        for (int h = 0; h < 4; ++h) unpack2<C>(words[h], v[k * 8 + 2 * h], v[k * 8 + 2 * h + 1]);
      }
    }
  }
};

// A lane takes every lanes-th piece of 16 bytes of a row, so that what the lanes write at once lies side by side (E elements side by side: 53 us instead of
// 39 for 19,400 tokens in float).
template <typename C, typename T, int AHEAD>
__global__ void __launch_bounds__(kRowsThreads, kCtas) read_kernel(const __grid_constant__ KvRowsCall c, RowsPlan p) {
  extern __shared__ int64_t place[];
  constexpr int V = kVec<T>;
  const int64_t token0 = static_cast<int64_t>(blockIdx.x) * p.tokens;
  const int lane = threadIdx.x % p.lanes, step = kRowsThreads / p.lanes, dim = c.cache.dim;
  const int tokens = static_cast<int>(min(static_cast<int64_t>(p.tokens), c.total - token0)), rows = tokens * 2 * c.cache.heads;
  find_places(c, token0, tokens, place);
  RowsWalk w(threadIdx.x / p.lanes, step, 2 * c.cache.heads);
  for (int i = threadIdx.x / p.lanes; i < rows; i += AHEAD * step) {
    uint2 raw[AHEAD][E / V];  // V codes, or elements of 16 bits, of a piece of the output
    uint2 more[AHEAD][E / V];
    float scale[AHEAD];
    int token[AHEAD], at[AHEAD];
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
      token[a] = w.token, at[a] = w.at;
      w.next();
      const bool values = at[a] >= c.cache.heads;
      const int64_t first = token[a] < tokens ? place[token[a]] : -1, row = first + static_cast<int64_t>(values ? at[a] - c.cache.heads : at[a]) * c.cache.page_size;
      const C *x = static_cast<const C *>(values ? c.cache.v : c.cache.k) + row * c.cache.ld;
      const int have = first < 0 ? 0 : dim;
      scale[a] = 0.0f;
      if constexpr (sizeof(C) == 1)
        if (have > 0) scale[a] = (values ? c.cache.v_scale : c.cache.k_scale)[row];
#pragma unroll
      for (int k = 0; k < E / V; ++k) {
        const int e = (k * p.lanes + lane) * V;
        if constexpr (sizeof(C) == 1) {
          raw[a][k] = load_codes<V>(x, e, have);
        } else {  // (as bytes: twice as many)
          raw[a][k] = load_codes<8>(reinterpret_cast<const int8_t *>(x), e * 2, have * 2);
          if constexpr (V == 8) more[a][k] = load_codes<8>(reinterpret_cast<const int8_t *>(x), e * 2 + 8, have * 2);
        }
      }
    }
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
      if (token[a] >= tokens) break;
      const bool values = at[a] >= c.cache.heads;
      T *out = static_cast<T *>(values ? c.v_out : c.k_out) + ((token0 + token[a]) * c.cache.heads + (values ? at[a] - c.cache.heads : at[a])) * c.cache.dim;
      float v[E];
#pragma unroll
      for (int k = 0; k < E / V; ++k) {
        float *to = v + k * V;
        if constexpr (sizeof(C) == 1) {
#pragma unroll
          for (int h = 0; h < V; ++h) to[h] = __fmul_rn(code_value((h < 4 ? raw[a][k].x : raw[a][k].y) ^ 0x80808080u, h % 4), scale[a]);
        } else {
          unpack2<C>(raw[a][k].x, to[0], to[1]), unpack2<C>(raw[a][k].y, to[2], to[3]);
          if constexpr (V == 8) unpack2<C>(more[a][k].x, to[4], to[5]), unpack2<C>(more[a][k].y, to[6], to[7]);
        }
      }
#pragma unroll
      for (int k = 0; k < E / V; ++k) store_piece<T>(out, (k * p.lanes + lane) * V, dim, v + k * V);
    }
  }
}

// The same where the rows that come out do not lie on 16 bytes: they follow one another, so that those of a pass go through shared memory, kept there as far
// from a 16-byte border as in the output, and out in pieces of 16 bytes (one element at a time: 61 us for 70 MB).
template <typename C, typename T, int AHEAD>
__global__ void __launch_bounds__(kRowsThreads, kCtas) read_through_kernel(const __grid_constant__ KvRowsCall c, RowsPlan p) {
  extern __shared__ int64_t place[];
  __shared__ __align__(16) T buf[AHEAD * kRowsThreads * E + kVec<T>];  // (a lane's E elements, and the border)
  const int64_t token0 = static_cast<int64_t>(blockIdx.x) * p.tokens;
  const int lane = threadIdx.x % p.lanes, group = threadIdx.x / p.lanes, step = kRowsThreads / p.lanes, e = lane * E, n = c.cache.dim - e;
  const int tokens = static_cast<int>(min(static_cast<int64_t>(p.tokens), c.total - token0)), rows = tokens * c.cache.heads;
  // A row's last 16 bytes are read whole, what lies behind its end with them, which goes no further (one by one: 19.2 us for 16.4 from 16 bits, 26 for 19.5
  // from codes); but not the cache's last row's, behind which its memory may end.
  const int64_t last = c.cache.pages * c.cache.heads * c.cache.page_size - 1;
  const int whole = reads_cached(n, sizeof(C), true), exact = reads_cached(n, sizeof(C), false);
  find_places(c, token0, tokens, place);
  for (int values = 0; values < 2; ++values) {
    const C *from = static_cast<const C *>(values ? c.cache.v : c.cache.k);
    const float *scales = values ? c.cache.v_scale : c.cache.k_scale;
    for (int i = 0; i < rows; i += AHEAD * step) {
      CachedRow<C> x[AHEAD];
#pragma unroll
      for (int a = 0; a < AHEAD; ++a) {
        const int r = i + group + a * step, token = r / c.cache.heads, head = r - token * c.cache.heads;
        const int64_t first = r < rows ? place[token] : -1, row = first + static_cast<int64_t>(head) * c.cache.page_size;
        x[a].load(from + (row * c.cache.ld + e), first < 0 ? 0 : row < last ? whole : exact, scales + row);
      }
      T *out = static_cast<T *>(values ? c.v_out : c.k_out) + (token0 * c.cache.heads + i) * c.cache.dim;
      const int off = static_cast<int>((reinterpret_cast<uintptr_t>(out) & 15u) / sizeof(T)), count = min(rows - i, AHEAD * step) * c.cache.dim;
#pragma unroll
      for (int a = 0; a < AHEAD; ++a) {
        float v[E];
        x[a].numbers(v);
        T *to = buf + off + (group + a * step) * c.cache.dim + e;
#pragma unroll
        for (int k = 0; k < E; ++k)
          if (k < n) to[k] = from_f32<T>(v[k]);
      }
      __syncthreads();
      constexpr int V = kVec<T>;
      for (int q = threadIdx.x * V; q < off + count; q += kRowsThreads * V) {
        if (q >= off && q + V <= off + count) {
          *reinterpret_cast<uint4 *>(out + (q - off)) = *reinterpret_cast<const uint4 *>(buf + q);
        } else {
#pragma unroll
          for (int k = 0; k < V; ++k)
            if (q + k >= off && q + k < off + count) out[q - off + k] = buf[q + k];
        }
      }
      __syncthreads();
    }
  }
}

// One wave of four CTAs to an SM, each with a share of the tokens: finding their places is a chain of three trips to L2 (with 4 tokens to a CTA, 4,500 CTAs
// of them, 19,400 prompt tokens took 77 us).  Few tokens: a CTA to each pass over its lanes.
template <class F>
cudaError_t plan_rows(const KvRowsCall &c, F &&launch) {
  RowsPlan p = {1, 1};
  while (p.lanes * E < c.cache.dim) p.lanes *= 2;
  const int64_t groups = kRowsThreads / p.lanes, rows = 2 * static_cast<int64_t>(c.cache.heads), ctas = kCtas * static_cast<int64_t>(sm_count());
  int64_t tokens = (c.total + ctas - 1) / ctas;
  if (tokens * rows < groups) tokens = groups / rows;
  p.tokens = static_cast<int>(tokens < 1 ? 1 : tokens > kMaxTokens ? kMaxTokens : tokens);
  launch(static_cast<unsigned>((c.total + p.tokens - 1) / p.tokens), p, static_cast<size_t>(p.tokens) * sizeof(int64_t), p.tokens * rows >= kAhead * groups);
  return cudaGetLastError();
}

// whether rows of these tensors (dim elements, their places so many elements apart) are pieces of 16 bytes
bool in_pieces(const void *k, const void *v, int64_t a, int64_t b, int64_t x, int64_t y, int dim, int size) {
  return ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v) | static_cast<uintptr_t>((a | b | x | y | dim) * size)) & 15u) == 0;
}

template <typename T, typename C>
cudaError_t append_of(const KvRowsCall &c, cudaStream_t st) {
  const bool wide = in_pieces(c.k, c.v, c.k_row, c.k_head, c.v_row, c.v_head, 0, sizeof(T));
  return plan_rows(c, [&](unsigned grid, const RowsPlan &p, size_t smem, bool many) {
    const auto kernel = wide ? (many ? append_kernel<T, C, 8 / sizeof(T), true> : append_kernel<T, C, 1, true>)
                             : many ? append_kernel<T, C, kAhead, false> : append_kernel<T, C, 1, false>;
    kernel<<<grid, kRowsThreads, smem, st>>>(c, p);
  });
}
template <typename C, typename T>
cudaError_t read_of(const KvRowsCall &c, cudaStream_t st) {
  const bool wide = in_pieces(c.k_out, c.v_out, 0, 0, 0, 0, c.cache.dim, sizeof(T));
  return plan_rows(c, [&](unsigned grid, const RowsPlan &p, size_t smem, bool many) {
    const auto kernel = wide ? (many ? read_kernel<C, T, kAhead> : read_kernel<C, T, 1>) : many ? read_through_kernel<C, T, kAhead> : read_through_kernel<C, T, 1>;
    kernel<<<grid, kRowsThreads, smem, st>>>(c, p);
  });
}
template <typename C>
cudaError_t read_from(const KvRowsCall &c, cudaStream_t st) {
  return c.dtype == 0 ? read_of<C, float>(c, st) : c.dtype == 1 ? read_of<C, __half>(c, st) : read_of<C, __nv_bfloat16>(c, st);
}

}  // namespace

cudaError_t launch_kv_append(const KvRowsCall &c, cudaStream_t st) {
  if (c.cache_dtype == 1) return append_of<__half, __half>(c, st);
  if (c.cache_dtype == 2) return append_of<__nv_bfloat16, __nv_bfloat16>(c, st);
  return c.dtype == 0 ? append_of<float, int8_t>(c, st) : c.dtype == 1 ? append_of<__half, int8_t>(c, st) : append_of<__nv_bfloat16, int8_t>(c, st);
}

cudaError_t launch_kv_read(const KvRowsCall &c, cudaStream_t st) {
  return c.cache_dtype == 3 ? read_from<int8_t>(c, st) : c.cache_dtype == 1 ? read_from<__half>(c, st) : read_from<__nv_bfloat16>(c, st);
}

}  // namespace aecct
