// kv_cache.cu -- keys and values of new tokens into a paged cache, quantised by eq. Quant as they are written, and
// back.
//
//   alpha = max(max_i |x_i|, 2^-100),  code_i = rint(x_i (127 / alpha)),  scale = alpha / 127    (a row of one token and head)
//   value_i = code_i scale
//
// Bound by memory: a row is read and written once.  A row has G lanes of a warp (a power of two, 8 elements each), which take its maximum
// by shuffles; a thread has kAhead rows on their way at once.  Where a row of tensors that lie anyhow has no 16-byte
// pieces, its elements are read one by one, by the same lanes.
#include <cuda_runtime.h>

#include <cstdint>

#include "aecct_internal.h"
#include "kv_pages.cuh"
#include "rowtypes.cuh"

namespace aecct {

namespace {

constexpr float kAlphaMin = 0x1p-100f;
constexpr int kRowsThreads = 256;
constexpr int E = 8;  // elements of a row to a lane
constexpr int kSearched = 1024, kMaxTokens = 512;  // of a CTA

struct RowsPlan {
  int lanes, tokens;  // lanes to a row; tokens of a CTA at most
  bool wide;          // rows of the call's tensors in pieces of 16 bytes
};

template <typename T>
__device__ __forceinline__ void load_row(const T *x, int n, bool wide, float (&v)[E]) {
  if (wide && n >= E) {
#pragma unroll
    for (int i = 0; i < E; i += kVec<T>) load_v<T, kVec<T>>(x + i, v + i);
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] = i < n ? to_f32(x[i]) : 0.0f;
  }
}
template <typename T>
__device__ __forceinline__ void store_row(T *x, int n, bool wide, const float (&v)[E]) {
  if (wide && n >= E) {
#pragma unroll
    for (int i = 0; i < E; i += kVec<T>) store_v<T, kVec<T>>(x + i, v + i);
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (i < n) x[i] = from_f32<T>(v[i]);
  }
}
__device__ __forceinline__ uint32_t codes_of(float a, float b, float c, float d) {  // (values of -127 .. 127; a NaN becomes 0)
  return (__float2int_rn(a) & 0xff) | (__float2int_rn(b) & 0xff) << 8 | (__float2int_rn(c) & 0xff) << 16 | static_cast<uint32_t>(__float2int_rn(d)) << 24;
}

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
template <typename T, typename C, int AHEAD>
__global__ void __launch_bounds__(kRowsThreads) append_kernel(const __grid_constant__ KvRowsCall c, RowsPlan p) {
  extern __shared__ int64_t place[];
  const int64_t token0 = static_cast<int64_t>(blockIdx.x) * p.tokens;
  const int lane = threadIdx.x % p.lanes, step = kRowsThreads / p.lanes, e = lane * E, n = c.cache.dim - e;
  const int tokens = static_cast<int>(min(static_cast<int64_t>(p.tokens), c.total - token0)), rows = tokens * 2 * c.cache.heads;
  const auto row_of = [&](int i, int &token, int &which, int &head) {
    token = i / (2 * c.cache.heads);
    const int h = i - token * 2 * c.cache.heads;
    which = h >= c.cache.heads, head = h - which * c.cache.heads;
  };
  bool found = false;
  for (int i0 = threadIdx.x / p.lanes; i0 - static_cast<int>(threadIdx.x / p.lanes) < rows; i0 += AHEAD * step) {
    float v[AHEAD][E];
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
      const int i = i0 + a * step;
      int token, which, head;
      row_of(i < rows ? i : 0, token, which, head);
      const int64_t r = token0 + token;
      const T *x = static_cast<const T *>(which ? c.v : c.k) + (which ? r * c.v_row + head * c.v_head : r * c.k_row + head * c.k_head);
      load_row<T>(x + e, i < rows ? n : 0, p.wide, v[a]);
    }
    if (!found) find_places(c, token0, tokens, place), found = true;  // (beside the first rows' loads)
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
      const int i = i0 + a * step;
      int token, which, head;
      row_of(i < rows ? i : 0, token, which, head);
      const int64_t at = i < rows ? place[token] : -1, row = at < 0 ? -1 : at + static_cast<int64_t>(head) * c.cache.page_size;
      C *out = static_cast<C *>(which ? c.cache.v : c.cache.k) + (row < 0 ? 0 : row * c.cache.ld + e);
      if constexpr (sizeof(C) == 1) {
        float m = 0.0f;
#pragma unroll
        for (int k = 0; k < E; ++k) {
          const float w = fabsf(v[a][k]);
          m = (w > m || w != w) ? w : m;  // (a NaN stays)
        }
        for (int o = p.lanes / 2; o > 0; o >>= 1) {
          const float w = __shfl_xor_sync(0xffffffffu, m, o);
          m = (w > m || w != w) ? w : m;
        }
        const float alpha = m < kAlphaMin ? kAlphaMin : m, by = __fdiv_rn(127.0f, alpha);
        if (row < 0) continue;
#pragma unroll
        for (int k = 0; k < E; ++k) v[a][k] = __fmul_rn(v[a][k], by);
        const uint2 w = make_uint2(codes_of(v[a][0], v[a][1], v[a][2], v[a][3]), codes_of(v[a][4], v[a][5], v[a][6], v[a][7]));
        if (n >= E) {
          *reinterpret_cast<uint2 *>(out) = w;  // (rows start on 16 bytes)
        } else {
#pragma unroll
          for (int k = 0; k < E; ++k)
            if (k < n) out[k] = static_cast<int8_t>((k < 4 ? w.x : w.y) >> (k % 4 * 8));
        }
        if (lane == 0) (which ? c.cache.v_scale : c.cache.k_scale)[row] = __fdiv_rn(alpha, 127.0f);
      } else {
        if (row >= 0) store_row<C>(out, n, true, v[a]);
      }
    }
  }
}

template <typename C, typename T, int AHEAD>
__global__ void __launch_bounds__(kRowsThreads) read_kernel(const __grid_constant__ KvRowsCall c, RowsPlan p) {
  extern __shared__ int64_t place[];
  const int64_t token0 = static_cast<int64_t>(blockIdx.x) * p.tokens;
  const int lane = threadIdx.x % p.lanes, step = kRowsThreads / p.lanes, e = lane * E, n = c.cache.dim - e;
  const int tokens = static_cast<int>(min(static_cast<int64_t>(p.tokens), c.total - token0)), rows = tokens * 2 * c.cache.heads;
  find_places(c, token0, tokens, place);
  for (int i0 = threadIdx.x / p.lanes; i0 < rows; i0 += AHEAD * step) {
    float v[AHEAD][E];
    T *out[AHEAD];
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
      const int i = i0 + a * step;
      if (i >= rows) break;
      // values after all of the keys: each tensor is written in order
      const int which = i >= tokens * c.cache.heads, j = i - which * tokens * c.cache.heads, token = j / c.cache.heads, head = j - token * c.cache.heads;
      const int64_t at = place[token], row = at < 0 ? -1 : at + static_cast<int64_t>(head) * c.cache.page_size;
      out[a] = static_cast<T *>(which ? c.v_out : c.k_out) + ((token0 + token) * c.cache.heads + head) * c.cache.dim + e;
      const C *x = static_cast<const C *>(which ? c.cache.v : c.cache.k) + (row < 0 ? 0 : row * c.cache.ld + e);
      if constexpr (sizeof(C) == 1) {
        const float scale = row < 0 ? 0.0f : (which ? c.cache.v_scale : c.cache.k_scale)[row];
        uint2 w = make_uint2(0, 0);
        if (row >= 0 && n >= E) {
          w = *reinterpret_cast<const uint2 *>(x);
        } else if (row >= 0) {
#pragma unroll
          for (int k = 0; k < E; ++k)
            if (k < n) (k < 4 ? w.x : w.y) |= static_cast<uint32_t>(static_cast<uint8_t>(x[k])) << (k % 4 * 8);
        }
#pragma unroll
        for (int k = 0; k < E; ++k) v[a][k] = __fmul_rn(static_cast<float>(static_cast<int8_t>((k < 4 ? w.x : w.y) >> (k % 4 * 8))), scale);
      } else {
        load_row<C>(x, row < 0 ? 0 : n, true, v[a]);
      }
    }
#pragma unroll
    for (int a = 0; a < AHEAD; ++a)
      if (i0 + a * step < rows) store_row<T>(out[a], n, p.wide, v[a]);
  }
}

// One wave of four CTAs to an SM, each with a share of the tokens: finding their places is a chain of three trips to L2 (with 4 tokens to a CTA, 4,500 CTAs
// of them, 18,000 prompt tokens took 77 us).  Few tokens: a CTA to each pass over its lanes.
template <class F>
cudaError_t plan_rows(const KvRowsCall &c, bool wide, F &&launch) {
  RowsPlan p = {1, 1, wide};
  while (p.lanes * E < c.cache.dim) p.lanes *= 2;
  const int64_t groups = kRowsThreads / p.lanes, rows = 2 * static_cast<int64_t>(c.cache.heads), ctas = 4 * static_cast<int64_t>(sm_count());
  int64_t tokens = (c.total + ctas - 1) / ctas;
  if (tokens * rows < groups) tokens = groups / rows;
  p.tokens = static_cast<int>(tokens < 1 ? 1 : tokens > kMaxTokens ? kMaxTokens : tokens);
  launch(static_cast<unsigned>((c.total + p.tokens - 1) / p.tokens), p, static_cast<size_t>(p.tokens) * sizeof(int64_t), p.tokens * rows >= 4 * groups);
  return cudaGetLastError();
}

// whether rows of these tensors (dim elements, their places so many elements apart) are pieces of 16 bytes
bool in_pieces(const void *k, const void *v, int64_t a, int64_t b, int64_t x, int64_t y, int dim, int size) {
  return ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v) | static_cast<uintptr_t>((a | b | x | y | dim) * size)) & 15u) == 0;
}

template <typename T, typename C>
cudaError_t append_of(const KvRowsCall &c, cudaStream_t st) {
  return plan_rows(c, in_pieces(c.k, c.v, c.k_row, c.k_head, c.v_row, c.v_head, 0, sizeof(T)), [&](unsigned grid, const RowsPlan &p, size_t smem, bool many) {
    if (many) append_kernel<T, C, 4><<<grid, kRowsThreads, smem, st>>>(c, p);
    else append_kernel<T, C, 1><<<grid, kRowsThreads, smem, st>>>(c, p);
  });
}
template <typename C, typename T>
cudaError_t read_of(const KvRowsCall &c, cudaStream_t st) {
  return plan_rows(c, in_pieces(c.k_out, c.v_out, 0, 0, 0, 0, c.cache.dim, sizeof(T)), [&](unsigned grid, const RowsPlan &p, size_t smem, bool many) {
    if (many) read_kernel<C, T, 4><<<grid, kRowsThreads, smem, st>>>(c, p);
    else read_kernel<C, T, 1><<<grid, kRowsThreads, smem, st>>>(c, p);
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
