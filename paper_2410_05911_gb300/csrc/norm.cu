// norm.cu -- the residual's addition, root-mean-square norm and eq. Quant (Sec. 4.1) of a token's row in
// one pass, and its gradients.
//
//   h = x + res                              rounded to the stream's type, in which it is kept
//   r = 1 / sqrt(mean_i h_i^2 + eps)
//   z_i = h_i g_i                            (32 bits), y_i = z_i r the norm's output
//   alpha_z = max(max_i |z_i|, 2^-100)
//   q_i = rint(z_i (127 / alpha_z)),  scale = alpha_z r / 127,  q_i scale ~ y_i
// The absmax quantiser cancels r, so the codes come from z alone: they hang on no sum, and are the same
// bits whatever order the row is added up in.
//
// The gradients pass the rounding straight through (dy is that of q_i scale and of y_i):
//   t_i = dy_i g_i,  dh_i = r t_i - h_i r^3 mean_j(t_j h_j) + dsum_i,  dg_i = sum over rows of dy_i h_i r
// and dx = dres = dh.  Squares, products and sums are in 32 bits; the middle term is (h_i r) (mean_j(t_j h_j) r) r, whose
// factors stay in range wherever the sum of squares does.
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>

#include "aecct_internal.h"
#include "rowtypes.cuh"
#include "sm103_ptx.cuh"

namespace aecct {

namespace {

constexpr float kAlphaMin = 0x1p-100f;  // 127 / alpha stays finite, and a row of zeros gets codes of zero
constexpr int kSmallThreads = 256;      // CTA of rows that fit a warp
// Elements of a row that a thread holds: few, so that many threads' loads are in flight; as many as it takes for a
// CTA of 1024 threads to hold the row (kNormMaxWidth: 32).
constexpr int kFew = 8, kSome = 16, kMany = 32;
static_assert(kNormMaxWidth == 1024 * kMany, "the widest row is a CTA of 1024 threads");

// The threads of a row: G consecutive lanes of a warp (d <= 32 E; BLOCK = 0), or a CTA of whole warps, at
// most BLOCK threads.  Thread t of the row holds elements (j G + t) V ... + V - 1 for j = 0 .. E / V - 1.
struct RowShape {
  int64_t rows;
  int d, G;
};

// sum of `a` and maximum of `b` (b >= 0) over the threads of a row, in every one of them.  `buf` alternates
// between calls, so that one barrier a call is enough.
template <int BLOCK>
__device__ __forceinline__ void row_reduce(float &a, float &b, int G, float2 *buf) {
  for (int o = (BLOCK ? 32 : G) >> 1; o > 0; o >>= 1) {
    a += __shfl_xor_sync(0xffffffffu, a, o);
    b = fmaxf(b, __shfl_xor_sync(0xffffffffu, b, o));
  }
  if constexpr (BLOCK) {
    const int warps = blockDim.x >> 5;
    if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = make_float2(a, b);
    __syncthreads();
    float2 s = (threadIdx.x & 31) < warps ? buf[threadIdx.x & 31] : make_float2(0.0f, 0.0f);
    for (int o = 16; o > 0; o >>= 1) {
      s.x += __shfl_xor_sync(0xffffffffu, s.x, o);
      s.y = fmaxf(s.y, __shfl_xor_sync(0xffffffffu, s.y, o));
    }
    a = s.x, b = s.y;
  }
}

template <typename T>
struct QuantArgs {
  RowShape s;
  const T *x, *res;
  int64_t ldx, ldr;
  const float *gain;
  float eps;
  T *sum;
  int8_t *codes;
  float *scale;
  T *values;
};

// The forward pass of rows that start on 16 bytes (or have at most 256 elements).  A row is read once and stays in
// registers: the sum of squares and the largest |z| come from one reduction, since the codes take no part of r, and the
// codes, the scale and the values follow without a second look at memory.  Bound by memory, with 9 bytes an element for 16-bit
// rows and all outputs: 8,192 rows of 4,096 in bfloat16 54 us (5.6 TB/s), 65,536 rows of 128 in float32 26 us (5.4 TB/s);
// 2,048 rows of 16,384 in bfloat16, a CTA of 1,024 threads each, 74 us (4.1 TB/s).  One row: 3.3 us, the launch and two trips to
// memory.
template <typename T, int V, int E, int BLOCK>
__global__ void __launch_bounds__(BLOCK ? BLOCK : kSmallThreads) rms_quant_kernel(const __grid_constant__ QuantArgs<T> a) {
  __shared__ float2 buf[2][32];
  constexpr int C = E / V;
  const int d = a.s.d, G = a.s.G;
  const int t = BLOCK ? threadIdx.x : threadIdx.x & (G - 1);
  const int per = BLOCK ? 1 : kSmallThreads / G;  // rows of a CTA at a time
  int parity = 0;
  for (int64_t first = static_cast<int64_t>(blockIdx.x) * per; first < a.s.rows; first += static_cast<int64_t>(gridDim.x) * per) {
    const int64_t row = first + (BLOCK ? 0 : threadIdx.x / G);
    const bool live = row < a.s.rows;
    float h[E];
#pragma unroll
    for (int j = 0; j < C; ++j) {
      const int i = (j * G + t) * V;
      if (live && i < d) {
        load_v<T, V>(a.x + row * a.ldx + i, h + j * V);
      } else {
#pragma unroll
        for (int e = 0; e < V; ++e) h[j * V + e] = 0.0f;
      }
    }
    if (a.res) {
#pragma unroll
      for (int j = 0; j < C; ++j) {
        const int i = (j * G + t) * V;
        if (live && i < d) {
          float r[V];
          load_v<T, V>(a.res + row * a.ldr + i, r);
#pragma unroll
          for (int e = 0; e < V; ++e) h[j * V + e] = to_f32(from_f32<T>(h[j * V + e] + r[e]));
          store_v<T, V>(a.sum + row * d + i, h + j * V);
        }
      }
    }
    float ss = 0.0f, top = 0.0f;
#pragma unroll
    for (int j = 0; j < C; ++j) {
      const int i = (j * G + t) * V;
      if (i < d) {
        float g[V];
        load_v<float, V == 1 ? 1 : 4>(a.gain + i, g);
        if constexpr (V == 8) load_v<float, 4>(a.gain + i + 4, g + 4);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          ss = fmaf(h[j * V + e], h[j * V + e], ss);
          h[j * V + e] *= g[e];
          top = fmaxf(top, fabsf(h[j * V + e]));
        }
      }
    }
    row_reduce<BLOCK>(ss, top, G, buf[parity]);
    parity ^= 1;
    const float alpha = fmaxf(top, kAlphaMin), inv = __fdiv_rn(127.0f, alpha);
    const float r = __fdiv_rn(1.0f, __fsqrt_rn(__fdiv_rn(ss, static_cast<float>(d)) + a.eps));
    const float sc = __fdiv_rn(alpha * r, 127.0f);
    if (!live) continue;  // (!BLOCK: no barrier follows)
    if (t == 0) a.scale[row] = sc;
#pragma unroll
    for (int j = 0; j < C; ++j) {
      const int i = (j * G + t) * V;
      if (i < d) {
        float y[V];
        uint32_t w[(V + 3) / 4] = {};
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const int q = __float2int_rn(h[j * V + e] * inv);  // (a NaN gives 0)
          w[e / 4] |= (static_cast<uint32_t>(q) & 0xFFu) << (8 * (e & 3));
          y[e] = static_cast<float>(q) * sc;
        }
        int8_t *c = a.codes + row * d + i;
        if constexpr (V == 1) *c = static_cast<int8_t>(w[0]);
        else if constexpr (V == 4) *reinterpret_cast<uint32_t *>(c) = w[0];
        else *reinterpret_cast<uint2 *>(c) = make_uint2(w[0], w[1]);
        if (a.values) store_v<T, V>(a.values + row * d + i, y);
      }
    }
  }
}

// E elements of a row as they lie in memory: V at a time (16 bytes, or one)
template <typename T, int V, int E>
struct RawRow {
  uint4 w[V == 1 ? 1 : E / V];
  T e[V == 1 ? E : 1];
  // elements (j G + t) V ... of the row at p, of d; what lies past its end, or in no row, is not read
  __device__ __forceinline__ void load(const T *p, bool live, int t, int G, int d) {
#pragma unroll
    for (int j = 0; j < E / V; ++j) {
      const int i = (j * G + t) * V;
      if (live && i < d) {
        if constexpr (V == 1) e[j] = p[i];
        else w[j] = *reinterpret_cast<const uint4 *>(p + i);
      } else {
        if constexpr (V == 1) e[j] = from_f32<T>(0.0f);
        else w[j] = make_uint4(0, 0, 0, 0);
      }
    }
  }
  __device__ __forceinline__ void get(int j, float (&v)[V]) const {
    if constexpr (V == 1) v[0] = to_f32(e[j]);
    else if constexpr (sizeof(T) == 4)
      v[0] = __uint_as_float(w[j].x), v[1] = __uint_as_float(w[j].y), v[2] = __uint_as_float(w[j].z), v[3] = __uint_as_float(w[j].w);
    else
      unpack2<T>(w[j].x, v[0], v[1]), unpack2<T>(w[j].y, v[2], v[3]), unpack2<T>(w[j].z, v[4], v[5]), unpack2<T>(w[j].w, v[6], v[7]);
  }
};

template <typename T>
struct GradArgs {
  RowShape s;
  const T *dy, *h, *dsum;
  int64_t lddy, ldh, ldd;
  const float *gain;
  float eps;
  T *dx;
  float *partial;  // [CTAs][d]: each CTA's sum of dy h r over its rows
};

// A CTA takes every gridDim-th row (or group of rows) and holds the next one's elements, in flight, while it works
// on one: the sums over a row and their barrier would otherwise stand between its loads and the next row's.
// Rows of up to 256 elements, by groups of lanes (65,536 rows of 128 in float32: 26 us, 5.2 TB/s), and rows too wide for
// the ring (ring_grad_kernel, which takes the others): past 16,384 elements, or two of them past its shared memory.  Those
// are bound by registers: 32 elements a thread of a CTA of 1,024 spill 1.4 to 3.1 KB (2,048 rows of 32,768 in bfloat16: 605 us,
// 0.9 TB/s).
template <typename T, int V, int E, int BLOCK>
__global__ void __launch_bounds__(BLOCK ? BLOCK : kSmallThreads) rms_quant_grad_kernel(const __grid_constant__ GradArgs<T> a) {
  __shared__ float2 buf[2][32];
  __shared__ float red[BLOCK ? 1 : kSmallThreads * E];
  constexpr int C = E / V;
  const int d = a.s.d, G = a.s.G;
  const int t = BLOCK ? threadIdx.x : threadIdx.x & (G - 1);
  const int per = BLOCK ? 1 : kSmallThreads / G;
  const int64_t step = static_cast<int64_t>(gridDim.x) * per;
  grid_trigger();
  float dg[E], g[E];
#pragma unroll
  for (int j = 0; j < C; ++j) {
    const int i = (j * G + t) * V;
#pragma unroll
    for (int e = 0; e < V; ++e) dg[j * V + e] = 0.0f, g[j * V + e] = i < d ? __ldg(a.gain + i + e) : 0.0f;
  }
  const float by = __fdiv_rn(1.0f, static_cast<float>(d));
  int parity = 0;
  int64_t row = static_cast<int64_t>(blockIdx.x) * per + (BLOCK ? 0 : threadIdx.x / G);
  RawRow<T, V, E> h, dy, ds;
  const auto load = [&](int64_t r) {
    const bool live = r < a.s.rows;
    h.load(a.h + r * a.ldh, live, t, G, d);
    dy.load(a.dy + r * a.lddy, live, t, G, d);
    if (a.dsum) ds.load(a.dsum + r * a.ldd, live, t, G, d);
  };
  load(row);
  for (int64_t first = static_cast<int64_t>(blockIdx.x) * per; first < a.s.rows; first += step, row += step) {
    float hv[E], tv[E], ss = 0.0f, th = 0.0f;  // tv: dy gain
#pragma unroll
    for (int j = 0; j < C; ++j) {
      float x[V], y[V];
      h.get(j, x), dy.get(j, y);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const int k = j * V + e;
        hv[k] = x[e], tv[k] = y[e] * g[k];
        ss = fmaf(x[e], x[e], ss), th = fmaf(tv[k], x[e], th);
      }
    }
    const RawRow<T, V, E> own = dy, sum = ds;
    load(row + step);
    for (int o = (BLOCK ? 32 : G) >> 1; o > 0; o >>= 1) {
      ss += __shfl_xor_sync(0xffffffffu, ss, o);
      th += __shfl_xor_sync(0xffffffffu, th, o);
    }
    if constexpr (BLOCK) {
      float2 *b = buf[parity];
      if ((threadIdx.x & 31) == 0) b[threadIdx.x >> 5] = make_float2(ss, th);
      __syncthreads();
      float2 s = (threadIdx.x & 31) < (blockDim.x >> 5) ? b[threadIdx.x & 31] : make_float2(0.0f, 0.0f);
      for (int o = 16; o > 0; o >>= 1) {
        s.x += __shfl_xor_sync(0xffffffffu, s.x, o);
        s.y += __shfl_xor_sync(0xffffffffu, s.y, o);
      }
      ss = s.x, th = s.y;
      parity ^= 1;
    }
    const float r = __fdiv_rn(1.0f, __fsqrt_rn(__fdiv_rn(ss, static_cast<float>(d)) + a.eps));
    const float c = th * r * by * r;  // (r^3 alone would leave the range for rows past 1e12 or under 1e-12)
    if (row < a.s.rows) {
#pragma unroll
      for (int j = 0; j < C; ++j) {
        const int i = (j * G + t) * V;
        if (i < d) {
          float o[V], y[V];
          own.get(j, y);
          if (a.dsum) sum.get(j, o);
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const int k = j * V + e;
            const float u = hv[k] * r, v = fmaf(-u, c, r * tv[k]);
            o[e] = a.dsum ? v + o[e] : v;
            dg[k] = fmaf(y[e], u, dg[k]);
          }
          store_v<T, V>(a.dx + row * d + i, o);
        }
      }
    }
  }
  // the CTA's sum over its groups of lanes, in order
  if constexpr (!BLOCK) {
    const int w = G * E;  // columns of a group (>= d)
#pragma unroll
    for (int j = 0; j < C; ++j)
#pragma unroll
      for (int e = 0; e < V; ++e) red[(threadIdx.x / G) * w + (j * G + t) * V + e] = dg[j * V + e];
    __syncthreads();
    for (int i = threadIdx.x; i < d; i += kSmallThreads) {
      float s = 0.0f;
      for (int k = 0; k < per; ++k) s += red[k * w + i];
      a.partial[static_cast<int64_t>(blockIdx.x) * d + i] = s;
    }
  } else {
#pragma unroll
    for (int j = 0; j < C; ++j) {
      const int i = (j * G + t) * V;
      if (i < d)
#pragma unroll
        for (int e = 0; e < V; ++e) a.partial[static_cast<int64_t>(blockIdx.x) * d + i + e] = dg[j * V + e];
    }
  }
}

// ----------------------------------------------------------------------------- rows through shared memory
// Rows of more than a warp's lanes hold come to shared memory by bulk copies, kRing rows ahead of the one that is
// worked on: what is in flight then does not hang on registers or threads, and a row that does not start on 16
// bytes is copied from the 16 bytes that it starts in, to the same place of a 16-byte line.  Copies stay within the
// tensor: at its very first and last row, elements outside of whole 16-byte lines are copied by threads.
constexpr int kRing = 4;  // rows in flight, fewer (two at least) where that many do not fit
constexpr int kNormWaitTries = 1 << 24;  // a wait that has looked so often (seconds) has lost its copy

template <typename T>
struct RowSource {
  const T *p;  // NULL: none
  int64_t ld;
};

// the bytes of a row of d elements at p that a bulk copy takes: [first, last)
template <typename T>
__device__ __forceinline__ void copy_range(const T *p, int d, bool first_row, bool last_row, uintptr_t &first, uintptr_t &last) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = a + d * sizeof(T);
  first = first_row ? (a + 15) & ~uintptr_t(15) : a & ~uintptr_t(15);
  last = last_row ? b & ~uintptr_t(15) : (b + 15) & ~uintptr_t(15);
  if (last < first) last = first;
}
// bytes of shared memory of a row
template <typename T>
__host__ __device__ constexpr int row_bytes(int d) { return (d * static_cast<int>(sizeof(T)) + 31) / 16 * 16; }

// one thread: the copies of a row's N sources into `stage`.  ALIGNED: every row starts and ends on 16 bytes
template <typename T, int N, bool ALIGNED = false>
__device__ __forceinline__ void copy_rows(const RowSource<T> (&src)[N], int64_t row, int64_t rows, int d, uint32_t stage, uint32_t bar) {
  if constexpr (ALIGNED) {
    const uint32_t bytes = d * sizeof(T);
    mbar_arrive_expect_tx(bar, (src[N - 1].p ? N : N - 1) * bytes);
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (src[k].p) bulk_g2s(stage + k * row_bytes<T>(d), src[k].p + row * src[k].ld, bytes, bar);
    return;
  }
  uintptr_t first[N], last[N];
  uint32_t bytes = 0;
#pragma unroll
  for (int k = 0; k < N; ++k)
    if (src[k].p) {
      copy_range(src[k].p + row * src[k].ld, d, row == 0, row == rows - 1, first[k], last[k]);
      bytes += static_cast<uint32_t>(last[k] - first[k]);
    }
  mbar_arrive_expect_tx(bar, bytes);
#pragma unroll
  for (int k = 0; k < N; ++k)
    if (src[k].p && last[k] > first[k]) {
      const uintptr_t line = reinterpret_cast<uintptr_t>(src[k].p + row * src[k].ld) & ~uintptr_t(15);
      bulk_g2s(stage + k * row_bytes<T>(d) + static_cast<uint32_t>(first[k] - line), reinterpret_cast<const void *>(first[k]),
               static_cast<uint32_t>(last[k] - first[k]), bar);
    }
}
// where source k's row lies in its stage
template <typename T, bool ALIGNED = false>
__device__ __forceinline__ T *row_in(uint8_t *stage, const RowSource<T> &src, int k, int64_t row, int d) {
  if constexpr (ALIGNED) return reinterpret_cast<T *>(stage + k * row_bytes<T>(d));
  return reinterpret_cast<T *>(stage + k * row_bytes<T>(d) + (reinterpret_cast<uintptr_t>(src.p + row * src.ld) & 15));
}
// all threads: the elements of the first and last row that no copy takes.  The row's place is filled by a copy later: a fence
// between the proxies orders these stores before its writes.
template <typename T, int N>
__device__ __forceinline__ void patch_rows(const RowSource<T> (&src)[N], int64_t row, int64_t rows, int d, uint8_t *stage) {
  if (row != 0 && row != rows - 1) return;
#pragma unroll
  for (int k = 0; k < N; ++k)
    if (src[k].p) {
      const T *p = src[k].p + row * src[k].ld;
      T *s = row_in(stage, src[k], k, row, d);
      uintptr_t first, last;
      copy_range(p, d, row == 0, row == rows - 1, first, last);
      const int from = static_cast<int>((static_cast<intptr_t>(first) - reinterpret_cast<intptr_t>(p)) / static_cast<int>(sizeof(T)));
      const int to = static_cast<int>((static_cast<intptr_t>(last) - reinterpret_cast<intptr_t>(p)) / static_cast<int>(sizeof(T)));
      // (no copy at all where the row lies within a line: from >= to)
      for (int i = threadIdx.x; i < d; i += blockDim.x)
        if (i < from || i >= to) s[i] = p[i];
    }
  fence_proxy_async_smem();
  __syncthreads();
}
// a wait for a copy, with an end: its rows are then wrong, and err says so
__device__ __forceinline__ void wait_copy(uint32_t bar, uint32_t parity, int *err) {
  for (int tries = 0; !mbar_try_wait(bar, parity); ++tries)
    if (tries > kNormWaitTries) {
      *err = 1;
      return;
    }
}

template <typename T>
struct RingGradArgs {
  RowSource<T> src[3];  // h, dy, dsum
  int64_t rows;
  int d;
  int ring;  // rows of the ring
  const float *gain;
  float eps;
  T *dx;
  float *partial;
  int *err;  // set to 1 by a wait that gave up
};

// One row a CTA at a time, the next ones on their way into a ring in shared memory by bulk copies, so that the sums over
// a row and their barriers stand between no loads; thread t holds the sums of dgain of elements (j blockDim + t) V ...
// (V = 1 where a row or its outputs do not start on 16 bytes).  Bound by memory: 8,192 rows of 4,096 in bfloat16 with
// `dsum` (8 bytes an element) 44 us and 6 us for dgain's join, 5.4 TB/s in all.  A row is read from shared memory once,
// its products kept in pairs: with two passes over it in single operations (328 instructions of a thread for 8 elements
// of 4,096) the instructions were the bound, 56 us for the same rows.  Rows past 8,192 elements, 32 of them a thread, spill
// up to 0.5 KB: 2,048 of 16,384 in bfloat16 77 us, 3.5 TB/s.
template <typename T, int V, int E>
__global__ void __launch_bounds__(512, E == kFew ? 2 : 1) ring_grad_kernel(const __grid_constant__ RingGradArgs<T> a) {
  extern __shared__ __align__(16) uint8_t ring[];
  __shared__ uint64_t bars[kRing];
  __shared__ __align__(16) f32x2 buf[2][16];  // a warp's sums, zeros where there is no warp
  constexpr int C = E / V, H = E / 2;
  const int d = a.d, t = threadIdx.x, G = blockDim.x;
  const int stage_bytes = (a.src[2].p ? 3 : 2) * row_bytes<T>(d);
  const uint32_t bar = smem_u32(bars), base = smem_u32(ring);
  if (t == 0) {
    for (int s = 0; s < a.ring; ++s) mbar_init(bar + 8 * s, 1);
    fence_mbar_init_cluster();
    for (int s = 0; s < a.ring; ++s) {
      const int64_t row = blockIdx.x + static_cast<int64_t>(s) * gridDim.x;
      if (row < a.rows) copy_rows<T, 3, (V > 1)>(a.src, row, a.rows, d, base + s * stage_bytes, bar + 8 * s);
    }
  }
  grid_trigger();
  if (t < 32) buf[t >> 4][t & 15] = 0;
  f32x2 dg[H], g[H];
  const float by = __fdiv_rn(1.0f, static_cast<float>(d));
#pragma unroll
  for (int k = 0; k < H; ++k) {
    float v[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int j = (2 * k + e) / V, i = (j * G + t) * V + (2 * k + e) % V;
      v[e] = i < d ? __ldg(a.gain + i) : 0.0f;
    }
    dg[k] = 0, g[k] = pair(v[0], v[1]);
  }
  __syncthreads();
  int s = 0, parity = 0, n = 0;
  T *out = a.dx + static_cast<int64_t>(blockIdx.x) * d;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, n ^= 1, out += static_cast<int64_t>(gridDim.x) * d) {
    uint8_t *stage = ring + s * stage_bytes;
    wait_copy(bar + 8 * s, parity, a.err);
    if constexpr (V == 1) patch_rows(a.src, row, a.rows, d, stage);
    f32x2 h[H], t2[H], y2[H];  // h, dy gain, dy
    f32x2 ss = 0, th = 0;
    {
      const T *hs = row_in<T, (V > 1)>(stage, a.src[0], 0, row, d), *ys = row_in<T, (V > 1)>(stage, a.src[1], 1, row, d);
      float x[E], y[E];
#pragma unroll
      for (int j = 0; j < C; ++j) {
        const int i = (j * G + t) * V;
        if (i < d) {
          load_v<T, V>(hs + i, x + j * V), load_v<T, V>(ys + i, y + j * V);
        } else {
#pragma unroll
          for (int e = 0; e < V; ++e) x[j * V + e] = y[j * V + e] = 0.0f;
        }
      }
#pragma unroll
      for (int k = 0; k < H; ++k) {
        h[k] = pair(x[2 * k], x[2 * k + 1]), y2[k] = pair(y[2 * k], y[2 * k + 1]);
        t2[k] = mul2(y2[k], g[k]);
        ss = fma2(h[k], h[k], ss), th = fma2(t2[k], h[k], th);
      }
    }
    // both sums side by side in a pair
    float s0, s1, h0, h1;
    unpair(ss, s0, s1), unpair(th, h0, h1);
    f32x2 sum = add2(pair(s0, h0), pair(s1, h1));
    for (int o = 16; o > 0; o >>= 1) sum = add2(sum, __shfl_xor_sync(0xffffffffu, sum, o));
    f32x2 *b = buf[n];
    if ((t & 31) == 0) b[t >> 5] = sum;
    __syncthreads();
    sum = 0;
#pragma unroll
    for (int w = 0; w < 16; w += 2) {
      const ulonglong2 v = *reinterpret_cast<const ulonglong2 *>(b + w);
      sum = add2(add2(sum, v.x), v.y);
    }
    float sq, dot;
    unpair(sum, sq, dot);
    const float r = rsqrtf(fmaf(sq, by, a.eps)), c = -(dot * r * by * r);  // (r^3 alone would leave the range)
    const f32x2 r2 = pair(r, r), c2 = pair(c, c);
    const T *ds = a.src[2].p ? row_in<T, (V > 1)>(stage, a.src[2], 2, row, d) : nullptr;
#pragma unroll
    for (int k = 0; k < H; ++k) h[k] = mul2(h[k], r2), dg[k] = fma2(y2[k], h[k], dg[k]);  // (h r from here on)
#pragma unroll
    for (int j = 0; j < C; ++j) {
      const int i = (j * G + t) * V;
      if (i < d) {
        float o[V];
        if (ds) {
          load_v<T, V>(ds + i, o);
        } else {
#pragma unroll
          for (int e = 0; e < V; ++e) o[e] = 0.0f;
        }
        if constexpr (V == 1) {
          float hh[2], tt[2];
          unpair(h[j / 2], hh[0], hh[1]), unpair(t2[j / 2], tt[0], tt[1]);
          o[0] = fmaf(tt[j & 1], r, fmaf(hh[j & 1], c, o[0]));
        } else {
#pragma unroll
          for (int e = 0; e < V; e += 2) {
            const int k = (j * V + e) / 2;
            unpair(fma2(t2[k], r2, fma2(h[k], c2, pair(o[e], o[e + 1]))), o[e], o[e + 1]);
          }
        }
        store_v<T, V>(out + i, o);
      }
    }
    __syncthreads();
    // (every thread is done with the row: its place takes another)
    if (t == 0) {
      const int64_t next = row + static_cast<int64_t>(a.ring) * gridDim.x;
      if (next < a.rows) copy_rows<T, 3, (V > 1)>(a.src, next, a.rows, d, base + s * stage_bytes, bar + 8 * s);
    }
    if (++s == a.ring) s = 0, parity ^= 1;
  }
#pragma unroll
  for (int k = 0; k < H; ++k) {
    float v[2];
    unpair(dg[k], v[0], v[1]);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int j = (2 * k + e) / V, i = (j * G + t) * V + (2 * k + e) % V;
      if (i < d) a.partial[static_cast<int64_t>(blockIdx.x) * d + i] = v[e];
    }
  }
}

template <typename T>
struct RingQuantArgs {
  RowSource<T> src[2];  // x, residual
  int64_t rows;
  int d, ring;
  const float *gain;
  float eps;
  T *sum;
  int8_t *codes;
  float *scale;
  T *values;
  int *err;
};

// The forward pass of rows that do not start on 16 bytes, or that its outputs' do not: an element at a time from shared
// memory, where bulk copies have brought the row with the aligned bytes around it (rms_quant_kernel reads aligned rows in
// 16-byte pieces).  Bound by the instructions of single elements and of their stores: 4,099 rows of 1,155 in bfloat16 15 us
// (2.8 TB/s), 8,192 rows of 4,097 112 us (2.7 TB/s).
template <typename T, int E>
__global__ void __launch_bounds__(512) ring_quant_kernel(const __grid_constant__ RingQuantArgs<T> a) {
  extern __shared__ __align__(16) uint8_t ring[];
  __shared__ uint64_t bars[kRing];
  __shared__ __align__(16) float2 buf[2][16];  // a warp's sum and maximum, zeros where there is no warp
  const int d = a.d, t = threadIdx.x, G = blockDim.x;
  const int stage_bytes = (a.src[1].p ? 2 : 1) * row_bytes<T>(d);
  const uint32_t bar = smem_u32(bars), base = smem_u32(ring);
  if (t == 0) {
    for (int s = 0; s < a.ring; ++s) mbar_init(bar + 8 * s, 1);
    fence_mbar_init_cluster();
    for (int s = 0; s < a.ring; ++s) {
      const int64_t row = blockIdx.x + static_cast<int64_t>(s) * gridDim.x;
      if (row < a.rows) copy_rows(a.src, row, a.rows, d, base + s * stage_bytes, bar + 8 * s);
    }
  }
  if (t < 32) buf[t >> 4][t & 15] = make_float2(0.0f, 0.0f);
  float g[E];
#pragma unroll
  for (int j = 0; j < E; ++j) g[j] = j * G + t < d ? __ldg(a.gain + j * G + t) : 0.0f;
  __syncthreads();
  int s = 0, parity = 0;
  int64_t n = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, ++n) {
    uint8_t *stage = ring + s * stage_bytes;
    wait_copy(bar + 8 * s, parity, a.err);
    patch_rows(a.src, row, a.rows, d, stage);
    const T *x = row_in(stage, a.src[0], 0, row, d);
    const T *res = a.src[1].p ? row_in(stage, a.src[1], 1, row, d) : nullptr;
    float z[E], ss = 0.0f, top = 0.0f;
#pragma unroll
    for (int j = 0; j < E; ++j) {
      const int i = j * G + t;
      z[j] = 0.0f;
      if (i < d) {
        float h = to_f32(x[i]);
        if (res) {
          const T sum = from_f32<T>(h + to_f32(res[i]));
          a.sum[row * d + i] = sum;
          h = to_f32(sum);
        }
        ss = fmaf(h, h, ss);
        z[j] = h * g[j];
        top = fmaxf(top, fabsf(z[j]));
      }
    }
    for (int o = 16; o > 0; o >>= 1) {
      ss += __shfl_xor_sync(0xffffffffu, ss, o);
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    }
    float2 *b = buf[n & 1];
    if ((t & 31) == 0) b[t >> 5] = make_float2(ss, top);
    __syncthreads();
    if (t == 0) {  // (every thread has read the row: its place takes another)
      const int64_t next = row + static_cast<int64_t>(a.ring) * gridDim.x;
      if (next < a.rows) copy_rows(a.src, next, a.rows, d, base + s * stage_bytes, bar + 8 * s);
    }
    float2 v = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int w = 0; w < 16; w += 2) {
      const float4 u = *reinterpret_cast<const float4 *>(b + w);
      v.x += u.x + u.z, v.y = fmaxf(v.y, fmaxf(u.y, u.w));
    }
    const float alpha = fmaxf(v.y, kAlphaMin), inv = __fdiv_rn(127.0f, alpha);
    const float r = __fdiv_rn(1.0f, __fsqrt_rn(__fdiv_rn(v.x, static_cast<float>(d)) + a.eps));
    const float sc = __fdiv_rn(alpha * r, 127.0f);
    if (t == 0) a.scale[row] = sc;
#pragma unroll
    for (int j = 0; j < E; ++j) {
      const int i = j * G + t;
      if (i < d) {
        const int q = __float2int_rn(z[j] * inv);  // (a NaN gives 0)
        a.codes[row * d + i] = static_cast<int8_t>(q);
        if (a.values) a.values[row * d + i] = from_f32<T>(static_cast<float>(q) * sc);
      }
    }
    if (++s == a.ring) s = 0, parity ^= 1;
  }
}

// out[i] = sum over k < parts of partial[k][i], in a fixed order: COLS columns a CTA, 1024 / COLS rows of them at a time
template <int COLS>
__global__ void __launch_bounds__(1024) join_columns_kernel(const float *partial, int parts, int64_t n, float *out) {
  constexpr int kRows = 1024 / COLS;
  __shared__ float s[kRows][COLS + 1];
  const int c = threadIdx.x % COLS, k0 = threadIdx.x / COLS, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t first = static_cast<int64_t>(blockIdx.x) * COLS;
  float v = 0.0f;
  grid_trigger();
  grid_wait();
  if (first + c < n)
#pragma unroll 4
    for (int k = k0; k < parts; k += kRows) v += partial[k * n + first + c];
  s[k0][c] = v;
  __syncthreads();
  if (warp >= COLS) return;
  v = 0.0f;  // column `warp` of the CTA
#pragma unroll
  for (int k = 0; k < kRows; k += 32) v += s[k + lane][warp];
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if (lane == 0 && first + warp < n) out[first + warp] = v;
}

bool on16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// threads of a row of d elements, E each: a power of two up to a warp, then whole warps
int row_threads(int d, int E) {
  int G = 1;
  while (G < 32 && G * E < d) G *= 2;
  return G * E >= d ? G : 32 * ((d + 32 * E - 1) / (32 * E));
}

// How rows go through shared memory: threads of a CTA, elements that each holds, rows of the ring, CTAs.  ring = 0:
// not at all, as two rows do not fit.
struct RingPlan {
  int threads, E, ring, blocks, smem;
};
constexpr int kRingSmem = 200 * 1024;  // of an SM
RingPlan ring_plan(int64_t rows, int d, int element_bytes, int sources) {
  RingPlan p = {};
  p.threads = (d + kFew * 32 - 1) / (kFew * 32) * 32;
  p.threads = p.threads < 64 ? 64 : p.threads > 512 ? 512 : p.threads;
  for (p.E = kFew; p.E * p.threads < d; p.E *= 2) {}
  const int stage = sources * ((d * element_bytes + 31) / 16 * 16);
  int ctas = 1024 / p.threads;
  while (ctas > 1 && ctas * 2 * stage > kRingSmem) --ctas;
  p.ring = kRingSmem / ctas / stage;
  if (p.ring > kRing) p.ring = kRing;
  if (p.ring < 2 || p.E > kMany) p.ring = 0;
  p.smem = p.ring * stage;
  const int64_t most = static_cast<int64_t>(sm_count()) * ctas;
  p.blocks = static_cast<int>(rows < most ? rows : most);
  return p;
}

template <class K, class A>
cudaError_t launch_ring(K *kernel, const A &a, const RingPlan &p, cudaStream_t st) {
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRingSmem);
  if (e != cudaSuccess) return e;
  kernel<<<p.blocks, p.threads, p.smem, st>>>(a);
  return cudaGetLastError();
}

template <typename T, int V, int E>
cudaError_t launch_quant(QuantArgs<T> a, cudaStream_t st) {
  a.s.G = row_threads(a.s.d, E);
  const bool block = a.s.G > 32;
  const int64_t per = block ? 1 : kSmallThreads / a.s.G;
  const int64_t grid = (a.s.rows + per - 1) / per;
  const unsigned blocks = static_cast<unsigned>(grid < (int64_t(1) << 30) ? grid : (int64_t(1) << 30));
  if constexpr (E == kFew) {
    rms_quant_kernel<T, V, E, 0><<<blocks, kSmallThreads, 0, st>>>(a);
  } else if constexpr (E == kSome) {
    if (!block) rms_quant_kernel<T, V, E, 0><<<blocks, kSmallThreads, 0, st>>>(a);
    else if (a.s.G <= 512) rms_quant_kernel<T, V, E, 512><<<blocks, a.s.G, 0, st>>>(a);
    else rms_quant_kernel<T, V, E, 1024><<<blocks, a.s.G, 0, st>>>(a);
  } else {
    rms_quant_kernel<T, V, E, 1024><<<blocks, a.s.G, 0, st>>>(a);
  }
  return cudaGetLastError();
}

template <typename T>
cudaError_t quant_of(const RmsQuantCall &c, cudaStream_t st) {
  QuantArgs<T> a = {{c.rows, c.d, 0}, static_cast<const T *>(c.x), static_cast<const T *>(c.res), c.ldx, c.ldr, c.gain, c.eps,
                    static_cast<T *>(c.sum), c.codes, c.scale, static_cast<T *>(c.values)};
  constexpr int V = kVec<T>;
  const bool vec = on16(c.x) && on16(c.res) && on16(c.sum) && on16(c.codes) && on16(c.values) && on16(c.gain) && c.d % V == 0 &&
                   c.ldx % V == 0 && c.ldr % V == 0;
  if (vec) return c.d <= 1024 * kSome ? launch_quant<T, V, kSome>(a, st) : launch_quant<T, V, kMany>(a, st);
  if (c.d <= 32 * kFew) return launch_quant<T, 1, kFew>(a, st);
  const RingPlan p = ring_plan(c.rows, c.d, sizeof(T), c.res ? 2 : 1);
  if (!p.ring) return launch_quant<T, 1, kMany>(a, st);
  const RingQuantArgs<T> r = {{{a.x, a.ldx}, {a.res, a.ldr}}, c.rows, c.d, p.ring, c.gain, c.eps, a.sum, c.codes, c.scale, a.values,
                              wait_status()};
  return p.E == kFew    ? launch_ring(ring_quant_kernel<T, kFew>, r, p, st)
         : p.E == kSome ? launch_ring(ring_quant_kernel<T, kSome>, r, p, st)
                        : launch_ring(ring_quant_kernel<T, kMany>, r, p, st);
}

// CTAs of the backward kernel that holds rows in registers: 1,024 threads an SM, no more than there are rows for
int grad_blocks(int64_t rows, int d) {
  const int G = row_threads(d, d <= 32 * kFew ? kFew : kMany), threads = G > 32 ? G : kSmallThreads;
  const int64_t per = G > 32 ? 1 : kSmallThreads / G;
  const int64_t most = static_cast<int64_t>(sm_count()) * (threads > 512 ? 1 : 1024 / threads);
  const int64_t need = (rows + per - 1) / per;
  return static_cast<int>(need < most ? need : most);
}

template <typename T, int V>
cudaError_t launch_grad(const RmsQuantGradCall &c, cudaStream_t st) {
  const T *h = static_cast<const T *>(c.h), *dy = static_cast<const T *>(c.dy), *ds = static_cast<const T *>(c.dsum);
  T *dx = static_cast<T *>(c.dx);
  const RingPlan p = c.d <= 32 * kFew ? RingPlan{} : ring_plan(c.rows, c.d, sizeof(T), ds ? 3 : 2);
  int blocks = p.ring ? p.blocks : grad_blocks(c.rows, c.d);
  cudaError_t e = cudaSuccess;
  if (blocks > 0 && p.ring) {
    const RingGradArgs<T> r = {{{h, c.ldh}, {dy, c.lddy}, {ds, c.ldd}}, c.rows, c.d, p.ring, c.gain, c.eps, dx, c.partial,
                               wait_status()};
    e = p.E == kFew    ? launch_ring(ring_grad_kernel<T, V, kFew>, r, p, st)
        : p.E == kSome ? launch_ring(ring_grad_kernel<T, V, kSome>, r, p, st)
                       : launch_ring(ring_grad_kernel<T, V, kMany>, r, p, st);
  } else if (blocks > 0) {
    GradArgs<T> a = {{c.rows, c.d, row_threads(c.d, c.d <= 32 * kFew ? kFew : kMany)}, dy, h, ds, c.lddy, c.ldh, c.ldd, c.gain, c.eps, dx, c.partial};
    if (c.d <= 32 * kFew) rms_quant_grad_kernel<T, V, kFew, 0><<<blocks, kSmallThreads, 0, st>>>(a);
    else rms_quant_grad_kernel<T, V, kMany, 1024><<<blocks, a.s.G, 0, st>>>(a);
    e = cudaGetLastError();
  }
  if (e != cudaSuccess) return e;
  return launch_join_columns(c.partial, blocks, c.d, c.dgain, st);
}

template <typename T>
cudaError_t grad_of(const RmsQuantGradCall &c, cudaStream_t st) {
  constexpr int V = kVec<T>;
  const bool vec = on16(c.dy) && on16(c.h) && on16(c.dsum) && on16(c.dx) && c.d % V == 0 && c.lddy % V == 0 && c.ldh % V == 0 &&
                   c.ldd % V == 0;
  return vec ? launch_grad<T, V>(c, st) : launch_grad<T, 1>(c, st);
}

}  // namespace

int sm_count() {
  static std::atomic<int> known[64];  // by device
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 1;
  if ((n = known[dev].load(std::memory_order_relaxed)) > 0) return n;
  if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 1;
  known[dev].store(n, std::memory_order_relaxed);
  return n;
}

// A wide CTA's loads are whole lines, a narrow one's are sectors of eight columns, but more SMs take part and each thread
// has fewer loads in a row: the narrowest of which there are at most two to an SM.  (A call with 912 parts of 1,370 columns:
// 21.6 us with 32 of them a CTA, 20.5 us with 8; 1,024 parts of 128: 7.9 and 6.5 us.)
cudaError_t launch_join_columns(const float *partial, int parts, int64_t n, float *out, cudaStream_t st) {
  const auto launch = [&](auto *kernel, int columns) {
    return launch_dependent(kernel, dim3(static_cast<unsigned>((n + columns - 1) / columns)), 1024, 0, st, partial, parts, n, out);
  };
  const int64_t ctas = 2 * static_cast<int64_t>(sm_count());
  return n <= 8 * ctas    ? launch(join_columns_kernel<8>, 8)
         : n <= 16 * ctas ? launch(join_columns_kernel<16>, 16)
                          : launch(join_columns_kernel<32>, 32);
}

cudaError_t launch_rms_quant(const RmsQuantCall &c, cudaStream_t st) {
  return c.dtype == 0 ? quant_of<float>(c, st) : c.dtype == 1 ? quant_of<__half>(c, st) : quant_of<__nv_bfloat16>(c, st);
}

// (for any type, and with a dsum or without)
int64_t rms_quant_grad_partials(int64_t rows, int d) {
  int most = grad_blocks(rows, d);
  for (int bytes = 2; bytes <= 4; bytes += 2)
    for (int sources = 2; sources <= 3; ++sources) {
      const RingPlan p = ring_plan(rows, d, bytes, sources);
      if (p.ring && p.blocks > most) most = p.blocks;
    }
  return static_cast<int64_t>(most) * d;
}

cudaError_t launch_rms_quant_grad(const RmsQuantGradCall &c, cudaStream_t st) {
  return c.dtype == 0 ? grad_of<float>(c, st) : c.dtype == 1 ? grad_of<__half>(c, st) : grad_of<__nv_bfloat16>(c, st);
}

}  // namespace aecct
