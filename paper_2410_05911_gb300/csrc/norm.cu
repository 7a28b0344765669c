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
// and dx = dres = dh.  Squares, products and sums are in 32 bits.
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>

#include "aecct_internal.h"
#include "rowtypes.cuh"

namespace aecct {

namespace {

constexpr float kAlphaMin = 0x1p-100f;  // 127 / alpha stays finite, and a row of zeros gets codes of zero
constexpr int kSmallThreads = 256;      // CTA of rows that fit a warp
constexpr int kPerThread = 16;          // elements of a row that a thread holds (kNormMaxWidth: twice that)
constexpr int kPerThreadWide = 32;
static_assert(kNormMaxWidth == 1024 * kPerThreadWide, "the widest row is a CTA of 1024 threads");

// The threads of a row: G consecutive lanes of a warp (d <= 32 E; BLOCK = 0), or a CTA of whole warps, at
// most BLOCK threads.  Thread t of
// the row holds elements (j G + t) V ... + V - 1 for j = 0 .. E / V - 1.
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

template <typename T, int V, int E, int BLOCK>
__global__ void __launch_bounds__(BLOCK ? BLOCK : kSmallThreads) rms_quant_grad_kernel(const __grid_constant__ GradArgs<T> a) {
  __shared__ float2 buf[2][32];
  __shared__ float red[BLOCK ? 1 : kSmallThreads * E];
  constexpr int C = E / V;
  const int d = a.s.d, G = a.s.G;
  const int t = BLOCK ? threadIdx.x : threadIdx.x & (G - 1);
  const int per = BLOCK ? 1 : kSmallThreads / G;
  float dg[E], g[E];
#pragma unroll
  for (int j = 0; j < C; ++j) {
    const int i = (j * G + t) * V;
#pragma unroll
    for (int e = 0; e < V; ++e) dg[j * V + e] = 0.0f, g[j * V + e] = i < d ? __ldg(a.gain + i + e) : 0.0f;
  }
  int parity = 0;
  for (int64_t first = static_cast<int64_t>(blockIdx.x) * per; first < a.s.rows; first += static_cast<int64_t>(gridDim.x) * per) {
    const int64_t row = first + (BLOCK ? 0 : threadIdx.x / G);
    const bool live = row < a.s.rows;
    float h[E], dy[E];
    float ss = 0.0f, th = 0.0f;
#pragma unroll
    for (int j = 0; j < C; ++j) {
      const int i = (j * G + t) * V;
      if (live && i < d) {
        load_v<T, V>(a.h + row * a.ldh + i, h + j * V);
        load_v<T, V>(a.dy + row * a.lddy + i, dy + j * V);
      } else {
#pragma unroll
        for (int e = 0; e < V; ++e) h[j * V + e] = 0.0f, dy[j * V + e] = 0.0f;
      }
    }
#pragma unroll
    for (int e = 0; e < E; ++e) ss = fmaf(h[e], h[e], ss), th = fmaf(dy[e] * g[e], h[e], th);
    // (both sums: the maximum's place is not used)
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
    const float c = r * r * r * __fdiv_rn(th, static_cast<float>(d));
    if (live) {
#pragma unroll
      for (int j = 0; j < C; ++j) {
        const int i = (j * G + t) * V;
        if (i < d) {
          float o[V];
          if (a.dsum) load_v<T, V>(a.dsum + row * a.ldd + i, o);
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const int k = j * V + e;
            const float v = fmaf(-h[k], c, r * (dy[k] * g[k]));
            o[e] = a.dsum ? v + o[e] : v;
            dg[k] = fmaf(dy[k], h[k] * r, dg[k]);
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

// dgain[i] = sum over the CTAs' partial sums, in a fixed order: 32 columns a CTA, 8 rows of them at a time
__global__ void __launch_bounds__(256) rms_quant_dgain_kernel(const float *partial, int parts, int d, float *dgain) {
  __shared__ float s[8][32];
  const int i = blockIdx.x * 32 + (threadIdx.x & 31), k0 = threadIdx.x >> 5;
  float v = 0.0f;
  if (i < d)
    for (int k = k0; k < parts; k += 8) v += partial[static_cast<int64_t>(k) * d + i];
  s[k0][threadIdx.x & 31] = v;
  __syncthreads();
  if (k0 == 0 && i < d) {
    for (int k = 1; k < 8; ++k) v += s[k][threadIdx.x];
    dgain[i] = v;
  }
}

bool on16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// threads of a row of d elements, E each: a power of two up to a warp, then whole warps
int row_threads(int d, int E) {
  int G = 1;
  while (G < 32 && G * E < d) G *= 2;
  return G * E >= d ? G : 32 * ((d + 32 * E - 1) / (32 * E));
}

template <typename T, int V, int E>
cudaError_t launch_quant(QuantArgs<T> a, cudaStream_t st) {
  a.s.G = row_threads(a.s.d, E);
  const bool block = a.s.G > 32;
  const int64_t per = block ? 1 : kSmallThreads / a.s.G;
  const int64_t grid = (a.s.rows + per - 1) / per;
  const unsigned blocks = static_cast<unsigned>(grid < (int64_t(1) << 30) ? grid : (int64_t(1) << 30));
  if constexpr (E == kPerThread) {
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
  if (c.d <= 1024 * kPerThread) return vec ? launch_quant<T, V, kPerThread>(a, st) : launch_quant<T, 1, kPerThread>(a, st);
  return vec ? launch_quant<T, V, kPerThreadWide>(a, st) : launch_quant<T, 1, kPerThreadWide>(a, st);
}

// CTAs of the backward kernel: what the GPU holds at once, no more than there are rows for
int grad_blocks(int64_t rows, int d, int E) {
  const int G = row_threads(d, E);
  const int threads = G > 32 ? G : kSmallThreads;
  const int64_t per = G > 32 ? 1 : kSmallThreads / G;
  const int64_t most = static_cast<int64_t>(sm_count()) * (threads > 512 ? 1 : 1024 / threads);
  const int64_t need = (rows + per - 1) / per;
  return static_cast<int>(need < most ? need : most);
}

template <typename T, int V, int E>
cudaError_t launch_grad(GradArgs<T> a, float *dgain, cudaStream_t st) {
  a.s.G = row_threads(a.s.d, E);
  const int blocks = grad_blocks(a.s.rows, a.s.d, E);
  if (blocks > 0) {
    if constexpr (E == kPerThread) {
      if (a.s.G <= 32) rms_quant_grad_kernel<T, V, E, 0><<<blocks, kSmallThreads, 0, st>>>(a);
      else if (a.s.G <= 512) rms_quant_grad_kernel<T, V, E, 512><<<blocks, a.s.G, 0, st>>>(a);
      else rms_quant_grad_kernel<T, V, E, 1024><<<blocks, a.s.G, 0, st>>>(a);
    } else {
      rms_quant_grad_kernel<T, V, E, 1024><<<blocks, a.s.G, 0, st>>>(a);
    }
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  rms_quant_dgain_kernel<<<(a.s.d + 31) / 32, 256, 0, st>>>(a.partial, blocks, a.s.d, dgain);
  return cudaGetLastError();
}

template <typename T>
cudaError_t grad_of(const RmsQuantGradCall &c, cudaStream_t st) {
  GradArgs<T> a = {{c.rows, c.d, 0}, static_cast<const T *>(c.dy), static_cast<const T *>(c.h), static_cast<const T *>(c.dsum),
                   c.lddy, c.ldh, c.ldd, c.gain, c.eps, static_cast<T *>(c.dx), c.partial};
  constexpr int V = kVec<T>;
  const bool vec = on16(c.dy) && on16(c.h) && on16(c.dsum) && on16(c.dx) && c.d % V == 0 && c.lddy % V == 0 && c.ldh % V == 0 &&
                   c.ldd % V == 0;
  if (c.d <= 1024 * kPerThread)
    return vec ? launch_grad<T, V, kPerThread>(a, c.dgain, st) : launch_grad<T, 1, kPerThread>(a, c.dgain, st);
  return vec ? launch_grad<T, V, kPerThreadWide>(a, c.dgain, st) : launch_grad<T, 1, kPerThreadWide>(a, c.dgain, st);
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

cudaError_t launch_rms_quant(const RmsQuantCall &c, cudaStream_t st) {
  return c.dtype == 0 ? quant_of<float>(c, st) : c.dtype == 1 ? quant_of<__half>(c, st) : quant_of<__nv_bfloat16>(c, st);
}

int64_t rms_quant_grad_partials(int64_t rows, int d) {
  return static_cast<int64_t>(grad_blocks(rows, d, d <= 1024 * kPerThread ? kPerThread : kPerThreadWide)) * d;
}

cudaError_t launch_rms_quant_grad(const RmsQuantGradCall &c, cudaStream_t st) {
  return c.dtype == 0 ? grad_of<float>(c, st) : c.dtype == 1 ? grad_of<__half>(c, st) : grad_of<__nv_bfloat16>(c, st);
}

}  // namespace aecct
