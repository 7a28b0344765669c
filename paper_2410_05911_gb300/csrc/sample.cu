// sample.cu -- the next token of a row of logits: temperature, top-k, top-p, min-p, and a given random number.
//
//   w_i = exp((x_i - max x) / temperature), as a whole number of 2^-44: sums of up to 2^19 of them are exact in 64 bits, so that
//   a cut or a choice hangs on no order of additions
#include <cuda_runtime.h>

#include <cmath>
#include <cstdint>

#include "aecct_internal.h"
#include "rowtypes.cuh"

namespace aecct {

namespace {

constexpr int kSampleThreads = 1024;

// logits in an order that whole numbers have; NaN below everything
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x == 0.0f ? 0.0f : x);
  return x != x ? 0u : (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key); }
constexpr uint32_t kNone = 0x007fffffu;  // the key of minus infinity: what is not above it never stays

__device__ unsigned long long block_sum(unsigned long long v, unsigned long long *buf) {
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
  __syncthreads();
  unsigned long long s = 0;
  for (int i = 0; i < kSampleThreads / 32; ++i) s += buf[i];
  return s;
}

__device__ __forceinline__ unsigned long long weight(uint32_t key, uint32_t top, double by) {
  if (key == top) return 1ull << 44;
  return __double2ull_rn(exp((static_cast<double>(logit_of(key)) - static_cast<double>(logit_of(top))) * by) * 0x1p44);
}

// a CTA to a row
template <typename T>
__global__ void __launch_bounds__(kSampleThreads) sample_kernel(SampleCall c) {
  __shared__ unsigned long long buf[32];
  __shared__ unsigned long long cut_u64;
  const int row = blockIdx.x;
  const T *x = static_cast<const T *>(c.logits) + row * c.ld;
  const float t = c.temperature ? c.temperature[row] : c.temperature_all, p = c.top_p ? c.top_p[row] : c.top_p_all;
  const float mp = c.min_p ? c.min_p[row] : c.min_p_all;
  const int k = c.top_k ? c.top_k[row] : c.top_k_all;
  const int per = (c.vocab + kSampleThreads - 1) / kSampleThreads, lo = threadIdx.x * per, hi = min(c.vocab, lo + per);  // a thread's tokens
  uint32_t top = 0;
  for (int i = lo; i < hi; ++i) top = max(top, key_of(to_f32(x[i])));
  top = __reduce_max_sync(0xffffffffu, top);
  if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = top;
  __syncthreads();
  for (int i = 0; i < kSampleThreads / 32; ++i) top = max(top, static_cast<uint32_t>(buf[i]));
  if (top <= kNone) {
    if (threadIdx.x == 0) c.tokens[row] = -1;
    return;
  }
  const double by = 1.0 / static_cast<double>(t);
  // the sum of f over the row's tokens
  const auto total = [&](auto f) {
    unsigned long long s = 0;
    for (int i = lo; i < hi; ++i) s += f(key_of(to_f32(x[i])));
    return block_sum(s, buf);
  };
  // A beginning of the descending order is "keys above `cut`, and the first `ties` of those that are the same".
  uint32_t cut = t > 0.0f ? kNone : top;
  int64_t ties = t > 0.0f ? 0 : 1;
  // the shortest beginning with at least `want` of f, among the one at hand
  const auto shorten = [&](auto f, auto enough) {
    uint32_t a = cut, z = top;  // the largest key v with enough in keys >= v, or `cut` itself
    while (a < z) {
      const uint32_t mid = a + (z - a + 1) / 2;
      if (enough(total([&](uint32_t key) { return key >= mid ? f(key) : 0ull; }))) a = mid;
      else z = mid - 1;
    }
    if (a == cut && ties == 0) return;  // (all of them)
    const unsigned long long above = total([&](uint32_t key) { return key > a ? f(key) : 0ull; }), one = f(a);
    const int64_t have = a == cut ? ties : INT64_MAX;
    int64_t n = 0, most = static_cast<int64_t>(total([&](uint32_t key) { return key == a ? 1ull : 0ull; }));
    if (most > have) most = have;
    int64_t l = 0, r = most;  // the fewest of the equal ones that are enough
    while (l < r) {
      const int64_t mid = (l + r) / 2;
      if (enough(above + mid * one)) r = mid;
      else l = mid + 1;
    }
    n = l;
    cut = a, ties = n;
  };
  const auto mass = [&](uint32_t key) { return key > kNone ? weight(key, top, by) : 0ull; };
  if (t > 0.0f) {
    if (top == 0xff800000u) cut = top - 1;  // plus infinity: only those
    if (k > 0) shorten([&](uint32_t key) { return 1ull; }, [&](unsigned long long n) { return n >= static_cast<unsigned long long>(k); });
    if (p < 1.0f) {
      // (the tokens at the cut: the first `ties` of them)
      const unsigned long long above = total([&](uint32_t key) { return key > cut ? mass(key) : 0ull; });
      const unsigned long long all = above + ties * mass(cut);
      const double want = static_cast<double>(p) * static_cast<double>(all);
      if (ties > 0) {
        const uint32_t c0 = cut;
        const int64_t t0 = ties;
        if (static_cast<double>(above) >= want) {
          cut = c0, ties = 0;
          shorten(mass, [&](unsigned long long n) { return n > 0 && static_cast<double>(n) >= want; });
        } else {
          int64_t l = 0, r = t0;
          while (l < r) {
            const int64_t mid = (l + r) / 2;
            if (static_cast<double>(above + mid * mass(c0)) >= want) r = mid;
            else l = mid + 1;
          }
          ties = l;
        }
      } else {
        shorten(mass, [&](unsigned long long n) { return n > 0 && static_cast<double>(n) >= want; });
      }
    }
  }
  // rank among the equal ones at the cut
  const auto scan = [&](unsigned long long v) {  // exclusive, over the threads
    __shared__ unsigned long long part[kSampleThreads];
    __syncthreads();
    part[threadIdx.x] = v;
    __syncthreads();
    unsigned long long s = 0;
    for (int i = 0; i < static_cast<int>(threadIdx.x); ++i) s += part[i];
    return s;
  };
  unsigned long long mine = 0;
  for (int i = lo; i < hi; ++i) mine += key_of(to_f32(x[i])) == cut;
  const unsigned long long rank0 = scan(mine);
  const double least = mp > 0.0f ? log(static_cast<double>(mp)) * static_cast<double>(t) : -INFINITY;
  const auto stays = [&](uint32_t key, unsigned long long &rank) {
    if (key <= kNone || key < cut) return false;
    if (key == cut && rank++ >= static_cast<unsigned long long>(ties)) return false;
    return key == top || static_cast<double>(logit_of(key)) - static_cast<double>(logit_of(top)) >= least;
  };
  const auto weight_of = [&](uint32_t key) { return t > 0.0f ? weight(key, top, by) : 1ull; };
  unsigned long long sum = 0, rank = rank0;
  int first = INT32_MAX, last = -1;
  for (int i = lo; i < hi; ++i) {
    const uint32_t key = key_of(to_f32(x[i]));
    if (stays(key, rank)) sum += weight_of(key), first = min(first, i), last = i;
  }
  const unsigned long long all = block_sum(sum, buf), before = scan(sum);
  const float u = c.u[row];
  const unsigned long long target = u > 0.0f ? static_cast<unsigned long long>(static_cast<double>(u) * static_cast<double>(all)) : 0ull;
  if (threadIdx.x == 0) cut_u64 = ~0ull;
  __syncthreads();
  if (!(u > 0.0f)) {
    if (first < INT32_MAX) atomicMin(&cut_u64, static_cast<unsigned long long>(first));
  } else if (!(u < 1.0f)) {
    if (last >= 0) atomicMin(&cut_u64, ~1ull - static_cast<unsigned long long>(last));
  } else {
    unsigned long long s = before;
    rank = rank0;
    for (int i = lo; i < hi; ++i) {
      const uint32_t key = key_of(to_f32(x[i]));
      if (!stays(key, rank)) continue;
      const unsigned long long w = weight_of(key);
      if (s <= target && s + w > target) atomicMin(&cut_u64, static_cast<unsigned long long>(i));
      s += w;
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) c.tokens[row] = static_cast<int64_t>(!(u > 0.0f) || u < 1.0f ? cut_u64 : ~1ull - cut_u64);
}

}  // namespace

cudaError_t launch_sample(const SampleCall &c, cudaStream_t st) {
  if (c.dtype == 0) sample_kernel<float><<<c.rows, kSampleThreads, 0, st>>>(c);
  else if (c.dtype == 1) sample_kernel<__half><<<c.rows, kSampleThreads, 0, st>>>(c);
  else sample_kernel<__nv_bfloat16><<<c.rows, kSampleThreads, 0, st>>>(c);
  return cudaGetLastError();
}

}  // namespace aecct
