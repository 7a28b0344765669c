// sample.cu -- the next token of a row of logits: temperature, top-k, top-p, min-p, and a given random number.
//
//   w_i = exp((x_i - top) / temperature) = 2^-(c (top - x_i)),  c = log2 e / temperature,  as a whole number of 2^-44
//
// Sums of up to 2^19 weights are exact in 64 bits, so that a cut or a choice hangs on no order of additions.  What stays is
// always "every logit above `cut`, and the first `ties` of those equal to it": top-k, top-p and min-p each move the cut up.
//
// No sort.  A cut is found from histograms: first over equal steps of c (top - x) (2,048 of 2^-6 octaves, or 512 of 2^-4, so that logits spread over the
// bins), which bound the mass of a bin by its edges, to 1.1% or 4.4%, from its count alone; then over the keys (logits as ordered whole numbers) between the
// bounds, until a bin is one key, whose mass is its count times its weight.  Weights are summed one by one only above the
// bounds, and for the whole.  Each of these is a pass over the row, which L2 holds: the row is read from memory once.
//
// A cluster of 1 to 8 CTAs takes a row, each a part of it, and reads the others' histograms and sums through distributed
// shared memory.
//
// Bound by instructions where rows are many and flat (128 rows of 131,072 logits, top-p 0.9: 72 us, of them some 32 for the weights of all logits, 11
// for the histogram of steps, 5 for the trip to memory; 4 of the 32 for what rounding takes from the difference to the largest logit), by the phases'
// trips and barriers where they are few (one row of 50,021, every filter: 17 us).  An exact weight of every logit is this design's choice: the
// definition needs exact sums next to a border only.  The kernels for 16-bit logits spill 4 bytes of their 64 registers.
#include <cuda_runtime.h>

#include <atomic>
#include <cmath>
#include <cstdint>

#include "aecct_internal.h"
#include "rowtypes.cuh"
#include "sample_weight.cuh"
#include "sm103_ptx.cuh"

namespace aecct {

namespace {

using u64 = unsigned long long;
constexpr int kList = 256;   // candidates of top-k that one CTA takes
constexpr int kFew = 128;    // logits between the bounds of a cut that one CTA puts in order
constexpr int kOctaves = 32;  // of weights that bins of equal steps cover
constexpr float kTemperatureMin = 0x1p-100f, kTemperatureMax = 0x1p100f;

__device__ const PowerTable kPowers;

// Logits in an order that whole numbers have, and back; no NaN comes here, and both zeros are one number.  A key has the bits that type T
// has (a number between two of them gets the key of one of them).
template <typename T>
struct KeyOf {
  static constexpr int kDrop = sizeof(T) == 4 ? 0 : std::is_same_v<T, __half> ? 13 : 16;
  static __device__ __forceinline__ uint32_t key(float x) {
    const uint32_t b = __float_as_uint(x == 0.0f ? 0.0f : x);
    return ((b & 0x80000000u) ? ~b : b | 0x80000000u) >> kDrop;
  }
  static __device__ __forceinline__ float logit(uint32_t key) {
    const uint32_t k = key << kDrop;
    return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~(k | ((1u << kDrop) - 1)));
  }
};

__device__ __forceinline__ u64 ld_cluster_u64(uint32_t addr) {
  u64 v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ uint2 ld_cluster_u32x2(uint32_t addr) {
  uint2 v;
  asm volatile("ld.shared::cluster.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr) : "memory");
  return v;
}

__device__ __forceinline__ uint32_t atom_cluster_add(uint32_t addr, uint32_t v) {
  uint32_t old;
  asm volatile("atom.shared::cluster.add.u32 %0, [%1], %2;" : "=r"(old) : "r"(addr), "r"(v) : "memory");
  return old;
}
__device__ __forceinline__ void st_cluster_u32(uint32_t addr, uint32_t v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}

template <int NT>
struct SampleShared {
  static constexpr int kBins = 2 * NT, kWarps = NT / 32;
  static constexpr int kNotes = NT == 1024 ? 1024 : 512;  // logits between the bounds of a cut that a warp puts down
  uint32_t power[kSteps][32];  // a copy to each lane's bank (with one, random entries took 3 to 4 reads)
  uint32_t count[2][kBins];
  u64 warp[32][3];  // (all 32 are read)
  u64 part[2][3];                // this CTA's sums, for the cluster
  u64 segment[2][32];  // a number of each warp's part of the row
  struct Hand {
    u64 passed, rank;
    int block, blocks;
  } hand;  // the part of the row that holds the token
  float notes[kWarps][kNotes];
  float list_logit[kList];
  uint32_t list_index[kList], listed;
  u64 list_weight[kList];
  uint32_t found[2];
  float settled;
  u64 found_sum[2];
  double least;          // temperature ln min_p
  float c, c_low, floor;  // log2 e / temperature, and the lowest logit that min_p leaves
};

// floor(f n) and whether something was cut off, for 0 < f < 1
__device__ __forceinline__ u64 times(float f, u64 n, bool &more) {
  const uint32_t b = __float_as_uint(f), e = b >> 23, m = e ? (b & 0x7fffffu) | 0x800000u : b & 0x7fffffu;
  const int shift = 150 - static_cast<int>(e ? e : 1);  // f = m 2^-shift, 24 <= shift <= 149
  const u64 low = m * n, high = __umul64hi(m, n);
  if (shift >= 64) {
    const int s = shift - 64;
    more = low != 0 || (s < 64 ? (high & ((1ull << s) - 1)) : high) != 0;
    return s < 64 ? high >> s : 0;
  }
  more = (low & ((1ull << shift) - 1)) != 0;
  return (low >> shift) | (high << (64 - shift));
}

template <typename T, int NT>
struct SampleRow {
  using Shared = SampleShared<NT>;
  static constexpr int kBins = Shared::kBins, kWarps = Shared::kWarps, kNotes = Shared::kNotes, kBinsPerOctave = kBins / kOctaves;
  static constexpr int V = 16 / sizeof(T);
  const T *x;
  int vocab, shift;         // shift: elements from the 16-byte border before x to x
  int block, blocks;        // this warp's blocks of V elements: block, ..., block + blocks - 1
  Shared &sh;
  const int lane, warp;
  const uint32_t rank, ctas;
  int noted = 0;           // logits put down by this warp
  int flip = 0, hist = 0;  // which of two places the next sum and the next histogram take

  float top, c, c_low, bin_by;  // log2 e / temperature in two floats; bins per logit
  float lowest;                 // logits below it never stay
  float most_off, bins_off;     // logits under the largest where weights end, and where bins end

  __device__ SampleRow(Shared &s, uint32_t r, uint32_t n) : sh(s), lane(threadIdx.x & 31), warp(threadIdx.x >> 5), rank(r), ctas(n) {}

  __device__ void sync() const {
    if (ctas > 1) cluster_sync_all();
    else __syncthreads();
  }

  // a block of V elements, NaN where the row has none
  __device__ __forceinline__ uint4 block_of(int q) const {
    const int64_t i = static_cast<int64_t>(q) * V - shift;
    if (i >= 0 && i + V <= vocab) return *reinterpret_cast<const uint4 *>(x + i);
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      w[k] = 0;
#pragma unroll
      for (int h = 0; h < V / 4; ++h) {
        const int64_t at = i + k * (V / 4) + h;
        uint32_t bits = sizeof(T) == 4 ? 0x7fffffffu : 0x7fffu;
        if (at >= 0 && at < vocab) {
          if constexpr (sizeof(T) == 4) bits = reinterpret_cast<const uint32_t *>(x)[at];
          else bits = reinterpret_cast<const uint16_t *>(x)[at];
        }
        w[k] |= bits << (h * 16);
      }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  static __device__ __forceinline__ void numbers(const uint4 &w, float (&v)[V]) {
    if constexpr (sizeof(T) == 4) {
      v[0] = __uint_as_float(w.x), v[1] = __uint_as_float(w.y), v[2] = __uint_as_float(w.z), v[3] = __uint_as_float(w.w);
    } else {
      unpack2<T>(w.x, v[0], v[1]), unpack2<T>(w.y, v[2], v[3]), unpack2<T>(w.z, v[4], v[5]), unpack2<T>(w.w, v[6], v[7]);
    }
  }
  // f(v, block) for blocks from, ..., from + n - 1 of V logits, 32 lanes' at once and in ascending order; blocks past the end hold NaN
  template <class F>
  __device__ __forceinline__ void blocks_of(int from, int n, F &&f) const {
    constexpr int kAhead = 2;
    for (int b = 0; b < n; b += 32 * kAhead) {
      uint4 w[kAhead];
#pragma unroll
      for (int a = 0; a < kAhead; ++a) w[a] = b + a * 32 + lane < n ? block_of(from + b + a * 32 + lane) : make_uint4(~0u, ~0u, ~0u, ~0u);
#pragma unroll
      for (int a = 0; a < kAhead; ++a) {
        if (b + a * 32 >= n) break;
        float v[V];
        numbers(w[a], v);
        f(v, from + b + a * 32 + lane);
      }
    }
  }
  // f(logit) for this warp's logits, those at or above `from` among them: blocks of the warp with none of these are left out
  template <class F>
  __device__ __forceinline__ void each(float from, F &&f) const {
    blocks_of(block, blocks, [&](const float (&v)[V], int) {
      float most = v[0];
#pragma unroll
      for (int e = 1; e < V; ++e) most = fmaxf(most, v[e]);
      if (!__any_sync(0xffffffffu, most >= from)) return;
#pragma unroll
      for (int e = 0; e < V; ++e) f(v[e]);
    });
  }
  // f(logit, index) for those from `from` to `upto`, which are few: 32 lanes with none of them are left out
  template <class F>
  __device__ __forceinline__ void between(float from, float upto, F &&f) const {
    blocks_of(block, blocks, [&](const float (&v)[V], int b) {
      float most = v[0];
#pragma unroll
      for (int e = 1; e < V; ++e) most = fmaxf(most, v[e]);
      if (!__any_sync(0xffffffffu, most >= from)) return;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const bool in = v[e] >= from && v[e] <= upto;
        if (__any_sync(0xffffffffu, in))
          if (in) f(v[e], b * V - shift + e);
      }
    });
  }

  __device__ __forceinline__ u64 weight(float v) const {
    return weight_of(v, top, c, c_low, most_off, [&](uint32_t j) { return sh.power[j][lane]; });
  }

  // puts down a logit between the bounds of a cut for the passes that follow: each warp its own
  __device__ __forceinline__ void note(bool in, float v) {
    const uint32_t who = __ballot_sync(0xffffffffu, in);
    if (who == 0) return;
    const int at = noted + __popc(who & ((1u << lane) - 1));
    if (in && at < kNotes) sh.notes[warp][at] = v;
    noted += __popc(who);
  }
  // f(logit) for the warp's logits from `from` to `upto`, all of which note() has seen
  template <class F>
  __device__ __forceinline__ void noted_between(float from, float upto, F &&f) const {
    if (noted > kNotes) {  // (too many to put down)
      between(from, upto, [&](float v, int) { f(v); });
      return;
    }
    __syncwarp();
    for (int i = lane; i < noted; i += 32) {
      const float v = sh.notes[warp][i];
      if (v >= from && v <= upto) f(v);
    }
  }

  // bounds of what weight() says of logits up to (from) one of which it says w: each is off by less than 2^-28 of itself and a unit
  static __device__ u64 above(u64 w) { return w + (w >> 27) + 2; }
  static __device__ u64 below(u64 w) { return w < 4 ? 0 : w - (w >> 27) - 2; }

  // sums over the row of three numbers
  __device__ void sums(u64 &a, u64 &b, u64 &c3) {
    for (int o = 16; o > 0; o >>= 1)
      a += __shfl_xor_sync(0xffffffffu, a, o), b += __shfl_xor_sync(0xffffffffu, b, o), c3 += __shfl_xor_sync(0xffffffffu, c3, o);
    if (lane == 0) sh.warp[warp][0] = a, sh.warp[warp][1] = b, sh.warp[warp][2] = c3;
    __syncthreads();
    if (warp == 0) {
      const bool in = lane < kWarps;
      a = in ? sh.warp[lane][0] : 0, b = in ? sh.warp[lane][1] : 0, c3 = in ? sh.warp[lane][2] : 0;
      for (int o = 16; o > 0; o >>= 1)
        a += __shfl_xor_sync(0xffffffffu, a, o), b += __shfl_xor_sync(0xffffffffu, b, o), c3 += __shfl_xor_sync(0xffffffffu, c3, o);
      if (lane == 0) sh.part[flip][0] = a, sh.part[flip][1] = b, sh.part[flip][2] = c3;
    }
    sync();
    a = b = c3 = 0;
    const uint32_t at = smem_u32(sh.part[flip]);
    for (uint32_t r = 0; r < ctas; ++r)
      a += ld_cluster_u64(mapa_cluster(at, r)), b += ld_cluster_u64(mapa_cluster(at + 8, r)), c3 += ld_cluster_u64(mapa_cluster(at + 16, r));
    flip ^= 1;
  }
  __device__ void sums(u64 &a, u64 &b) {
    u64 none = 0;
    sums(a, b, none);
  }
  __device__ float maximum(float v) {
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    if (lane == 0) sh.warp[warp][0] = __float_as_uint(v);
    __syncthreads();
    v = __uint_as_float(static_cast<uint32_t>(sh.warp[lane % kWarps][0]));
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    if (threadIdx.x == 0) sh.part[flip][0] = __float_as_uint(v);
    sync();
    for (uint32_t r = 0; r < ctas; ++r)
      v = fmaxf(v, __uint_as_float(static_cast<uint32_t>(ld_cluster_u64(mapa_cluster(smem_u32(sh.part[flip]), r)))));
    flip ^= 1;
    return v;
  }
  __device__ u64 lanes_before(u64 v) const {
    u64 s = v;
    for (int d = 1; d < 32; d <<= 1) {
      const u64 w = __shfl_up_sync(0xffffffffu, s, d);
      if (lane >= d) s += w;
    }
    return s - v;
  }
  // sum over the threads before this one, in its CTA, and over all (the row's bins lie in thread order in every CTA)
  __device__ u64 before(u64 v, u64 &all) {
    const u64 s = lanes_before(v) + v;
    __syncthreads();
    if (lane == 31) sh.warp[warp][0] = s;
    __syncthreads();
    const u64 w = lane < kWarps ? sh.warp[lane][0] : 0, e = lanes_before(w);
    all = __shfl_sync(0xffffffffu, e + w, 31);
    return __shfl_sync(0xffffffffu, e, warp) + s - v;
  }

  // counts of the row's logits by bin, which count_all(counts) adds for this warp's part; this thread's are bins 2 i and 2 i + 1
  template <class F>
  __device__ uint2 histogram(F &&count_all) {
    uint32_t *count = sh.count[hist];
    for (int i = threadIdx.x; i < kBins; i += NT) count[i] = 0;
    __syncthreads();
    count_all(count);
    sync();
    uint2 n = {0, 0};
    const uint32_t at = smem_u32(count + 2 * threadIdx.x);
    for (uint32_t r = 0; r < ctas; ++r) {
      const uint2 m = ld_cluster_u32x2(mapa_cluster(at, r));
      n.x += m.x, n.y += m.y;
    }
    hist ^= 1;
    return n;
  }
  // The bin of equal steps of a logit that is not below `lowest`: the nearest whole number of steps, off by less than 2^-11 of one (three
  // roundings of a number below 2^11).
  __device__ __forceinline__ int step_bin(float v) const {
    return static_cast<int>(__float_as_uint(fmaf(fminf(fmaxf(top - v, 0.0f), bins_off), bin_by, 12582912.0f)) - 0x4b400000u);
  }
  // a logit that no logit of a bin >= b is above, and one that none of a bin <= b is below
  __device__ float bin_high(int b) const { return b <= 1 ? top : fminf(top, __fsub_ru(top, __fmul_rd(static_cast<float>(b - 1), __frcp_rd(bin_by)))); }
  __device__ float bin_low(int b) const {
    return b >= kBins - 2 ? lowest : fmaxf(lowest, __fsub_rd(top, __fmul_ru(static_cast<float>(b + 2), __frcp_ru(bin_by))));
  }
  // the weight of its upper edge
  __device__ u64 bin_power(int b) const {
    const int j = b == 0 ? 0 : (2 * b - 1) * (kSteps / kBinsPerOctave) / 2;
    static_assert(kSteps / kBinsPerOctave % 2 == 0, "half a bin is a step of the table");
    return (static_cast<u64>(sh.power[j % kSteps][lane]) << 14) >> (j / kSteps);
  }

  // The whole choice among the listed candidates, which hold the first k: a thread to each, in the descending order that counting gives.
  __device__ void choose(int k, float p, float min_p, float u, int64_t *token) {
    const int n = static_cast<int>(sh.listed), i = threadIdx.x;
    int rank_here = 0;
    const float v0 = i < n ? sh.list_logit[i] : 0.0f;
    const uint32_t i0 = i < n ? sh.list_index[i] : 0;
    if ((i & ~31) < n)
      for (int j = 0; j < n; ++j) {
        const float v = sh.list_logit[j];
        rank_here += v > v0 || (v == v0 && sh.list_index[j] < i0);
      }
    __syncthreads();
    if (i < n) sh.list_logit[rank_here] = v0, sh.list_index[rank_here] = i0;
    __syncthreads();
    const int most = min(n, k);
    const float v = i < most ? sh.list_logit[i] : -INFINITY;
    u64 w = i < most ? weight(v) : 0, all, want = ~0ull;
    const u64 passed = before(w, all);
    if (p < 1.0f) {
      want = 1;
      if (p > 0.0f) {
        bool cut_off;
        want = times(p, all, cut_off);
        want += cut_off;
      }
    }
    const bool stays = i < most && (i == 0 || passed < want) && !(min_p > 0.0f && v < sh.floor);
    const bool ends = !(u > 0.0f) || !(u < 1.0f);
    w = !stays ? 0 : ends ? 1 : w;
    before(w, all);
    u64 target = 0;
    if (!(u < 1.0f) && u > 0.0f) {
      target = all - 1;
    } else if (!ends) {
      bool cut_off;
      target = times(u, all, cut_off);
    }
    // the same in the order of the row
    if (i < most) sh.list_weight[i] = w;
    __syncthreads();
    if ((i & ~31) < most) {
      const uint32_t index = i < most ? sh.list_index[i] : 0;
      u64 at = 0;
      for (int j = 0; j < most; ++j) at += sh.list_index[j] < index ? sh.list_weight[j] : 0;
      if (stays && at <= target && target < at + w) *token = index;
    }
  }
  // The cut of the mass among the listed logits, one of which it is, `passed` being that of the logits above them: to every CTA of the row.
  __device__ void settle(u64 passed, u64 want) {
    const int n = static_cast<int>(sh.listed), i = threadIdx.x;
    const float v0 = i < n ? sh.list_logit[i] : 0.0f;
    int rank_here = 0;
    if ((i & ~31) < n)
      for (int j = 0; j < n; ++j) {
        const float v = sh.list_logit[j];
        rank_here += v > v0 || (v == v0 && j < i);
      }
    __syncthreads();
    if (i < n) sh.list_logit[rank_here] = v0;
    __syncthreads();
    const float v = i < n ? sh.list_logit[i] : 0.0f;
    const u64 w = i < n ? weight(v) : 0;
    u64 all;
    const u64 at = passed + before(w, all);
    if (i < n && (i == 0 || at < want) && (at + w >= want || i == n - 1)) {  // (one of them)
      uint32_t ties = 1;
      while (ties <= static_cast<uint32_t>(i) && sh.list_logit[i - ties] == v) ++ties;
      for (uint32_t r = 0; r < ctas; ++r) {
        st_cluster_f32(mapa_cluster(smem_u32(&sh.settled), r), v);
        st_cluster_u32(mapa_cluster(smem_u32(sh.found), r), ties);
      }
    }
  }
  // the bin that one thread has found, and the sum before it
  __device__ void publish(uint32_t bin, u64 sum) { sh.found[0] = bin, sh.found_sum[0] = sum; }
};

template <typename T, int NT>
__global__ void __launch_bounds__(NT, NT == 1024 ? 1 : 4) sample_kernel(SampleCall call) {
  using Shared = SampleShared<NT>;
  constexpr int kBins = Shared::kBins, kWarps = Shared::kWarps;
  extern __shared__ __align__(16) unsigned char smem[];
  Shared &sh = *reinterpret_cast<Shared *>(smem);
  const uint32_t ctas = call.ctas, rank = ctas > 1 ? cluster_ctarank() : 0;
  const int row = blockIdx.x / ctas, tid = threadIdx.x;
  SampleRow<T, NT> r(sh, rank, ctas);
  constexpr int V = SampleRow<T, NT>::V;
  using K = KeyOf<T>;
  r.x = static_cast<const T *>(call.logits) + row * call.ld, r.vocab = call.vocab;
  r.shift = static_cast<int>((reinterpret_cast<uintptr_t>(r.x) & 15u) / sizeof(T));
  {
    const int blocks = (call.vocab + r.shift + V - 1) / V, per = (blocks + ctas * kWarps - 1) / (ctas * kWarps);
    r.block = static_cast<int>(rank * kWarps + r.warp) * per;
    r.blocks = max(0, min(per, blocks - r.block));
  }
  for (int i = r.warp; i < kSteps; i += kWarps) sh.power[i][r.lane] = kPowers.e[i];
  const float t = call.temperature ? call.temperature[row] : call.temperature_all;
  const float p = call.top_p ? call.top_p[row] : call.top_p_all, min_p = call.min_p ? call.min_p[row] : call.min_p_all, u = call.u[row];
  const int k = call.top_k ? call.top_k[row] : call.top_k_all;

  const bool greedy = !(t > 0.0f);
  if (tid == 0) sh.hand.blocks = 0, sh.listed = 0;
  if (tid == 0) {  // (a double operation of all the threads takes as long as 300 others)
    const float kept = fminf(fmaxf(t, kTemperatureMin), kTemperatureMax);
    const double c = 1.4426950408889634074 / static_cast<double>(kept);
    sh.c = static_cast<float>(c), sh.c_low = static_cast<float>(c - static_cast<double>(sh.c));
    sh.least = min_p > 0.0f ? log(static_cast<double>(min_p)) * static_cast<double>(kept) : 0.0;
  }
  float most = -INFINITY;
  r.blocks_of(r.block, r.blocks, [&](const float (&v)[V], int) {
#pragma unroll
    for (int e = 0; e < V; ++e) most = fmaxf(most, v[e]);
  });
  r.top = most = r.maximum(most);
  if (most == -INFINITY) {  // (the same in every CTA of the row)
    if (rank == 0 && tid == 0) call.tokens[row] = -1;
    if (ctas > 1) cluster_sync_all();
    return;
  }
  if (tid == 0) {  // logits under top + temperature ln min_p go; the largest stays
    const float v = __double2float_ru(static_cast<double>(most) + sh.least);
    sh.floor = v < most ? v : most;
  }
  __syncthreads();
  r.c = sh.c, r.c_low = sh.c_low;
  r.most_off = __fdiv_rd(45.0f, r.c);
  r.bin_by = r.c * SampleRow<T, NT>::kBinsPerOctave;
  r.bins_off = __fdiv_rd(kBins - 0.75f, r.bin_by);
  r.lowest = most == INFINITY ? INFINITY : -3.402823466e38f;

  float cut = r.lowest;       // what stays: logits above it,
  u64 ties = ~0ull;           // and the first of those equal to it
  if (greedy) cut = most, ties = 1;
  // this lane's mass of the logits above `known`, where a pass has summed it
  u64 above = 0;
  float known = INFINITY;
  const bool by_count = !greedy && k > 0 && k < call.vocab, by_mass = !greedy && p < 1.0f;
  if (by_count || by_mass) {
    const uint2 n = r.histogram([&](uint32_t *count) {
      r.each(r.lowest, [&](float v) {
        if (v >= r.lowest) atomicAdd(count + r.step_bin(v), 1u);
      });
    });
    const u64 m0 = n.x * r.bin_power(2 * tid), m1 = n.y * r.bin_power(2 * tid + 1);
    u64 counts = 0, masses = 0;
    const u64 n0 = r.before(static_cast<u64>(n.x) + n.y, counts);  // logits before this thread's bins
    int last = kBins - 1;                                          // the bin of the k-th
    if (by_count && counts > static_cast<u64>(k)) {
      const u64 want = static_cast<u64>(k);
      if (n0 < want && n0 + n.x + n.y >= want) r.publish(2 * tid + (n0 + n.x < want), 0);
      __syncthreads();
      last = static_cast<int>(sh.found[0]);
      // few candidates (the logits up to that bin): to one CTA, and through
      if (2 * tid == (last & ~1)) sh.found_sum[1] = n0 + n.x + (last & 1 ? n.y : 0);
      __syncthreads();
      if (sh.found_sum[1] <= kList) {
        r.between(r.bin_low(last), INFINITY, [&](float v, int i) {
          if (r.step_bin(v) > last) return;
          const uint32_t at = atom_cluster_add(mapa_cluster(smem_u32(&sh.listed), 0), 1u);
          st_cluster_f32(mapa_cluster(smem_u32(sh.list_logit + at), 0), v);
          st_cluster_u32(mapa_cluster(smem_u32(sh.list_index + at), 0), static_cast<uint32_t>(i));
        });
        r.sync();
        if (rank == 0) r.choose(k, p, min_p, u, call.tokens + row);
        return;
      }
      // down to one key
      uint32_t high = K::key(r.bin_high(last)), low = K::key(r.bin_low(last));
      bool first = true;
      u64 passed = 0;
      for (int step = 0; step < 4; ++step) {  // (each leaves a 512th of the keys at most)
        int shift = 0;
        while ((high - low) >> shift >= kBins) ++shift;
        u64 over = 0, none = 0;
        const float upto = K::logit(high), from = fmaxf(r.lowest, K::logit(low));
        const uint2 m = r.histogram([&](uint32_t *count) {
          r.between(from, first ? INFINITY : upto, [&](float v, int) {
            if (v > upto) ++over;
            else atomicAdd(count + ((high - K::key(v)) >> shift), 1u);
          });
        });
        if (first) r.sums(over, none), passed = over;
        first = false;
        u64 all;
        const u64 at = passed + r.before(static_cast<u64>(m.x) + m.y, all);
        if (at < want && at + m.x + m.y >= want) r.publish(2 * tid + (at + m.x < want), at + m.x < want ? at + m.x : at);
        __syncthreads();
        const uint32_t b = sh.found[0];
        passed = sh.found_sum[0];
        __syncthreads();
        if (shift == 0) {
          cut = K::logit(high - b), ties = want - passed;
          break;
        }
        high -= b << shift;
        low = max(low, high - ((1u << shift) - 1));
      }
    }
    if (by_mass) {
      // Upper bounds up to a bin: the cut is not before the first that reaches p of the least that the whole may be.  Lower ones: it is not after
      // the first that reaches p of the most.  And the same from the other end, which says more where p is near 1: what lies behind the cut is at
      // most 1 - p of the whole, and with the cut's own bin more than that.
      constexpr float kOver = 1.0f + 0x1p-14f;  // for the bins' own errors, and these roundings
      const float ratio = exp2f(-1.0f / SampleRow<T, NT>::kBinsPerOctave);  // of a bin's lower bound to its upper one
      const bool x0 = 2 * tid <= last, x1 = 2 * tid + 1 <= last;
      const u64 before = r.before((x0 ? m0 : 0) + (x1 ? m1 : 0), masses);
      // (what the last bin holds may be anything from nothing to its bound)
      if (2 * tid == (last & ~1)) sh.found_sum[1] = last & 1 ? before + m0 : before;
      if (tid == 0) sh.found[0] = 0, sh.found[1] = static_cast<uint32_t>(last);
      __syncthreads();
      const float sure = static_cast<float>(sh.found_sum[1]), most_all = static_cast<float>(masses) * kOver, least_all = fmaxf(sure * ratio, 0x1p44f) / kOver;
      const float want_low = p * least_all, want_high = p * most_all, rest_low = (1.0f - p) * least_all, rest_high = (1.0f - p) * most_all;
      for (int i = 0; i < 2; ++i) {
        const int b = 2 * tid + i;
        const float hi = static_cast<float>(i == 0 ? before + m0 : before + m0 + m1);
        if (b >= last) continue;
        // not in this bin or before it: all up to it is too little, or all behind it too much
        if (hi * kOver < want_low || fmaxf(sure - hi, 0.0f) * (ratio / kOver) > rest_high + sure * 0x1p-20f) atomicMax(&sh.found[0], static_cast<uint32_t>(b + 1));
        // not after it: all up to it is enough, or all behind it no more than may be
        if (hi * (ratio / kOver) >= want_high || (static_cast<float>(masses) - hi) * kOver + most_all * 0x1p-20f <= rest_low) atomicMin(&sh.found[1], static_cast<uint32_t>(b));
      }
      __syncthreads();
      uint32_t high = K::key(r.bin_high(static_cast<int>(sh.found[0]))), low = max(K::key(r.bin_low(static_cast<int>(sh.found[1]))), K::key(cut));
      // (46 steps of the logarithm under the largest logit, weights are 0)
      low = max(low, K::key(fmaxf(r.lowest, __fsub_rd(most, __fmul_ru(46.0f, __frcp_ru(r.c))))));
      high = max(high, low);
      // the whole mass, and that above the bounds
      u64 whole = 0, passed = 0;
      const float over = K::logit(high);
      const float under = K::logit(low);
      const bool some = ties != ~0ull;  // (of those at the cut)
      r.each(cut, [&](float v) {
        const u64 w = r.weight(some ? v > cut ? v : -INFINITY : v >= cut ? v : -INFINITY);
        whole += w;
        if (v > over) passed += w;
        r.note(v <= over && v >= under, v);
      });
      above = passed;
      u64 notes = r.lane == 0 ? r.noted : 0;
      r.sums(whole, passed, notes);
      if (ties != ~0ull) whole += ties * r.weight(cut);
      u64 want = 1;
      if (p > 0.0f) {
        bool cut_off;
        want = times(p, whole, cut_off);
        want += cut_off;
      }
      // Few logits between the bounds: one CTA puts them in order instead of histograms of their keys, of which logits of 32 bits take up to four (one
      // row of 50,021 28 us for 33, 512 rows of 1,000 21 for 24.5; with up to 256 of them, rows of 131,072 took 64 for 62).
      const bool few = notes > 0 && notes <= kFew;  // (the same in every CTA)
      static_assert(kFew <= SampleRow<T, NT>::kNotes && kFew <= kList && kFew <= NT, "all of them were put down, and a thread takes each");
      if (few) {
        if (r.noted > 0) {
          uint32_t at = 0;
          if (r.lane == 0) at = atom_cluster_add(mapa_cluster(smem_u32(&sh.listed), 0), static_cast<uint32_t>(r.noted));
          at = __shfl_sync(0xffffffffu, at, 0);
          __syncwarp();
          for (int i = r.lane; i < r.noted; i += 32) st_cluster_f32(mapa_cluster(smem_u32(sh.list_logit + at + i), 0), sh.notes[r.warp][i]);
        }
        r.sync();
        if (rank == 0) r.settle(passed, want);
        r.sync();
        const float v = sh.settled;
        const u64 n = sh.found[0];
        ties = v == cut && ties < n ? ties : n, cut = v;
        known = over;
      }
      for (int step = 0; step < 33 && !few; ++step) {  // (each leaves half of the keys at most)
        int shift = 0;
        while ((high - low) >> shift >= kBins) ++shift;
        const float upto = K::logit(high), from = fmaxf(r.lowest, K::logit(low));
        const uint2 m = r.histogram(
            [&](uint32_t *count) { r.noted_between(from, upto, [&](float v) { atomicAdd(count + ((high - K::key(v)) >> shift), 1u); }); });
        u64 up[2], down[2];
        for (int i = 0; i < 2; ++i) {
          const uint32_t b = 2 * tid + i, off = b << shift;
          const bool in = b <= (high - low) >> shift;
          const uint32_t k1 = in ? high - off : high, k0 = in && k1 - low >= (1u << shift) - 1 ? k1 - ((1u << shift) - 1) : in ? low : high;
          u64 count = in ? (i == 0 ? m.x : m.y) : 0;
          if (shift == 0) {
            if (K::logit(k1) == cut && count > ties) count = ties;
            up[i] = down[i] = count ? count * r.weight(K::logit(k1)) : 0;
          } else {
            up[i] = count ? count * r.above(r.weight(K::logit(k1))) : 0, down[i] = count ? count * r.below(r.weight(K::logit(k0))) : 0;
          }
        }
        u64 all;
        const u64 a = passed + r.before(up[0] + up[1], all), d = shift == 0 ? a : passed + r.before(down[0] + down[1], all);
        const uint32_t bins = ((high - low) >> shift);
        if (tid == 0) sh.found[0] = sh.found[1] = bins, sh.found_sum[0] = passed;
        __syncthreads();
        if (a < want && a + up[0] + up[1] >= want) {
          const bool second = a + up[0] < want;
          r.publish(2 * tid + second, second ? a + up[0] : a);
        }
        if (d < want && d + down[0] + down[1] >= want) sh.found[1] = 2 * tid + (d + down[0] < want);
        __syncthreads();
        const uint32_t b0 = sh.found[0], b1 = sh.found[1];
        const u64 sum = sh.found_sum[0];
        __syncthreads();
        if (shift == 0) {
          const float v = K::logit(high - b0);
          const u64 w = r.weight(v), n = (want - sum + w - 1) / w;
          ties = v == cut && ties < n ? ties : n, cut = v;
          known = upto;
          break;
        }
        // between the bounds; where that is more than half of what it was (they may say little of a few wide bins), the half of it that the cut is in
        const uint32_t range = high - low, next = high - (b0 << shift), least = b1 >= bins ? low : max(low, high - (((b1 + 1) << shift) - 1));
        const bool halve = next - least > range / 2;
        const uint32_t mid = least + (next - least) / 2;
        if (b0 > 0 || halve) {
          u64 more = 0, half = 0;
          const float border = K::logit(next), middle = K::logit(halve ? mid : next);
          r.noted_between(middle, upto, [&](float v) {
            if (v > middle) (v > border ? more : half) += r.weight(v);
          });
          above += more;
          const u64 half_here = half;
          r.sums(more, half);
          passed += more;
          high = next, low = least;
          if (halve) {
            if (passed + half >= want) low = mid + 1;
            else passed += half, above += half_here, high = mid;
          }
        } else {
          low = least;
        }
      }
    }
  }
  if (!greedy && min_p > 0.0f && sh.floor > cut) cut = sh.floor, ties = ~0ull;
  if (known < cut) known = INFINITY;

  const auto segments = [&](u64 mine, u64 &all) {  // sum over the warps before this one in the row, and over all
    __syncthreads();
    if (r.lane == 0) sh.segment[r.flip][r.warp] = mine;
    r.sync();
    u64 s = 0;
    all = 0;
    for (uint32_t q = 0; q < ctas; ++q) {
      u64 v = r.lane < kWarps ? ld_cluster_u64(mapa_cluster(smem_u32(&sh.segment[r.flip][r.lane]), q)) : 0, w = v;
      for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
      all += v;
      if (q < rank) s += v;
      if (q == rank) {
        w = r.lane < r.warp ? w : 0;
        for (int o = 16; o > 0; o >>= 1) w += __shfl_xor_sync(0xffffffffu, w, o);
        s += w;
      }
    }
    r.flip ^= 1;
    return s;
  };
  const auto warp_sum = [&](u64 v) {
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
  };
  // This warp's mass, in the order of the row: the equal ones that stay are the first of the row.  u at an end takes the first or the last
  // that stays, whatever their weights are.
  const bool ends = greedy || !(u > 0.0f) || !(u < 1.0f);
  const auto weight = [&](float v) { return ends ? 1ull : r.weight(v); };
  if (ends) known = INFINITY;
  u64 mine = 0, equal = 0, all;
  if (known < INFINITY) {
    mine = above;
    r.noted_between(cut, known, [&](float v) {
      if (v > cut) mine += r.weight(v);
      else ++equal;
    });
  } else {
    r.each(cut, [&](float v) {
      if (v > cut) mine += weight(v);
      equal += v == cut;
    });
  }
  mine = warp_sum(mine), equal = warp_sum(equal);
  const u64 one = weight(cut);
  u64 earlier = 0;  // equal ones before this warp
  if (ties != ~0ull) {
    earlier = segments(equal, all);
    if (all <= ties) ties = ~0ull;
  }
  const u64 left = ties > earlier ? ties - earlier : 0;  // equal ones that stay from this warp on
  mine += (equal < left ? equal : left) * one;
  u64 passed = segments(mine, all), target = 0;
  if (!(u < 1.0f) && u > 0.0f) {
    target = all - 1;
  } else if (!ends) {
    bool cut_off;
    target = times(u, all, cut_off);
  }
  // The warp with the token's place hands its part of the row to all warps of its CTA.
  if (r.lane == 0 && passed <= target && target < passed + mine) sh.hand = {passed, earlier, r.block, r.blocks};
  __syncthreads();
  if (sh.hand.blocks > 0) {
    const int per = (sh.hand.blocks + 32 * kWarps - 1) / (32 * kWarps) * 32, from = sh.hand.block + r.warp * per;
    const int blocks = max(0, min(per, sh.hand.blocks - r.warp * per));
    mine = equal = 0;
    r.blocks_of(from, blocks, [&](const float (&v)[V], int) {
#pragma unroll
      for (int e = 0; e < V; ++e) mine += v[e] > cut ? weight(v[e]) : 0, equal += v[e] == cut;
    });
    mine = warp_sum(mine), equal = warp_sum(equal);
    if (r.lane == 0) sh.warp[r.warp][0] = mine, sh.warp[r.warp][1] = equal;
    __syncthreads();
    // (lane i for warp i)
    equal = r.lane < kWarps ? sh.warp[r.lane][1] : 0;
    const u64 ranks = sh.hand.rank + r.lanes_before(equal), stay = ties > ranks ? ties - ranks : 0;
    mine = (r.lane < kWarps ? sh.warp[r.lane][0] : 0) + (equal < stay ? equal : stay) * one;
    const u64 masses = sh.hand.passed + r.lanes_before(mine);
    if (__shfl_sync(0xffffffffu, masses <= target && target < masses + mine, r.warp)) {
      passed = __shfl_sync(0xffffffffu, masses, r.warp), earlier = __shfl_sync(0xffffffffu, ranks, r.warp);
      r.blocks_of(from, blocks, [&](const float (&v)[V], int block) {
        uint32_t equals = 0;
#pragma unroll
        for (int e = 0; e < V; ++e) equals += v[e] == cut;
        const u64 here = earlier + r.lanes_before(equals);
        // the equal ones that stay are the first of this block
        const int first = here >= ties ? 0 : ties - here < V ? static_cast<int>(ties - here) : V;
        u64 w[V], sum = 0;
        int met = 0;
#pragma unroll
        for (int e = 0; e < V; ++e) w[e] = v[e] > cut ? weight(v[e]) : v[e] == cut && met++ < first ? one : 0, sum += w[e];
        u64 at = passed + r.lanes_before(sum);
        const u64 next = at + sum, next_rank = here + equals;
#pragma unroll
        for (int e = 0; e < V; ++e) {
          if (at <= target && target < at + w[e]) call.tokens[row] = static_cast<int64_t>(block) * V - r.shift + e;
          at += w[e];
        }
        passed = __shfl_sync(0xffffffffu, next, 31), earlier = __shfl_sync(0xffffffffu, next_rank, 31);
      });
    }
  }
  if (ctas > 1) cluster_sync_all();  // (no CTA ends while another one reads its sums)
}

template <typename T, int NT>
cudaError_t launch(const SampleCall &c, cudaStream_t st, int *clusters = nullptr) {
  using Shared = SampleShared<NT>;
  cudaError_t e = cudaFuncSetAttribute(sample_kernel<T, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(Shared));
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = static_cast<unsigned>(c.ctas), attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(c.rows) * static_cast<unsigned>(c.ctas));
  cfg.blockDim = dim3(NT);
  cfg.dynamicSmemBytes = sizeof(Shared);
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (clusters) return cudaOccupancyMaxActiveClusters(clusters, sample_kernel<T, NT>, &cfg);
  return cudaLaunchKernelEx(&cfg, sample_kernel<T, NT>, c);
}

constexpr int kLong = 1024, kShort = 256;  // threads of a CTA

// rows of 2^i CTAs of NT threads that the current device holds at once
template <int NT>
int rows_at_once(int i) {
  static std::atomic<int> known[64][4];  // by device
  int device = 0, n = 0;
  if (cudaGetDevice(&device) != cudaSuccess || device < 0 || device >= 64) return 0;
  if ((n = known[device][i].load(std::memory_order_relaxed)) == 0) {
    SampleCall c = {};
    c.rows = 1, c.ctas = 1 << i;
    if (launch<float, NT>(c, nullptr, &n) != cudaSuccess) n = 0;
    known[device][i].store(n, std::memory_order_relaxed);
  }
  return n;
}

// CTAs to a row: as long as all rows' run at once, and each has 8 logits to a thread (one row of 50,021: 27.3 us with 4 CTAs and 30.6 with 8 at
// top-p alone, 36.5 with one; 15.6 with either, 20.7 with one, at top-k; of 131,072 in 16 bits 36.7, 38.5 and 67)
template <int NT>
int ctas_of(const SampleCall &c) {
  int i = 0;
  while (i < 3 && c.rows <= rows_at_once<NT>(i + 1) && c.vocab >= (2 << i) * 8 * NT) ++i;
  return 1 << i;
}

template <int NT>
cudaError_t launch_of(SampleCall c, cudaStream_t st) {
  c.ctas = ctas_of<NT>(c);
  if (c.dtype == 0) return launch<float, NT>(c, st);
  if (c.dtype == 1) return launch<__half, NT>(c, st);
  return launch<__nv_bfloat16, NT>(c, st);
}

}  // namespace

cudaError_t launch_sample(const SampleCall &c, cudaStream_t st) {
  // Short rows, and rows that CTAs of 1,024 threads, one to an SM, would take in three rounds or more: CTAs of 256 threads, of which an SM holds
  // four (512 rows of 1,000 logits 18 us, 62 in the long ones; of 30,000 85 and 118; but 160 rows of 131,072 168 and 131, and 305 of them 315 and 195,
  // where the rule takes the slower side).
  if (c.vocab <= 4 * kLong || c.rows > 2 * sm_count()) return launch_of<kShort>(c, st);
  return launch_of<kLong>(c, st);
}

}  // namespace aecct
