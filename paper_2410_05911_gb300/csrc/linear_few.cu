// linear_few.cu -- the AAP linear layer (linear.cu has the formulas) for the few tokens of a decoding step.
//
// The work is to read the weights once, a quarter of a byte each: there is nothing in it for the tensor cores, whose
// operands would have to be converted, stored and waited for.  A word's 16 2-bit weights are the selectors of a byte
// permutation in two masked halves, which makes 4 words of bytes 0, 1 and -1 (field 10 is 0), and each of those
// is 4 products with codes of the same order in one instruction, in integers: exact, however K is split.
//
// A warp takes 4 rows of weights by 2,048 k at a time, its lanes neighbouring 16s of them, so that the codes are put
// in order once for 4 rows; a CTA's warps split a longer row, up to 8 ways, and join it in shared memory.
//
// 1 token, 4,096 x 4,096: 3.6 us, most of it the launch and one trip to memory (2.7 us at 128 x 512); 16,384 x 4,096:
// 8.3 us, 2 TB/s of weights, bound by the integer instructions (a 4-product instruction takes some 5 cycles of a
// scheduler, so that mma.sync was no better: 14.6 us, and half-precision fragments 5.6 us at 4,096 x 4,096).
#include <cuda_runtime.h>

#include <cstdint>

#include "linear_gemm.cuh"

namespace aecct {

namespace {

constexpr int kFewWarps = 8, kFewRows = 4, kFewSpan = 2048;  // rows of a warp; k of its step

// y of up to TOKENS tokens; parts: warps on a row
template <int TOKENS>
__global__ void __launch_bounds__(kFewWarps * 32, TOKENS == 1 ? 3 : 2)
    few_kernel(const int8_t *codes, int64_t ldc, int codes_in, const uint8_t *packed, int weights_in, int M, int64_t N, int64_t K,
               int parts, const OutY out) {
  __shared__ int sums[kFewWarps][kFewRows * TOKENS];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, part = warp & (parts - 1), group = warp / parts;
  const int rows = kFewWarps / parts * kFewRows;  // of the CTA
  const int64_t row0 = static_cast<int64_t>(blockIdx.x) * rows;
  // this thread's output, and what it takes beside the sum
  const int orow = threadIdx.x % rows, token = threadIdx.x / rows;
  const int64_t n = row0 + orow;
  const bool owns = token < M && n < N;
  const float factor = owns ? out.factor(token) : 0.0f, add = owns ? out.add(n) : 0.0f;

  const uint8_t *w0[kFewRows], *limit = packed + (N * K >> 2);
#pragma unroll
  for (int r = 0; r < kFewRows; ++r) {
    const int64_t row = row0 + group * kFewRows + r;  // (past the last one: that one again)
    w0[r] = packed + ((row < N ? row : N - 1) * K >> 2);
  }
  const int8_t *codes_end = codes + (M - 1) * ldc + K;
  // Rows of whole 16s of k: every load of a step is issued before the first is used.  Those past K read the row's
  // first codes and weights, and take them as zero codes.
  const bool whole = codes_in == 16 && weights_in >= 4;
  int acc[kFewRows][TOKENS] = {};
  for (int k0 = part * kFewSpan + lane * 16; k0 < K; k0 += parts * kFewSpan) {
    uint32_t w[kFewRows][4], c[4][TOKENS][4];
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int k = k0 + g * 512;
      if (whole) {
        const int at = k < K ? k : 0;
#pragma unroll
        for (int r = 0; r < kFewRows; ++r) w[r][g] = __ldg(reinterpret_cast<const uint32_t *>(w0[r] + (at >> 2)));
#pragma unroll
        for (int m = 0; m < TOKENS; ++m) {
          const uint4 v = __ldg(reinterpret_cast<const uint4 *>(codes + (m < M ? m : M - 1) * ldc + at));
          c[g][m][0] = v.x, c[g][m][1] = v.y, c[g][m][2] = v.z, c[g][m][3] = v.w;
        }
      } else {
#pragma unroll
        for (int r = 0; r < kFewRows; ++r) {
          uint32_t v[1];
          load_weights<1>(w0[r] + (k >> 2), static_cast<int>(K) - k, weights_in, packed, limit, v);
          w[r][g] = v[0];
        }
#pragma unroll
        for (int m = 0; m < TOKENS; ++m)
          load_codes(codes + (m < M ? m : M - 1) * ldc + k, static_cast<int>(K) - k, codes_in, codes, codes_end, c[g][m]);
      }
    }
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const bool in = k0 + g * 512 < K;
      int q[TOKENS][4];
#pragma unroll
      for (int m = 0; m < TOKENS; ++m)
#pragma unroll
        for (int s = 0; s < 4; ++s)  // the even k of 8, those of the other 8, the odd ones
          q[m][s] = in ? static_cast<int>(__byte_perm(c[g][m][2 * (s & 1)], c[g][m][2 * (s & 1) + 1], s < 2 ? 0x6420 : 0x7531)) : 0;
#pragma unroll
      for (int r = 0; r < kFewRows; ++r) {
        const uint32_t even = w[r][g] & 0x33333333u, odd = (w[r][g] >> 2) & 0x33333333u;
        const int t[4] = {static_cast<int>(__byte_perm(0xFF000100u, 0, even)), static_cast<int>(__byte_perm(0xFF000100u, 0, even >> 16)),
                          static_cast<int>(__byte_perm(0xFF000100u, 0, odd)), static_cast<int>(__byte_perm(0xFF000100u, 0, odd >> 16))};
#pragma unroll
        for (int m = 0; m < TOKENS; ++m)
#pragma unroll
          for (int s = 0; s < 4; ++s) acc[r][m] = __dp4a(q[m][s], t[s], acc[r][m]);
      }
    }
  }
#pragma unroll
  for (int m = 0; m < TOKENS; ++m)
#pragma unroll
    for (int r = 0; r < kFewRows; ++r) {
      const int v = __reduce_add_sync(0xffffffffu, acc[r][m]);
      if (lane == 0) sums[warp][r * TOKENS + m] = v;
    }
  __syncthreads();
  if (!owns) return;
  int v = 0;
  for (int p = 0; p < parts; ++p) v += sums[orow / kFewRows * parts + p][orow % kFewRows * TOKENS + token];
  put_element(out.y, out.dtype, token * out.ld + n, fmaf(static_cast<float>(v), factor, add));
}

template <int TOKENS>
cudaError_t launch_few(const AapLinearCall &c, const OutY &out, cudaStream_t st) {
  int parts = 1;
  while (parts < kFewWarps && parts * kFewSpan < c.K) parts *= 2;
  const int64_t rows = kFewWarps / parts * kFewRows;
  few_kernel<TOKENS><<<static_cast<unsigned>((c.N + rows - 1) / rows), kFewWarps * 32, 0, st>>>(
      c.codes, c.ldc, codes_unit(c.codes, c.ldc, c.K), c.packed, weights_unit(c.packed, c.K), static_cast<int>(c.M), c.N, c.K, parts, out);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_aap_linear_few(const AapLinearCall &c, cudaStream_t st) {
  const OutY out = {c.y, c.dtype, c.N, c.scale, c.w_scale, c.bias};
  return c.M == 1 ? launch_few<1>(c, out, st) : c.M == 2 ? launch_few<2>(c, out, st) : launch_few<4>(c, out, st);
}

}  // namespace aecct
