// attend.cu -- one new token of each sequence over its keys and values in a paged cache: the choice of a kernel (attend.cuh), and
// the join of what passed a CTA's border.
#include <cuda_runtime.h>

#include <cmath>
#include <cstdint>

#include "attend.cuh"

namespace aecct {

namespace {

constexpr int kJoinThreads = 128;

// Query head blockIdx.y of the piece that begins in CTA blockIdx.x and goes on in those after it.  And a row of zeros for
// sequences that have no key: no tile of theirs is in the list.
__global__ void __launch_bounds__(kJoinThreads) attend_join_kernel(const __grid_constant__ AttendArgs a, AttendPlan plan) {
  grid_wait();
  const int tid = threadIdx.x, lane = tid & 31, head = blockIdx.y;
  if (head == 0) {
    for (int base = (blockIdx.x * kJoinThreads + tid) & ~31; base < a.seqs.batch; base += gridDim.x * kJoinThreads) {
      const int b = base + lane;
      bool none = false;
      if (b < a.seqs.batch) {
        const int n = sequence_length(a.seqs, b, a.cache.page_size);
        none = n == 0 || (a.first && a.first[b] >= n);
      }
      for (uint32_t left = __ballot_sync(0xffffffffu, none); left; left &= left - 1) {
        const int64_t row = static_cast<int64_t>(base + __ffs(left) - 1) * a.q_heads;
        for (int64_t i = lane; i < static_cast<int64_t>(a.q_heads) * a.cache.dim; i += 32) store_out(a, row * a.cache.dim + i, 0.0f);
        if (a.lse)
          for (int i = lane; i < a.q_heads; i += 32) a.lse[row + i] = -INFINITY;
      }
    }
  }
  const auto ends_at = [&](int c) { return c < static_cast<int>(gridDim.x) ? a.piece[c * 2].ends != 0 : true; };
  const AttendPiece p = a.piece[blockIdx.x * 2 + 1];
  bool ends = ends_at(blockIdx.x + 1 + lane);
  if (p.b < 0) return;
  const int part = p.j % a.parts;
  if (head >= min(plan.heads, a.group - part * plan.heads)) return;
  // the CTAs up to the one where it ends
  int count = 1;
  for (int c = blockIdx.x + 1;;) {
    const uint32_t found = __ballot_sync(0xffffffffu, ends);
    if (found) {
      count += c - static_cast<int>(blockIdx.x) - 1 + __ffs(found);
      break;
    }
    c += 32;
    ends = ends_at(c + lane);
  }
  const auto from = [&](int k) { return a.partial + ((blockIdx.x + k) * 2 + (k == 0 ? 1 : 0)) * static_cast<int64_t>(plan.part); };
  const int row = 2 * plan.heads + head * plan.width;
  float top = -INFINITY, l = 0.0f, v[2] = {0.0f, 0.0f};
  // 32 parts at a time, a lane to each for what it is scaled by; 8 parts' rows on their way at once
  for (int k0 = 0; k0 < count; k0 += 32) {
    const int parts = min(32, count - k0);
    float mine = lane < parts ? from(k0 + lane)[head] : -INFINITY;
    const float sum = lane < parts ? from(k0 + lane)[plan.heads + head] : 0.0f;
    for (int k1 = 0; k1 < parts; k1 += 8) {
      float x[8][2];
#pragma unroll
      for (int k = 0; k < 8; ++k)
#pragma unroll
        for (int i = 0; i < 2; ++i) x[k][i] = k1 + k < parts && tid + i * kJoinThreads < plan.width ? from(k0 + k1 + k)[row + tid + i * kJoinThreads] : 0.0f;
      if (k1 == 0) {
        float most = fmaxf(top, mine);
        for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
        const float base = most == -INFINITY ? 0.0f : most, old = exp2_fast(top - base);
        mine = exp2_fast(mine - base);
        float s = sum * mine;
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        l = fmaf(l, old, s), v[0] *= old, v[1] *= old, top = most;
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float by = __shfl_sync(0xffffffffu, mine, k1 + k);
        v[0] = fmaf(x[k][0], by, v[0]), v[1] = fmaf(x[k][1], by, v[1]);
      }
    }
  }
  const int64_t at = static_cast<int64_t>(p.b) * a.q_heads + p.j / a.parts * a.group + part * plan.heads + head;
  for (int i = 0; i < 2; ++i) {
    const int e = tid + i * kJoinThreads;
    if (e < a.cache.dim) store_out(a, at * a.cache.dim + e, share(v[i], l));
  }
  if (tid == 0 && a.lse) a.lse[at] = lse_of(top, l);
}

// One piece of 16 bits for a weight is under the rounding of a bfloat16 result (2^-11 of it and 2^-8, each at most half a step); a
// half or float result takes two, and so does a cache in bfloat16, whose weights have that type's 8 bits.
cudaError_t run(int dim, int group, int dtype, int cache_dtype, const AttendArgs *a, AttendPlan *plan, cudaStream_t st) {
  if (cache_dtype == 1) return run_attend_half(dim, group, a, plan, st);
  if (cache_dtype == 2) return run_attend_bf16(dim, group, a, plan, st);
  return dtype == 2 ? run_attend_codes(dim, group, a, plan, st) : run_attend_pieces(dim, group, a, plan, st);
}

int64_t piece_bytes(const AttendPlan &p) { return (2 * static_cast<int64_t>(p.ctas) * p.part * static_cast<int64_t>(sizeof(float)) + 15) / 16 * 16; }

}  // namespace

int64_t attend_workspace(int, int q_heads, int heads, int dim, int dtype, int cache_dtype) {
  AttendPlan p = {};
  run(dim, q_heads / heads, dtype, cache_dtype, nullptr, &p, nullptr);
  return piece_bytes(p) + 2 * static_cast<int64_t>(p.ctas) * static_cast<int64_t>(sizeof(AttendPiece));
}

cudaError_t launch_attend(const AttendCall &c, cudaStream_t st) {
  const int group = c.q_heads / c.cache.heads;
  AttendPlan p = {};
  run(c.cache.dim, group, c.dtype, c.cache_dtype, nullptr, &p, st);
  AttendArgs a = {c.cache, c.seqs, c.first, c.q, c.ld_row, c.ld_head, group, c.q_heads, c.dtype, (group + p.heads - 1) / p.heads, c.scale * kLog2e, c.out,
                  c.lse, static_cast<float *>(c.workspace), reinterpret_cast<AttendPiece *>(static_cast<char *>(c.workspace) + piece_bytes(p)), 0};
  // A cluster to each piece where all run at once and no warp has more than 4 tiles, as far as the table says: the most CTAs that have a tile for
  // each warp.  (Beyond that, the longest sequence would have its cluster work while others are done.)
  const int64_t pieces = static_cast<int64_t>(c.seqs.batch) * c.cache.heads * a.parts;
  const int64_t tiles = (static_cast<int64_t>(c.seqs.columns) * c.cache.page_size + p.tile - 1) / p.tile;
  for (int i = 0; i < 4; ++i)
    if (pieces <= p.at_once[i] && tiles <= 4 * static_cast<int64_t>(p.warps << i) && (i == 0 || tiles > p.warps << (i - 1))) a.ctas = 1 << i;
  // A warp to each piece where there are more, of 6 tiles at most, or of 16 where most warps have one (512 pieces of 4 tiles 11 us, dealt out 16; of 8
  // 17.6 and 16.3, of 16 30 and 21; 2,048 pieces of 16 tiles 48 and 54).
  if (a.ctas == 0 && pieces <= INT32_MAX / 2 && (tiles <= 6 || (tiles <= 16 && 4 * pieces >= 3 * static_cast<int64_t>(p.ctas) * p.warps))) a.ctas = -1;
  const cudaError_t e = run(c.cache.dim, group, c.dtype, c.cache_dtype, &a, &p, st);
  if (e != cudaSuccess || a.ctas != 0) return e;
  return launch_dependent(attend_join_kernel, dim3(p.ctas, p.heads), kJoinThreads, 0, st, a, p);
}

}  // namespace aecct
