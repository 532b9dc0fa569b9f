// The joining of an attention's chunks along the cache: out = sum_k 2^(m_k - m) o_k / sum_k
// 2^(m_k - m) l_k over the chunks' maxima m_k, sums l_k and weighted sums o_k, in a fixed order.
#pragma once

#include "nq_attend.hpp"

namespace nq {
namespace {

// DIM / 4 threads take a row of a block: all chunks of it, W rows a workgroup (THREADS 256), or,
// where there are few rows of many chunks, every W-th chunk, the W shares then joined in LDS
// (THREADS 1024: 32 rows of 256 chunks of 128 entries took 10.3 us with 256).  BR: rows of a block;
// tiles of 2^SHIFT tokens, PER of them a step of the chunks.
template <int DIM, int BR, int SHIFT, int PER, int THREADS>
__global__ __launch_bounds__(THREADS) void join_kernel(AttendArgs a, int parts) {
  constexpr bool SPREAD = THREADS > 256;
  constexpr int L = DIM / 4, W = THREADS / L;
  __shared__ __attribute__((aligned(16))) float sums[SPREAD ? W : 1][DIM];
  __shared__ float tops[W], totals[W];
  const int c = (int)threadIdx.x % L, w = (int)threadIdx.x / L;
  const uint32_t id = SPREAD ? blockIdx.x : blockIdx.x * W + w;
  if (!SPREAD && id >= (uint32_t)parts) return;
  const Place at = place_of(a, id);
  const int head = at.head, b = at.b, x = at.part % a.rows, rb = at.part / a.rows;
  const Sequence sq = sequence_of(a, b);
  const RowBlock blk = row_block<BR>(a, sq, rb);
  if (x >= blk.rows) return;
  const Tiles tiles = tiles_of<SHIFT>(a, blk.p_lo, blk.p_hi, sq.end);
  const int steps = (tiles.count + PER - 1) / PER;
  const int n = (steps + a.steps - 1) / a.steps;
  float big = -INFINITY, total = 0.0f;
  f32x4 sum = {};
  auto add = [&](float m, float l, f32x4 v) {
    const float next = fmaxf(big, m), ref = next == -INFINITY ? 0.0f : next;
    const float fo = __builtin_amdgcn_exp2f(big - ref), fn = __builtin_amdgcn_exp2f(m - ref);
    total = total * fo + l * fn;
    sum = sum * fo + v * fn;
    big = next;
  };
  constexpr int AHEAD = 4;                      // partial rows in flight
  constexpr int STEP = SPREAD ? W : 1;
  const float* __restrict__ first = partial(a, b, head, rb, x, 0, DIM);
  for (int k = SPREAD ? w : 0; k < n; k += AHEAD * STEP) {
    float m[AHEAD], l[AHEAD];
    f32x4 v[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int kk = k + i * STEP < n ? k + i * STEP : k;
      const float* y = first + (int64_t)kk * (DIM + 4);
      m[i] = y[0];
      l[i] = y[1];
      v[i] = *reinterpret_cast<const f32x4*>(y + 4 + 4 * c);
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
      if (k + i * STEP < n) add(m[i], l[i], v[i]);
  }
  if constexpr (SPREAD) {
    *reinterpret_cast<f32x4*>(&sums[w][4 * c]) = sum;
    if (c == 0) {
      tops[w] = big;
      totals[w] = total;
    }
    __syncthreads();
    if (w != 0) return;
#pragma unroll
    for (int k = 1; k < W; ++k)
      add(tops[k], totals[k], *reinterpret_cast<const f32x4*>(&sums[k][4 * c]));
  }
  const int r = blk.r0 + x, i = query_of(a, r), hq = head * (int)a.by_group.n + r - i * (int)a.by_group.n;
  const int64_t token = sq.first + i;
  store_out(a.out, a.dtype, token * a.out_token + hq * a.out_head + 4 * c, sum * inverse_sum(total));
  if (a.lse && c == 0) a.lse[token * a.q_heads + hq] = log_sum(big, total);
}

template <int DIM, int BR, int SHIFT, int PER>
hipError_t launch_join(const AttendArgs& a, hipStream_t st) {
  const int parts = a.rows * a.blocks * a.heads * a.seqs;
  constexpr int W = 1024 / DIM;
  if (a.chunks > 8 && parts < 1024) {
    hipLaunchKernelGGL((join_kernel<DIM, BR, SHIFT, PER, 1024>), dim3((unsigned)parts), dim3(1024), 0,
                       st, a, parts);
  } else {
    hipLaunchKernelGGL((join_kernel<DIM, BR, SHIFT, PER, 256>), dim3((unsigned)((parts + W - 1) / W)),
                       dim3(256), 0, st, a, parts);
  }
  return hipGetLastError();
}

}  // namespace
}  // namespace nq
