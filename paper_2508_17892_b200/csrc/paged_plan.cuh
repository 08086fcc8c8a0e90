// Device side of the work split: where a CTA's share begins.
#pragma once
#include "paged_batch.cuh"

namespace ilre {

// Units of the whole batch: all threads of the CTA; `tmp` holds 34 entries in shared memory.  *mine: the units of
// the sequences that this thread looked at (its own one, if the batch has no more than the CTA threads).
__device__ __forceinline__ long long plan_total(const PagedBatch& b, const TileShape& ts, long long* tmp, long long* mine) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_warps = (blockDim.x + 31) >> 5;
  long long sum = 0;
  for (int i = threadIdx.x; i < b.n_seqs; i += blockDim.x) sum += seq_units(b, ts, i);
  *mine = sum;
  for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
  if (lane == 0) tmp[warp] = sum;
  __syncthreads();
  long long total = 0;
  for (int w = 0; w < n_warps; ++w) total += tmp[w];
  __syncthreads();
  return total;
}

// The sequence that unit u0 lies in, and its first unit, into *out (valid behind a barrier).
__device__ __forceinline__ void plan_find(const PagedBatch& b, const TileShape& ts, long long mine, long long u0,
                                          long long* tmp, PlanStart* out) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_warps = (blockDim.x + 31) >> 5;
  long long base = 0;
  for (int i0 = 0; i0 < b.n_seqs; i0 += blockDim.x) {
    const int i = i0 + threadIdx.x;
    const long long n = (i < b.n_seqs) ? (b.n_seqs <= static_cast<int>(blockDim.x) ? mine : seq_units(b, ts, i)) : 0;
    long long incl = n;
    for (int o = 1; o < 32; o <<= 1) {
      const long long v = __shfl_up_sync(0xFFFFFFFFu, incl, o);
      if (lane >= o) incl += v;
    }
    if (lane == 31) tmp[warp] = incl;
    __syncthreads();
    long long before = base;
    for (int w = 0; w < n_warps; ++w) {
      if (w < warp) before += tmp[w];
      base += tmp[w];
    }
    const long long begin = before + incl - n;
    if (n > 0 && begin <= u0 && u0 < begin + n) { out->seq = i; out->seq_begin = begin; }
    __syncthreads();
    if (base > u0) break;
  }
}

// The units [u0, u1) as a share of its own: all threads; *out is valid behind the next barrier.
__device__ __forceinline__ void plan_range(const PagedBatch& b, const TileShape& ts, long long total, int n_cta,
                                           long long mine, long long u0, long long u1, long long* tmp, PlanStart* out) {
  if (threadIdx.x == 0) { out->total = total; out->n_cta = n_cta; out->u0 = u0; out->u1 = u1; out->seq = 0; out->seq_begin = 0; }
  __syncthreads();
  if (u0 < u1) plan_find(b, ts, mine, u0, tmp, out);
}

// This CTA's share.
__device__ __forceinline__ void plan_start(const PagedBatch& b, const TileShape& ts, int min_units, long long* tmp,
                                           PlanStart* out) {
  long long mine;
  const long long total = plan_total(b, ts, tmp, &mine);
  const int n_cta = share_ctas(total, gridDim.x, min_units), c = blockIdx.x;
  const bool has = total > 0 && c < n_cta;
  plan_range(b, ts, total, n_cta, mine, has ? share_begin(total, n_cta, c) : 0, has ? share_begin(total, n_cta, c + 1) : 0, tmp, out);
}

// The last unit of the share that CTA blockIdx.x of `grid` had; nothing for the last share of all.
__device__ __forceinline__ void plan_last(const PagedBatch& b, const TileShape& ts, int grid, int min_units, long long* tmp,
                                          PlanStart* out) {
  long long mine;
  const long long total = plan_total(b, ts, tmp, &mine);
  const int n_cta = share_ctas(total, grid, min_units), c = blockIdx.x;
  const bool has = total > 0 && c + 1 < n_cta;
  const long long end = has ? share_begin(total, n_cta, c + 1) : 0;
  plan_range(b, ts, total, n_cta, mine, has ? end - 1 : 0, end, tmp, out);
}

}  // namespace ilre
