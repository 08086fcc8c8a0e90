// Device side of the work split: where a CTA's share begins.
#pragma once
#include "paged_batch.cuh"

namespace ilre {

// All threads of the CTA; `tmp` holds 34 entries in shared memory, *out is valid after it returns.
__device__ __forceinline__ void plan_start(const PagedBatch& b, const TileShape& ts, int min_units, long long* tmp,
                                           PlanStart* out) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_warps = (blockDim.x + 31) >> 5;
  long long mine = 0;
  for (int i = threadIdx.x; i < b.n_seqs; i += blockDim.x) mine += seq_units(b, ts, i);
  long long sum = mine;
  for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
  if (lane == 0) tmp[warp] = sum;
  __syncthreads();
  long long total = 0;
  for (int w = 0; w < n_warps; ++w) total += tmp[w];
  const int n_cta = share_ctas(total, gridDim.x, min_units);
  const bool has = total > 0 && static_cast<int>(blockIdx.x) < n_cta;
  const long long u0 = has ? share_begin(total, n_cta, blockIdx.x) : 0;
  if (threadIdx.x == 0) {
    out->total = total; out->n_cta = n_cta;
    out->u0 = u0; out->u1 = has ? share_begin(total, n_cta, blockIdx.x + 1) : 0;
    out->seq = 0; out->seq_begin = 0;
  }
  __syncthreads();
  if (has) {
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
}

}  // namespace ilre
