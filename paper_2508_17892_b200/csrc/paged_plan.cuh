// Device side of the work split: where a CTA's share begins.
#pragma once
#include "paged_batch.cuh"

namespace ilre {

static constexpr int kPlanTmp = 36;

// Units of the whole batch: all threads of the CTA; `tmp` holds kPlanTmp entries in shared memory.  *mine: the units of
// the sequences that this thread looked at (its own one, if the batch has no more than the CTA threads).
template <class Tiles>
__device__ __forceinline__ long long plan_total(const PagedBatch& b, const TileShape& ts, long long* tmp, long long* mine) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_warps = (blockDim.x + 31) >> 5;
  long long sum = 0;
  for (int i = threadIdx.x; i < b.n_seqs; i += blockDim.x) sum += seq_units<Tiles>(b, ts, i);
  *mine = sum;
  for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
  if (lane == 0) tmp[warp] = sum;
  __syncthreads();
  long long total = 0;
  for (int w = 0; w < n_warps; ++w) total += tmp[w];
  __syncthreads();
  return total;
}

// The items of units u0 and u1 - 1 into *out (valid behind a barrier).
template <class Tiles>
__device__ __forceinline__ void plan_find(const PagedBatch& b, const TileShape& ts, long long mine, long long u0,
                                          long long u1, long long* tmp, PlanStart* out) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_warps = (blockDim.x + 31) >> 5;
  long long* found = tmp + 32;             // (sequence, first unit) of u0 and of u1 - 1
  long long base = 0;
  for (int i0 = 0; i0 < b.n_seqs; i0 += blockDim.x) {
    const int i = i0 + threadIdx.x;
    const long long n = (i < b.n_seqs) ? (b.n_seqs <= static_cast<int>(blockDim.x) ? mine : seq_units<Tiles>(b, ts, i)) : 0;
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
    if (n > 0 && begin <= u0 && u0 < begin + n) { found[0] = i; found[1] = begin; }
    if (n > 0 && begin < u1 && u1 <= begin + n) { found[2] = i; found[3] = begin; }
    __syncthreads();
    if (base >= u1) break;
  }
  if (warp < 2) {
    const int seq = static_cast<int>(found[2 * warp]);
    const SeqSpan span = load_span(b, seq);
    const Item x = locate_by_head<Tiles>(ts, seq, span, head_units<Tiles>(b, ts, span), found[2 * warp + 1], warp ? u1 - 1 : u0);
    if (lane == 0) { if (warp) out->last = x; else out->first = x; }
  }
}

// The same for a batch of at most 32 sequences: one load of the lengths and no barrier, each of two warps for itself.
template <class Tiles>
__device__ __forceinline__ void plan_small(const PagedBatch& b, const TileShape& ts, int min_units, PlanStart* out) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (warp >= 2) return;
  SeqSpan span = {0, 0, 0};
  long long per_head = 0;
  if (lane < b.n_seqs) {
    span = load_span(b, lane);
    per_head = head_units<Tiles>(b, ts, span);
  }
  const long long n = per_head * ts.heads;
  long long incl = n;
  for (int o = 1; o < 32 && o < b.n_seqs; o <<= 1) {
    const long long v = __shfl_up_sync(0xFFFFFFFFu, incl, o);
    if (lane >= o) incl += v;
  }
  const long long total = __shfl_sync(0xFFFFFFFFu, incl, b.n_seqs - 1);
  const int n_cta = share_ctas(total, gridDim.x, min_units), c = blockIdx.x;
  const bool has = total > 0 && c < n_cta;
  const long long u0 = has ? share_begin(total, n_cta, c) : 0, u1 = has ? share_begin(total, n_cta, c + 1) : 0;
  if (threadIdx.x == 0) { out->total = total; out->n_cta = n_cta; out->u0 = u0; out->u1 = u1; }
  if (!has) return;
  const long long at = warp ? u1 - 1 : u0, begin = incl - n;
  const int seq = __ffs(__ballot_sync(0xFFFFFFFFu, begin <= at && at < incl)) - 1;
  span = SeqSpan{__shfl_sync(0xFFFFFFFFu, span.q0, seq), __shfl_sync(0xFFFFFFFFu, span.n, seq), __shfl_sync(0xFFFFFFFFu, span.kv, seq)};
  const Item x = locate_by_head<Tiles>(ts, seq, span, __shfl_sync(0xFFFFFFFFu, per_head, seq), __shfl_sync(0xFFFFFFFFu, begin, seq), at);
  if (lane == 0) { if (warp) out->last = x; else out->first = x; }
}

// This CTA's share: all threads; *out is valid behind the next barrier.
template <class Tiles>
__device__ __forceinline__ void plan_start(const PagedBatch& b, const TileShape& ts, int min_units, long long* tmp,
                                           PlanStart* out) {
  if (b.n_seqs <= 32) return plan_small<Tiles>(b, ts, min_units, out);
  long long mine;
  const long long total = plan_total<Tiles>(b, ts, tmp, &mine);
  const int n_cta = share_ctas(total, gridDim.x, min_units), c = blockIdx.x;
  const bool has = total > 0 && c < n_cta;
  const long long u0 = has ? share_begin(total, n_cta, c) : 0, u1 = has ? share_begin(total, n_cta, c + 1) : 0;
  if (threadIdx.x == 0) { out->total = total; out->n_cta = n_cta; out->u0 = u0; out->u1 = u1; }
  if (has) plan_find<Tiles>(b, ts, mine, u0, u1, tmp, out);
}

}  // namespace ilre
