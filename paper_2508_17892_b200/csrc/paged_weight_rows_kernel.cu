// Accumulated attention weight of few query rows (decoding): w[t, g] += sum over at most 16 rows (token, head of g) that
// see t of 2^(s c2 - lse2).
//
// Bound by HBM, 256 bytes of keys for 32 flop per row and key.  As in the attention of few rows the batch's key tiles
// are cut into equal shares over two CTAs per SM, a warp of TMA loads keeps three 32 KB stages in flight per CTA and each of
// four warps has 32 keys of a stage: S = Q K^T by mma.m16n8k16, the exponentials, and the rows' sum by shuffles.  A tile's
// weights are complete in its warp, so there is nothing to join.
#include "launch.cuh"
#include "paged_mma.cuh"
#include "paged_plan.cuh"
#include "paged_weight_kernels.cuh"

namespace ilre {

namespace {

constexpr int kStages = 3;
constexpr int kKeys = 128;                               // of a stage
constexpr int kHalfBytes = kKeys * 128, kStageBytes = 2 * kHalfBytes;
constexpr int kWarps = 4;
constexpr int kThreads = 32 * (kWarps + 1);

struct Tail {
  uint64_t full[kStages], empty[kStages];
  PlanStart plan;
  long long tmp[kPlanTmp];
  int abort_flag;
  int issued;
};

template <bool kF16>
__global__ void __launch_bounds__(kThreads, 2)
paged_weight_rows_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ PagedWeightParams p,
                         const TileShape ts) {
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t ring = smem_u32(smem);
  Tail* tail = reinterpret_cast<Tail*>(smem + kStages * kStageBytes);
  volatile int* abort_flag = &tail->abort_flag;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const PagedBatch& b = p.batch;

  if (threadIdx.x == 0) {
    tail->abort_flag = tail->issued = 0;
    for (int s = 0; s < kStages; ++s) {
      mbar_init(smem_u32(&tail->full[s]), 1);
      mbar_init(smem_u32(&tail->empty[s]), kWarps);
    }
    fence_mbar_init();
    tma_prefetch_desc(&map_k);
  }
  __syncthreads();
  grid_dep_wait();
  grid_dep_launch();
  if (threadIdx.x == 0 && (ring & 1023u)) {
    tail->abort_flag = 1;
    report(b.status, kDevSmemAlign);
  }
  plan_start<HeadTiles>(b, ts, 1, tail->tmp, &tail->plan);
  __syncthreads();
  PieceWalk<HeadTiles> w;
  bool more = *abort_flag == 0 && w.begin(b, ts, tail->plan), ok = more;

  if (warp == kWarps) {
    const int ps = 1 << b.page_shift;
    const int box_rows = min(ps, kKeys), n_box = kKeys / box_rows;
    const int half = lane & 1, bx = lane >> 1;
    const bool active = bx < n_box;
    const uint32_t off = half * kHalfBytes + bx * box_rows * 128;
    int it = 0;
    // entries two tiles ahead; rows at and behind kv need none: zeros, not read
    auto needs = [&](int t) { return active && t < w.p.t1 && t * kKeys + bx * box_rows < w.p.span.kv; };
    auto entry_at = [&](int t) -> int { return needs(t) ? table_entry(b, w.p.seq, t * kKeys + bx * box_rows) : 0; };
    while (more && ok) {
      int e0 = entry_at(w.p.t0), e1 = entry_at(w.p.t0 + 1);
      for (int t = w.p.t0; t < w.p.t1; ++t, ++it) {
        const int s = it % kStages;
        const int row = t * kKeys + bx * box_rows, e2 = entry_at(t + 2);
        ok = warp_wait(&tail->empty[s], ((it / kStages) & 1) ^ 1, abort_flag, b.status, kDevWaitKEmpty);
        if (!ok) break;
        const int page = needs(t) ? checked_page(b, e0) : b.n_pages;
        const uint32_t bar = smem_u32(&tail->full[s]);
        if (lane == 0) {
          mbar_arrive_expect_tx(bar, kStageBytes);
          tail->issued = it + 1;
        }
        __syncwarp();
        if (active) tma_load_4d(ring + s * kStageBytes + off, &map_k, half * 64, w.p.head, row & (ps - 1), page, bar);
        e0 = e1;
        e1 = e2;
      }
      if (ok) more = w.next(b, ts, tail->plan);
    }
  } else {
    const int r0 = lane >> 2, c0 = (lane & 3) * 2;       // rows r0, r0 + 8; columns c0, c0 + 1 (+ 8 j)
    const int mat = lane >> 3, mr = lane & 7;
    const int tok_0 = r0 / p.group, tok_1 = (r0 + 8) / p.group;
    int it = 0;
    while (more && ok) {
      const SeqSpan span = w.p.span;
      const int seq = w.p.seq, head = w.p.head, pre = span.kv - span.n;
      // the rows' queries (zero rows where there is none) and lse in log2 units (+inf where there is none or it saw nothing)
      uint32_t qa[8][4];
      float lse2[2];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int tok = x ? tok_1 : tok_0, r = r0 + 8 * x;
        const bool valid = tok < span.n && tok < ts.tq;
        const long long at = static_cast<long long>(span.q0) + tok;
        const int h = head * p.group + r - tok * p.group;
        const uint32_t* src = reinterpret_cast<const uint32_t*>(static_cast<const uint16_t*>(p.q) + (valid ? at * p.q_stride + h * 128 : 0));
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) {
          qa[ks][x] = valid ? src[ks * 8 + (c0 >> 1)] : 0u;
          qa[ks][2 + x] = valid ? src[ks * 8 + 4 + (c0 >> 1)] : 0u;
        }
        const float v = valid ? p.lse[at * p.n_q + h] : -INFINITY;
        lse2[x] = v == -INFINITY ? INFINITY : v * 1.44269504f;
      }
      const int lim0 = pre + tok_0, lim1 = pre + tok_1;
      for (int t = w.p.t0; t < w.p.t1; ++t, ++it) {
        const int s = it % kStages, key0 = t * kKeys + warp * 32;
        // lanes r0 = j of n-tile j (eight keys) will write keys key0 + 8 j + c0 and the next, of one page
        const int key = key0 + 8 * r0 + c0;
        const bool writes = r0 < 4 && key < span.kv;
        const int entry = writes ? table_entry(b, seq, key) : 0;
        ok = warp_wait(&tail->full[s], (it / kStages) & 1, abort_flag, b.status, kDevWaitKFull);
        if (!ok) break;
        float sc[4][4] = {};
        if (key0 < span.kv) {
          const uint32_t base = ring + s * kStageBytes;
#pragma unroll
          for (int ks = 0; ks < 8; ++ks) {
            const int c16 = (ks & 3) * 2 + (mat & 1);
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              const int krow = warp * 32 + x * 16 + (mat >> 1) * 8 + mr;
              uint32_t kb[4];
              ldsm4(base + (ks >> 2) * kHalfBytes + krow * 128 + ((c16 ^ (krow & 7)) << 4), kb);
              mma16816<kF16>(sc[2 * x], qa[ks], kb[0], kb[1]);
              mma16816<kF16>(sc[2 * x + 1], qa[ks], kb[2], kb[3]);
            }
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&tail->empty[s]));
        if (key0 >= span.kv) continue;
        const bool edge = key0 + 31 > pre;
        float mine0 = 0.f, mine1 = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float a[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int k = key0 + 8 * j + c0 + i;
            float x = ex2_approx(fmaf(sc[j][i], p.c2, -lse2[0])), y = ex2_approx(fmaf(sc[j][2 + i], p.c2, -lse2[1]));
            if (edge) {
              x = k <= lim0 ? x : 0.f;
              y = k <= lim1 ? y : 0.f;
            }
            a[i] = x + y;
            a[i] += __shfl_xor_sync(0xFFFFFFFFu, a[i], 4);
            a[i] += __shfl_xor_sync(0xFFFFFFFFu, a[i], 8);
            a[i] += __shfl_xor_sync(0xFFFFFFFFu, a[i], 16);
          }
          if (r0 == j) { mine0 = a[0]; mine1 = a[1]; }
        }
        if (writes) {
          const int page = checked_page(b, entry);
          if (page < b.n_pages) {
            float* dst = p.w + ((static_cast<long long>(page) * p.n_kv + head) << b.page_shift) + (key & ((1 << b.page_shift) - 1));
            atomicAdd(dst, mine0);
            if (key + 1 < span.kv) atomicAdd(dst + 1, mine1);
          }
        }
      }
      more = w.next(b, ts, tail->plan);
    }
  }
  __syncthreads();
  if (*abort_flag && threadIdx.x == 0) {                 // given up: no load may outlive the CTA
    int no_flag = 0;
    for (int i = max(0, tail->issued - kStages); i < tail->issued; ++i)
      mbar_wait(smem_u32(&tail->full[i % kStages]), (i / kStages) & 1, &no_flag, b.status, kDevWaitKFull);
  }
}

constexpr size_t kSmem = kStages * kStageBytes + sizeof(Tail);

}  // namespace

cudaError_t init_paged_weight_rows() {
  const cudaError_t e = cudaFuncSetAttribute(paged_weight_rows_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kSmem));
  if (e != cudaSuccess) return e;
  return cudaFuncSetAttribute(paged_weight_rows_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kSmem));
}

cudaError_t launch_paged_weight_rows(const CUtensorMap& map_k, const PagedWeightParams& p, bool f16, int n_sm, cudaStream_t st) {
  auto k = f16 ? paged_weight_rows_kernel<true> : paged_weight_rows_kernel<false>;
  const TileShape ts = {p.n_kv, 16 / p.group, 7, 0};
  return launch_after_previous(k, 2 * n_sm, kThreads, kSmem, st, map_k, p, ts);
}

}  // namespace ilre
