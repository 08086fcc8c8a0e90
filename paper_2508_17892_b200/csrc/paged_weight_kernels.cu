// Accumulated attention weight: w[t, g] += sum over the rows (token, head of g) that see t of 2^(s c2 - lse2).
//
// The contraction is turned round, S^T = K Q^T, so that a key is a lane of tensor memory: a thread owns one key and
// adds up its columns without exchanging anything.  A unit of work is 128 keys by up to 128 query rows; an item is a
// key tile, its units the row tiles that see it, and the items' units are cut into one equal share per SM
// (paged_batch.cuh).  Whole items add their sums to the pool; the pieces of a cut item go to a workspace and the last
// one to arrive adds them up in the order of the CTAs, so a call's result does not depend on who was last.
//
// What bounds it: with few rows (decoding) the reading of the keys, 256 bytes for 256 flop per row; with many the
// exponentials, one per logit, of which a quarter are polynomials on the FMA pipe.  One warp loads (a key tile per
// item, a row tile per unit), one thread issues the MMAs into four accumulators, sixteen warps in four groups have an
// accumulator each.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "launch.cuh"
#include "paged_plan.cuh"
#include "paged_weight_kernels.cuh"

namespace ilre {

namespace {

constexpr int kKeySlots = 4, kRowSlots = 3, kAccs = 4;
constexpr int kTileBytes = 128 * 128 * 2, kHalf = kTileBytes / 2;
constexpr int kGroups = 4;                               // of four warps, one per accumulator
constexpr int kThreads = 64 + kGroups * 128;             // warp 0 loads, 1 MMAs, the others sum
constexpr int kPolyPairs = 4;                            // of 16 pairs of exponentials, those on the FMA pipe

struct WeightTail {
  uint64_t k_full[kKeySlots], k_empty[kKeySlots], q_full[kRowSlots], q_empty[kRowSlots], d_full[kAccs], d_empty[kAccs];
  PlanStart plan;
  float lse[kGroups][128];                               // [group][row], log2 units; then the group's sums [key]
  uint32_t tmem_base;
  int abort_flag;
  int k_issued, q_issued;
  int last[kGroups];
};
constexpr size_t kSmem = static_cast<size_t>(kKeySlots + kRowSlots) * kTileBytes + sizeof(WeightTail);
static_assert(kSmem <= 232448, "shared memory");

__device__ __forceinline__ void sync_group(int group) { asm volatile("bar.sync %0, 128;" ::"r"(2 + group) : "memory"); }
__device__ __forceinline__ void sync_sums() { asm volatile("bar.sync 1, %0;" ::"n"(kGroups * 128) : "memory"); }

// This thread's sum over kCols columns (at most 32) of its key: all of them, or those in [lo, hi).
template <int kCols, bool kMasked>
__device__ __forceinline__ float2 column_sum(float2 sum, const float (&v)[kCols], const float* lse2, float c2, int lo, int hi) {
#pragma unroll
  for (int j = 0; j < kCols; j += 4) {
    const float4 n = *reinterpret_cast<const float4*>(lse2 + j);
    const float2 a = ffma2(make_float2(v[j], v[j + 1]), make_float2(c2, c2), make_float2(-n.x, -n.y));
    const float2 b = ffma2(make_float2(v[j + 2], v[j + 3]), make_float2(c2, c2), make_float2(-n.z, -n.w));
    auto poly = [](int pair) { return ((pair + 1) * kPolyPairs) / 16 > (pair * kPolyPairs) / 16; };
    float2 ea = poly((j >> 1) & 15) ? exp2_poly2(a) : make_float2(ex2_approx(a.x), ex2_approx(a.y));
    float2 eb = poly(((j >> 1) + 1) & 15) ? exp2_poly2(b) : make_float2(ex2_approx(b.x), ex2_approx(b.y));
    if (kMasked) {
      ea.x = (j >= lo && j < hi) ? ea.x : 0.f;
      ea.y = (j + 1 >= lo && j + 1 < hi) ? ea.y : 0.f;
      eb.x = (j + 2 >= lo && j + 2 < hi) ? eb.x : 0.f;
      eb.y = (j + 3 >= lo && j + 3 < hi) ? eb.y : 0.f;
    }
    sum = fadd2(sum, fadd2(ea, eb));
  }
  return sum;
}

template <bool kF16>
__global__ void __launch_bounds__(kThreads, 1)
paged_weights_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                     const __grid_constant__ PagedWeightParams p, const TileShape ts, const int n_cols) {
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t k_s = smem_u32(smem), q_s = k_s + kKeySlots * kTileBytes;
  WeightTail* tail = reinterpret_cast<WeightTail*>(smem + (kKeySlots + kRowSlots) * kTileBytes);
  volatile int* abort_flag = &tail->abort_flag;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const PagedBatch& b = p.batch;
  const int tile_rows = ts.tq * p.group;                 // rows that a load brings, <= n_cols

  if (threadIdx.x == 0) {
    tail->abort_flag = 0;
    tail->k_issued = tail->q_issued = 0;
    for (int s = 0; s < kKeySlots; ++s) { mbar_init(smem_u32(&tail->k_full[s]), 1); mbar_init(smem_u32(&tail->k_empty[s]), 1); }
    for (int s = 0; s < kRowSlots; ++s) { mbar_init(smem_u32(&tail->q_full[s]), 1); mbar_init(smem_u32(&tail->q_empty[s]), 1); }
    for (int s = 0; s < kAccs; ++s) { mbar_init(smem_u32(&tail->d_full[s]), 1); mbar_init(smem_u32(&tail->d_empty[s]), 4); }
    fence_mbar_init();
  }
  // rows that no load brings: zeros, for good
  for (int i = threadIdx.x; i < kRowSlots * 2 * (n_cols - tile_rows) * 8; i += kThreads) {
    const int part = i & 7, row = tile_rows + (i >> 3) % (n_cols - tile_rows), half = (i >> 3) / (n_cols - tile_rows);
    *reinterpret_cast<uint4*>(smem + kKeySlots * kTileBytes + half * kHalf + row * 128 + part * 16) = make_uint4(0, 0, 0, 0);
  }
  fence_proxy_async_smem();
  if (warp == 1) {
    tmem_alloc(smem_u32(&tail->tmem_base), 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = tail->tmem_base;
  grid_dep_wait();
  grid_dep_launch();
  if (threadIdx.x == 0 && (k_s & 1023u)) {
    tail->abort_flag = 1;
    report(b.status, kDevSmemAlign);
  }
  plan_start<KeyTiles>(b, ts, 1, reinterpret_cast<long long*>(&tail->lse), &tail->plan);
  __syncthreads();
  const PlanStart& plan = tail->plan;
  const bool run = *abort_flag == 0;
  PieceWalk<KeyTiles> w;
  bool more = run && w.begin(ts, plan), ok = more;
  auto first_tile = [&](const Piece& pc) { return KeyTiles{pc.span.n, pc.span.kv, ts.tq, ts.tk_shift}.first(pc.qt); };

  if (warp == 0) {
    const int ps = 1 << b.page_shift;
    const int box_rows = min(ps, 128), n_box = 128 / box_rows;
    const int half = lane & 1, bx = lane >> 1;
    const bool active = bx < n_box;
    const uint32_t off = half * kHalf + bx * box_rows * 128;
    int n_key = 0, n_row = 0;
    // the entry of the next piece's keys is asked for a piece ahead (where the piece is the next key tile of the head)
    auto needs = [&](int kt, const Piece& pc) { return active && kt * 128 + bx * box_rows < pc.span.kv; };
    int e_next = 0, next_kt = -1, next_seq = -1;
    while (more && ok) {
      const Piece& pc = w.p;
      int entry = 0;
      if (needs(pc.qt, pc)) entry = (next_kt == pc.qt && next_seq == pc.seq) ? e_next : table_entry(b, pc.seq, pc.qt * 128 + bx * box_rows);
      next_kt = pc.qt + 1; next_seq = pc.seq;
      e_next = needs(next_kt, pc) ? table_entry(b, pc.seq, next_kt * 128 + bx * box_rows) : 0;
      int s = n_key % kKeySlots;
      ok = warp_wait(&tail->k_empty[s], ((n_key / kKeySlots) & 1) ^ 1, abort_flag, b.status, kDevWaitKEmpty);
      if (!ok) break;
      const int page = needs(pc.qt, pc) ? checked_page(b, entry) : b.n_pages;
      uint32_t bar = smem_u32(&tail->k_full[s]);
      if (lane == 0) { mbar_arrive_expect_tx(bar, kTileBytes); tail->k_issued = n_key + 1; }
      __syncwarp();
      if (active)
        tma_load_4d(k_s + s * kTileBytes + off, &map_k, half * 64, pc.head, (pc.qt * 128 + bx * box_rows) & (ps - 1), page, bar);
      ++n_key;
      const int r_first = first_tile(pc);
      for (int t = pc.t0; t < pc.t1; ++t, ++n_row) {
        s = n_row % kRowSlots;
        ok = warp_wait(&tail->q_empty[s], ((n_row / kRowSlots) & 1) ^ 1, abort_flag, b.status, kDevWaitQFull);
        if (!ok) break;
        if (lane == 0) {
          bar = smem_u32(&tail->q_full[s]);
          mbar_arrive_expect_tx(bar, 2 * tile_rows * 128);
          tail->q_issued = n_row + 1;
          for (int h = 0; h < 2; ++h)
            tma_load_3d(q_s + s * kTileBytes + h * kHalf, &map_q, h * 64, pc.head * p.group, pc.span.q0 + (r_first + t) * ts.tq, bar);
        }
      }
      if (ok) more = w.next(b, ts, plan);
    }
  } else if (warp == 1) {
    if (lane == 0) {
      const uint32_t idesc = kF16 ? umma_idesc_bf16(128, n_cols) & ~((1u << 7) | (1u << 10)) : umma_idesc_bf16(128, n_cols);
      int n_key = 0, n_row = 0;
      while (more && ok) {
        const int ks = n_key % kKeySlots;
        ok = mbar_wait(smem_u32(&tail->k_full[ks]), (n_key / kKeySlots) & 1, abort_flag, b.status, kDevWaitKFull);
        for (int t = w.p.t0; t < w.p.t1 && ok; ++t, ++n_row) {
          const int qs = n_row % kRowSlots, ds = n_row % kAccs;
          ok = mbar_wait(smem_u32(&tail->d_empty[ds]), ((n_row / kAccs) & 1) ^ 1, abort_flag, b.status, kDevWaitAccEmpty) &&
               mbar_wait(smem_u32(&tail->q_full[qs]), (n_row / kRowSlots) & 1, abort_flag, b.status, kDevWaitQFull);
          if (!ok) break;
          tc_fence_after();
#pragma unroll
          for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int st = 0; st < 4; ++st)
              umma_bf16(tmem_base + ds * 128, umma_desc_sw128(k_s + ks * kTileBytes + kb * kHalf + st * 32),
                        umma_desc_sw128(q_s + qs * kTileBytes + kb * kHalf + st * 32), idesc, (kb | st) != 0);
          umma_commit(smem_u32(&tail->d_full[ds]));
          umma_commit(smem_u32(&tail->q_empty[qs]));
        }
        if (!ok) break;
        umma_commit(smem_u32(&tail->k_empty[ks]));
        ++n_key;
        more = w.next(b, ts, plan);
      }
    }
  } else {
    const int group = (warp - 2) >> 2, quad = warp & 3;
    const int key_lane = quad * 32 + lane;               // this thread's key of the tile
    const int gi = threadIdx.x - 64 - group * 128;       // its number in the group
    const int row_tok = gi / p.group, row_head = gi - row_tok * p.group;
    const uint32_t lane_base = tmem_base + (static_cast<uint32_t>(quad * 32) << 16);
    int n_row = 0;                                       // units before this piece
    while (more) {
      const Piece& pc = w.p;
      const int n = pc.t1 - pc.t0, r_first = first_tile(pc), pre = pc.span.kv - pc.span.n;
      const int key = pc.qt * 128 + key_lane;
      int entry = 0;
      if (key < pc.span.kv) entry = table_entry(b, pc.seq, key);
      // lse of this thread's row of tile t, in log2 units; +inf where there is no row or it sees nothing
      auto row_lse = [&](int t) -> float {
        const int tok = (r_first + t) * ts.tq + row_tok;
        if (gi >= tile_rows || tok >= pc.span.n) return INFINITY;
        const float v = p.lse[(static_cast<long long>(pc.span.q0) + tok) * p.n_q + pc.head * p.group + row_head];
        return v == -INFINITY ? INFINITY : v * 1.44269504f;
      };
      int u = (group - n_row) & (kGroups - 1);           // unit i is group i % kGroups'
      float lse_next = u < n ? row_lse(pc.t0 + u) : 0.f;
      float2 sum2 = make_float2(0.f, 0.f);
      for (; u < n && ok; u += kGroups) {
        float* lse2 = tail->lse[group];
        sync_group(group);                               // its last readers are done
        lse2[gi] = lse_next;
        if (u + kGroups < n) lse_next = row_lse(pc.t0 + u + kGroups);
        sync_group(group);
        const int ds = (n_row + u) % kAccs;
        ok = warp_wait(&tail->d_full[ds], ((n_row + u) / kAccs) & 1, abort_flag, b.status, kDevWaitAccFull);
        if (!ok) break;
        tc_fence_after();
        // column c is row (token c / group, head c % group) of the tile: seen from column lo on, rows up to hi
        const int tok0 = (r_first + pc.t0 + u) * ts.tq;
        const int hi = min(ts.tq, pc.span.n - tok0) * p.group;
        const int lo = (key - pre - tok0) * p.group;
        const bool masked = hi < tile_rows || pc.qt * 128 + 127 > pre + tok0;
        const uint32_t d = lane_base + ds * 128;
        // (loops that are not unrolled: the code stays in the instruction cache, the other groups cover the waits)
        if (n_cols == 16) {
          float v[16];
          tmem_ld16(d, v);
          tmem_ld_wait();
          sum2 = masked ? column_sum<16, true>(sum2, v, lse2, p.c2, lo, hi) : column_sum<16, false>(sum2, v, lse2, p.c2, 0, 0);
        } else if (masked) {
#pragma unroll 1
          for (int c = 0; c < n_cols; c += 32) {
            float v[32];
            tmem_ld32(d + c, v);
            tmem_ld_wait();
            sum2 = column_sum<32, true>(sum2, v, lse2 + c, p.c2, lo - c, hi - c);
          }
        } else {
#pragma unroll 1
          for (int c = 0; c < n_cols; c += 32) {
            float v[32];
            tmem_ld32(d + c, v);
            tmem_ld_wait();
            sum2 = column_sum<32, false>(sum2, v, lse2 + c, p.c2, 0, 0);
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&tail->d_empty[ds]));
      }
      float sum = sum2.x + sum2.y;
      // ---- one sum per key: the groups' shares, then to the pool, or to the workspace where the item is cut
      const bool whole = pc.t0 == 0 && pc.t1 == pc.n_tiles;
      int owner = 0;
      if (n == 1) {
        owner = n_row & (kGroups - 1);
      } else {
        sync_group(group);
        tail->lse[group][key_lane] = sum;
        sync_sums();
        if (group == 0)
          for (int g = 1; g < kGroups; ++g) sum += tail->lse[g][key_lane];
        sync_sums();
      }
      if (group == owner) {
        bool write = whole;
        if (!whole) {
          const int c0 = share_of(plan.total, plan.n_cta, pc.item), c1 = share_of(plan.total, plan.n_cta, pc.item + pc.n_tiles - 1);
          p.part[(blockIdx.x * 2 + (pc.t0 > 0 ? 0 : 1)) * 128 + key_lane] = sum;
          __threadfence();
          sync_group(group);
          if (gi == 0) {                                 // wraps to 0 with the last arrival
            tail->last[group] = atomicInc(p.arrived + c0, c1 - c0) == static_cast<uint32_t>(c1 - c0);
            __threadfence();
          }
          sync_group(group);
          write = tail->last[group] != 0;
          if (write) {
            sum = 0.f;
            for (int c = c0; c <= c1; ++c) sum += __ldcg(p.part + (c * 2 + (c == c0)) * 128 + key_lane);
          }
        }
        if (write && ok && key < pc.span.kv) {
          const int page = checked_page(b, entry);
          if (page < b.n_pages)
            atomicAdd(p.w + ((static_cast<long long>(page) * p.n_kv + pc.head) << b.page_shift) + (key & ((1 << b.page_shift) - 1)), sum);
        }
      }
      n_row += n;
      more = w.next(b, ts, plan);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (*abort_flag && threadIdx.x == 0) {                 // given up: no load may outlive the CTA
    int no_flag = 0;
    for (int i = max(0, tail->k_issued - kKeySlots); i < tail->k_issued; ++i)
      mbar_wait(smem_u32(&tail->k_full[i % kKeySlots]), (i / kKeySlots) & 1, &no_flag, b.status, kDevWaitKFull);
    for (int i = max(0, tail->q_issued - kRowSlots); i < tail->q_issued; ++i)
      mbar_wait(smem_u32(&tail->q_full[i % kRowSlots]), (i / kRowSlots) & 1, &no_flag, b.status, kDevWaitQFull);
  }
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, 512);
  }
}

}  // namespace

int weight_tile_tokens(int group, int max_q_len) {
  const int most = 128 / group;
  return max_q_len < most ? (max_q_len < 1 ? 1 : max_q_len) : most;
}

cudaError_t launch_paged_weights(const CUtensorMap& map_q, const CUtensorMap& map_k, const PagedWeightParams& p, bool f16,
                                 int n_sm, cudaStream_t st) {
  auto k = f16 ? paged_weights_kernel<true> : paged_weights_kernel<false>;
  const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kSmem));
  if (e != cudaSuccess) return e;
  const TileShape ts = {p.n_kv, weight_tile_tokens(p.group, p.batch.max_q_len), 7};
  const int rows = ts.tq * p.group, n_cols = rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 ? 64 : 128;
  return launch_after_previous(k, n_sm, kThreads, kSmem, st, map_q, map_k, p, ts, n_cols);
}

}  // namespace ilre
