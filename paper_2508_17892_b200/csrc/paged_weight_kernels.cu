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

#include <cstddef>

#include "launch.cuh"
#include "paged_plan.cuh"
#include "paged_weight_kernels.cuh"

namespace ilre {

namespace {

constexpr int kMaxKeySlots = 6, kMaxRowSlots = 6, kAccs = 4, kTiles = 7;         // kTiles x 32 KB for both rings
constexpr int kTileBytes = 128 * 128 * 2, kHalf = kTileBytes / 2;
constexpr int kGroups = 4;                               // of four warps, one per accumulator
constexpr int kThreads = 64 + kGroups * 128;             // warp 0 loads, 1 MMAs, the others sum
constexpr int kPolyPairs = 4;                            // of 16 pairs of exponentials, those on the FMA pipe

// A piece as the loading warp hands it to the others.  The ring is safe without a barrier of its own: a place is
// written again 16 pieces later, behind the wait for the MMAs of a piece at most 6 before, which waited for accumulators that
// every group has read, of pieces at least 3 behind the place's.
struct Job {
  int kt, row_tile, count, flags;          // key tile, first row tile, units (0: the end); kCut, kOfFirst
  int q0, n, kv, place;                    // span; head + n_kv * sequence
};
constexpr int kJobs = 16, kCut = 1, kOfFirst = 2;

// A place in a ring, and the parity of the phase that completes it; no division on the way round.
struct RingPos {
  int slot = 0;
  uint32_t phase = 0;
  __device__ __forceinline__ void step(int slots) {
    if (++slot == slots) { slot = 0; phase ^= 1u; }
  }
};

struct WeightTail {
  uint64_t k_full[kMaxKeySlots], k_empty[kMaxKeySlots], q_full[kMaxRowSlots], q_empty[kMaxRowSlots], d_full[kAccs], d_empty[kAccs];
  uint64_t sums_full, sums_empty;                        // the groups' sums in `lse`: written, read
  PlanStart plan;
  Job job[kJobs];
  int published;                                         // pieces handed over so far
  alignas(16) float lse[kGroups][128];                               // [group][row], log2 units; then the group's sums [key]
  uint32_t tmem_base;
  int abort_flag;
  int k_issued, q_issued;
  int last[kGroups];
};
static_assert(offsetof(WeightTail, lse) % 16 == 0, "read four at a time");
constexpr size_t kSmem = static_cast<size_t>(kTiles) * kTileBytes + sizeof(WeightTail);
static_assert(kSmem <= 232448, "shared memory");

// Barrier of a group that also agrees on going on: when a bounded wait was given up in one of its warps, all of them
// learn it here and leave together.
__device__ __forceinline__ bool agree(int group, bool ok) {
  uint32_t all;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %2, 0;\n\tbar.red.and.pred q, %1, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
               : "=r"(all) : "r"(1 + group), "r"(ok ? 1u : 0u) : "memory");
  return all != 0;
}

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

// Columns of an accumulator (query rows of a tile, 16, 32, 64 or 128) and the slots of the two rings.  Few rows: the
// room goes to the keys, since what is in flight bounds the rate (32 KB per key tile, a step of eight requests behind
// 20000-32768 rows: RINGS_US).
struct WeightRings {
  int n_cols, key_slots, row_slots;
};

template <bool kF16>
__global__ void __launch_bounds__(kThreads, 1)
paged_weights_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                     const __grid_constant__ PagedWeightParams p, const TileShape ts, const WeightRings rings) {
  extern __shared__ __align__(1024) uint8_t smem[];
  const int n_cols = rings.n_cols, key_slots = rings.key_slots, row_slots = rings.row_slots;
  const uint32_t q_half = n_cols * 128, q_bytes = 2 * q_half;
  const uint32_t k_s = smem_u32(smem), q_s = k_s + key_slots * kTileBytes;
  WeightTail* tail = reinterpret_cast<WeightTail*>(smem + kTiles * kTileBytes);
  volatile int* abort_flag = &tail->abort_flag;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const PagedBatch& b = p.batch;
  const int tile_rows = ts.tq * p.group;                 // rows that a load brings, <= n_cols

  if (threadIdx.x == 0) {
    tail->abort_flag = 0;
    tail->k_issued = tail->q_issued = tail->published = 0;
    for (int s = 0; s < key_slots; ++s) { mbar_init(smem_u32(&tail->k_full[s]), 1); mbar_init(smem_u32(&tail->k_empty[s]), 1); }
    for (int s = 0; s < row_slots; ++s) { mbar_init(smem_u32(&tail->q_full[s]), 1); mbar_init(smem_u32(&tail->q_empty[s]), 1); }
    for (int s = 0; s < kAccs; ++s) { mbar_init(smem_u32(&tail->d_full[s]), 1); mbar_init(smem_u32(&tail->d_empty[s]), 4); }
    mbar_init(smem_u32(&tail->sums_full), 4 * (kGroups - 1));
    mbar_init(smem_u32(&tail->sums_empty), 4);
    fence_mbar_init();
  }
  // rows that no load brings: zeros, for good
  for (int i = threadIdx.x; i < row_slots * 2 * (n_cols - tile_rows) * 8; i += kThreads) {
    const int part = i & 7, row = tile_rows + (i >> 3) % (n_cols - tile_rows), half = (i >> 3) / (n_cols - tile_rows);
    *reinterpret_cast<uint4*>(smem + key_slots * kTileBytes + half * q_half + row * 128 + part * 16) = make_uint4(0, 0, 0, 0);
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
  bool ok = run;
  // job i: a whole warp; false when the wait was given up
  auto take_job = [&](int i, Job* job) -> bool {
    if (!warp_wait_count(&tail->published, i + 1, abort_flag, b.status, kDevWaitKFull)) return false;
    __threadfence_block();
    *job = tail->job[i % kJobs];
    return true;
  };

  if (warp == 0) {
    const int ps = 1 << b.page_shift;
    const int box_rows = min(ps, 128), n_box = 128 / box_rows;
    const int half = lane & 1, bx = lane >> 1;
    const bool active = bx < n_box;
    const uint32_t off = half * kHalf + bx * box_rows * 128;
    PieceWalk<KeyTiles> w;
    bool more = ok && w.begin(b, ts, plan);
    int n_key = 0, n_row = 0;
    RingPos kp, qp;
    auto publish = [&](const Job& job) {
      if (lane == 0) {
        tail->job[n_key % kJobs] = job;
        __threadfence_block();
        *reinterpret_cast<volatile int*>(&tail->published) = n_key + 1;
      }
      __syncwarp();
    };
    // the entry of the next piece's keys is asked for a piece ahead (where the piece is the next key tile of the head)
    auto needs = [&](int kt, const Piece& pc) { return active && kt * 128 + bx * box_rows < pc.span.kv; };
    int e_next = 0, next_kt = -1, next_seq = -1;
    while (more && ok) {
      const Piece& pc = w.p;
      int entry = 0;
      if (needs(pc.qt, pc)) entry = (next_kt == pc.qt && next_seq == pc.seq) ? e_next : table_entry(b, pc.seq, pc.qt * 128 + bx * box_rows);
      next_kt = pc.qt + 1; next_seq = pc.seq;
      e_next = needs(next_kt, pc) ? table_entry(b, pc.seq, next_kt * 128 + bx * box_rows) : 0;
      ok = warp_wait(&tail->k_empty[kp.slot], kp.phase ^ 1u, abort_flag, b.status, kDevWaitKEmpty);
      if (!ok) break;
      const int r_first = KeyTiles{pc.span.n, pc.span.kv, ts.tq, ts.tk_shift, 0}.first(pc.qt) + pc.t0;
      const bool cut = pc.t0 > 0 || pc.t1 < pc.n_tiles;
      publish(Job{pc.qt, r_first, pc.t1 - pc.t0, (cut ? kCut : 0) | (pc.item == plan.first.begin ? kOfFirst : 0), pc.span.q0,
                  pc.span.n, pc.span.kv, pc.head + p.n_kv * pc.seq});
      const int page = needs(pc.qt, pc) ? checked_page(b, entry) : b.n_pages;
      uint32_t bar = smem_u32(&tail->k_full[kp.slot]);
      if (lane == 0) { mbar_arrive_expect_tx(bar, kTileBytes); tail->k_issued = n_key + 1; }
      __syncwarp();
      if (active)
        tma_load_4d(k_s + kp.slot * kTileBytes + off, &map_k, half * 64, pc.head, (pc.qt * 128 + bx * box_rows) & (ps - 1), page, bar);
      ++n_key;
      kp.step(key_slots);
      for (int t = 0; t < pc.t1 - pc.t0; ++t, ++n_row, qp.step(row_slots)) {
        ok = warp_wait(&tail->q_empty[qp.slot], qp.phase ^ 1u, abort_flag, b.status, kDevWaitQFull);
        if (!ok) break;
        if (lane == 0) {
          bar = smem_u32(&tail->q_full[qp.slot]);
          mbar_arrive_expect_tx(bar, 2 * tile_rows * 128);
          tail->q_issued = n_row + 1;
          for (int h = 0; h < 2; ++h)
            tma_load_3d(q_s + qp.slot * q_bytes + h * q_half, &map_q, h * 64, pc.head * p.group, pc.span.q0 + (r_first + t) * ts.tq, bar);
        }
      }
      if (ok) more = w.next(b, ts, plan);
    }
    if (ok) {                                            // the end, behind the same wait as a piece
      ok = warp_wait(&tail->k_empty[kp.slot], kp.phase ^ 1u, abort_flag, b.status, kDevWaitKEmpty);
      if (ok) publish(Job{0, 0, 0, 0, 0, 0, 0, 0});
    }
  } else if (warp == 1) {
    {
      const uint32_t idesc = kF16 ? umma_idesc_bf16(128, n_cols) & ~((1u << 7) | (1u << 10)) : umma_idesc_bf16(128, n_cols);
      RingPos kp, qp, dp;
      Job job;
      for (int n_key = 0; ok && (ok = take_job(n_key, &job)) && job.count; ++n_key) {
        if (lane == 0) {
          ok = mbar_wait(smem_u32(&tail->k_full[kp.slot]), kp.phase, abort_flag, b.status, kDevWaitKFull);
          for (int t = 0; t < job.count && ok; ++t, qp.step(row_slots), dp.step(kAccs)) {
            ok = mbar_wait(smem_u32(&tail->d_empty[dp.slot]), dp.phase ^ 1u, abort_flag, b.status, kDevWaitAccEmpty) &&
                 mbar_wait(smem_u32(&tail->q_full[qp.slot]), qp.phase, abort_flag, b.status, kDevWaitQFull);
            if (!ok) break;
            tc_fence_after();
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
              for (int st = 0; st < 4; ++st)
                umma_bf16(tmem_base + dp.slot * 128, umma_desc_sw128(k_s + kp.slot * kTileBytes + kb * kHalf + st * 32),
                          umma_desc_sw128(q_s + qp.slot * q_bytes + kb * q_half + st * 32), idesc, (kb | st) != 0);
            umma_commit(smem_u32(&tail->d_full[dp.slot]));
            umma_commit(smem_u32(&tail->q_empty[qp.slot]));
          }
          if (ok) umma_commit(smem_u32(&tail->k_empty[kp.slot]));
        }
        kp.step(key_slots);
        ok = __all_sync(0xFFFFFFFFu, ok);
      }
    }
  } else {
    const int group = (warp - 2) >> 2, quad = warp & 3;
    const int key_lane = quad * 32 + lane;               // this thread's key of the tile
    const int gi = threadIdx.x - 64 - group * 128;       // its number in the group
    const int row_tok = gi / p.group, row_head = gi - row_tok * p.group;
    const uint32_t lane_base = tmem_base + (static_cast<uint32_t>(quad * 32) << 16);
    int n_row = 0;                                       // units before this piece
    Job job;
    uint32_t n_joined = 0;                               // pieces whose sums the groups have put together
    for (int n_piece = 0;; n_row += job.count, ++n_piece) {
      ok = agree(group, ok && take_job(n_piece, &job));
      if (!ok || job.count == 0) break;
      const int n = job.count, pre = job.kv - job.n;
      int u = (group - n_row) & (kGroups - 1);           // unit i is group i % kGroups'
      if (n == 1 && u > 0) continue;
      const int seq = job.place / p.n_kv, head = job.place - seq * p.n_kv;
      const int key = job.kt * 128 + key_lane;
      int entry = 0;
      if (key < job.kv) entry = table_entry(b, seq, key);
      // lse of this thread's row of tile t, in log2 units; +inf where there is no row or it sees nothing
      auto row_lse = [&](int t) -> float {
        const int tok = (job.row_tile + t) * ts.tq + row_tok;
        if (gi >= tile_rows || tok >= job.n) return INFINITY;
        const float v = p.lse[(static_cast<long long>(job.q0) + tok) * p.n_q + head * p.group + row_head];
        return v == -INFINITY ? INFINITY : v * 1.44269504f;
      };
      float lse_next = u < n ? row_lse(u) : 0.f;
      float2 sum2 = make_float2(0.f, 0.f);
      for (; u < n; u += kGroups) {
        float* lse2 = tail->lse[group];
        ok = agree(group, ok);                           // its last readers are done
        if (!ok) break;
        lse2[gi] = lse_next;
        if (u + kGroups < n) lse_next = row_lse(u + kGroups);
        ok = agree(group, ok);
        if (!ok) break;
        const int ds = (n_row + u) % kAccs;
        ok = warp_wait(&tail->d_full[ds], ((n_row + u) / kAccs) & 1, abort_flag, b.status, kDevWaitAccFull);
        if (!ok) continue;                               // (the next barrier tells the others)
        tc_fence_after();
        // column c is row (token c / group, head c % group) of the tile: seen from column lo on, rows up to hi
        const int tok0 = (job.row_tile + u) * ts.tq;
        const int hi = min(ts.tq, job.n - tok0) * p.group;
        const int lo = (key - pre - tok0) * p.group;
        const bool masked = hi < tile_rows || job.kt * 128 + 127 > pre + tok0;
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
      const bool whole = !(job.flags & kCut);
      int owner = 0;
      if (n == 1) {
        owner = group;
      } else {
        ok = agree(group, ok);
        if (!ok) break;
        if (group > 0) {
          tail->lse[group][key_lane] = sum;
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&tail->sums_full));
          ok = warp_wait(&tail->sums_empty, n_joined & 1u, abort_flag, b.status, kDevWaitAccEmpty);
        } else {
          ok = warp_wait(&tail->sums_full, n_joined & 1u, abort_flag, b.status, kDevWaitAccFull);
          for (int g = 1; g < kGroups; ++g) sum += tail->lse[g][key_lane];
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&tail->sums_empty));
        }
        ++n_joined;
      }
      if (group == owner) {
        bool write = whole;
        if (!whole) {
          const Item& x = (job.flags & kOfFirst) ? plan.first : plan.last;
          const int c0 = share_of(plan.total, plan.n_cta, x.begin), c1 = share_of(plan.total, plan.n_cta, x.begin + x.n_tiles - 1);
          p.part[(blockIdx.x * 2 + (blockIdx.x == c0)) * 128 + key_lane] = sum;
          ok = agree(group, ok);
          if (!ok) break;
          if (gi == 0) tail->last[group] = arrive_last(p.arrived + c0, c1 - c0 + 1);
          ok = agree(group, ok);
          if (!ok) break;
          write = tail->last[group] != 0;
          if (write) {
            sum = 0.f;
            for (int c = c0; c <= c1; ++c) sum += __ldcg(p.part + (c * 2 + (c == c0)) * 128 + key_lane);
          }
        }
        if (write && ok && key < job.kv) {
          const int page = checked_page(b, entry);
          if (page < b.n_pages)
            atomicAdd(p.w + ((static_cast<long long>(page) * p.n_kv + head) << b.page_shift) + (key & ((1 << b.page_shift) - 1)), sum);
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (*abort_flag && threadIdx.x == 0) {                 // given up: no load may outlive the CTA
    int no_flag = 0;
    for (int i = max(0, tail->k_issued - key_slots); i < tail->k_issued; ++i)
      mbar_wait(smem_u32(&tail->k_full[i % key_slots]), (i / key_slots) & 1, &no_flag, b.status, kDevWaitKFull);
    for (int i = max(0, tail->q_issued - row_slots); i < tail->q_issued; ++i)
      mbar_wait(smem_u32(&tail->q_full[i % row_slots]), (i / row_slots) & 1, &no_flag, b.status, kDevWaitQFull);
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

cudaError_t init_paged_weights() {
  const cudaError_t e = cudaFuncSetAttribute(paged_weights_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kSmem));
  if (e != cudaSuccess) return e;
  return cudaFuncSetAttribute(paged_weights_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kSmem));
}

cudaError_t launch_paged_weights(const CUtensorMap& map_q, const CUtensorMap& map_k, const PagedWeightParams& p, bool f16,
                                 int n_sm, cudaStream_t st) {
  auto k = f16 ? paged_weights_kernel<true> : paged_weights_kernel<false>;
  const TileShape ts = {p.n_kv, weight_tile_tokens(p.group, p.batch.max_q_len), 7, 0};
  const int rows = ts.tq * p.group;
  WeightRings r;
  r.n_cols = rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 ? 64 : 128;
  r.key_slots = r.n_cols == 16 ? kMaxKeySlots : r.n_cols == 32 ? 5 : 4;
  r.row_slots = (kTiles - r.key_slots) * kTileBytes / (r.n_cols * 256);
  if (r.row_slots > kMaxRowSlots) r.row_slots = kMaxRowSlots;
  return launch_after_previous(k, n_sm, kThreads, kSmem, st, map_q, map_k, p, ts, r);
}

}  // namespace ilre
