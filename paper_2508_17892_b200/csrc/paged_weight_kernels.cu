// Accumulated attention weight: w[t, g] += sum over the rows (token, head of g) that see t of 2^(s c2 - lse2).
//
// The contraction is turned round, S^T = K Q^T, so that a key is a lane of tensor memory: a thread owns one key and
// adds up its columns without exchanging anything.  An item of work is 256 keys of a head, its units the tiles of up
// to 64 query rows that see any of them (128 where one token has more than 64 heads); the units are cut into one equal
// share per SM (paged_batch.cuh).  Whole items add their sums to the pool; the pieces of a cut item go to a workspace and
// the last one to arrive adds them up in the order of the CTAs, so a call's result does not depend on who was last.
//
// What bounds it: the exponentials, one per logit, 16 per SM and cycle.  Everything else is arranged around keeping the
// special-function units fed: one warp loads (256 keys per item, a row tile per unit), two threads issue the MMAs, and
// four groups of four warps (the parity of the unit by the half of the keys) have two accumulators each, so that the next
// unit's logits are there when a group has summed up this one's.  256 x 64 logits then take 1225 cycles, 84 % of the
// units' rate; a fourth of them as polynomials on the FMA pipe made it slower.  A 4160-token prompt (32 / 8 heads): 99 us,
// 720 TFLOP/s.  (One unit at a time per group, 128 rows: 122 us; two groups that take 128 logits to registers: 129 us.)
//
// Nothing is rounded to fewer than 32 bits: logits, exponents, the approximate exponential (2 ulp) and sums.  Against 64 bits
// that prompt's weights are 4.4e-7 off (exp of torch in 32 bits 0.8e-7).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cstddef>

#include "launch.cuh"
#include "paged_plan.cuh"
#include "paged_weight_kernels.cuh"

namespace ilre {

namespace {

constexpr int kKeySlots = 2, kMaxRowSlots = 6, kAccs = 8;
constexpr int kTileBytes = 128 * 128 * 2, kHalf = kTileBytes / 2;
constexpr int kKeyBytes = 2 * kTileBytes;                // 256 keys
constexpr int kRowBytes = 2 * kTileBytes;                // the row ring
constexpr int kRingBytes = kKeySlots * kKeyBytes + kRowBytes;
constexpr int kGroups = 4;                               // of four warps: (unit parity, half of the keys)
constexpr int kIssuers = 2;                              // threads that issue MMAs, every other unit each
// What an item costs beside its units, in units: a 4160-token prompt takes 109, 103, 99, 101 us with 0, 3, 6, 9.
constexpr int kItemUnits = 6;
constexpr int kFirstSum = 1 + kIssuers;                  // warp 0 loads, then the issuers, the others sum
constexpr int kThreads = 32 * kFirstSum + kGroups * 128;

// A piece as the loading warp hands it to the others.  The ring is safe without a barrier of its own: a place is
// written again 16 pieces later, behind the wait for both threads' MMAs of the piece two before that, which waited for
// accumulators that every group has read, of pieces at least 9 behind the place's.
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
  uint64_t k_full[kKeySlots], k_empty[kKeySlots], q_full[kMaxRowSlots], q_empty[kMaxRowSlots], d_full[kAccs], d_empty[kAccs];
  uint64_t sums_full[2], sums_empty[2];                  // the odd units' sums of a half, in `lse`: written, read
  PlanStart plan;
  Job job[kJobs];
  int published;                                         // pieces handed over so far
  alignas(16) float lse[kGroups * 4][2][128];            // [warp][parity][row], log2 units; then the group's sums [key]
  uint32_t tmem_base;
  int abort_flag;
  int k_issued, q_issued;
  int last[kGroups];
};
static_assert(offsetof(WeightTail, lse) % 16 == 0, "read four at a time");
constexpr size_t kSmem = static_cast<size_t>(kRingBytes) + sizeof(WeightTail);
static_assert(kSmem <= 232448, "shared memory");

// Barrier of a group that also agrees on going on: when a bounded wait was given up in one of its warps, all of them
// learn it here and leave together.
__device__ __forceinline__ bool agree(int group, bool ok) {
  uint32_t all;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %2, 0;\n\tbar.red.and.pred q, %1, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
               : "=r"(all) : "r"(1 + group), "r"(ok ? 1u : 0u) : "memory");
  return all != 0;
}

// This thread's sum over 32 columns of its key.
__device__ __forceinline__ float2 column_sum(float2 sum, const float (&v)[32], const float* lse2, float c2) {
#pragma unroll
  for (int j = 0; j < 32; j += 4) {
    const float4 n = *reinterpret_cast<const float4*>(lse2 + j);
    const float2 a = ffma2(make_float2(v[j], v[j + 1]), make_float2(c2, c2), make_float2(-n.x, -n.y));
    const float2 b = ffma2(make_float2(v[j + 2], v[j + 3]), make_float2(c2, c2), make_float2(-n.z, -n.w));
    sum = fadd2(sum, fadd2(make_float2(ex2_approx(a.x), ex2_approx(a.y)), make_float2(ex2_approx(b.x), ex2_approx(b.y))));
  }
  return sum;
}

template <bool kF16, int kCols>
__global__ void __launch_bounds__(kThreads, 1)
paged_weights_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                     const __grid_constant__ PagedWeightParams p, const TileShape ts) {
  extern __shared__ __align__(1024) uint8_t smem[];
  constexpr int n_cols = kCols;
  constexpr uint32_t q_half = n_cols * 128, q_bytes = 2 * q_half;
  // even: an issuing thread asks for every other place and so sees all of its phases
  constexpr int row_slots = kRowBytes / q_bytes < kMaxRowSlots ? kRowBytes / q_bytes : kMaxRowSlots, key_slots = kKeySlots;
  static_assert(row_slots % 2 == 0, "row ring");
  // accumulators of a group: with two the next unit's logits are computed while it sums up this one's
  constexpr int bufs = kCols == 128 ? 1 : 2, per_lane = kCols / 32;
  const uint32_t k_s = smem_u32(smem), q_s = k_s + key_slots * kKeyBytes;
  WeightTail* tail = reinterpret_cast<WeightTail*>(smem + kRingBytes);
  volatile int* abort_flag = &tail->abort_flag;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const PagedBatch& b = p.batch;
  const int tile_rows = ts.tq * p.group;                 // rows that a load brings, <= n_cols

  if (threadIdx.x == 0) {
    tail->abort_flag = 0;
    tail->k_issued = tail->q_issued = tail->published = 0;
    for (int s = 0; s < key_slots; ++s) { mbar_init(smem_u32(&tail->k_full[s]), 1); mbar_init(smem_u32(&tail->k_empty[s]), kIssuers); }
    for (int s = 0; s < row_slots; ++s) { mbar_init(smem_u32(&tail->q_full[s]), 1); mbar_init(smem_u32(&tail->q_empty[s]), 1); }
    for (int s = 0; s < kAccs; ++s) { mbar_init(smem_u32(&tail->d_full[s]), 1); mbar_init(smem_u32(&tail->d_empty[s]), 4); }
    for (int h = 0; h < 2; ++h) { mbar_init(smem_u32(&tail->sums_full[h]), 4); mbar_init(smem_u32(&tail->sums_empty[h]), 4); }
    fence_mbar_init();
    tma_prefetch_desc(&map_q);
    tma_prefetch_desc(&map_k);
  }
  // rows that no load brings: zeros, for good
  for (int i = threadIdx.x; i < row_slots * 2 * (n_cols - tile_rows) * 8; i += kThreads) {
    const int part = i & 7, row = tile_rows + (i >> 3) % (n_cols - tile_rows), half = (i >> 3) / (n_cols - tile_rows);
    *reinterpret_cast<uint4*>(smem + key_slots * kKeyBytes + half * q_half + row * 128 + part * 16) = make_uint4(0, 0, 0, 0);
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
    const int box_rows = min(ps, 128), n_box = 256 / box_rows;
    const int half = lane & 1, bx = lane >> 1;
    const bool active = bx < n_box;
    const int box_row = bx * box_rows;                   // of the 256
    const uint32_t off = (box_row >> 7) * kTileBytes + half * kHalf + (box_row & 127) * 128;
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
    auto needs = [&](int kt, const Piece& pc) { return active && kt * 256 + box_row < pc.span.kv; };
    int e_next = 0, next_kt = -1, next_seq = -1;
    while (more && ok) {
      const Piece& pc = w.p;
      int entry = 0;
      if (needs(pc.qt, pc)) entry = (next_kt == pc.qt && next_seq == pc.seq) ? e_next : table_entry(b, pc.seq, pc.qt * 256 + box_row);
      next_kt = pc.qt + 1; next_seq = pc.seq;
      e_next = needs(next_kt, pc) ? table_entry(b, pc.seq, next_kt * 256 + box_row) : 0;
      ok = warp_wait(&tail->k_empty[kp.slot], kp.phase ^ 1u, abort_flag, b.status, kDevWaitKEmpty);
      if (!ok) break;
      const int r_first = KeyTiles{pc.span.n, pc.span.kv, ts.tq, ts.tk_shift, ts.extra}.first(pc.qt) + pc.t0;
      const bool cut = pc.t0 > 0 || pc.t1 < pc.n_tiles;
      publish(Job{pc.qt, r_first, pc.t1 - pc.t0, (cut ? kCut : 0) | (pc.item == plan.first.begin ? kOfFirst : 0), pc.span.q0,
                  pc.span.n, pc.span.kv, pc.head + p.n_kv * pc.seq});
      const int page = needs(pc.qt, pc) ? checked_page(b, entry) : b.n_pages;
      uint32_t bar = smem_u32(&tail->k_full[kp.slot]);
      if (lane == 0) { mbar_arrive_expect_tx(bar, kKeyBytes); tail->k_issued = n_key + 1; }
      __syncwarp();
      if (active)
        tma_load_4d(k_s + kp.slot * kKeyBytes + off, &map_k, half * 64, pc.head, (pc.qt * 256 + box_row) & (ps - 1), page, bar);
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
  } else if (warp < kFirstSum) {
    {
      constexpr uint32_t idesc = kF16 ? umma_idesc_f16(128, n_cols) : umma_idesc_bf16(128, n_cols);
      // An issuing thread is held until the tensor pipe takes its instructions, and its waits and commits leave the
      // pipe idle (128 keys by 128 rows take it some 500 cycles, one thread 1340): two of them take turns.
      const int parity = warp - 1;                       // of its units, and the accumulators 2 parity, 2 parity + 1
      RingPos kp, qp;
      RingPos dp;
      int n_row = 0;
      Job job;
      for (int n_key = 0; ok && (ok = take_job(n_key, &job)) && job.count; ++n_key) {
        if (lane == 0) {
          ok = mbar_wait(smem_u32(&tail->k_full[kp.slot]), kp.phase, abort_flag, b.status, kDevWaitKFull);
          for (int t = 0; t < job.count && ok; ++t, ++n_row, qp.step(row_slots)) {
            if ((n_row & 1) != parity) continue;
            ok = mbar_wait(smem_u32(&tail->q_full[qp.slot]), qp.phase, abort_flag, b.status, kDevWaitQFull);
#pragma unroll
            for (int h = 0; h < 2 && ok; ++h) {
              const int acc = (2 * parity + h) * bufs + dp.slot;
              ok = mbar_wait(smem_u32(&tail->d_empty[acc]), dp.phase ^ 1u, abort_flag, b.status, kDevWaitAccEmpty);
              if (!ok) break;
              tc_fence_after();
#pragma unroll
              for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int st = 0; st < 4; ++st)
                  umma_bf16(tmem_base + acc * kCols,
                            umma_desc_sw128(k_s + kp.slot * kKeyBytes + h * kTileBytes + kb * kHalf + st * 32),
                            umma_desc_sw128(q_s + qp.slot * q_bytes + kb * q_half + st * 32), idesc, (kb | st) != 0);
              umma_commit(smem_u32(&tail->d_full[acc]));
            }
            if (ok) umma_commit(smem_u32(&tail->q_empty[qp.slot]));
            dp.step(bufs);
          }
          if (ok) umma_commit(smem_u32(&tail->k_empty[kp.slot]));
        }
        kp.step(key_slots);
        ok = __all_sync(0xFFFFFFFFu, ok);
      }
    }
  } else {
    const int group = (warp - kFirstSum) >> 2, quad = warp & 3, half = group & 1, parity = group >> 1;
    const int key_lane = quad * 32 + lane;               // this thread's key of the half
    const int gi = threadIdx.x - 32 * kFirstSum - group * 128;       // its number in the group
    int row_tok[per_lane], row_off[per_lane];            // the rows whose lse this lane fetches for its warp
#pragma unroll
    for (int i = 0; i < per_lane; ++i) {
      const int row = lane + 32 * i, tok = row / p.group;
      row_off[i] = tok * p.n_q + row - tok * p.group;
      row_tok[i] = row < tile_rows ? tok : 1 << 30;
    }
    float (&my_lse)[2][128] = tail->lse[warp - kFirstSum];
    int n_mine = 0;                                      // units of this warp so far
    RingPos dp;
    const uint32_t lane_base = tmem_base + (static_cast<uint32_t>(quad * 32) << 16);
    int n_row = 0;                                       // units before this piece
    Job job;
    uint32_t n_joined = 0;                               // pieces whose sums the groups have put together
    for (int n_piece = 0;; n_row += job.count, ++n_piece) {
      ok = agree(group, ok && take_job(n_piece, &job));
      if (!ok || job.count == 0) break;
      const int n = job.count, pre = job.kv - job.n;
      int u = (parity - n_row) & 1;                      // the piece's units of this group's parity
      if (n == 1 && u > 0) continue;
      const int seq = job.place / p.n_kv, head = job.place - seq * p.n_kv;
      const int key = job.kt * 256 + half * 128 + key_lane;
      int entry = 0;
      if (key < job.kv) entry = table_entry(b, seq, key);
      // lse of the lane's rows of the piece's unit t (-inf where there is no row); left alone until the next unit, which
      // does not wait for it then
      float lse_next[per_lane];
      auto row_lse = [&](int t) {
        const int tok0 = (job.row_tile + t) * ts.tq, left = job.n - tok0;
        const float* at = p.lse + (static_cast<long long>(job.q0) + tok0) * p.n_q + head * p.group;
#pragma unroll
        for (int i = 0; i < per_lane; ++i) lse_next[i] = row_tok[i] < left ? at[row_off[i]] : -INFINITY;
      };
      // in log2 units, +inf where there is no row or it sees nothing: its probabilities come out as 0
      auto log2_units = [](float v) { return v == -INFINITY ? INFINITY : v * 1.44269504f; };
      if (u < n) row_lse(u);
      float2 sum2 = make_float2(0.f, 0.f);
      for (; u < n && ok; u += 2, ++n_mine, dp.step(bufs)) {
        float* lse2 = my_lse[n_mine & 1];
#pragma unroll
        for (int i = 0; i < per_lane; ++i) lse2[lane + 32 * i] = log2_units(lse_next[i]);
        if (u + 2 < n) row_lse(u + 2);
        __syncwarp();
        const int acc = group * bufs + dp.slot;
        ok = warp_wait(&tail->d_full[acc], dp.phase, abort_flag, b.status, kDevWaitAccFull);
        if (!ok) break;                                  // (the next barrier tells the others)
        tc_fence_after();
        // column c is row (token c / group, head c % group) of the tile: seen from column lo on, rows up to hi
        const int tok0 = (job.row_tile + u) * ts.tq;
        const int hi = min(ts.tq, job.n - tok0) * p.group;
        // (clamped first: 32 heads times the distance of a row 67 million back would pass 32 bits.  Above, the distance
        // stays below a key tile and a row tile, since the unit sees some of the keys)
        const int lo = max(key - pre - tok0, 0) * p.group;
        const bool masked = hi < tile_rows || job.kt * 256 + half * 128 + 127 > pre + tok0;
        const uint32_t d = lane_base + acc * kCols;
        // (not unrolled: the code stays in the instruction cache, the other groups cover the waits)
#pragma unroll 1
        for (int c = 0; c < kCols; c += 32) {
          float v[32];
          tmem_ld32(d + c, v);
          tmem_ld_wait();
          if (c == kCols - 32) {                         // the accumulator is free for the group's next unit
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&tail->d_empty[acc]));
          }
          if (masked) {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = (c + j >= lo && c + j < hi) ? v[j] : -INFINITY;
          }
          sum2 = column_sum(sum2, v, lse2 + c, p.c2);
        }
      }
      float sum = sum2.x + sum2.y;
      // ---- one sum per key: the even and the odd units', then to the pool, or to the workspace where the item is cut
      const bool whole = !(job.flags & kCut);
      int owner = half;
      if (n == 1) {
        owner = group;
      } else {
        ok = agree(group, ok);
        if (!ok) break;
        if (parity == 1) {
          tail->lse[4 * group][0][key_lane] = sum;
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&tail->sums_full[half]));
          ok = warp_wait(&tail->sums_empty[half], n_joined & 1u, abort_flag, b.status, kDevWaitAccEmpty);
        } else {
          ok = warp_wait(&tail->sums_full[half], n_joined & 1u, abort_flag, b.status, kDevWaitAccFull);
          sum += tail->lse[4 * (group + 2)][0][key_lane];
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&tail->sums_empty[half]));
        }
        ++n_joined;
      }
      if (group == owner) {
        bool write = whole;
        if (!whole) {
          const Item& x = (job.flags & kOfFirst) ? plan.first : plan.last;
          const int c0 = share_of(plan.total, plan.n_cta, x.tiles_at(ts)), c1 = share_of(plan.total, plan.n_cta, x.end(ts) - 1);
          p.part[((blockIdx.x * 2 + (blockIdx.x == c0)) * 2 + half) * 128 + key_lane] = sum;
          ok = agree(group, ok);
          if (!ok) break;
          if (gi == 0) tail->last[group] = arrive_last(p.arrived + 2 * c0 + half, c1 - c0 + 1);
          ok = agree(group, ok);
          if (!ok) break;
          write = tail->last[group] != 0;
          if (write) {
            sum = 0.f;
            for (int c = c0; c <= c1; ++c) sum += __ldcg(p.part + ((c * 2 + (c == c0)) * 2 + half) * 128 + key_lane);
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
  const int most = group <= 64 ? 64 / group : 1;
  return max_q_len < most ? (max_q_len < 1 ? 1 : max_q_len) : most;
}

typedef void (*WeightKernel)(CUtensorMap, CUtensorMap, PagedWeightParams, TileShape);
static WeightKernel weight_kernel(bool f16, int n_cols) {
  if (f16) return n_cols == 32 ? paged_weights_kernel<true, 32> : n_cols == 64 ? paged_weights_kernel<true, 64> : paged_weights_kernel<true, 128>;
  return n_cols == 32 ? paged_weights_kernel<false, 32> : n_cols == 64 ? paged_weights_kernel<false, 64> : paged_weights_kernel<false, 128>;
}

cudaError_t init_paged_weights() {
  for (int f16 = 0; f16 < 2; ++f16)
    for (int n_cols = 32; n_cols <= 128; n_cols *= 2) {
      const cudaError_t e = cudaFuncSetAttribute(weight_kernel(f16 != 0, n_cols), cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                 static_cast<int>(kSmem));
      if (e != cudaSuccess) return e;
    }
  return cudaSuccess;
}

cudaError_t launch_paged_weights(const CUtensorMap& map_q, const CUtensorMap& map_k, const PagedWeightParams& p, bool f16,
                                 int n_sm, cudaStream_t st) {
  const TileShape ts = {p.n_kv, weight_tile_tokens(p.group, p.batch.max_q_len), 8, kItemUnits};
  const int rows = ts.tq * p.group, n_cols = rows <= 32 ? 32 : rows <= 64 ? 64 : 128;
  return launch_after_previous(weight_kernel(f16, n_cols), n_sm, kThreads, kSmem, st, map_q, map_k, p, ts);
}

}  // namespace ilre
