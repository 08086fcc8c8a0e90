// Attention of few query rows over the paged cache (decoding: one new token of a group of up to 16 heads), single pass:
//   o = sum_t p_t v_t / sum_t p_t,  p_t = 2^((q.k_t) log2(e)/sqrt(d) - m),  m the running maximum.
//
// Bound by HBM: every key and value is read once for all heads of its group, 512 bytes for 4 x group x 128 flop.
// So the work is cut by keys (paged_batch.cuh: equal shares of 64-key tiles over two CTAs per SM, whatever the
// sequences' lengths), a warp of TMA loads keeps three 32 KB stages in flight per CTA, and the arithmetic only has to
// stay out of the way: 16 query rows are the M of mma.m16n8k16, each of four warps takes 16 keys of a stage
// and keeps its own maximum, sum and output in registers, so that nothing is exchanged until a piece ends.
// (A tcgen05 tile has 128 rows; with 4 to 16 of them used its detour through tensor memory and barriers between
// warps costs more than it saves.)  The pieces of an item that several CTAs share are joined by the last of them
// to arrive, in the order of the CTAs: the result does not depend on who was last.
#include "launch.cuh"
#include "paged_attn_kernels.cuh"
#include "paged_mma.cuh"
#include "paged_plan.cuh"

namespace ilre {

namespace {

constexpr int kStages = 3;
constexpr int kHalfBytes = kRowKeys * 128;               // 64 keys x 64 channels of 2 bytes
constexpr int kTileBytes = 2 * kHalfBytes;               // keys or values of a stage
constexpr int kStageBytes = 2 * kTileBytes;
constexpr int kWarps = 4;                                // consumers
constexpr int kThreads = 32 * (kWarps + 1);
constexpr int kMergeFloats = kRowTile * 128;             // output of one warp on its way to another
constexpr int kJoinFlight = 8;                           // partial results in flight
constexpr int kMinUnits = 3;                             // 64-key tiles that a CTA gets at least (4160 rows: 2 11.8 us, 3 11.2, 4 13.6; 32768 rows alike)

struct RowTail {
  uint64_t full[kStages];
  uint64_t empty[kStages];
  PlanStart plan;
  long long tmp[kPlanTmp];
  float2 ml[kWarps][kRowTile];
  int abort_flag;
  int last;
  int issued;                                            // stages whose loads have begun
};

__device__ __forceinline__ void sync_consumers() { asm volatile("bar.sync 1, %0;" ::"n"(32 * kWarps) : "memory"); }

template <bool kF16>
__global__ void __launch_bounds__(kThreads, kRowCtasPerSm)
paged_rows_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                  const __grid_constant__ PagedAttnParams p, const TileShape ts) {
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t ring = smem_u32(smem);
  float* merge = reinterpret_cast<float*>(smem + kStages * kStageBytes);          // two warps' outputs
  RowTail* tail = reinterpret_cast<RowTail*>(smem + kStages * kStageBytes + 2 * kMergeFloats * 4);
  volatile int* abort_flag = &tail->abort_flag;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const PagedBatch& b = p.batch;
  constexpr float kShift = kF16 ? kRowShift : 0.f;

  if (threadIdx.x == 0) {
    tail->abort_flag = tail->issued = 0;
    for (int s = 0; s < kStages; ++s) {
      mbar_init(smem_u32(&tail->full[s]), 1);
      mbar_init(smem_u32(&tail->empty[s]), kWarps);
    }
    fence_mbar_init();
    tma_prefetch_desc(&map_k);
    tma_prefetch_desc(&map_v);
  }
  __syncthreads();
  grid_dep_wait();
  grid_dep_launch();
  if (threadIdx.x == 0 && (ring & 1023u)) {
    tail->abort_flag = 1;
    report(b.status, kDevSmemAlign);
  }
  plan_start<HeadTiles>(b, ts, kMinUnits, tail->tmp, &tail->plan);
  __syncthreads();
  const PlanStart& plan = tail->plan;
  PieceWalk<HeadTiles> w;
  if (!w.begin(b, ts, plan)) return;
  bool ok = *abort_flag == 0;

  if (warp == kWarps) {
    // ---- loads: one lane per box, a box is 64 channels of the rows that one page has in the tile
    const int ps = 1 << b.page_shift;
    const int box_rows = min(ps, kRowKeys), n_box = kRowKeys / box_rows;
    const int half = lane & 1, is_v = (lane >> 1) & 1, bx = lane >> 2;            // lanes 4 n_box and up rest
    const bool active = bx < n_box;
    const uint32_t off = is_v * kTileBytes + half * kHalfBytes + bx * box_rows * 128;
    int it = 0;
    bool more = true;
    // Entries two tiles ahead; rows at and behind kv need none: zeros, not read.
    auto needs = [&](int t) { return active && t < w.p.t1 && t * kRowKeys + bx * box_rows < w.p.span.kv; };
    auto entry_at = [&](int t) -> int { return needs(t) ? table_entry(b, w.p.seq, t * kRowKeys + bx * box_rows) : 0; };
    while (more && ok) {
      int e0 = entry_at(w.p.t0), e1 = entry_at(w.p.t0 + 1);
      for (int t = w.p.t0; t < w.p.t1; ++t, ++it) {
        const int s = it % kStages;
        const int row = t * kRowKeys + bx * box_rows, e2 = entry_at(t + 2);
        ok = warp_wait(&tail->empty[s], ((it / kStages) & 1) ^ 1, abort_flag, b.status, kDevWaitKEmpty);
        if (!ok) break;
        const int page = needs(t) ? checked_page(b, e0) : b.n_pages;
        const uint32_t bar = smem_u32(&tail->full[s]);
        if (lane == 0) {
          mbar_arrive_expect_tx(bar, kStageBytes);
          tail->issued = it + 1;
        }
        __syncwarp();
        if (active)
          tma_load_4d(ring + s * kStageBytes + off, is_v ? &map_v : &map_k, half * 64, w.p.head, row & (ps - 1), page, bar);
        e0 = e1;
        e1 = e2;
      }
      if (ok) more = w.next(b, ts, tail->plan);
    }
  } else {

    // ---- consumers: warp `warp` has keys 16 warp .. 16 warp + 15 of every stage
    const int r0 = lane >> 2, c0 = (lane & 3) * 2;         // this thread's rows r0, r0 + 8; columns c0, c0 + 1 (+ 8 j)
    const int mat = lane >> 3, mr = lane & 7;              // ldmatrix: matrix and row that this lane addresses
    int it = 0;
    do {
      const Piece& pc = w.p;
      const int h_first = pc.head * p.group;
      const int tok0 = pc.qt * ts.tq, n_row = min(ts.tq, pc.span.n - tok0) * p.group;
      const int pre = pc.span.kv - pc.span.n + tok0;       // token i of the tile sees rows up to pre + i
      // row r is token r / group of the tile, head r % group of the group
      auto row_valid = [&](int r) { return r < n_row; };
      auto row_tok = [&](int r) -> long long { return static_cast<long long>(pc.span.q0) + tok0 + r / p.group; };
      uint32_t qa[8][4];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int r = r0 + 8 * x;
        const bool valid = row_valid(r);
        const uint32_t* src = reinterpret_cast<const uint32_t*>(
            static_cast<const uint16_t*>(p.q) + (valid ? row_tok(r) * p.q_stride + (h_first + r % p.group) * 128 : 0));
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) {
          qa[ks][x] = valid ? src[ks * 8 + (c0 >> 1)] : 0u;
          qa[ks][2 + x] = valid ? src[ks * 8 + 4 + (c0 >> 1)] : 0u;
        }
      }
      const int lim0 = pre + r0 / p.group, lim1 = pre + (r0 + 8) / p.group;
      float o[16][4];
#pragma unroll
      for (int j = 0; j < 16; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f;
      float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;

      for (int t = pc.t0; t < pc.t1; ++t, ++it) {
        const int s = it % kStages;
        ok = ok && warp_wait(&tail->full[s], (it / kStages) & 1, abort_flag, b.status, kDevWaitKFull);
        if (!ok) continue;
        const uint32_t ks_base = ring + s * kStageBytes, vs_base = ks_base + kTileBytes;
        const int key0 = t * kRowKeys + warp * 16;
        if (key0 < pc.span.kv) {                           // else all of this warp's keys are behind the sequence
          float sc[2][4] = {};
          // S = Q K^T: matrices (keys 0-7 | 8-15) x (channels 0-7 | 8-15) of each 16-channel step
          const int krow = warp * 16 + (mat >> 1) * 8 + mr;
#pragma unroll
          for (int ks = 0; ks < 8; ++ks) {
            const int c16 = (ks & 3) * 2 + (mat & 1);
            uint32_t kb[4];
            ldsm4(ks_base + (ks >> 2) * kHalfBytes + krow * 128 + ((c16 ^ (krow & 7)) << 4), kb);
            mma16816<kF16>(sc[0], qa[ks], kb[0], kb[1]);
            mma16816<kF16>(sc[1], qa[ks], kb[2], kb[3]);
          }
          float x0[4] = {sc[0][0] * p.c2, sc[0][1] * p.c2, sc[1][0] * p.c2, sc[1][1] * p.c2};
          float x1[4] = {sc[0][2] * p.c2, sc[0][3] * p.c2, sc[1][2] * p.c2, sc[1][3] * p.c2};
          const bool edge = key0 + 15 > pre;               // some row does not see some of these keys
          if (edge) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int key = key0 + (i >> 1) * 8 + c0 + (i & 1);
              x0[i] = key <= lim0 ? x0[i] : -INFINITY;
              x1[i] = key <= lim1 ? x1[i] : -INFINITY;
            }
          }
          float a0 = fmaxf(fmax3(x0[0], x0[1], x0[2]), x0[3]), a1 = fmaxf(fmax3(x1[0], x1[1], x1[2]), x1[3]);
          a0 = fmaxf(a0, __shfl_xor_sync(0xFFFFFFFFu, a0, 1));
          a1 = fmaxf(a1, __shfl_xor_sync(0xFFFFFFFFu, a1, 1));
          a0 = fmaxf(a0, __shfl_xor_sync(0xFFFFFFFFu, a0, 2));
          a1 = fmaxf(a1, __shfl_xor_sync(0xFFFFFFFFu, a1, 2));
          const float n0 = fmaxf(m0, a0), n1 = fmaxf(m1, a1);
          const float z0 = n0 == -INFINITY ? 0.f : n0, z1 = n1 == -INFINITY ? 0.f : n1;
          if (__any_sync(0xFFFFFFFFu, n0 != m0 || n1 != m1)) {
            const float f0 = ex2_approx(m0 - z0), f1 = ex2_approx(m1 - z1);          // m = -inf: 0
            l0 *= f0; l1 *= f1;
#pragma unroll
            for (int j = 0; j < 16; ++j) { o[j][0] *= f0; o[j][1] *= f0; o[j][2] *= f1; o[j][3] *= f1; }
            m0 = n0; m1 = n1;
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {                    // (the shift behind the difference: it is 0 at most, exactly)
            x0[i] = ex2_approx(kF16 ? (x0[i] - z0) + kShift : x0[i] - z0);
            x1[i] = ex2_approx(kF16 ? (x1[i] - z1) + kShift : x1[i] - z1);
          }
          l0 += (x0[0] + x0[1]) + (x0[2] + x0[3]);
          l1 += (x1[0] + x1[1]) + (x1[2] + x1[3]);
          const uint32_t pa[4] = {pack2<kF16>(x0[0], x0[1]), pack2<kF16>(x1[0], x1[1]), pack2<kF16>(x0[2], x0[3]),
                                  pack2<kF16>(x1[2], x1[3])};
          // O += P V: matrices (keys 0-7 | 8-15) x (channels 0-7 | 8-15), transposed on the way in
          const int vrow = warp * 16 + (mat & 1) * 8 + mr;
          const int dead = key0 + 16 - pc.span.kv;         // keys behind the sequence: whatever they hold counts as 0
          uint32_t keep0 = ~0u, keep1 = ~0u;
          if (dead > 0) {
            keep0 = (key0 + c0 < pc.span.kv ? 0xFFFFu : 0u) | (key0 + c0 + 1 < pc.span.kv ? 0xFFFF0000u : 0u);
            keep1 = (key0 + 8 + c0 < pc.span.kv ? 0xFFFFu : 0u) | (key0 + 9 + c0 < pc.span.kv ? 0xFFFF0000u : 0u);
          }
#pragma unroll
          for (int j2 = 0; j2 < 8; ++j2) {
            const int c16 = (j2 & 3) * 2 + (mat >> 1);
            uint32_t vb[4];
            ldsm4_trans(vs_base + (j2 >> 2) * kHalfBytes + vrow * 128 + ((c16 ^ (vrow & 7)) << 4), vb);
            mma16816<kF16>(o[2 * j2], pa, vb[0] & keep0, vb[1] & keep1);
            mma16816<kF16>(o[2 * j2 + 1], pa, vb[2] & keep0, vb[3] & keep1);
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&tail->empty[s]));
      }
      l0 += __shfl_xor_sync(0xFFFFFFFFu, l0, 1); l1 += __shfl_xor_sync(0xFFFFFFFFu, l1, 1);
      l0 += __shfl_xor_sync(0xFFFFFFFFu, l0, 2); l1 += __shfl_xor_sync(0xFFFFFFFFu, l1, 2);

      // ---- the four warps' results into one: common maximum, then outputs scaled to it and added 2+3 -> 0+1 -> 0
      if ((lane & 3) == 0) { tail->ml[warp][r0] = make_float2(m0, l0); tail->ml[warp][r0 + 8] = make_float2(m1, l1); }
      sync_consumers();
      float M0 = -INFINITY, M1 = -INFINITY;
#pragma unroll
      for (int x = 0; x < kWarps; ++x) { M0 = fmaxf(M0, tail->ml[x][r0].x); M1 = fmaxf(M1, tail->ml[x][r0 + 8].x); }
      const float z0 = M0 == -INFINITY ? 0.f : M0, z1 = M1 == -INFINITY ? 0.f : M1;
      float L0 = 0.f, L1 = 0.f;
#pragma unroll
      for (int x = 0; x < kWarps; ++x) {
        L0 += tail->ml[x][r0].y * ex2_approx(tail->ml[x][r0].x - z0);
        L1 += tail->ml[x][r0 + 8].y * ex2_approx(tail->ml[x][r0 + 8].x - z1);
      }
      const float f0 = ex2_approx(m0 - z0), f1 = ex2_approx(m1 - z1);
#pragma unroll
      for (int j = 0; j < 16; ++j) { o[j][0] *= f0; o[j][1] *= f0; o[j][2] *= f1; o[j][3] *= f1; }
#pragma unroll
      for (int step = 2; step >= 1; step >>= 1) {
        if (warp >= step && warp < 2 * step) {
          float4* dst = reinterpret_cast<float4*>(merge + (warp - step) * kMergeFloats);
#pragma unroll
          for (int j = 0; j < 16; ++j) dst[j * 32 + lane] = make_float4(o[j][0], o[j][1], o[j][2], o[j][3]);
        }
        sync_consumers();
        if (warp < step) {
          const float4* src = reinterpret_cast<const float4*>(merge + warp * kMergeFloats);
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const float4 v = src[j * 32 + lane];
            o[j][0] += v.x; o[j][1] += v.y; o[j][2] += v.z; o[j][3] += v.w;
          }
        }
        sync_consumers();
      }
      const bool whole = pc.t0 == 0 && pc.t1 == pc.n_tiles;
      const int slot = blockIdx.x * 2 + (pc.t0 > 0 ? 0 : 1);   // an item that began before this share, or one that goes on
      if (warp == 0) {
        if (whole) {
          const float i0 = L0 > 0.f ? 1.f / L0 : (L0 == 0.f ? 0.f : L0), i1 = L1 > 0.f ? 1.f / L1 : (L1 == 0.f ? 0.f : L1);
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const int r = r0 + 8 * x;
            if (!row_valid(r) || !ok) continue;
            const long long at = row_tok(r) * p.n_q + h_first + r % p.group;
            uint32_t* dst = reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(p.out) + at * 128);
#pragma unroll
            for (int j = 0; j < 16; ++j)
              dst[j * 4 + (c0 >> 1)] = x ? pack2<kF16>(o[j][2] * i1, o[j][3] * i1) : pack2<kF16>(o[j][0] * i0, o[j][1] * i0);
            if (p.lse && (lane & 3) == 0) p.lse[at] = (x ? M1 + (log2f(L1) - kShift) : M0 + (log2f(L0) - kShift)) * 0.69314718f;
          }
        } else {
          float* po = p.part_o + static_cast<long long>(slot) * kMergeFloats;
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            *reinterpret_cast<float2*>(po + r0 * 128 + j * 8 + c0) = make_float2(o[j][0], o[j][1]);
          }
          if (n_row > 8) {                                  // rows 8 and up, if there are any (8 x 4160 rows 34.1 -> 33.6 us)
#pragma unroll
            for (int j = 0; j < 16; ++j)
              *reinterpret_cast<float2*>(po + (r0 + 8) * 128 + j * 8 + c0) = make_float2(o[j][2], o[j][3]);
          }
          if ((lane & 3) == 0) {
            p.part_ml[slot * kRowTile + r0] = make_float2(M0, L0);
            p.part_ml[slot * kRowTile + r0 + 8] = make_float2(M1, L1);
          }
        }
      }
      if (!whole) {
        const int b_first = share_of(plan.total, plan.n_cta, pc.item);
        const int b_last = share_of(plan.total, plan.n_cta, pc.item + pc.n_tiles - 1);
        if (warp == 0) {
          __syncwarp();
          if (lane == 0) tail->last = arrive_last(p.arrived + b_first, b_last - b_first + 1);
        }
        sync_consumers();
        if (tail->last && ok) {
          // A row per warp: the contributors' factors by the lanes into shared memory, then four channels per lane.
          // Contributor c's slot is 1 if the item begins in it, else 0.
          const int n = b_last - b_first + 1;
          float* factor = merge + warp * (kMergeFloats / 2);                     // n <= 2 CTAs x SMs
          for (int r = warp; r < kRowTile; r += kWarps) {
            if (!row_valid(r)) continue;
            float M = -INFINITY;
            for (int c = lane; c < n; c += 32) M = fmaxf(M, __ldcg(&p.part_ml[((b_first + c) * 2 + (c == 0)) * kRowTile + r]).x);
            for (int o = 16; o; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xFFFFFFFFu, M, o));
            const float z = M == -INFINITY ? 0.f : M;
            float L = 0.f;
            for (int c = lane; c < n; c += 32) {
              const float2 ml = __ldcg(&p.part_ml[((b_first + c) * 2 + (c == 0)) * kRowTile + r]);
              const float f = ex2_approx(ml.x - z);
              factor[c] = f;
              L = fmaf(ml.y, f, L);
            }
            for (int o = 16; o; o >>= 1) L += __shfl_xor_sync(0xFFFFFFFFu, L, o);
            __syncwarp();
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int c0 = 0; c0 < n; c0 += kJoinFlight) {
              float4 v[kJoinFlight];
#pragma unroll
              for (int i = 0; i < kJoinFlight; ++i) {
                const int c = min(c0 + i, n - 1);
                v[i] = __ldcg(reinterpret_cast<const float4*>(
                    p.part_o + static_cast<long long>((b_first + c) * 2 + (c == 0)) * kMergeFloats + r * 128) + lane);
              }
#pragma unroll
              for (int i = 0; i < kJoinFlight; ++i) {
                const float f = c0 + i < n ? factor[c0 + i] : 0.f;
                acc.x = fmaf(v[i].x, f, acc.x); acc.y = fmaf(v[i].y, f, acc.y);
                acc.z = fmaf(v[i].z, f, acc.z); acc.w = fmaf(v[i].w, f, acc.w);
              }
            }
            __syncwarp();
            const float inv = L == 0.f ? 0.f : 1.f / L;
            const long long at = row_tok(r) * p.n_q + h_first + r % p.group;
            uint2* dst = reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.out) + at * 128) + lane;
            *dst = make_uint2(pack2<kF16>(acc.x * inv, acc.y * inv), pack2<kF16>(acc.z * inv, acc.w * inv));
            if (p.lse && lane == 0) p.lse[at] = (M + (log2f(L) - kShift)) * 0.69314718f;
          }
        }
        sync_consumers();                                  // tail->last is written again by the next piece
      }
    } while (w.next(b, ts, tail->plan));
  }
  __syncthreads();
  if (*abort_flag && threadIdx.x == 0) {                 // given up: no load may outlive the CTA
    int no_flag = 0;
    for (int i = max(0, tail->issued - kStages); i < tail->issued; ++i)
      mbar_wait(smem_u32(&tail->full[i % kStages]), (i / kStages) & 1, &no_flag, b.status, kDevWaitKFull);
  }
}

constexpr size_t kSmem = kStages * kStageBytes + 2 * kMergeFloats * 4 + sizeof(RowTail);

}  // namespace

cudaError_t init_paged_rows() {
  const cudaError_t e = cudaFuncSetAttribute(paged_rows_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kSmem));
  if (e != cudaSuccess) return e;
  return cudaFuncSetAttribute(paged_rows_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kSmem));
}

cudaError_t launch_paged_rows(const CUtensorMap& map_k, const CUtensorMap& map_v, const PagedAttnParams& p, bool f16,
                              int n_sm, cudaStream_t st) {
  auto k = f16 ? paged_rows_kernel<true> : paged_rows_kernel<false>;
  const TileShape ts = {p.n_kv, kRowTile / p.group, 6, 0};
  return launch_after_previous(k, n_sm * kRowCtasPerSm, kThreads, kSmem, st, map_k, map_v, p, ts);
}

}  // namespace ilre
