// Attention of a chunk of new tokens over the paged cache, and the joining of its cut items.
//
// A work item is one kv head and 256 query rows: two streams of 128 rows, a row being a (token, head of the group)
// pair, so that a key tile serves all heads of the group.  Both contractions run on the tensor cores: S = Q K^T
// into tensor memory, O += P V with P written to shared memory by the softmax warps (four per stream, a thread per
// row).  While the softmax of one stream works on its S tile the tensor cores serve the other.  Keys and values
// arrive in 128-key tiles through one TMA ring; a lane of the loading warp fetches the rows that one page has in the
// tile.  The output is kept against a reference maximum that moves only when it is outrun by 2^8.
//
// What bounds it: the exponentials, one per logit, and the tensor pipe, of about the same length (2048 cycles per unit,
// which takes 2900; a part of the exponentials as polynomials on the FMA pipe makes it slower, 431 -> 436 -> 451 us with 0, 2
// and 4 of 16 pairs for 1024 tokens behind 31744 rows).  So nothing may leave either idle: the batch's key tiles are cut
// into equal shares, one per SM (paged_batch.cuh), and a CTA runs its pieces as one stream of tiles: ring, barriers and
// tensor memory go on from piece to piece, the next piece's first logits are computed while the last one's output is
// written.  An item that the cut divides leaves 32-bit partial outputs, which a second kernel joins in the order of the
// CTAs.
#include "launch.cuh"
#include "paged_attn_kernels.cuh"
#include "paged_mma.cuh"
#include "paged_plan.cuh"

namespace ilre {

namespace {

constexpr int kStages = 3;
constexpr int kTileBytes = 128 * 128 * 2;
constexpr int kHalf = kTileBytes / 2;                    // 128 rows x 64 channels
constexpr int kThreads = 352;                            // warp 0 loads, 1 S MMAs, 2 PV MMAs, 3..6 / 7..10 softmax
constexpr int kSoftmaxWarps = 4;
constexpr int kEarly = 2;                                // of a tile's four groups, those before the wait for P
// What an item costs beside its tiles, in tiles.  Ragged batch of 12 sequences, 4096 tokens alone: 0 136 / 180 us, 2
// 108 / 135, 3 107 / 135, 4 110 / 138.
constexpr int kItemUnits = 3;
// Logits against the reference take one multiply-add, whose constant is the reference in powers of two, rounded: off by up to
// 2^-24 of it.  Every probability of the row is off by the same power then, which cancels, until it is too large for
// its type (a logit of 10^9: 2^32 times).  So from here on (2^-5 powers) the reference is taken off first.  The test costs
// a 128-key tile 1 % (4096 tokens alone 134.4 -> 136.8 us, 1024 behind 31744 rows 420.6 -> 425.6); two adds a logit always
// would cost 2 to 3 %.
constexpr float kFarLogit = 524288.f;
constexpr int kMinUnits = 4;                             // that a CTA gets at least (64 tokens behind 4096 rows: 2 25.8 us, 4 24.9)

struct ChunkTail {
  uint64_t q_full, q_empty;
  uint64_t kv_full[kStages];
  uint64_t kv_empty[kStages];
  uint64_t s_full[2], s_empty[2], p_full[2], p_empty[2], o_full[2];      // per stream
  PlanStart plan;
  PieceWalk<HeadTiles> walk[2 * kSoftmaxWarps];          // one per softmax warp
  uint32_t tmem_base;
  int abort_flag;
  int v_landed;                                          // value tiles that the PV thread has seen arrive
  int q_issued, kv_issued;                               // loads begun
};
constexpr size_t kSmem = static_cast<size_t>(4 + kStages) * kTileBytes + sizeof(ChunkTail);
static_assert(kSmem <= 232448, "shared memory");

template <bool kF16>
__global__ void __launch_bounds__(kThreads, 1)
paged_chunk_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                   const __grid_constant__ CUtensorMap map_v, const __grid_constant__ PagedAttnParams p,
                   const TileShape ts) {
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t q_s = smem_u32(smem);
  const uint32_t ring_s = q_s + 2 * kTileBytes;
  const uint32_t p_s = ring_s + kStages * kTileBytes;
  uint8_t* p_ptr = smem + (2 + kStages) * kTileBytes;
  ChunkTail* tail = reinterpret_cast<ChunkTail*>(smem + (4 + kStages) * kTileBytes);
  volatile int* abort_flag = &tail->abort_flag;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const PagedBatch& b = p.batch;
  const int tok = ts.tq / 2;                             // tokens of a stream

  if (threadIdx.x == 0) {
    tail->abort_flag = 0;
    tail->v_landed = 0;
    tail->q_issued = tail->kv_issued = 0;
    mbar_init(smem_u32(&tail->q_full), 1);
    mbar_init(smem_u32(&tail->q_empty), 1);
    for (int s = 0; s < kStages; ++s) {
      mbar_init(smem_u32(&tail->kv_full[s]), 1);
      mbar_init(smem_u32(&tail->kv_empty[s]), 1);
    }
    for (int x = 0; x < 2; ++x) {
      mbar_init(smem_u32(&tail->s_full[x]), 1);
      mbar_init(smem_u32(&tail->s_empty[x]), kSoftmaxWarps);
      mbar_init(smem_u32(&tail->p_full[x]), kSoftmaxWarps);
      mbar_init(smem_u32(&tail->p_empty[x]), 1);
      mbar_init(smem_u32(&tail->o_full[x]), 1);
    }
    fence_mbar_init();
    tma_prefetch_desc(&map_q);
    tma_prefetch_desc(&map_k);
    tma_prefetch_desc(&map_v);
  }
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
  if (threadIdx.x == 0 && (q_s & 1023u)) {
    tail->abort_flag = 1;
    report(b.status, kDevSmemAlign);
  }
  plan_start<HeadTiles>(b, ts, kMinUnits, reinterpret_cast<long long*>(p_ptr), &tail->plan);
  __syncthreads();
  if (threadIdx.x == 0) {                                // the item that begins here and goes on in other shares
    const PlanStart& s = tail->plan;
    ChunkJoin j = {-1, 0, 0, 0};
    if (s.u0 < s.u1 && s.last.tiles_at(ts) >= s.u0 && s.last.tiles_at(ts) < s.u1 && s.last.end(ts) > s.u1) {
      j.c_last = share_of(s.total, s.n_cta, s.last.end(ts) - 1);
      j.token = s.last.span.q0 + s.last.qt * ts.tq;
      j.n_tok = min(ts.tq, s.last.span.n - s.last.qt * ts.tq);
      j.head = s.last.head;
    }
    p.join[blockIdx.x] = j;
  }
  const bool run = *abort_flag == 0;
  auto streams = [&](const Piece& pc) { return pc.span.n - pc.qt * ts.tq > tok ? 2 : 1; };

  // TMEM columns: S of stream x at 128 x, O of stream x at 256 + 128 x.
  // Ring order of a piece of n tiles: K_0, K_1, V_0, K_2, V_1, ..., K_{n-1}, V_{n-2}, V_{n-1}: keys run one tile ahead,
  // because S of the next tile is issued while the softmax of the current one is still running.
  auto k_item = [](int i) -> int { return i == 0 ? 0 : 2 * i - 1; };
  auto v_item = [](int i, int n) -> int { return i < n - 1 ? 2 * i + 2 : 2 * n - 1; };

  if (warp == 0) {
    const int ps = 1 << b.page_shift;
    const int box_rows = min(ps, 128), n_box = 128 / box_rows;
    const int half = lane & 1, bx = lane >> 1;
    const bool active = bx < n_box;
    const uint32_t off = half * kHalf + bx * box_rows * 128;
    PieceWalk<HeadTiles> w;
    bool ok = run && w.begin(b, ts, tail->plan), more = ok;
    int it = 0, n_piece = 0;
    while (more && ok) {
      const Piece& pc = w.p;
      const int n = pc.t1 - pc.t0, n_str = streams(pc);
      auto tile_of_item = [&](int i, bool* is_k) -> int {
        *is_k = i == 0 || ((i & 1) && i != 2 * n - 1);
        return pc.t0 + (i == 0 ? 0 : i == 2 * n - 1 ? n - 1 : *is_k ? (i + 1) / 2 : i / 2 - 1);
      };
      // Table entries: of the key tile to come and of the value tile behind it (the one before), the former asked for a
      // tile ahead.  Rows at and behind kv need none: zeros, not read.
      auto needs = [&](int t) { return active && t < pc.t1 && t * 128 + bx * box_rows < pc.span.kv; };
      auto entry_at = [&](int t) -> int { return needs(t) ? table_entry(b, pc.seq, t * 128 + bx * box_rows) : 0; };
      int e_k = entry_at(pc.t0), e_v = e_k, e_next = entry_at(pc.t0 + 1);
      ok = warp_wait(&tail->q_empty, (n_piece & 1) ^ 1, abort_flag, b.status, kDevWaitQFull);
      if (!ok) break;
      if (lane == 0) {
        const uint32_t qf = smem_u32(&tail->q_full);
        const int row0 = pc.span.q0 + pc.qt * ts.tq;
        mbar_arrive_expect_tx(qf, n_str * 2 * tok * p.group * 128);
        for (int x = 0; x < n_str; ++x)
          for (int h = 0; h < 2; ++h)
            tma_load_3d(q_s + x * kTileBytes + h * kHalf, &map_q, h * 64, pc.head * p.group, row0 + x * tok, qf);
      }
      ++n_piece;
      if (lane == 0) tail->q_issued = n_piece;
      for (int i = 0; i < 2 * n; ++i, ++it) {
        bool is_k;
        const int t = tile_of_item(i, &is_k);
        const int row = t * 128 + bx * box_rows, s = it % kStages;
        ok = warp_wait(&tail->kv_empty[s], ((it / kStages) & 1) ^ 1, abort_flag, b.status, kDevWaitKEmpty);
        if (!ok) break;
        const int page = needs(t) ? checked_page(b, is_k ? e_k : e_v) : b.n_pages;
        const uint32_t bar = smem_u32(&tail->kv_full[s]);
        if (lane == 0) {
          mbar_arrive_expect_tx(bar, kTileBytes);
          tail->kv_issued = it + 1;
        }
        __syncwarp();
        if (active)
          tma_load_4d(ring_s + s * kTileBytes + off, is_k ? &map_k : &map_v, half * 64, pc.head, row & (ps - 1), page, bar);
        // order K_0, K_1, V_0, K_2, V_1, ...: V_t comes behind K_{t+1}, whose entry then is the next V's
        if (i == 0 || !is_k) {
          if (i > 0) e_v = e_k;
          e_k = e_next;
          e_next = entry_at(t + (i == 0 ? 2 : 3));
        }
      }
      if (ok) more = w.next(b, ts, tail->plan);
    }
  } else if (warp == 1 || warp == 2) {
    // Two MMA-issuing threads, one for every S = Q K^T, one for every O += P V; each polls its streams' barriers and
    // issues what is ready.  A test of a ring slot's phase tells its two latest phases apart, so an item may be
    // asked for only once the item before it in its slot, three items earlier, is known to have arrived: the PV
    // thread knows (P of its tile is made from that tile's keys), the S thread asks for the count of value tiles.
    if (lane == 0 && run) {
      constexpr uint32_t idesc_s = kF16 ? umma_idesc_f16(128, 128) : umma_idesc_bf16(128, 128);
      constexpr uint32_t idesc_o = idesc_s | (1u << 16);                   // B = V: channels contiguous
      const bool s_role = (warp == 1);
      volatile int* v_landed = &tail->v_landed;
      PieceWalk<HeadTiles> w;
      bool ok = w.begin(b, ts, tail->plan), more = ok;
      int it0 = 0, tile0 = 0, n_prev = 2, n_piece = 0;
      uint32_t done[2] = {0, 0};                         // tiles of each stream so far
      int landed = 0;
      while (more && ok) {
        const int n = w.p.t1 - w.p.t0, n_str = streams(w.p);
        if (s_role) {
          ok = mbar_wait(smem_u32(&tail->q_full), n_piece & 1, abort_flag, b.status, kDevWaitQFull);
          tc_fence_after();
        }
        auto slot = [&](int item) { return (it0 + item) % kStages; };
        auto ring_ready = [&](int item) {
          return mbar_test_wait(smem_u32(&tail->kv_full[slot(item)]), ((it0 + item) / kStages) & 1);
        };
        int next[2] = {0, n_str == 2 ? 0 : n};
        int released = 0;
        long long t_idle = 0;
        uint32_t spins = 0;
        while (ok && (next[0] < n || next[1] < n)) {
          bool progress = false;
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const int i = next[x];
            if (i >= n) continue;
            const uint32_t par = (done[x] + i) & 1u;
            if (s_role) {
              // needs the stream's S before it read out of tensor memory, and the key tile
              const int need = tile0 + i - (i == 0 && n_prev == 1 ? 1 : 2);
              if (mbar_test_wait(smem_u32(&tail->s_empty[x]), par ^ 1u) && *v_landed >= need && ring_ready(k_item(i))) {
                tc_fence_after();
                const uint32_t k_s = ring_s + slot(k_item(i)) * kTileBytes, qx = q_s + x * kTileBytes;
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                  for (int ks = 0; ks < 4; ++ks)
                    umma_bf16(tmem_base + x * 128, umma_desc_sw128(qx + kb * kHalf + ks * 32),
                              umma_desc_sw128(k_s + kb * kHalf + ks * 32), idesc_s, (kb | ks) != 0);
                umma_commit(smem_u32(&tail->s_full[x]));
                next[x] = i + 1;
                progress = true;
                while (released < min(next[0], next[1])) {
                  umma_commit(smem_u32(&tail->kv_empty[slot(k_item(released))]));
                  ++released;
                }
              }
            } else {
              // needs P written and the value tile
              if (mbar_test_wait(smem_u32(&tail->p_full[x]), par) && ring_ready(v_item(i, n))) {
                if (tile0 + i + 1 > landed) *v_landed = landed = tile0 + i + 1;
                tc_fence_after();
                const uint32_t v_s = ring_s + slot(v_item(i, n)) * kTileBytes, px = p_s + x * kTileBytes;
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                  for (int ks = 0; ks < 4; ++ks)
                    umma_bf16(tmem_base + 256 + x * 128, umma_desc_sw128(px + kb * kHalf + ks * 32),
                              umma_desc_sw128_mn(v_s + (kb * 64 + ks * 16) * 128, kHalf, 1024), idesc_o, (i | kb | ks) != 0);
                umma_commit(smem_u32(&tail->p_empty[x]));
                next[x] = i + 1;
                progress = true;
                if (i + 1 == n) umma_commit(smem_u32(&tail->o_full[x]));
                while (released < min(next[0], next[1])) {
                  umma_commit(smem_u32(&tail->kv_empty[slot(v_item(released, n))]));
                  ++released;
                }
              }
            }
          }
          if (progress) {
            spins = 0;
          } else {
            if (spins == 0) t_idle = clock64();
            if ((++spins & 0x3FF) == 0) {
              if (*abort_flag) {
                ok = false;
              } else if (clock64() - t_idle > kWaitCycleLimit) {
                *abort_flag = 1;
                atomicCAS(b.status, 0, kDevWaitAccFull);
                ok = false;
              }
            }
          }
        }
        if (!ok) break;
        if (s_role) umma_commit(smem_u32(&tail->q_empty));
        done[0] += n;
        if (n_str == 2) done[1] += n;
        it0 += 2 * n;
        tile0 += n;
        n_prev = n;
        ++n_piece;
        more = w.next(b, ts, tail->plan);
      }
    }
  } else {
    // Softmax warps of stream x: warp w reads TMEM lane quadrant w % 4, so a thread owns one query row: its 128
    // logits of the tile, its reference and sum, its row of P and of O.
    const int x = (warp - 3) / kSoftmaxWarps;
    const int quad = warp & 3;
    const int row = quad * 32 + lane;
    const int my_tok = row / p.group, my_head = row - my_tok * p.group;
    const uint32_t lane_base = tmem_base + (static_cast<uint32_t>(quad * 32) << 16);
    const uint32_t s_tm = lane_base + x * 128, o_tm = lane_base + 256 + x * 128;
    uint8_t* p_mine = p_ptr + x * kTileBytes;
    const float c2 = p.c2;
    PieceWalk<HeadTiles>* walk = &tail->walk[warp - 3];
    uint32_t n_tile = 0, n_out = 0;                      // of this stream so far
    uint32_t items = 0;                                  // ring items before this piece
    bool ok = run;
    bool more;
    if (lane == 0) more = walk->begin(b, ts, tail->plan);
    more = __shfl_sync(0xFFFFFFFFu, more, 0);
    __syncwarp();
    while (more && ok) {
      const int n = walk->p.t1 - walk->p.t0, k_first = walk->p.t0 * 128, kv = walk->p.span.kv;
      const int tok0 = walk->p.qt * ts.tq + x * tok;     // first token of the stream
      if (tok0 < walk->p.span.n) {
        const int pre = kv - walk->p.span.n + tok0;      // what its first token sees
        const int limit = pre + my_tok;
        constexpr float kShift = kF16 ? kChunkShift : 0.f;
        float ref = -INFINITY, l = 0.f;
        for (int i = 0; i < n && ok; ++i, ++n_tile) {
          ok = warp_wait(&tail->s_full[x], n_tile & 1u, abort_flag, b.status, kDevWaitAccFull);
          if (!ok) break;
          float vv[4][32];
#define V(i) vv[(i) >> 5][(i) & 31]
          tc_fence_after();
          tmem_ld32(s_tm, vv[0]);
          tmem_ld32(s_tm + 32, vv[1]);
          tmem_ld32(s_tm + 64, vv[2]);
          tmem_ld32(s_tm + 96, vv[3]);
          tmem_ld_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&tail->s_empty[x]));
          const int k0 = k_first + i * 128;
          if (k0 + 127 > pre) {
#pragma unroll
            for (int j = 0; j < 128; ++j) V(j) = (k0 + j <= limit) ? V(j) : -INFINITY;
          }
          float m0 = fmax3(V(0), V(1), V(2)), m1 = fmax3(V(3), V(4), V(5));
#pragma unroll
          for (int j = 6; j < 126; j += 4) {
            m0 = fmax3(m0, V(j), V(j + 1));
            m1 = fmax3(m1, V(j + 2), V(j + 3));
          }
          const float cm = fmax3(m0, m1, fmaxf(V(126), V(127)));
          float scale = 1.f;
          if ((cm - ref) * c2 > kChunkSlack || ref == -INFINITY) {
            scale = (ref == -INFINITY) ? 0.f : ex2_approx((ref - cm) * c2);
            ref = (cm == -INFINITY) ? ref : cm;
          }
          float nr = (ref == -INFINITY) ? 0.f : fmaf(-ref, c2, kShift);
          if (__builtin_expect(__any_sync(0xFFFFFFFFu, fabsf(nr) > kFarLogit), 0)) {
            const float r = (ref == -INFINITY) ? 0.f : ref;
#pragma unroll
            for (int j = 0; j < 128; j += 2) {
              const float2 v = fadd2(make_float2(V(j), V(j + 1)), make_float2(-r, -r));
              V(j) = v.x;
              V(j + 1) = v.y;
            }
            nr = kShift;
          }
          float2 sum2 = make_float2(0.f, 0.f);
          auto exponentials = [&](int g32, uint32_t (&wd)[16]) {
#pragma unroll
            for (int j = 0; j < 32; j += 2) {
              const float2 a = ffma2(make_float2(V(g32 * 32 + j), V(g32 * 32 + j + 1)), make_float2(c2, c2),
                                     make_float2(nr, nr));
              const float2 pp = make_float2(ex2_approx(a.x), ex2_approx(a.y));
              sum2 = fadd2(sum2, pp);
              wd[j >> 1] = pack2<kF16>(pp.x, pp.y);
            }
          };
          auto store = [&](int g32, const uint32_t (&wd)[16]) {
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              const int c16 = g32 * 4 + c;
              *reinterpret_cast<uint4*>(p_mine + (c16 >> 3) * kHalf + row * 128 + (((c16 & 7) ^ (row & 7)) << 4)) =
                  make_uint4(wd[c * 4], wd[c * 4 + 1], wd[c * 4 + 2], wd[c * 4 + 3]);
            }
          };
          uint32_t early[kEarly][16];
#pragma unroll
          for (int g32 = 0; g32 < kEarly; ++g32) {
            exponentials(g32, early[g32]);
#pragma unroll
            for (int j = 0; j < 16; ++j) asm volatile("" : "+r"(early[g32][j]));     // not after the wait
          }
          ok = warp_wait(&tail->p_empty[x], (n_tile & 1u) ^ 1u, abort_flag, b.status, kDevWaitAccEmpty);
          if (!ok) break;
#pragma unroll
          for (int g32 = 0; g32 < 4; ++g32) {
            uint32_t wd[16];
            if (g32 < kEarly) {
              store(g32, early[g32 < kEarly ? g32 : 0]);
            } else {
              exponentials(g32, wd);
              store(g32, wd);
            }
          }
          l = fmaf(l, scale, sum2.x + sum2.y);
          if (i > 0 && __any_sync(0xFFFFFFFFu, scale != 1.f)) {
            tc_fence_after();
#pragma unroll 1
            for (int q4 = 0; q4 < 4; ++q4) {
              float o[32];
              tmem_ld32(o_tm + q4 * 32, o);
              tmem_ld_wait();
#pragma unroll
              for (int j = 0; j < 32; ++j) o[j] *= scale;
              tmem_st32(o_tm + q4 * 32, o);
            }
            tmem_st_wait();
            tc_fence_before();
          }
#undef V
          if (k0 + 128 > kv && (kv & ((1 << b.page_shift) - 1))) {
            // The sequence ends inside a page: whatever the page holds behind it must not reach the tensor cores (0
            // times NaN).  Both streams write the same zeros before either hands its P over.
            const int item = items + v_item(i, n);
            // (the value tiles before it first, for the same reason as the S thread's)
            ok = warp_wait_count(&tail->v_landed, items / 2 + i, abort_flag, b.status, kDevWaitKFull) &&
                 warp_wait(&tail->kv_full[item % kStages], (item / kStages) & 1u, abort_flag, b.status, kDevWaitKFull);
            if (!ok) break;
            uint8_t* v_ptr = smem + 2 * kTileBytes + (item % kStages) * kTileBytes;
            const int first = max(kv - k0, 0);
            for (int j = first * 8 + row; j < 128 * 8; j += 128) {
              *reinterpret_cast<uint4*>(v_ptr + j * 16) = make_uint4(0, 0, 0, 0);
              *reinterpret_cast<uint4*>(v_ptr + kHalf + j * 16) = make_uint4(0, 0, 0, 0);
            }
          }
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&tail->p_full[x]));
        }
        ok = ok && warp_wait(&tail->o_full[x], n_out & 1u, abort_flag, b.status, kDevWaitAccFull);
        ++n_out;
        if (ok) {
          tc_fence_after();
          const int valid_tok = min(tok, walk->p.span.n - tok0);
          const long long tok_at = static_cast<long long>(walk->p.span.q0) + tok0;
          const int head0 = walk->p.head * p.group;
          if (walk->p.t0 == 0 && walk->p.t1 == walk->p.n_tiles) {
            // O / sum through this warp's rows of the P buffer (its MMAs are done), out in whole rows of 256 bytes
            const float inv_l = l == 0.f ? 0.f : 1.f / l;
#pragma unroll 2
            for (int q4 = 0; q4 < 4; ++q4) {
              float v[32];
              tmem_ld32(o_tm + q4 * 32, v);
              tmem_ld_wait();
              uint32_t wd[16];
#pragma unroll
              for (int j = 0; j < 32; j += 2) wd[j >> 1] = pack2<kF16>(v[j] * inv_l, v[j + 1] * inv_l);
#pragma unroll
              for (int c = 0; c < 4; ++c)
                *reinterpret_cast<uint4*>(p_mine + (q4 >> 1) * kHalf + row * 128 + ((((q4 & 1) * 4 + c) ^ (row & 7)) << 4)) =
                    make_uint4(wd[4 * c], wd[4 * c + 1], wd[4 * c + 2], wd[4 * c + 3]);
            }
            tc_fence_before();
            __syncwarp();
            const int c16 = lane & 15, row0 = quad * 32 + (lane >> 4), step_t = 2 / p.group, step_h = 2 - step_t * p.group;
            int rt = row0 / p.group, rh = row0 - rt * p.group;
            uint4* dst = static_cast<uint4*>(p.out) + (tok_at * p.n_q + head0) * 16 + c16;
#pragma unroll
            for (int r8 = 0; r8 < 2; ++r8) {
              uint4 v[8];
#pragma unroll
              for (int k = 0; k < 8; ++k) {
                const int r = row0 + 2 * (r8 * 8 + k);
                v[k] = *reinterpret_cast<const uint4*>(p_mine + (c16 >> 3) * kHalf + r * 128 + (((c16 & 7) ^ (r & 7)) << 4));
              }
#pragma unroll
              for (int k = 0; k < 8; ++k) {
                if (rt < valid_tok) dst[(static_cast<long long>(rt) * p.n_q + rh) * 16] = v[k];
                rt += step_t;
                rh += step_h;
                if (rh >= p.group) { rh -= p.group; ++rt; }
              }
            }
            __syncwarp();
            if (p.lse && my_tok < valid_tok)
              p.lse[(tok_at + my_tok) * p.n_q + head0 + my_head] =
                  l == 0.f ? -INFINITY : (ref * c2 + (log2f(l) - kShift)) * 0.69314718f;
          } else {
            // partial: [channel / 4][row][4], so that the lanes' stores join
            const long long slot = blockIdx.x * 2 + (walk->p.t0 > 0 ? 0 : 1);
            float4* po = reinterpret_cast<float4*>(p.chunk_o) + slot * (kChunkRows * 32) + x * 128 + row;
#pragma unroll 1
            for (int q4 = 0; q4 < 4; ++q4) {
              float v[32];
              tmem_ld32(o_tm + q4 * 32, v);
              tmem_ld_wait();
#pragma unroll
              for (int c = 0; c < 8; ++c)
                po[(q4 * 8 + c) * kChunkRows] = make_float4(v[4 * c], v[4 * c + 1], v[4 * c + 2], v[4 * c + 3]);
            }
            tc_fence_before();
            p.chunk_ml[slot * kChunkRows + x * 128 + row] = make_float2(ref * c2, l);
          }
        }
      }
      if (!ok) break;
      items += 2 * n;
      __syncwarp();
      if (lane == 0) more = walk->next(b, ts, tail->plan);
      more = __shfl_sync(0xFFFFFFFFu, more, 0);
      __syncwarp();
    }
  }
  tc_fence_before();
  __syncthreads();
  if (*abort_flag && threadIdx.x == 0) {                 // given up: no load may outlive the CTA
    const long long limit = kWaitCycleLimit;
    int no_flag = 0;
    if (tail->q_issued) mbar_wait(smem_u32(&tail->q_full), (tail->q_issued - 1) & 1, &no_flag, b.status, kDevWaitQFull, limit);
    for (int it = max(0, tail->kv_issued - kStages); it < tail->kv_issued; ++it)
      mbar_wait(smem_u32(&tail->kv_full[it % kStages]), (it / kStages) & 1, &no_flag, b.status, kDevWaitKFull, limit);
  }
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, 512);
  }
}

// Joins the pieces of the item that begins in share blockIdx.x and goes on behind it, if there is one: 32 of its rows
// (lane = row), a warp per 8 channels.  Bound by latency, so the contributors' statistics are fetched side by side.
// Most items have two or three contributors: two outputs of a thread in flight and three CTAs per SM serve them better
// than eight and one (a ragged batch of 12 sequences 115 -> 107 us in all, 4096 tokens alone 143 -> 135; four and two
// 108 and 137).  Contributor c's slot is 1 if the item begins in its share, else 0.
constexpr int kJoinRows = 32, kJoinThreads = 512, kJoinFlight = 2, kMaxCtas = 192;

template <bool kF16>
__global__ void __launch_bounds__(kJoinThreads, 3)
paged_join_kernel(const __grid_constant__ PagedAttnParams p, int tok) {
  __shared__ float2 ml[kMaxCtas][kJoinRows];
  grid_dep_wait();
  grid_dep_launch();
  const ChunkJoin j = p.join[blockIdx.x];
  const int c0 = blockIdx.x, n = j.c_last - c0 + 1;
  if (j.c_last < 0) return;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, row = blockIdx.y * kJoinRows + lane;
  for (int c = warp; c < n; c += kJoinThreads / 32)
    ml[c][lane] = p.chunk_ml[((c0 + c) * 2 + (c == 0)) * kChunkRows + row];
  __syncthreads();
  const int rt = (row & 127) / p.group, rh = (row & 127) - rt * p.group, my_tok = (row >> 7) * tok + rt;
  if (rt >= tok || my_tok >= j.n_tok) return;
  float M = -INFINITY, L = 0.f;
  for (int c = 0; c < n; ++c) M = fmaxf(M, ml[c][lane].x);
  const float z = M == -INFINITY ? 0.f : M;
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f), b = a;
  const float4* po = reinterpret_cast<const float4*>(p.chunk_o) + 2 * warp * kChunkRows + row;
  for (int c = 0; c < n; c += kJoinFlight) {
    float4 va[kJoinFlight], vb[kJoinFlight];
#pragma unroll
    for (int f = 0; f < kJoinFlight; ++f) {
      const int cc = min(c + f, n - 1);
      const float4* at = po + static_cast<long long>((c0 + cc) * 2 + (cc == 0)) * (kChunkRows * 32);
      va[f] = at[0];
      vb[f] = at[kChunkRows];
    }
#pragma unroll
    for (int f = 0; f < kJoinFlight; ++f) {
      if (c + f >= n) break;
      const float2 x = ml[c + f][lane];
      const float s = ex2_approx(x.x - z);
      if (s != 0.f || isnan(x.y)) {                      // where the row saw nothing, O may hold anything
        L = fmaf(x.y, s, L);
        a.x = fmaf(va[f].x, s, a.x); a.y = fmaf(va[f].y, s, a.y); a.z = fmaf(va[f].z, s, a.z); a.w = fmaf(va[f].w, s, a.w);
        b.x = fmaf(vb[f].x, s, b.x); b.y = fmaf(vb[f].y, s, b.y); b.z = fmaf(vb[f].z, s, b.z); b.w = fmaf(vb[f].w, s, b.w);
      }
    }
  }
  const float inv = L == 0.f ? 0.f : 1.f / L;
  const long long at = (static_cast<long long>(j.token) + my_tok) * p.n_q + j.head * p.group + rh;
  reinterpret_cast<uint4*>(p.out)[at * 16 + warp] =
      make_uint4(pack2<kF16>(a.x * inv, a.y * inv), pack2<kF16>(a.z * inv, a.w * inv), pack2<kF16>(b.x * inv, b.y * inv),
                 pack2<kF16>(b.z * inv, b.w * inv));
  if (p.lse && warp == 0) p.lse[at] = L == 0.f ? -INFINITY : (M + (log2f(L) - (kF16 ? kChunkShift : 0.f))) * 0.69314718f;
}

}  // namespace

cudaError_t init_paged_chunk() {
  const cudaError_t e = cudaFuncSetAttribute(paged_chunk_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kSmem));
  if (e != cudaSuccess) return e;
  return cudaFuncSetAttribute(paged_chunk_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kSmem));
}

cudaError_t launch_paged_chunk(const CUtensorMap& map_q, const CUtensorMap& map_k, const CUtensorMap& map_v,
                               const PagedAttnParams& p, bool f16, int n_sm, cudaStream_t st) {
  auto k = f16 ? paged_chunk_kernel<true> : paged_chunk_kernel<false>;
  if (n_sm > kMaxCtas) return cudaErrorInvalidConfiguration;
  const TileShape ts = {p.n_kv, 2 * (128 / p.group), 7, kItemUnits};
  const cudaError_t e = launch_after_previous(k, n_sm, kThreads, kSmem, st, map_q, map_k, map_v, p, ts);
  if (e != cudaSuccess) return e;
  auto j = f16 ? paged_join_kernel<true> : paged_join_kernel<false>;
  return launch_after_previous(j, dim3(n_sm, kChunkRows / kJoinRows), kJoinThreads, 0, st, p, 128 / p.group);
}

}  // namespace ilre
