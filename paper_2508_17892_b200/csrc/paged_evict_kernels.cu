// Eviction: of the rows between the sinks and the recent ones the `want` rows of largest weight (equal weights: the
// lower row), then the kept rows' way to the front.
//
// Selection: one cluster of CTAs per list (a kv head of a sequence, or a sequence).  Each CTA reads its part of the
// list's weights once, as numbers that order like them, and keeps them in shared memory; three histograms (11, 11
// and 10 bits, added up over the cluster through its shared memory) narrow the threshold down until its bin
// is kept as a whole (one request of 4608 rows 13.8 us in all; 15.1 with all three always), and prefix counts give
// every row above it, and the first rows equal to it, its place in the ascending output.  Bound by latency: a list is
// some 10^4 numbers, so what counts is that they are read once and that few barriers follow.
//
// Moving, to other pages: every row is its own, so CTAs of 64 rows of a head copy them all at once.  In place:
// the kept rows ascend, so kept row i comes from a row >= i, and rows may move as long as none is written before every
// row up to it has been read.  A CTA then has one 64-byte column of the keys or values of one head (columns are
// independent) and goes through the rows in ascending batches: all reads of a batch, a barrier, all its writes.
// Later batches read at or behind their own begin only.
#include "launch.cuh"
#include "paged_weight_kernels.cuh"

namespace ilre {

namespace {

constexpr int kSelThreads = 512;
constexpr int kSelCluster = 8;                           // CTAs of a list, at most
constexpr int kSelFlight = 4;
constexpr int kSelBins = 2048;
constexpr int kSelKeep = 44032;                          // keys of a CTA that shared memory takes, at most
constexpr int kMoveThreads = 256;
constexpr int kMoveRows = 64;                            // rows of a CTA that copies to other pages
constexpr int kMoveCols = 8;                             // columns of a head: 4 of keys, 4 of values

// Row t's key: larger is heavier; the sum over the heads is formed in double and rounded once, so its value does
// not hang on an order.
__device__ __forceinline__ uint32_t weight_key(const EvictParams& p, int list, int t, int entry) {
  const int page = checked_page(p.batch, entry);
  if (page >= p.batch.n_pages) return float_to_ordered(0.f);      // its rows' weights count as zeros
  const int row = t & ((1 << p.batch.page_shift) - 1);
  const float* w = p.w + ((static_cast<long long>(page) * p.n_kv) << p.batch.page_shift) + row;
  float x;
  if (p.per_head) {
    x = w[static_cast<long long>(list) << p.batch.page_shift];
  } else {
    double s = 0.0;
#pragma unroll 8
    for (int g = 0; g < p.n_kv; ++g) s += w[static_cast<long long>(g) << p.batch.page_shift];
    x = static_cast<float>(s);
  }
  return isnan(x) ? 0xFFFFFFFFu : float_to_ordered(x + 0.f);
}

struct SelShared {
  uint32_t hist[3][kSelBins];
  uint32_t warp_sum[kSelThreads / 32];
  uint32_t above, equal;                                 // of this CTA's part
  uint32_t bin, left, held;                              // held: rows of the bin
};

__device__ __forceinline__ uint32_t ld_cluster(const uint32_t* mine, uint32_t rank) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(cluster_addr(smem_u32(mine), rank)) : "memory");
  return v;
}
__device__ __forceinline__ uint4 ld_cluster4(const uint32_t* mine, uint32_t rank) {
  uint4 v;
  asm volatile("ld.shared::cluster.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(cluster_addr(smem_u32(mine), rank)) : "memory");
  return v;
}

// Sum of `v` over the threads before this one; all threads of the CTA.
__device__ __forceinline__ uint32_t scan_before(uint32_t v, uint32_t* warp_sum) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t incl = v;
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t x = __shfl_up_sync(0xFFFFFFFFu, incl, o);
    if (lane >= o) incl += x;
  }
  if (lane == 31) warp_sum[warp] = incl;
  __syncthreads();
  uint32_t before = incl - v;
  for (int w = 0; w < warp; ++w) before += warp_sum[w];
  __syncthreads();
  return before;
}

__global__ void __launch_bounds__(kSelThreads)
evict_select_kernel(const __grid_constant__ EvictParams p, int keep, int n_cta) {
  extern __shared__ __align__(16) uint32_t keys[];       // [keep], then SelShared
  SelShared& s = *reinterpret_cast<SelShared*>(keys + keep);
  const int lists = p.per_head ? p.n_kv : 1;
  const int which = blockIdx.x / n_cta, rank = blockIdx.x % n_cta;
  const int seq = which / lists, list = which % lists;
  for (int i = threadIdx.x; i < 3 * kSelBins; i += kSelThreads) s.hist[0][i] = 0;
  grid_dep_wait();
  grid_dep_launch();
  int32_t* kept = p.kept + static_cast<long long>(which) * p.budget;
  const int kv = p.batch.kv_len[seq];
  const bool ok = kv >= 0 && kv <= (static_cast<long long>(p.batch.max_blocks) << p.batch.page_shift);
  if (!ok && threadIdx.x == 0) report(p.batch.status, kDevBadLengths);
  const int n_keep = ok ? min(kv, p.budget) : 0;
  if (threadIdx.x == 0 && rank == 0 && list == 0) p.n_keep[seq] = ok ? n_keep : -1;
  if (!ok || kv <= p.budget) {                           // the whole cluster
    for (int i = rank * kSelThreads + threadIdx.x; i < p.budget; i += n_cta * kSelThreads) kept[i] = i < n_keep ? i : -1;
    // A sequence left out has no rows; the batch's own array keeps what it says, so that the next call reports it too.
    // (The kernels that move rows write the other lengths.)
    if (!ok && p.new_len != p.batch.kv_len && threadIdx.x == 0 && rank == 0 && list == 0) p.new_len[seq] = 0;
    return;
  }
  for (int i = rank * kSelThreads + threadIdx.x; i < p.n_sink; i += n_cta * kSelThreads) kept[i] = i;
  for (int i = rank * kSelThreads + threadIdx.x; i < p.n_recent; i += n_cta * kSelThreads)
    kept[p.budget - p.n_recent + i] = kv - p.n_recent + i;
  const uint32_t want = p.budget - p.n_sink - p.n_recent;
  if (want == 0) return;
  const int middle = kv - p.n_recent - p.n_sink;         // > want
  const int part = (middle + n_cta - 1) / n_cta;
  const int lo = p.n_sink + min(rank * part, middle), n = p.n_sink + min((rank + 1) * part, middle) - lo;
  auto key_at = [&](int i) { return i < keep ? keys[i] : weight_key(p, list, lo + i, table_entry(p.batch, seq, lo + i)); };
  __syncthreads();
  for (int ib = threadIdx.x; ib < n; ib += kSelThreads * kSelFlight) {        // four rows of a thread in flight
    int entry[kSelFlight];
    uint32_t k[kSelFlight];
#pragma unroll
    for (int j = 0; j < kSelFlight; ++j)
      entry[j] = ib + j * kSelThreads < n ? table_entry(p.batch, seq, lo + ib + j * kSelThreads) : 0;
#pragma unroll
    for (int j = 0; j < kSelFlight; ++j)
      k[j] = ib + j * kSelThreads < n ? weight_key(p, list, lo + ib + j * kSelThreads, entry[j]) : 0;
#pragma unroll
    for (int j = 0; j < kSelFlight; ++j) {
      const int i = ib + j * kSelThreads;
      if (i >= n) break;
      if (i < keep) keys[i] = k[j];
      atomicAdd(&s.hist[0][k[j] >> 21], 1u);
    }
  }
  uint32_t left = want, prefix = 0;                      // rows to take among those whose leading bits are `prefix`
  int low = 0;                                           // bits behind the prefix
#pragma unroll 1
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = pass == 2 ? 1024 : kSelBins;
    if (pass > 0)
      for (int i = threadIdx.x; i < n; i += kSelThreads) {
        const uint32_t k = key_at(i);
        const uint32_t up = pass == 1 ? k >> 21 : k >> 10;
        if (up == prefix) atomicAdd(&s.hist[pass][(k >> shift) & (bins - 1)], 1u);
      }
    cluster_sync_all();
    // thread 0 has the heaviest four bins; the bin in which the count from above reaches `left`
    const int b0 = bins - 4 - 4 * static_cast<int>(threadIdx.x);
    uint4 c = make_uint4(0, 0, 0, 0);
    if (b0 >= 0)
#pragma unroll 4
      for (uint32_t r = 0; r < static_cast<uint32_t>(n_cta); ++r) {
        const uint4 v = ld_cluster4(&s.hist[pass][b0], r);
        c.x += v.x; c.y += v.y; c.z += v.z; c.w += v.w;
      }
    uint32_t before = scan_before(c.x + c.y + c.z + c.w, s.warp_sum);
    const uint32_t in_bin[4] = {c.w, c.z, c.y, c.x};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (before < left && left <= before + in_bin[j]) { s.bin = b0 + 3 - j; s.left = left - before; s.held = in_bin[j]; }
      before += in_bin[j];
    }
    __syncthreads();
    left = s.left;
    prefix = pass == 0 ? s.bin : pass == 1 ? (prefix << 11) | s.bin : (prefix << 10) | s.bin;
    low = shift;
    if (left == s.held) break;                           // the whole bin is kept: its rows need no order
    __syncthreads();
  }
  // `prefix` is the threshold, `left` the rows equal to it (but for the low bits) that are kept.  Each thread a run of consecutive rows.
  const int run = (n + kSelThreads - 1) / kSelThreads, i0 = min(static_cast<int>(threadIdx.x) * run, n), i1 = min(i0 + run, n);
  uint32_t above = 0, equal = 0;
  for (int i = i0; i < i1; ++i) {
    const uint32_t k = key_at(i) >> low;
    above += k > prefix;
    equal += k == prefix;
  }
  const uint32_t above_before = scan_before(above, s.warp_sum), equal_before = scan_before(equal, s.warp_sum);
  if (threadIdx.x == kSelThreads - 1) { s.above = above_before + above; s.equal = equal_before + equal; }
  cluster_sync_all();
  const int lane = threadIdx.x & 31;                     // the CTAs before this one: a lane of every warp asks one
  uint32_t a = lane < rank ? ld_cluster(&s.above, lane) : 0, e = lane < rank ? ld_cluster(&s.equal, lane) : 0;
  a = __reduce_add_sync(0xFFFFFFFFu, a) + above_before;
  e = __reduce_add_sync(0xFFFFFFFFu, e) + equal_before;
  cluster_sync_all();                                    // no CTA leaves while its counts are read
  for (int i = i0; i < i1; ++i) {
    const uint32_t k = key_at(i) >> low;
    const bool is_above = k > prefix, is_equal = k == prefix;
    if (is_above || (is_equal && e < left)) kept[p.n_sink + a + min(e, left)] = lo + i;
    a += is_above;
    e += is_equal;
  }
}

__device__ __forceinline__ int dst_page(const EvictParams& p, int seq, int i) {
  return checked_page(p.batch, p.dst_table[static_cast<long long>(seq) * p.dst_blocks + (i >> p.batch.page_shift)]);
}
__device__ __forceinline__ const int32_t* kept_rows(const EvictParams& p, int seq, int g) {
  return p.kept + (static_cast<long long>(seq) * (p.per_head ? p.n_kv : 1) + (p.per_head ? g : 0)) * p.budget;
}

// To other pages: a CTA has 64 rows of a head, its threads find their places, then 16 of them move a row.
__global__ void __launch_bounds__(kMoveThreads)
evict_copy_kernel(const __grid_constant__ EvictParams p) {
  __shared__ int src_page[kMoveRows], src_row[kMoveRows], to_page[kMoveRows];
  const int g = blockIdx.x % p.n_kv, i0 = static_cast<int>(blockIdx.x / p.n_kv) * kMoveRows, seq = blockIdx.z;
  grid_dep_wait();
  grid_dep_launch();
  const PagedBatch& b = p.batch;
  const int n = p.n_keep[seq], mask = (1 << b.page_shift) - 1;
  if (g == 0 && i0 == 0 && threadIdx.x == 0 && n >= 0) p.new_len[seq] = n;
  if (i0 >= n) return;
  if (threadIdx.x < kMoveRows) {
    const int i = i0 + threadIdx.x;
    int sp = -1, src = 0, dp = 0;
    if (i < n) {
      src = kept_rows(p, seq, g)[i];
      dp = dst_page(p, seq, i);
      sp = page_of(b, seq, src);
      if (sp >= b.n_pages || dp >= b.n_pages) sp = -1;
    }
    src_page[threadIdx.x] = sp; src_row[threadIdx.x] = src & mask; to_page[threadIdx.x] = dp;
    if (sp >= 0)
      p.w[((static_cast<long long>(dp) * p.n_kv + g) << b.page_shift) + (i & mask)] =
          p.w[((static_cast<long long>(sp) * p.n_kv + g) << b.page_shift) + (src & mask)];
  }
  __syncthreads();
  const int lane = threadIdx.x & 15;
  constexpr int kStep = kMoveThreads / 16, kTurns = kMoveRows / kStep;
  const uint4* k = static_cast<const uint4*>(p.k);
  const uint4* v = static_cast<const uint4*>(p.v);
  uint4 xk[kTurns], xv[kTurns];
#pragma unroll
  for (int t = 0; t < kTurns; ++t) {
    const int r = t * kStep + (threadIdx.x >> 4), sp = src_page[r];
    if (sp >= 0) {
      const long long at = (static_cast<long long>(src_row[r]) * p.n_kv + g) * 16 + lane;
      xk[t] = k[sp * (p.k_page_stride >> 3) + at];
      xv[t] = v[sp * (p.v_page_stride >> 3) + at];
    }
  }
#pragma unroll
  for (int t = 0; t < kTurns; ++t) {
    const int r = t * kStep + (threadIdx.x >> 4);
    if (src_page[r] >= 0) {
      const long long at = (static_cast<long long>((i0 + r) & mask) * p.n_kv + g) * 16 + lane;
      static_cast<uint4*>(p.k)[to_page[r] * (p.k_page_stride >> 3) + at] = xk[t];
      static_cast<uint4*>(p.v)[to_page[r] * (p.v_page_stride >> 3) + at] = xv[t];
    }
  }
}

// In place: CTA x of a head has column x of its keys or values, the last one its weights.  Rows that stay lead the list
// (kept[i] = i) and are passed over.  kMoveFlight: rows of a thread in flight, 8 where the launch leaves SMs
// to spare and a CTA's own rate counts, 2 where many CTAs share them (one request of 4608 rows 36 us with 8, 42 with 2; 16
// prompts of 6000 to 14000 rows 209 with 8, 137 with 2: 32 registers, so that all its CTAs run as one wave).
template <int kMoveFlight>
__global__ void __launch_bounds__(kMoveThreads)
evict_move_kernel(const __grid_constant__ EvictParams p) {
  const int col = blockIdx.x, g = blockIdx.y, seq = blockIdx.z;
  grid_dep_wait();
  grid_dep_launch();
  const int n = p.n_keep[seq];
  if (n < 0) return;
  const PagedBatch& b = p.batch;
  if (col == 0 && g == 0 && threadIdx.x == 0) p.new_len[seq] = n;
  const int32_t* kept = kept_rows(p, seq, g);
  int first = 0;                                         // kept[i] - i never falls: the first row that moves
  for (int hi = n; first < hi;) {
    const int mid = (first + hi) >> 1;
    if (kept[mid] > mid) hi = mid; else first = mid + 1;
  }
  const int mask = (1 << b.page_shift) - 1;
  if (col == kMoveCols) {
    for (int i0 = first; i0 < n; i0 += kMoveThreads) {
      const int i = i0 + threadIdx.x;
      float x = 0.f;
      float* dst = nullptr;
      if (i < n) {
        const int src = kept[i], sp = page_of(b, seq, src), dp = page_of(b, seq, i);
        if (sp < b.n_pages && dp < b.n_pages) {
          x = p.w[((static_cast<long long>(sp) * p.n_kv + g) << b.page_shift) + (src & mask)];
          dst = p.w + ((static_cast<long long>(dp) * p.n_kv + g) << b.page_shift) + (i & mask);
        }
      }
      __syncthreads();
      if (dst) *dst = x;
    }
    return;
  }
  const bool is_v = col >= kMoveCols / 2;
  uint4* pool = static_cast<uint4*>(is_v ? p.v : p.k);
  const long long page_stride = (is_v ? p.v_page_stride : p.k_page_stride) >> 3;
  const int part = (col % (kMoveCols / 2)) * 4 + (threadIdx.x & 3);
  constexpr int kRows = kMoveThreads / 4;
  auto at = [&](int page, int row) -> uint4* { return pool + page * page_stride + (static_cast<long long>(row & mask) * p.n_kv + g) * 16 + part; };
  // where the rows of a batch come from and go to; the next batch's are looked up while this one's rows are on their way
  int src[kMoveFlight], sp[kMoveFlight], dp[kMoveFlight];
  auto look_up = [&](int i0) {
#pragma unroll
    for (int f = 0; f < kMoveFlight; ++f) {
      const int i = i0 + f * kRows + (threadIdx.x >> 2);
      src[f] = i < n ? kept[i] : -1;
    }
#pragma unroll
    for (int f = 0; f < kMoveFlight; ++f) {
      const int i = i0 + f * kRows + (threadIdx.x >> 2);
      sp[f] = src[f] >= 0 ? table_entry(b, seq, src[f]) : 0;
      dp[f] = src[f] >= 0 ? table_entry(b, seq, i) : 0;
    }
  };
  look_up(first);
  for (int i0 = first; i0 < n; i0 += kRows * kMoveFlight) {
    uint4 x[kMoveFlight];
    uint4* dst[kMoveFlight];
#pragma unroll
    for (int f = 0; f < kMoveFlight; ++f) {
      dst[f] = nullptr;
      if (src[f] >= 0) {
        const int from = checked_page(b, sp[f]), to = checked_page(b, dp[f]);
        if (from < b.n_pages && to < b.n_pages) {
          x[f] = *at(from, src[f]);
          dst[f] = at(to, i0 + f * kRows + (threadIdx.x >> 2));
        }
      }
    }
    look_up(i0 + kRows * kMoveFlight);
    __syncthreads();
#pragma unroll
    for (int f = 0; f < kMoveFlight; ++f)
      if (dst[f]) *dst[f] = x[f];
  }
}

}  // namespace

long long evict_copy_blocks(const EvictParams& p) {
  const long long rows = static_cast<long long>(p.batch.max_blocks) << p.batch.page_shift, n = p.budget < rows ? p.budget : rows;
  return (n < 1 ? 1 : (n + kMoveRows - 1) / kMoveRows) * p.n_kv;
}

cudaError_t init_evict() {
  return cudaFuncSetAttribute(evict_select_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              static_cast<int>(kSelKeep * 4 + sizeof(SelShared)));
}

cudaError_t launch_evict(const EvictParams& p, int n_sm, cudaStream_t st) {
  const int lists = p.per_head ? p.n_kv : 1;
  const long long rows = static_cast<long long>(p.batch.max_blocks) << p.batch.page_shift;
  // Few CTAs for short lists: what a CTA reads of the others' histograms grows with their number (24 KB each, the
  // longest step: one request of 4608 rows, eight lists, with all three 18.9 us with 8 CTAs, 15.0 with 2, then 13.8 with
  // 2, 16.0 with 1; 16 lists of 6000 to 14000 rows 115 with 8, 108 with 4).  The table's width is all that the host
  // knows of the lists: 4608 rows in a table of 16384 take 13.4, in one of 32768, with 8 CTAs, 16.3.
  const int n_cta = rows <= 8192 ? 2 : rows <= 16384 ? 4 : kSelCluster;
  const long long part = (rows + n_cta - 1) / n_cta;
  const int keep = static_cast<int>(part < kSelKeep ? (part + 3) & ~3ll : kSelKeep);
  const size_t smem = static_cast<size_t>(keep) * 4 + sizeof(SelShared);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(p.batch.n_seqs) * lists * n_cta);
  cfg.blockDim = dim3(kSelThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = n_cta;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, evict_select_kernel, p, keep, n_cta);
  if (e != cudaSuccess) return e;
  if (p.dst_table)
    return launch_after_previous(evict_copy_kernel, dim3(static_cast<unsigned>(evict_copy_blocks(p)), 1, p.batch.n_seqs),
                                 kMoveThreads, 0, st, p);
  const dim3 grid(kMoveCols + 1, p.n_kv, p.batch.n_seqs);
  const bool many = static_cast<long long>(grid.x) * grid.y * grid.z > 2ll * n_sm;
  return launch_after_previous(many ? evict_move_kernel<2> : evict_move_kernel<8>, grid, kMoveThreads, 0, st, p);
}

}  // namespace ilre
