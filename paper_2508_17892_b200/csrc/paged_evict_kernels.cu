// Eviction: of the rows between the sinks and the recent ones the `middle` rows of largest weight (equal weights:
// the lower row), then the kept rows' way to the front.
//
// Selection: one CTA per list (a kv head of a sequence, or a sequence).  The weights' bits order as unsigned numbers
// (after a monotone map), so the threshold is found a byte at a time from histograms; the rows above it and the
// first rows equal to it are written in ascending order from prefix counts.
//
// Compaction: the kept rows ascend, so kept row i comes from a row >= i and rows may move to the front in place
// as long as no row is written before every row up to it has been read.  A CTA has one 64-byte column of the
// keys or values of one head (columns are independent) and goes through the rows in ascending batches: all
// reads of a batch, a barrier, all its writes.  Later batches read at or behind their own begin only.
#include "launch.cuh"
#include "paged_weight_kernels.cuh"

namespace ilre {

namespace {

constexpr int kSelThreads = 1024;
constexpr int kMoveThreads = 256;
constexpr int kMoveFlight = 8;                           // rows of a thread in flight
constexpr int kMoveCols = 8;                             // CTAs of a head: 4 columns of keys, 4 of values

// Row t's key: larger is heavier; the sum over the heads is formed in double and rounded once, so its value does
// not hang on an order.
__device__ __forceinline__ uint32_t weight_key(const EvictParams& p, int seq, int list, int t) {
  const int page = page_of(p.batch, seq, t);
  if (page >= p.batch.n_pages) return 0;
  const int row = t & ((1 << p.batch.page_shift) - 1);
  const float* w = p.w + ((static_cast<long long>(page) * p.n_kv) << p.batch.page_shift) + row;
  float x;
  if (p.per_head) {
    x = w[static_cast<long long>(list) << p.batch.page_shift];
  } else {
    double s = 0.0;
    for (int g = 0; g < p.n_kv; ++g) s += w[static_cast<long long>(g) << p.batch.page_shift];
    x = static_cast<float>(s);
  }
  return isnan(x) ? 0xFFFFFFFFu : float_to_ordered(x + 0.f);
}

__global__ void __launch_bounds__(kSelThreads)
evict_select_kernel(const EvictParams p) {
  __shared__ uint32_t hist[256];
  __shared__ uint32_t s_prefix, s_need;
  __shared__ int wsum[2][32];
  const int lists = p.per_head ? p.n_kv : 1;
  const int seq = blockIdx.x / lists, list = blockIdx.x % lists;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  grid_dep_wait();
  int32_t* kept = p.kept + static_cast<long long>(blockIdx.x) * p.budget;
  const int kv = p.batch.kv_len[seq];
  const bool ok = kv >= 0 && kv <= (static_cast<long long>(p.batch.max_blocks) << p.batch.page_shift);
  if (!ok && threadIdx.x == 0) report(p.batch.status, kDevBadLengths);
  const int n_keep = ok ? min(kv, p.budget) : 0;
  if (threadIdx.x == 0 && list == 0) p.n_keep[seq] = ok ? n_keep : -1;
  if (!ok || kv <= p.budget) {
    for (int i = threadIdx.x; i < p.budget; i += kSelThreads) kept[i] = i < n_keep ? i : -1;
    return;
  }
  const int lo = p.n_sink, hi = kv - p.n_recent, want = p.budget - p.n_sink - p.n_recent;
  uint32_t prefix = 0;
  int need = want;                                       // rows still to take among those with this prefix
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = threadIdx.x; i < 256; i += kSelThreads) hist[i] = 0;
    __syncthreads();
    for (int t = lo + threadIdx.x; t < hi; t += kSelThreads) {
      const uint32_t key = weight_key(p, seq, list, t);
      if (shift == 24 || (key >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(key >> shift) & 255u], 1u);
    }
    __syncthreads();
    if (threadIdx.x == 0) {
      uint32_t left = need;
      int bin = 255;
      while (bin > 0 && hist[bin] < left) left -= hist[bin--];
      s_prefix = prefix | (static_cast<uint32_t>(bin) << shift);
      s_need = left;
    }
    __syncthreads();
    prefix = s_prefix;
    need = s_need;
    __syncthreads();
  }
  // ascending output: sinks, the middle rows above the threshold or among the first `need` equal to it, recent rows
  for (int i = threadIdx.x; i < p.n_sink; i += kSelThreads) kept[i] = i;
  for (int i = threadIdx.x; i < p.n_recent; i += kSelThreads) kept[p.budget - p.n_recent + i] = hi + i;
  int above = 0, equal = 0;                              // rows before this round's, of either kind
  for (int t0 = lo; t0 < hi; t0 += kSelThreads) {
    const int t = t0 + threadIdx.x;
    const uint32_t key = t < hi ? weight_key(p, seq, list, t) : 0;
    const bool is_above = t < hi && key > prefix, is_equal = t < hi && key == prefix;
    const uint32_t ma = __ballot_sync(0xFFFFFFFFu, is_above), me = __ballot_sync(0xFFFFFFFFu, is_equal);
    if (lane == 0) { wsum[0][warp] = __popc(ma); wsum[1][warp] = __popc(me); }
    __syncthreads();
    int a = above, e = equal;
    for (int w = 0; w < 32; ++w) {
      if (w < warp) { a += wsum[0][w]; e += wsum[1][w]; }
      above += wsum[0][w]; equal += wsum[1][w];
    }
    const uint32_t below = (1u << lane) - 1u;
    a += __popc(ma & below);
    e += __popc(me & below);
    if (is_above || (is_equal && e < need)) kept[p.n_sink + a + min(e, need)] = t;
    __syncthreads();
  }
}

__global__ void __launch_bounds__(kMoveThreads)
evict_move_kernel(const EvictParams p) {
  const int col = blockIdx.x, g = blockIdx.y, seq = blockIdx.z;
  grid_dep_wait();
  const int n = p.n_keep[seq];
  if (n < 0) return;
  const PagedBatch& b = p.batch;
  const int32_t* kept = p.kept + (static_cast<long long>(seq) * (p.per_head ? p.n_kv : 1) + (p.per_head ? g : 0)) * p.budget;
  const bool in_place = p.dst_table == nullptr;
  const int mask = (1 << b.page_shift) - 1;
  auto dst_page = [&](int i) -> int {
    if (in_place) return page_of(b, seq, i);
    const int page = p.dst_table[static_cast<long long>(seq) * p.dst_blocks + (i >> b.page_shift)];
    if (page >= 0 && page < b.n_pages) return page;
    report(b.status, kDevBadPage);
    return b.n_pages;
  };
  const bool is_v = col >= kMoveCols / 2;
  uint4* pool = static_cast<uint4*>(is_v ? p.v : p.k);
  const long long page_stride = (is_v ? p.v_page_stride : p.k_page_stride) >> 3;
  const int part = (col % (kMoveCols / 2)) * 4 + (threadIdx.x & 3);
  constexpr int kRows = kMoveThreads / 4;
  auto at = [&](int page, int row) -> uint4* { return pool + page * page_stride + (static_cast<long long>(row & mask) * p.n_kv + g) * 16 + part; };
  for (int i0 = 0; i0 < n; i0 += kRows * kMoveFlight) {
    uint4 x[kMoveFlight];
    uint4* dst[kMoveFlight];
#pragma unroll
    for (int f = 0; f < kMoveFlight; ++f) {
      const int i = i0 + f * kRows + (threadIdx.x >> 2);
      dst[f] = nullptr;
      if (i < n) {
        const int src = kept[i];
        if (!in_place || src != i) {
          const int sp = page_of(b, seq, src), dp = dst_page(i);
          if (sp < b.n_pages && dp < b.n_pages) { x[f] = *at(sp, src); dst[f] = at(dp, i); }
        }
      }
    }
    __syncthreads();
#pragma unroll
    for (int f = 0; f < kMoveFlight; ++f)
      if (dst[f]) *dst[f] = x[f];
  }
  if (col != 0) return;
  // the weights of this head, in the same manner
  if (g == 0 && threadIdx.x == 0) p.new_len[seq] = n;
  for (int i0 = 0; i0 < n; i0 += kMoveThreads) {
    const int i = i0 + threadIdx.x;
    float x = 0.f;
    float* dst = nullptr;
    if (i < n) {
      const int src = kept[i], sp = page_of(b, seq, src), dp = dst_page(i);
      if (sp < b.n_pages && dp < b.n_pages) {
        x = p.w[((static_cast<long long>(sp) * p.n_kv + g) << b.page_shift) + (src & mask)];
        dst = p.w + ((static_cast<long long>(dp) * p.n_kv + g) << b.page_shift) + (i & mask);
      }
    }
    __syncthreads();
    if (dst) *dst = x;
  }
}

}  // namespace

cudaError_t launch_evict(const EvictParams& p, int n_sm, cudaStream_t st) {
  (void)n_sm;
  const int lists = p.per_head ? p.n_kv : 1;
  evict_select_kernel<<<p.batch.n_seqs * lists, kSelThreads, 0, st>>>(p);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  evict_move_kernel<<<dim3(kMoveCols, p.n_kv, p.batch.n_seqs), kMoveThreads, 0, st>>>(p);
  return cudaGetLastError();
}

}  // namespace ilre
