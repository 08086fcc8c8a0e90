// A batch over the paged cache as the kernels see it, and the arithmetic that splits its work.
//
// The lengths live on the device, so no launch knows them: every kernel is launched with a fixed grid and each
// CTA works out its share.  Work is counted in units (one tile of keys for one tile of query rows); the units of
// the whole batch, in the order (sequence, head, query tile, key tile), are cut into equal contiguous shares.
// A share begins and ends anywhere, so an item (one head's query tile) may be cut: its pieces leave partial
// results that are joined afterwards.  What is counted here must be counted alike by every role of every CTA.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace ilre {

// Sum of floor((a i + b) / m) for i = 0 .. n-1 (a, b >= 0, m >= 1): Euclid's algorithm on the lattice points
// below the line.
__host__ __device__ inline long long floor_sum(long long n, long long m, long long a, long long b) {
  long long ans = 0;
  while (true) {
    if (a >= m) { ans += n * (n - 1) / 2 * (a / m); a %= m; }
    if (b >= m) { ans += n * (b / m); b %= m; }
    const long long y = a * n + b;
    if (y < m) return ans;
    n = y / m;
    b = y % m;
    const long long t = m; m = a; a = t;
  }
}

// One head of one sequence: n query tokens in tiles of `tq`, the last of them seeing all kv rows, keys in tiles
// of `tk`.  Every query tile has at least one key tile (a tile that sees nothing still writes its output).
struct HeadTiles {
  int n, kv, tq, tk;
  __host__ __device__ int n_qt() const { return (n + tq - 1) / tq; }
  __host__ __device__ int key_tiles(int qt) const {
    const long long last = static_cast<long long>(qt + 1) * tq;
    const long long seen = static_cast<long long>(kv) - n + (last < n ? last : n);
    return seen <= 0 ? 1 : static_cast<int>((seen + tk - 1) / tk);
  }
  // key tiles of the query tiles before qt, qt <= n_qt() - 1
  __host__ __device__ long long before(int qt) const {
    const long long pre = static_cast<long long>(kv) - n;
    long long blind = pre < 0 ? -pre / tq : 0;            // tiles that see nothing
    if (blind > qt) blind = qt;
    return blind + floor_sum(qt - blind, tk, tq, pre + (blind + 1) * tq + tk - 1);
  }
  __host__ __device__ long long units() const {
    if (n <= 0) return 0;
    const int last = n_qt() - 1;
    return before(last) + key_tiles(last);
  }
  // the query tile that unit u of this head belongs to
  __host__ __device__ int tile_of(long long u) const {
    int lo = 0, hi = n_qt() - 1;                           // largest qt with before(qt) <= u
    while (lo < hi) {
      const int mid = lo + (hi - lo + 1) / 2;
      if (before(mid) <= u) lo = mid; else hi = mid - 1;
    }
    return lo;
  }
};

// Shares: CTA b of n has the units [total b / n, total (b + 1) / n).
__host__ __device__ inline long long share_begin(long long total, int n, int b) { return total * b / n; }
__host__ __device__ inline int share_of(long long total, int n, long long u) {
  return static_cast<int>(((u + 1) * n - 1) / total);
}
// CTAs that get a share: all, or fewer so that none has less than min_units.
__host__ __device__ inline int share_ctas(long long total, int grid, int min_units) {
  const long long n = total / min_units;
  return n < 1 ? 1 : n < grid ? static_cast<int>(n) : grid;
}

// Codes of the device status word beside those of the waits.
enum : int { kDevBadLengths = 32, kDevBadPage = 33 };

struct PagedBatch {
  int n_seqs, n_tokens, max_q_len, max_blocks;
  int page_shift;                          // log2(page_size)
  int n_pages;
  int q_from, q_to;                        // sequences of fewer or more new tokens are another kernel's
  const int32_t* q_start;
  const int32_t* kv_len;
  const int32_t* table;
  int* status;
};

struct SeqSpan {
  int q0, n, kv;                           // first token, new tokens, cached rows; n = 0 where out of range
};

// The first fault stays until the host reads it.
__host__ __device__ __forceinline__ void report(int* status, int code) {
#ifdef __CUDA_ARCH__
  atomicCAS(status, 0, code);
#else
  if (*status == 0) *status = code;
#endif
}

__host__ __device__ __forceinline__ SeqSpan load_span(const PagedBatch& b, int i) {
  const int a = b.q_start[i], e = b.q_start[i + 1], kv = b.kv_len[i];
  const bool ok = a >= 0 && e >= a && e <= b.n_tokens && e - a <= b.max_q_len && kv >= 0 &&
                  kv <= (static_cast<long long>(b.max_blocks) << b.page_shift);
  if (!ok) report(b.status, kDevBadLengths);
  return ok ? SeqSpan{a, e - a, kv} : SeqSpan{0, 0, 0};
}

__host__ __device__ __forceinline__ bool in_range(const PagedBatch& b, int n) { return n >= b.q_from && n <= b.q_to; }

// Page of row t, n_pages (past the pool's end: a TMA load reads zeros there) if the table's entry is none.
__host__ __device__ __forceinline__ int page_of(const PagedBatch& b, int seq, int t) {
  const int page = b.table[static_cast<long long>(seq) * b.max_blocks + (t >> b.page_shift)];
  if (page >= 0 && page < b.n_pages) return page;
  report(b.status, kDevBadPage);
  return b.n_pages;
}

// Tiles of the batch's heads: `heads` work columns per sequence (kv heads, or parts of their groups).
struct TileShape {
  int heads, tq, tk;
};

__host__ __device__ __forceinline__ long long seq_units(const PagedBatch& b, const TileShape& ts, int i) {
  const SeqSpan s = load_span(b, i);
  if (!in_range(b, s.n)) return 0;
  return HeadTiles{s.n, s.kv, ts.tq, ts.tk}.units() * ts.heads;
}

struct PlanStart {
  long long total;                         // units of the batch
  long long u0, u1;                        // this CTA's share (empty: u0 == u1)
  long long seq_begin;                     // first unit of sequence `seq`
  int seq;                                 // the sequence that u0 lies in
  int n_cta;                               // CTAs that have a share
};

// A run of key tiles [t0, t1) of one query tile of one head: what a CTA works on at a time.
struct Piece {
  SeqSpan span;
  int seq, head, qt;
  int t0, t1, n_tiles;                     // n_tiles: of the whole item
  long long item;                          // the item's first unit
};

// The pieces of a CTA's share, one after another.
struct PieceWalk {
  long long u, end;
  HeadTiles tiles;
  int n_qt;
  Piece p;

  // Positions on the first piece; false if the share is empty.
  __host__ __device__ __forceinline__ bool begin(const PagedBatch& b, const TileShape& ts, const PlanStart& s) {
    u = s.u0; end = s.u1;
    if (u >= end) return false;
    p.seq = s.seq;
    p.span = load_span(b, p.seq);
    tiles = HeadTiles{p.span.n, p.span.kv, ts.tq, ts.tk};
    n_qt = tiles.n_qt();
    const long long per_head = tiles.units(), off = u - s.seq_begin;
    p.head = static_cast<int>(off / per_head);
    const long long in_head = off - p.head * per_head;
    p.qt = n_qt == 1 ? 0 : tiles.tile_of(in_head);
    p.t0 = static_cast<int>(in_head - tiles.before(p.qt));
    p.item = u - p.t0;
    p.n_tiles = tiles.key_tiles(p.qt);
    close();
    return true;
  }
  __host__ __device__ __forceinline__ void close() {
    const long long left = end - p.item;
    p.t1 = left < p.n_tiles ? static_cast<int>(left) : p.n_tiles;
    u = p.item + p.t1;
  }
  __host__ __device__ __forceinline__ bool next(const PagedBatch& b, const TileShape& ts) {
    if (u >= end) return false;
    if (++p.qt == n_qt) {
      p.qt = 0;
      if (++p.head == ts.heads) {
        p.head = 0;
        do {                               // units are left, so a sequence with work follows
          if (++p.seq >= b.n_seqs) return false;
          p.span = load_span(b, p.seq);
        } while (p.span.n == 0 || !in_range(b, p.span.n));
        tiles = HeadTiles{p.span.n, p.span.kv, ts.tq, ts.tk};
        n_qt = tiles.n_qt();
      }
    }
    p.t0 = 0;
    p.item = u;
    p.n_tiles = tiles.key_tiles(p.qt);
    close();
    return true;
  }
};

}  // namespace ilre
