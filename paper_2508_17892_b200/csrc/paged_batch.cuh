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

// Zeros below the lowest set bit of x > 0, at most `most`.
__host__ __device__ inline int low_zeros(int x, int most) {
#ifdef __CUDA_ARCH__
  const int z = __ffs(x) - 1;
#else
  const int z = __builtin_ctz(static_cast<unsigned>(x));
#endif
  return z < most ? z : most;
}

// One head of one sequence: n query tokens in tiles of `tq`, the last of them seeing all kv rows, keys in tiles
// of 2^tk_shift.  Every query tile has at least one key tile (a tile that sees nothing still writes its output).
// Lengths stay below 2^31 - 2048, so what a tile sees fits 32 bits; sums take 64.
//
// An item costs more than its key tiles (its queries arrive, its output leaves): `extra` units in front of them stand
// for that, so that CTAs with many short items get fewer tiles.
struct HeadTiles {
  int n, kv, tq, tk_shift, extra;
  __host__ __device__ int n_qt() const { return n <= tq ? (n > 0) : static_cast<int>(static_cast<unsigned>(n + tq - 1) / tq); }
  __host__ __device__ int key_tiles(int qt) const {
    const long long last = static_cast<long long>(qt + 1) * tq;
    const int seen = kv - n + (last < n ? static_cast<int>(last) : n);
    return seen <= 0 ? 1 : static_cast<int>((static_cast<unsigned>(seen) + (1u << tk_shift) - 1) >> tk_shift);
  }
  // Key tiles of the query tiles before qt <= n_qt() - 1.  Tile i behind those that see nothing counts
  // f(i) = (b + i tq) >> tk_shift, and with tq = odd 2^z: f(i) = (c + i odd) >> p_shift, c = b >> z.  Over a period of
  // P = 2^p_shift the remainders are each number below P once, so its sum is c + (odd - 1)(P - 1) / 2, and
  // f(i + P) = f(i) + odd: k whole periods in closed form and a rest of less than P terms (P is 2 for tq = 64 and 128 keys).
  __host__ __device__ long long before(int qt) const {
    if (qt == 0) return 0;
    const int pre = kv - n;
    const int blind = pre < 0 ? static_cast<int>(static_cast<unsigned>(-pre) / tq) : 0;  // tiles that see nothing
    if (blind >= qt) return static_cast<long long>(qt) * (1 + extra);
    const int z = low_zeros(tq, tk_shift), p_shift = tk_shift - z, P = 1 << p_shift, terms = qt - blind;
    const unsigned c = (static_cast<unsigned>(pre + (blind + 1) * tq) + (1u << tk_shift) - 1) >> z, odd = tq >> z;
    const int k = terms >> p_shift, r = terms & (P - 1);
    const long long whole = c + ((odd - 1) * (P - 1) >> 1);
    unsigned rest = 0;                     // less than 128 numbers below 2^25
    for (int i = 0; i < r; ++i) rest += (c + i * odd) >> p_shift;
    return blind + k * whole + static_cast<long long>(odd) * P * (static_cast<long long>(k) * (k - 1) / 2) + rest +
           static_cast<long long>(odd) * k * r + static_cast<long long>(qt) * extra;
  }
  __host__ __device__ bool empty() const { return n <= 0; }
  __host__ __device__ long long units() const {
    if (empty()) return 0;
    const int last = n_qt() - 1;
    return before(last) + key_tiles(last) + extra;
  }
  // the query tile that unit u of this head belongs to: the largest qt with before(qt) <= u
  __host__ __device__ int tile_of(long long u) const {
    int lo = 0, hi = n_qt() - 1;
    while (lo < hi) {
      const int mid = lo + (hi - lo + 1) / 2;
      if (before(mid) <= u) lo = mid; else hi = mid - 1;
    }
    return lo;
  }
};

// The same split seen from the keys, for sums over the query rows: an item is a tile of 2^tk_shift keys, its units are
// the tiles of `tq` query tokens that see any of them.  (The names are HeadTiles': "query tile" is the item's
// number, "key tiles" are its units.)
struct KeyTiles {
  int n, kv, tq, tk_shift, extra;
  __host__ __device__ int n_qt() const { return static_cast<int>((static_cast<unsigned>(kv) + (1u << tk_shift) - 1) >> tk_shift); }
  __host__ __device__ int row_tiles() const { return n <= tq ? 1 : static_cast<int>(static_cast<unsigned>(n + tq - 1) / tq); }
  // the first row tile that sees a key of tile kt
  __host__ __device__ int first(int kt) const {
    const int tok = (kt << tk_shift) - (kv - n);
    return tok <= 0 || n <= tq ? 0 : static_cast<int>(static_cast<unsigned>(tok) / tq);
  }
  __host__ __device__ int key_tiles(int kt) const { return row_tiles() - first(kt); }
  // Units of the key tiles before kt: all row tiles less those that see none, first(i) = (b + i 2^tk_shift) / tq from
  // key tile `seen` on; with tq = P 2^z and s = 2^(tk_shift - z) that is (c + i s) / P, c = b >> z, whose sum over a period
  // of P tiles is c + (s - 1)(P - 1) / 2 (the remainders are each number below P once; P = 1 where tq is a power of two).
  __host__ __device__ long long before(int kt) const {
    if (kt == 0) return 0;
    const int pre = kv - n;
    const int seen = pre <= 0 ? 0 : static_cast<int>((static_cast<unsigned>(pre) + (1u << tk_shift) - 1) >> tk_shift);
    const long long all = static_cast<long long>(kt) * (row_tiles() + extra);
    if (seen >= kt) return all;
    const int z = low_zeros(tq, tk_shift), P = tq >> z, s = 1 << (tk_shift - z), terms = kt - seen;
    const unsigned c = static_cast<unsigned>((seen << tk_shift) - pre) >> z;
    const int k = P == 1 ? terms : terms / P, r = terms - k * P;
    const long long whole = c + ((s - 1) * (P - 1) >> 1);
    long long rest = 0;
    for (int i = 0; i < r; ++i) rest += (c + static_cast<unsigned>(i) * s) / P;     // (no term where P = 1)
    return all - (k * whole + static_cast<long long>(s) * P * (static_cast<long long>(k) * (k - 1) / 2) + rest +
                  static_cast<long long>(s) * k * r);
  }
  __host__ __device__ bool empty() const { return n <= 0 || kv <= 0; }
  __host__ __device__ long long units() const {
    if (empty()) return 0;
    const int last = n_qt() - 1;
    return before(last) + key_tiles(last) + extra;
  }
  __host__ __device__ int tile_of(long long u) const {
    int lo = 0, hi = n_qt() - 1;
    while (lo < hi) {
      const int mid = lo + (hi - lo + 1) / 2;
      if (before(mid) <= u) lo = mid; else hi = mid - 1;
    }
    return lo;
  }
};

// x / d of positive numbers; a 64-bit division only where it needs one (it takes some hundred cycles).
__host__ __device__ inline long long div_pos(long long x, long long d) {
  if (((x | d) >> 32) == 0) return static_cast<unsigned>(x) / static_cast<unsigned>(d);
  return x / d;
}

// Shares: CTA b of n has the units [total b / n, total (b + 1) / n).
__host__ __device__ inline long long share_begin(long long total, int n, int b) { return div_pos(total * b, n); }
__host__ __device__ inline int share_of(long long total, int n, long long u) {
  return static_cast<int>(div_pos((u + 1) * n - 1, total));
}
// CTAs that get a share: all, or fewer so that none has less than min_units.
__host__ __device__ inline int share_ctas(long long total, int grid, int min_units) {
  const long long n = div_pos(total, min_units);
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

// Page of row t, n_pages (past the pool's end: a TMA load reads zeros there) if the table's entry is none.  In two
// steps for loops that ask for an entry well before they need it (the check waits for the load).
__host__ __device__ __forceinline__ int table_entry(const PagedBatch& b, int seq, int t) {
  return b.table[static_cast<long long>(seq) * b.max_blocks + (t >> b.page_shift)];
}
__host__ __device__ __forceinline__ int checked_page(const PagedBatch& b, int entry) {
  if (entry >= 0 && entry < b.n_pages) return entry;
  report(b.status, kDevBadPage);
  return b.n_pages;
}
__host__ __device__ __forceinline__ int page_of(const PagedBatch& b, int seq, int t) {
  return checked_page(b, table_entry(b, seq, t));
}

// Tiles of the batch's heads: `heads` work columns per sequence (kv heads, or parts of their groups).
struct TileShape {
  int heads, tq, tk_shift, extra;
};

template <class Tiles>
__host__ __device__ __forceinline__ long long head_units(const PagedBatch& b, const TileShape& ts, const SeqSpan& s) {
  return in_range(b, s.n) ? Tiles{s.n, s.kv, ts.tq, ts.tk_shift, ts.extra}.units() : 0;
}
template <class Tiles>
__host__ __device__ __forceinline__ long long seq_units(const PagedBatch& b, const TileShape& ts, int i) {
  return head_units<Tiles>(b, ts, load_span(b, i)) * ts.heads;
}

// The query tile of one head that a unit lies in.
struct Item {
  SeqSpan span;
  int seq, head, qt, n_tiles;              // n_tiles: key tiles
  long long begin;                         // its first unit
  int n_qt;                                // query tiles of the head
  __host__ __device__ long long tiles_at(const TileShape& ts) const { return begin + ts.extra; }
  __host__ __device__ long long end(const TileShape& ts) const { return begin + ts.extra + n_tiles; }
};

// The query tile of a head's unit, and the units before it.  On the device all lanes of a warp ask together and try 32
// tiles at a time.
template <class Tiles>
__host__ __device__ __forceinline__ int find_tile(const Tiles& t, long long u, long long* before) {
#ifdef __CUDA_ARCH__
  const int lane = threadIdx.x & 31;
  int lo = 0, n = t.n_qt();                // in [lo, lo + n)
  *before = 0;
  while (n > 1) {
    const int step = (n + 31) >> 5, qt = lo + lane * step;
    const long long mine = lane * step < n ? t.before(qt) : 0;
    const int k = 31 - __clz(__ballot_sync(0xFFFFFFFFu, lane * step < n && mine <= u));      // lane 0's is true
    *before = __shfl_sync(0xFFFFFFFFu, mine, k);
    n = min(step, n - k * step);
    lo += k * step;
  }
  return lo;
#else
  const int qt = t.tile_of(u);
  *before = t.before(qt);
  return qt;
#endif
}

// The item of unit `at` of the sequence `seq` of `per_head` units a head, the first of which is seq_begin.
template <class Tiles>
__host__ __device__ __forceinline__ Item locate_by_head(const TileShape& ts, int seq, const SeqSpan& span,
                                                        long long per_head, long long seq_begin, long long at) {
  Item x;
  x.seq = seq;
  x.span = span;
  const Tiles tiles{span.n, span.kv, ts.tq, ts.tk_shift, ts.extra};
  const long long off = at - seq_begin;
  x.head = static_cast<int>(div_pos(off, per_head));
  const long long in_head = off - x.head * per_head;
  long long before;
  x.qt = find_tile(tiles, in_head, &before);
  x.begin = at - in_head + before;
  x.n_tiles = tiles.key_tiles(x.qt);
  x.n_qt = tiles.n_qt();
  return x;
}

// The same of a sequence of `units` units.
template <class Tiles>
__host__ __device__ __forceinline__ Item locate(const TileShape& ts, int seq, const SeqSpan& span, long long units,
                                                long long seq_begin, long long at) {
  return locate_by_head<Tiles>(ts, seq, span, div_pos(units, ts.heads), seq_begin, at);
}

struct PlanStart {
  long long total;                         // units of the batch
  long long u0, u1;                        // this CTA's share (empty: u0 == u1)
  Item first, last;                        // the items of u0 and u1 - 1
  int n_cta;                               // CTAs that have a share
};

// A run of key tiles [t0, t1) of one item: what a CTA works on at a time.
struct Piece {
  SeqSpan span;
  int seq, head, qt;
  int t0, t1, n_tiles;                     // n_tiles: of the whole item
  long long item;                          // the item's first unit
};

// The pieces of a CTA's share: the last one first, then the others in order.  The last piece begins at its item's
// first keys and the first one usually goes on where another CTA's stops, so that in this order the CTAs that work
// on query tiles of one sequence pass over its keys side by side, and one of them brings each key tile into L2 for
// all (1024 tokens behind 31744 rows: in the order of the units 588 us, so 480).
template <class Tiles>
struct PieceWalk {
  long long u, end;                        // units that follow the current piece
  bool last;                               // the current piece is the share's last one
  int n_qt;
  Piece p;

  // Positions on the first piece; false if the share has none.
  __host__ __device__ __forceinline__ bool begin(const PagedBatch& b, const TileShape& ts, const PlanStart& s) {
    if (s.u0 >= s.u1) return false;
    last = true;
    end = s.u1;
    return open(ts, s.last, s.last.begin < s.u0 ? s.u0 : s.last.begin) || next(b, ts, s);
  }
  // The item from unit `at` on; false if the share has none of its tiles.
  __host__ __device__ __forceinline__ bool open(const TileShape& ts, const Item& x, long long at) {
    p.span = x.span; p.seq = x.seq; p.head = x.head; p.qt = x.qt; p.n_tiles = x.n_tiles; p.item = x.begin;
    n_qt = x.n_qt;
    return close(ts, at);
  }
  __host__ __device__ __forceinline__ bool close(const TileShape& ts, long long at) {
    const long long from = at - p.item - ts.extra, left = end - p.item - ts.extra;
    p.t0 = from > 0 ? static_cast<int>(from) : 0;
    p.t1 = left < 0 ? 0 : left < p.n_tiles ? static_cast<int>(left) : p.n_tiles;
    u = p.item + ts.extra + p.n_tiles;
    if (u > end) u = end;
    return p.t0 < p.t1;
  }
  __host__ __device__ __forceinline__ bool next(const PagedBatch& b, const TileShape& ts, const PlanStart& s) {
    if (last) {
      last = false;
      end = s.last.begin;
      if (s.u0 >= end) return false;
      if (open(ts, s.first, s.u0)) return true;
    }
    while (u < end) {
      if (++p.qt == n_qt) {
        p.qt = 0;
        if (++p.head == ts.heads) {
          p.head = 0;
          do {                             // units are left, so a sequence with work follows
            if (++p.seq >= b.n_seqs) return false;
            p.span = load_span(b, p.seq);
          } while (!in_range(b, p.span.n) || Tiles{p.span.n, p.span.kv, ts.tq, ts.tk_shift, ts.extra}.empty());
          n_qt = Tiles{p.span.n, p.span.kv, ts.tq, ts.tk_shift, ts.extra}.n_qt();
        }
      }
      p.item = u;
      p.n_tiles = Tiles{p.span.n, p.span.kv, ts.tq, ts.tk_shift, ts.extra}.key_tiles(p.qt);
      if (close(ts, u)) return true;
    }
    return false;
  }
};

}  // namespace ilre
