"""How the paged kernels split a batch: the header's arithmetic, compiled with the host compiler and
checked against counting.  No GPU."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2508_17892_b200", "csrc")
CUDA = os.environ.get("CUDA_HOME", "/usr/local/cuda")

BODY = r"""
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>
#include "paged_batch.cuh"
using namespace ilre;
static int bad = 0;
#define CHECK(c) do { if (!(c) && bad++ < 10) std::printf("line %d: %s\n", __LINE__, #c); } while (0)


const int tqs[] = {1, 2, 4, 16, 50, 64, 256}, tks[] = {6, 7};
struct Q : HeadTiles {
  Q(int n, int kv, int tq, int tk, int extra) : HeadTiles{n, kv, tq, tk, extra} {}
  static bool counts(int) { return true; }
};
struct K : KeyTiles {
  K(int n, int kv, int tq, int tk, int extra) : KeyTiles{n, kv, tq, tk, extra} {}
  static bool counts(int kv) { return kv > 0; }
};

template <class Tiles>
void batches(std::mt19937& rng) {
  auto pick = [&](int lo, int hi) { return lo + static_cast<int>(rng() % static_cast<unsigned>(hi - lo + 1)); };
  // whole batches: the shares of all CTAs cover every (sequence, head, query tile, key tile) once, in order; the
  // CTAs that an item's ends belong to are the ones that walk over them; sequences out of range get nothing
  for (int round = 0; round < 1500; ++round) {
    const int n = pick(1, 9), page_shift = pick(4, 7), max_blocks = pick(1, 40), max_q = pick(1, 90);
    const int most = max_blocks << page_shift;
    std::vector<int> q_start(n + 1, 0), kv(n), table(n * max_blocks, 0);
    for (int i = 0; i < n; ++i) {
      q_start[i + 1] = q_start[i] + (pick(0, 4) ? pick(0, max_q) : 0);
      kv[i] = pick(0, most);
      if (pick(0, 30) == 0) kv[i] = pick(0, 1) ? most + 1 : -1;
    }
    if (pick(0, 15) == 0) q_start[pick(0, n)] = pick(0, 1) ? -3 : 100000;
    int status = 0;
    PagedBatch b{n, pick(0, 5) ? q_start[n] : q_start[n] + 3, max_q, max_blocks, page_shift, 1, 0, 1 << 30, q_start.data(), kv.data(),
                 table.data(), &status};
    const TileShape ts{pick(1, 5), tqs[rng() % 7], tks[rng() % 2], pick(0, 3)};
    std::vector<long long> units(n), begin(n + 1, 0);
    for (int i = 0; i < n; ++i) {
      const long long len = static_cast<long long>(q_start[i + 1]) - q_start[i];
      const bool ok = q_start[i] >= 0 && len >= 0 && q_start[i + 1] <= b.n_tokens && len <= max_q && kv[i] >= 0 && kv[i] <= most;
      units[i] = seq_units<Tiles>(b, ts, i);
      CHECK(ok || units[i] == 0);
      CHECK(!ok || len == 0 || (units[i] > 0) == Tiles::counts(kv[i]));
      if (!ok) CHECK(status == kDevBadLengths);
      begin[i + 1] = begin[i] + units[i];
    }
    const long long total = begin[n];
    if (!total) continue;
    const int grid = pick(1, 60), n_cta = share_ctas(total, grid, pick(1, 4));
    CHECK(n_cta >= 1 && n_cta <= grid);
    long long u = 0;
    int seq = -1, head = 0, qt = 0, tile = 0, c_begin = 0;
    for (int c = 0; c < n_cta; ++c) {
      PlanStart s;
      s.total = total; s.n_cta = n_cta;
      s.u0 = share_begin(total, n_cta, c); s.u1 = share_begin(total, n_cta, c + 1);
      CHECK(s.u0 == u && s.u1 > s.u0);
      u = s.u1;
      int a = 0, z = 0;
      while (begin[a + 1] <= s.u0) ++a;
      while (begin[z + 1] < s.u1) ++z;
      s.first = locate<Tiles>(ts, a, load_span(b, a), units[a], begin[a], s.u0);
      s.last = locate<Tiles>(ts, z, load_span(b, z), units[z], begin[z], s.u1 - 1);
      PieceWalk<Tiles> w;
      std::vector<Piece> pieces;            // the last one comes first
      for (bool more = w.begin(b, ts, s); more; more = w.next(b, ts, s)) pieces.push_back(w.p);
      std::sort(pieces.begin(), pieces.end(), [](const Piece& x, const Piece& y) { return x.item < y.item; });
      for (const Piece& p : pieces) {
        CHECK(p.t0 < p.t1 && p.t1 <= p.n_tiles && p.item + ts.extra + p.t0 >= s.u0 && p.item + ts.extra + p.t1 <= s.u1);
        if (p.t0 == 0) {                    // a new item: the next in order
          CHECK(tile == 0);
          if (p.seq != seq) { CHECK(p.seq > seq && p.head == 0 && p.qt == 0); seq = p.seq; head = qt = 0; }
          CHECK(p.head == head && p.qt == qt);
          c_begin = c;
          // what the joining goes by
          const Item x{p.span, p.seq, p.head, p.qt, p.n_tiles, p.item};
          CHECK(share_of(total, n_cta, x.tiles_at(ts)) == c);
          const bool listed = s.last.tiles_at(ts) >= s.u0 && s.last.tiles_at(ts) < s.u1 && s.last.end(ts) > s.u1;
          CHECK((x.end(ts) > s.u1) == (listed && s.last.begin == p.item));
        } else {
          CHECK(p.t0 == tile && p.seq == seq && p.head == head && p.qt == qt && c > c_begin);
        }
        CHECK(share_of(total, n_cta, p.item + ts.extra + p.t0) == c && share_of(total, n_cta, p.item + ts.extra + p.t1 - 1) == c);
        tile = p.t1 == p.n_tiles ? 0 : p.t1;
        if (tile == 0) {
          Tiles h{p.span.n, p.span.kv, ts.tq, ts.tk_shift, ts.extra};
          if (++qt == h.n_qt()) { qt = 0; ++head; }
        }
      }
    }
    CHECK(u == total && tile == 0);
    int last = n - 1;
    while (units[last] == 0) --last;
    CHECK(seq == last && head == ts.heads && qt == 0);
  }
}

int main() {
  std::mt19937 rng(7);
  auto pick = [&](int lo, int hi) { return lo + static_cast<int>(rng() % static_cast<unsigned>(hi - lo + 1)); };
  // one head: units, their prefix sums and the tile of each unit
  for (int i = 0; i < 4000; ++i) {
    HeadTiles h{pick(1, 400), pick(0, 3) ? pick(0, 2000) : pick(0, 5), tqs[rng() % 7], tks[rng() % 2], pick(0, 1) * 3};
    long long at = 0;
    for (int qt = 0; qt < h.n_qt(); ++qt) {
      const int last = std::min((qt + 1) * h.tq, h.n), seen = h.kv - h.n + last;
      CHECK(h.key_tiles(qt) == (seen <= 0 ? 1 : (seen + (1 << h.tk_shift) - 1) >> h.tk_shift));
      CHECK(h.before(qt) == at);
      for (long long u = at; u < at + h.key_tiles(qt) + h.extra; u += 3) CHECK(h.tile_of(u) == qt);
      at += h.key_tiles(qt) + h.extra;
    }
    CHECK(h.units() == at);
  }
  // the same from the keys: the row tiles that see a key of the tile
  const int tts[] = {1, 2, 3, 18, 25, 32, 42, 128};
  for (int i = 0; i < 4000; ++i) {
    KeyTiles h{pick(1, 400), pick(1, 3) > 1 ? pick(1, 2000) : pick(1, 5), tts[rng() % 8], 7, pick(0, 1) * 3};
    long long at = 0;
    for (int kt = 0; kt < h.n_qt(); ++kt) {
      int seen = 0;
      for (int r = 0; r * h.tq < h.n; ++r) {
        const int last = std::min((r + 1) * h.tq, h.n) - 1;            // its last token sees the most
        if (h.kv - h.n + last >= kt * 128) ++seen;
      }
      CHECK(seen >= 1 && h.key_tiles(kt) == seen && h.first(kt) == h.row_tiles() - seen);
      CHECK(h.before(kt) == at);
      for (long long u = at; u < at + seen + h.extra; u += 3) CHECK(h.tile_of(u) == kt);
      at += seen + h.extra;
    }
    CHECK(h.units() == at);
  }
  // far lengths: no overflow
  HeadTiles far{1 << 30, 2147481000, 64, 7, 3};
  CHECK(far.units() > 0 && far.before(far.n_qt() - 1) < far.units());
  CHECK(far.tile_of(far.units() - 1) == far.n_qt() - 1);
  KeyTiles far_k{1 << 30, 2147481000, 18, 7, 3};
  CHECK(far_k.tile_of(far_k.units() - 1) == far_k.n_qt() - 1 && far_k.key_tiles(far_k.n_qt() - 1) >= 1);

  batches<Q>(rng);
  batches<K>(rng);
  // pages out of range
  int table[4] = {0, 5, -1, 2}, kv = 64, q0[2] = {0, 1}, status = 0;
  PagedBatch b{1, 1, 1, 4, 4, 5, 0, 1 << 30, q0, &kv, table, &status};
  CHECK(page_of(b, 0, 15) == 0 && page_of(b, 0, 63) == 2 && status == 0);
  CHECK(page_of(b, 0, 16) == 5 && status == kDevBadPage);
  status = 0;
  CHECK(page_of(b, 0, 32) == 5 && status == kDevBadPage);
  std::printf("%d\n", bad);
  return bad != 0;
}
"""


def test_shares_cover_every_unit_once(tmp_path):
    src, exe = tmp_path / "plan.cpp", tmp_path / "plan"
    src.write_text("#include <algorithm>\n" + BODY)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=undefined", "-I", CSRC,
                           "-I", os.path.join(CUDA, "include"), "-x", "c++", str(src), "-o", str(exe)])
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-2000:]
