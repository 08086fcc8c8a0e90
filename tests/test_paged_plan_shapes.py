"""The split of a batch at the shapes that the kernels run with: every tile of query tokens that a group of 1 to 128 heads
gives, the kernels' key tiles and item costs, near lengths by counting, far ones by differences.  No GPU."""
import os
import re
import subprocess

from test_paged_plan import BODY, CSRC, CUDA

SHAPES = r"""
template <class Tiles>
void shape(std::mt19937& rng, int tq, int shift, int extra) {
  auto pick = [&](int lo, int hi) { return lo + static_cast<int>(rng() % static_cast<unsigned>(hi - lo + 1)); };
  for (int i = 0; i < 60; ++i) {                   // the first tiles one by one, whatever lies behind them
    const int n = pick(1, 900), kv = pick(0, 3) ? pick(1, 5000) : pick(1, 9);
    Tiles h{n, kv, tq, shift, extra};
    long long at = 0;
    for (int t = 0; t < h.n_qt(); ++t) {
      CHECK(h.before(t) == at);
      CHECK(h.key_tiles(t) >= 1);
      at += h.key_tiles(t) + extra;
    }
    CHECK(h.units() == at);
  }
  for (int i = 0; i < 60; ++i) {                   // far: neighbours, anywhere
    const int n = pick(0, 1) ? pick(1, 1 << 30) : pick(1, 3000), kv = pick(1, 3) > 1 ? 2147481599 - pick(0, 1 << 20) : pick(1, 1 << 30);
    Tiles h{n, kv, tq, shift, extra};
    for (int j = 0; j < 8; ++j) {
      const int t = pick(0, h.n_qt() - 1);
      const long long a = h.before(t), z = t + 1 < h.n_qt() ? h.before(t + 1) : h.units();
      CHECK(a >= 0 && z - a == h.key_tiles(t) + extra);
      CHECK(h.tile_of(a) == t && h.tile_of(z - 1) == t);
    }
  }
}
// by the definition: tile kt of 2^shift keys is seen by the row tiles whose last token sees its first key
void key_counts(std::mt19937& rng, int tq, int shift, int extra) {
  auto pick = [&](int lo, int hi) { return lo + static_cast<int>(rng() % static_cast<unsigned>(hi - lo + 1)); };
  for (int i = 0; i < 40; ++i) {
    KeyTiles h{pick(1, 900), pick(1, 5000), tq, shift, extra};
    for (int kt = 0; kt < h.n_qt(); ++kt) {
      int seen = 0;
      for (int r = 0; r * tq < h.n; ++r) seen += h.kv - h.n + std::min((r + 1) * tq, h.n) - 1 >= kt << shift;
      CHECK(seen == h.key_tiles(kt) && h.first(kt) == h.row_tiles() - seen);
    }
  }
}
"""

MAIN = r"""
int main() {
  std::mt19937 rng(11);
  for (int group = 1; group <= 128; ++group) {
    if (group <= 16) shape<HeadTiles>(rng, 16 / group, 6, 0);              // attention of few rows
    if (group <= 16) shape<HeadTiles>(rng, 16 / group, 7, 0);              // weights of few rows
    shape<HeadTiles>(rng, 2 * (128 / group), 7, @CHUNK@);                  // attention of chunks
    const int most = group <= 64 ? 64 / group : 1;
    for (int tq : {most, (most + 1) / 2, most > 2 ? most - 1 : 1}) {       // weights; fewer tokens where no sequence has more
      shape<KeyTiles>(rng, tq, 8, @WEIGHT@);
      key_counts(rng, tq, 8, @WEIGHT@);
    }
  }
  batches<Q>(rng);
  batches<K>(rng);
  std::printf("%d\n", bad);
  return bad != 0;
}
"""


def _constant(source, name):
    return re.search(r"constexpr int %s = (\d+);" % name, open(os.path.join(CSRC, source)).read()).group(1)


def test_the_kernels_shapes(tmp_path):
    wide = BODY[:BODY.index("int main()")]
    for old, new in (("tqs[] = {1, 2, 4, 16, 50, 64, 256}, tks[] = {6, 7}", "tqs[] = {1, 3, 5, 16, 42, 64, 256}, tks[] = {7, 8}"),
                     ("tks[rng() % 2], pick(0, 3)}", "tks[rng() % 2], pick(3, 6)}")):
        assert wide.count(old) == 1
        wide = wide.replace(old, new)
    main = MAIN.replace("@CHUNK@", _constant("paged_chunk_kernel.cu", "kItemUnits"))
    main = main.replace("@WEIGHT@", _constant("paged_weight_kernels.cu", "kItemUnits"))
    src, exe = tmp_path / "shapes.cpp", tmp_path / "shapes"
    src.write_text("#include <algorithm>\n" + wide + SHAPES + main)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=undefined", "-I", CSRC,
                           "-I", os.path.join(CUDA, "include"), "-x", "c++", str(src), "-o", str(exe)])
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-2000:]
