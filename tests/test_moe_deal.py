"""How the products grouped by expert are dealt out (csrc/moe_deal.cuh), followed on the host: every row of every expert belongs to exactly one piece of work for
every feature, both CTAs of a pair load what the product of a piece reads, and nothing changes up to the most rows that 32 bits can number."""
import os
import random
import shutil
import subprocess

import pytest

from paper_2310_17723_b200 import build as B

HARNESS = r"""
#include "moe_deal.cuh"
#include <cstdio>
#include <cstdlib>
#include <vector>
using namespace hero;
// usage: deal <pair> <rows of the tensor> <feature tiles> <CTAs or pairs> <list: print pieces, sum: check that they follow one another> <offsets...>
template <bool PAIR> static int go(int R, int num_nt, int groups, bool list, int E, char** at) {
  using Rows = MoeRows<PAIR>;
  std::vector<int> first(E + 1), tiles(E + 1);
  int run = 0;
  for (int e = 0; e <= E; ++e) first[e] = atoi(at[e]);
  for (int e = 0; e < E; ++e) {
    const int k = moe_tiles<PAIR>(first[e], first[e + 1], R);
    tiles[e] = run;
    if (k < 0) printf("bad %d\n", e);
    else run += k;
  }
  tiles[E] = run;
  MoeDeal d;
  d.init(E, num_nt, first.data(), tiles.data(), groups);
  int next = first[0];
  long long pieces = 0;
  for (int u = 0; u < d.units; ++u) {
    const MoeTile w = d.at<PAIR>(u, 0);
    if (w.rows <= 0) continue;
    ++pieces;
    const int n = (w.rows + Rows::STEP - 1) / Rows::STEP * Rows::STEP;      // what the product reads
    if (w.rows > Rows::MT || n > Rows::MT) { printf("too many rows %d\n", w.rows); return 1; }
    int have = 0;
    for (int rank = 0; rank < (PAIR ? 2 : 1); ++rank) {
      const MoeShare s = moe_share<PAIR>(w, rank);
      if (s.n > 0) have += s.n;
      const int boxes = s.n > 0 ? (s.n + Rows::BOX - 1) / Rows::BOX * Rows::BOX : 0;
      if (s.lo != rank * n / 2 || s.fours * 4 < s.n || s.fours * 4 > Rows::ROWS || s.fours < Rows::WARPS || boxes > Rows::ROWS) { printf("share\n"); return 1; }
    }
    if (have != w.rows) { printf("shares bring %d of %d rows\n", have, w.rows); return 1; }
    if (list) printf("%d %d %d %d %d %d %d\n", u, w.e, w.row0, w.rows, w.nt, w.part, w.split);
    else if (w.row0 != next) { printf("piece %d begins at %d, not %d\n", u, w.row0, next); return 1; }
    next = w.row0 + w.rows;
  }
  if (!list) printf("%lld pieces up to row %d\n", pieces, next);
  return 0;
}
int main(int argc, char** argv) {
  const bool list = argv[5][0] == 'l';
  auto f = atoi(argv[1]) ? go<true> : go<false>;
  return f(atoi(argv[2]), atoi(argv[3]), atoi(argv[4]), list, argc - 7, argv + 6);
}
"""


@pytest.fixture(scope="module")
def deal(tmp_path_factory):
    d = tmp_path_factory.mktemp("deal")
    (d / "deal.cpp").write_text(HARNESS)
    compiler = shutil.which(os.environ.get("CXX", "g++"))
    assert compiler, "a C++ compiler is needed"
    subprocess.run([compiler, "-std=c++17", "-O2", "-Wall", "-Werror", "-ftrapv", "-I", B.CSRC, "-o", str(d / "deal"),
                    str(d / "deal.cpp")], check=True)

    def run(pair, R, num_nt, groups, how, offset):
        out = subprocess.run([str(d / "deal"), *map(str, (int(pair), R, num_nt, groups, how, *offset))], capture_output=True, text=True)
        assert out.returncode == 0, out.stdout + out.stderr
        return out.stdout.splitlines()
    return run


@pytest.mark.parametrize("pair", [False, True])
def test_every_row_belongs_to_one_piece_for_every_feature(deal, pair):
    g = random.Random(1)
    for _ in range(60):
        E, num_nt, groups = g.choice([1, 2, 7, 33, 64, 512]), g.randint(1, 9), g.choice([1, 3, 74, 296])
        counts = [g.choice([0, 1, 15, 16, 17, 31, 32, 33, 64, 255, 256, 257, g.randint(0, 1500)]) if g.random() < 0.7 else 0 for _ in range(E)]
        offset = [0]
        for c in counts:
            offset.append(offset[-1] + c)
        quarters = {}                                          # (feature tile, quarter) -> rows
        for line in deal(pair, offset[-1] + g.choice([0, 9]), num_nt, groups, "list", offset):
            u, e, row0, rows, nt, part, split = map(int, line.split())
            assert offset[e] <= row0 and row0 + rows <= offset[e + 1] and (split == 0 or not pair)
            for q in range(part * (4 >> split), (part + 1) * (4 >> split)):
                quarters.setdefault((nt, q), []).append((row0, rows))
        for nt in range(num_nt):
            for q in range(4):
                at = 0
                for row0, rows in sorted(quarters.get((nt, q), [])):
                    assert row0 == at
                    at += rows
                assert at == offset[-1]


MOST = 2 ** 31 - 1


@pytest.mark.parametrize("offset", [[0, MOST], [0, MOST - 255], [0, MOST - 256], [0, 5, MOST], [0, MOST - 5, MOST], [0, 0, MOST, MOST], [0, 2 ** 30 + 1, MOST - 100]])
@pytest.mark.parametrize("pair", [False, True])
def test_rows_up_to_the_last_that_32_bits_can_number(deal, pair, offset):
    mt = 256 if pair else 32
    words = deal(pair, MOST, 1, 1, "sum", offset)[-1].split()
    assert int(words[0]) == sum(-(-(b - a) // mt) for a, b in zip(offset, offset[1:])) and int(words[-1]) == offset[-1]


@pytest.mark.parametrize("pair", [False, True])
def test_rows_outside_the_tensor_are_no_work(deal, pair):
    assert deal(pair, 100, 1, 4, "list", [-1, 5])[0] == "bad 0"
    assert deal(pair, 100, 1, 4, "list", [0, 101])[0] == "bad 0"
    assert deal(pair, 100, 1, 4, "list", [50, 20, 20])[0] == "bad 0"
    assert len(deal(pair, 100, 1, 4, "list", [50, 20, 20])) == 1
    assert len(deal(pair, 100, 1, 1, "list", [0, 0])) == 0
