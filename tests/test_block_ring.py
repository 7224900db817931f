"""The order of a warp's copies in the few-rows attention over the block cache (csrc/block_ring.cuh), followed on the host: every copy
that was asked for is waited for before its stage is used again or the warp goes on, and after a wait that ran out nothing more is
asked for or computed, in that group and in all later ones."""
import os
import shutil
import subprocess

import pytest

from paper_2310_17723_b200 import build as B

HARNESS = r"""
#include "block_ring.cuh"
#include <cstdio>
#include <cstdlib>
// usage: ring <fail at wait number, -1: never> <steps of each group...>; prints one line per event
template <int STAGES> static void go(int fail, int groups, char** steps) {
  hero::CopyRing<STAGES> ring;
  int waits = 0;
  for (int g = 0; g < groups; ++g) {
    const int mine = ring.steps_of(atoi(steps[g]));
    auto request = [&](int n, int stage) { if (n < mine) printf("request %d %d %d\n", g, n, stage); };
    auto wait = [&](bool go, int stage, unsigned phase) {
      if (go) printf("wait %d %d %u\n", g, stage, phase);
      return go && waits++ != fail;
    };
    ring.open(request);
    for (int n = 0; n < mine && ring.arrive(n, mine, wait); ++n) {
      printf("step %d %d %d\n", g, n, ring.stage);
      ring.leave(n, request);
    }
    printf("group %d %d\n", g, ring.ok ? 1 : 0);
  }
}
int main(int argc, char** argv) {
  if (argc == 1) {
    for (int i = 0; i < 4; ++i) printf("%g\n", hero::part_maximum(i & 1, i & 2, -3.5f));
    return 0;
  }
  if (atoi(argv[1]) == 2) go<2>(atoi(argv[2]), argc - 3, argv + 3);
  else go<4>(atoi(argv[2]), argc - 3, argv + 3);
}
"""


@pytest.fixture(scope="module")
def ring(tmp_path_factory):
    d = tmp_path_factory.mktemp("ring")
    (d / "ring.cpp").write_text(HARNESS)
    compiler = shutil.which(os.environ.get("CXX", "g++"))
    assert compiler, "a C++ compiler is needed"
    subprocess.run([compiler, "-std=c++17", "-Wall", "-Werror", "-I", B.CSRC, "-o", str(d / "ring"), str(d / "ring.cpp")], check=True)

    def run(stages=None, fail=None, groups=()):
        if stages is None:
            return subprocess.run([str(d / "ring")], check=True, capture_output=True, text=True).stdout.split()
        out = subprocess.run([str(d / "ring"), str(stages), str(fail), *map(str, groups)], check=True, capture_output=True, text=True).stdout
        return [(w[0], *map(int, w[1:])) for w in (line.split() for line in out.splitlines())]
    return run


@pytest.mark.parametrize("stages", [2, 4])
@pytest.mark.parametrize("groups", [[0], [1], [3, 0, 1, 9], [7, 2, 4, 4, 1], [16, 33]])
def test_every_copy_is_waited_for_and_nothing_follows_a_wait_that_ran_out(ring, stages, groups):
    total = sum(groups)
    for fail in range(-1, total):
        at, phase = 0, 0                           # the ring's place: copies fill stages in order, each wait is for the oldest
        pending, stepped, waits, dead = [], [], 0, False
        for what, g, *rest in ring(stages, fail, groups):
            if what == "request":
                n, stage = rest
                assert not dead and len(pending) < stages
                assert stage not in [s for _, s in pending]
                pending.append(((g, n), stage))
            elif what == "wait":
                stage, parity = rest
                assert pending and (stage, parity) == (at, phase) and pending[0][1] == stage
                waiting = pending.pop(0)
                at, phase = (at + 1) % stages, phase ^ (at + 1 == stages)
                dead = dead or waits == fail
                waits += 1
            elif what == "step":
                assert not dead and ((g, rest[0]), rest[1]) == waiting
                stepped.append((g, rest[0]))
            else:
                assert not pending and rest == [0 if dead else 1]
        want = [(g, n) for g, steps in enumerate(groups) for n in range(steps)]
        assert stepped == (want if fail < 0 else want[:fail])


def test_a_part_that_is_not_complete_makes_its_row_nan_whatever_the_workspace_held(ring):
    # (complete, seen) = (0, 0), (1, 0), (0, 1), (1, 1)
    parts = [float(x) for x in ring()]
    assert parts[0] != parts[0] and parts[2] != parts[2] and parts[1] == -float("inf") and parts[3] == -3.5
