// The order of a warp's copies through its ring of shared-memory stages, and what becomes of a part of a row's keys, apart from what moves and
// what is computed, so that both can be compiled for the host too and followed there through waits that run out.
#pragma once
#include <cmath>

#if defined(__CUDACC__)
#define HERO_RING_FN __host__ __device__ __forceinline__
#else
#define HERO_RING_FN inline
#endif

namespace hero {

// A group is `steps` copies, of which up to STAGES are in flight.  Position and parity go on from group to group.  wait(go, stage, parity)
// is false where a copy did not arrive within its bound (and, without waiting, where go is false); from then on the warp asks for
// nothing and computes nothing (ok is false): the copies that it had asked for are waited for, each within its bound, before its stages
// are put to another use.  request(n, stage) does nothing for n >= steps.
template <int STAGES>
struct CopyRing {
  int stage = 0;
  unsigned phase = 0;
  bool ok = true;

  HERO_RING_FN void advance() {
    if (++stage == STAGES) { stage = 0; phase ^= 1; }
  }
  // the steps that a group of so many is to have
  HERO_RING_FN int steps_of(int steps) const { return ok ? steps : 0; }
  // the group's first copies
  template <class Request>
  HERO_RING_FN void open(Request request) const {
#if defined(__CUDACC__)
#pragma unroll
#endif
    for (int i = 0; i < STAGES; ++i) request(i, (stage + i) % STAGES);
  }
  // before step n: false where its copy did not arrive, and the group ends there
  template <class Wait>
  HERO_RING_FN bool arrive(int n, int steps, Wait wait) {
    ok = wait(ok, stage, phase);
    if (ok) return true;
    for (int i = 1; i < STAGES && n + i < steps; ++i) {
      advance();
      wait(true, stage, phase);
    }
    return false;
  }
  // after step n, once its stage has been read
  template <class Request>
  HERO_RING_FN void leave(int n, Request request) {
    request(n + STAGES, stage);
    advance();
  }
};

// What a part of a row's keys tells the join beside its sum: its maximum; minus infinity where the row saw none of them; NaN, which makes the
// row NaN, where copies or products did not arrive, so that what the workspace happened to hold is never taken for a result.
HERO_RING_FN float part_maximum(bool complete, bool seen, float maximum) { return complete ? (seen ? maximum : -INFINITY) : NAN; }

}  // namespace hero
