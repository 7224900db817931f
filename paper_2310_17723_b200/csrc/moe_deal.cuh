// How the products grouped by expert are dealt out (hero_moe_linear), apart from what copies and computes, so that it can be compiled for the host too
// and followed there over sizes that no test fills memory with.
#pragma once

#if defined(__CUDACC__)
#define HERO_MOE_FN __host__ __device__ __forceinline__
#else
#define HERO_MOE_FN inline
#endif

namespace hero {

// Rows of a tile: of a CTA pair, or of a single CTA.
template <bool PAIR>
struct MoeRows {
  static constexpr int MT = PAIR ? 256 : 32;              // at most
  static constexpr int ROWS = PAIR ? MT / 2 : MT;         // ... that a CTA loads
  static constexpr int STEP = PAIR ? 32 : 16;             // granularity of the N side
  static constexpr int WARPS = PAIR ? 8 : 2;              // warps that gather rows
  static constexpr int BOX = PAIR ? 64 : 16;              // rows of a copy where A is in order
};

HERO_MOE_FN int moe_least(int a, int b) { return a < b ? a : b; }

// A piece of work: rows of an expert (0: none) and a tile of features, or a part of it (single CTAs: part `part` of 1 << split parts).
struct MoeTile { int e, row0, rows, nt, part, split; };

// Row tiles of an expert with the sorted rows lo .. hi - 1 of R; -1: no such rows.  (The sum that would round up passes 32 bits for R near 2^31.)
template <bool PAIR>
HERO_MOE_FN int moe_tiles(int lo, int hi, int R) {
  constexpr int MT = MoeRows<PAIR>::MT;
  if (lo < 0 || hi < lo || hi > R) return -1;
  return (hi - lo) / MT + ((hi - lo) % MT != 0 ? 1 : 0);
}

// The launch's tiles are dealt out in rounds, one for each CTA (or pair).  Where the last round has tiles for a half or a quarter of them only, these are cut
// in two or four, each part for a CTA of its own: single CTAs by features (a part brings its share of the weights, which is what their
// time goes to), pairs by rows (a product over fewer rows takes less time, one over fewer features does not).
struct MoeDeal {
  const int* first; const int* tiles;         // first sorted row, first row tile of each expert (shared memory, [E + 1])
  int E, num_nt, full, split, units;          // tiles of the full rounds, parts (log2) of the others, units in all
  HERO_MOE_FN void init(int E_, int num_nt_, const int* first_, const int* tiles_, int groups) {
    first = first_; tiles = tiles_; E = E_; num_nt = num_nt_;
    const int all = tiles[E] * num_nt, rest = all % groups;
    full = all - rest;
    split = rest * 4 <= groups ? 2 : rest * 2 <= groups ? 1 : 0;
    units = full + (rest << split);
  }
  // the last expert whose first row tile is not behind rt; the whole warp calls
  HERO_MOE_FN int expert_of(int rt, int lane) const {
#if defined(__CUDA_ARCH__)
    // by sixteens, then among sixteen
    int base = 0;
    if (E > 32) base = 16 * (__popc(__ballot_sync(0xffffffffu, 16 * lane < E && tiles[moe_least(16 * lane, E)] <= rt)) - 1);
    const int e = base + lane;
    return base + __popc(__ballot_sync(0xffffffffu, (E <= 32 || lane < 16) && e < E && tiles[moe_least(e, E)] <= rt)) - 1;
#else
    int e = 0;
    while (e + 1 < E && tiles[e + 1] <= rt) ++e;
    return e;
#endif
  }
  // unit u < units; the whole warp calls
  template <bool PAIR>
  HERO_MOE_FN MoeTile at(int u, int lane) const {
    constexpr int STEP = MoeRows<PAIR>::STEP;
    MoeTile r;
    r.part = 0; r.split = 0;
    int t = u;
    if (u >= full) { r.split = split; t = full + ((u - full) >> split); r.part = (u - full) & ((1 << split) - 1); }
    const int rt = (int)((unsigned)t / (unsigned)num_nt);
    r.nt = t - rt * num_nt;
    r.e = expert_of(rt, lane);
    const int lo = first[r.e], n = first[r.e + 1] - lo, k = tiles[r.e + 1] - tiles[r.e], i = rt - tiles[r.e];
    // an even share of the expert's rows
    const int per = (int)(((k == 1 ? (unsigned)n : ((unsigned)n + (unsigned)k - 1) / (unsigned)k) + STEP - 1) / STEP * STEP);
    r.row0 = lo + i * per;
    r.rows = moe_least(per, n - i * per);     // may be 0 or less where a share rounds up: such a unit is skipped
    if (PAIR && r.split) {
      const int sub = (((r.rows + (1 << r.split) - 1) >> r.split) + STEP - 1) / STEP * STEP, skip = r.part * sub;
      r.rows = moe_least(sub, r.rows - skip);
      if (r.rows > 0) r.row0 += skip;
      r.part = r.split = 0;
    }
    return r;
  }
};

// Rows of a tile that a CTA loads, in groups of four: of a pair, each has half of the N side.  Every row warp takes part in every stage, with a group
// that nobody needs if there are too few: a warp without one could fall two uses of a stage behind, where a barrier's parity repeats.
struct MoeShare { int lo, n, fours; };        // first row in the tile, rows (0 or less: none), groups
template <bool PAIR>
HERO_MOE_FN MoeShare moe_share(const MoeTile& w, int rank) {
  constexpr int STEP = MoeRows<PAIR>::STEP, WARPS = MoeRows<PAIR>::WARPS;
  const int half = (w.rows + STEP - 1) / STEP * (STEP / (PAIR ? 2 : 1));
  MoeShare s;
  s.lo = rank * half;
  s.n = moe_least(half, w.rows - s.lo);
  const int fours = (s.n + 3) >> 2;
  s.fours = fours < WARPS ? WARPS : fours;
  return s;
}

}  // namespace hero
