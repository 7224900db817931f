// Attention over the 8-bit block cache (hero_block_attention): o = softmax(scale q K^T) V, causal in a sequence's new rows.
#include "block_attention.cuh"
#include "block_ring.cuh"
#include <cmath>

namespace hero {

// ------------------------------------------------------------------------------------------------------------------
// Few rows per key / value head (decode steps, drafts).  Every cached byte is read once and meets at most 24 query rows (25 to 32 rows
// are two tiles of 16, each of which reads it), so the kernel is built to keep loads in flight and the chains between them short;
// up to 8 rows it is bound by HBM, with 24 by the latency of 8 warps per SM (issue slots 36 %, DRAM 37 %, tensor pipe 30 %).  Each warp walks steps of 32
// tokens of its own (two halves of 16, each within a page) through a ring that bulk tensor copies fill: keys and values of a half are
// one box each of a map over [pages][heads][tokens][features], swizzled so that the fragment loads below do not collide.
// The operands need no transposition because a contraction's index may be permuted at will as long as both sides agree:
//   S^T [16 tokens x 8 rows] = K Q^T: lane (g, t) of mma.m16n8k16 holds features 64 c + 16 t .. + 15 of tokens g and g + 8 (one 16-byte
//       load each); the four k slots it has in step (c, j) stand for features 64 c + 16 t + 4 j .. + 3, for K and Q alike.
//   O^T [features x 8 rows] = V^T P^T: lane (g, t) holds DH / 8 consecutive features of tokens 2t, 2t + 1, 2t + 8, 2t + 9; rows g and g + 8
//       of M tile j stand for features (DH / 8) g + 2 j and + 1.  P^T is S^T's fragment, transposed by movmatrix.
// Rows are the N dimension (8, the smallest there is), so a single query row does not pad a tile to 16.  Codes become FP16
// exactly (INT8: byte permute into 1024 + u, subtract; e4m3: conversion instruction).  A query row is scaled by a power of two
// into FP16: a feature is off by at most 2^-39 of the row's largest (and exact from 2^-31 of it on).  The page's key scale multiplies the
// scores; the value scale enters P relative to the largest one the warp has met.  P is rounded to FP16, because the matrix instruction
// takes 16 bits on both sides and FP16 has eight times BF16's precision: half a step, 2^-11, for each probability, 2.0e-4 ->
// 2.9e-4 against 64 bits in F16 outputs (one token on 384), nothing in BF16 ones.  It is formed with a factor 2^11, so a probability times its
// page's relative scale is in FP16's normal range down to 2^-25 and rounded by 2^-36 of the largest value scale below that.  The
// running maximum moves only when a score exceeds it by more than 4 in the exponent (P <= 2^15), so that most steps need no
// reduction over tokens.
// Work is dealt out in units of one step of one (sequence, row tile, key / value head).  The lengths are on the device, so each CTA of
// one full GPU takes an equal, consecutive share of all units, whatever the lengths are: ragged batches, a long document
// and many short ones end at the same time.  A group of units cut by a share's end leaves partial results in the workspace (at
// most two per CTA), which a second kernel joins.  Short sequences take one CTA per group and no second kernel.
constexpr int ROWS_WARPS = 4;
constexpr int rows_ctas(int nt) { return nt == 3 ? 2 : 3; }   // resident per SM (NT = 3: 255 registers a thread)
// what a group costs beside its steps (page numbers and queries in, partial results joined and out), in steps; with too low a figure
// the share that holds a batch's shortest sequences ends last (4 for all: 116 us, these: 56 us on ragged drafts for 16 sequences; 45 and 39 on
// ragged steps for 32)
__host__ __device__ constexpr int rows_group_units(int nt) { return 8 + 5 * nt; }
constexpr int ROWS_MIN_UNITS = 16;              // units of a share, at least
constexpr int ROWS_KEPT = 256;                  // sequences whose lengths and rows a CTA keeps in shared memory while it walks its share
constexpr int ROWS_DIRECT_STEPS = 16;           // up to this many steps (512 tokens) a group is one CTA's

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// one half (16 tokens) of a page: box {DH, 16, 1, 1} of the map over {features, tokens of a page, heads, pages}
__device__ __forceinline__ void load_half(uint32_t dst, const CUtensorMap* m, int token, int head, int page, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(m)), "r"(0), "r"(token), "r"(head), "r"(page), "r"(bar) : "memory");
}

template <int DH, int NT>
struct RowsSmem {
  static constexpr int STAGES = DH == 128 ? 2 : 4;                          // ring depth in steps of 32 tokens
  static constexpr int HALF = 16 * DH;                                      // bytes of 16 keys (or values)
  static constexpr int STAGE = 4 * HALF;                                    // keys of both halves, values of both halves
  static constexpr int RING = STAGES * STAGE;                               // per warp; afterwards its partial O
  static constexpr int OROW = DH + 8;                                       // floats between rows of a partial O (no bank conflicts)
  static constexpr int PARTIAL = 8 * NT * OROW * 4;
  static constexpr int WARP = ((RING > PARTIAL ? RING : PARTIAL) + 1023) / 1024 * 1024;
  static constexpr int OFF_SCALES = ROWS_WARPS * WARP;                      // float2 [warps][stages][2]: key and value scale of a half
  static constexpr int OFF_BARS = OFF_SCALES + ROWS_WARPS * STAGES * 16;    // uint64 [warps][stages]
  static constexpr int OFF_ML = OFF_BARS + ROWS_WARPS * STAGES * 8;         // float [2][warps][8 NT]
  static constexpr int OFF_PLACE = OFF_ML + ROWS_WARPS * 8 * NT * 8 + 16;   // (behind them: float [warps]) Place, long long [warps], SeqRows [ROWS_KEPT]
  static constexpr int OFF_SEQ = OFF_PLACE + 80 + ROWS_WARPS * 8;
  static constexpr int BYTES = 1024 + OFF_SEQ + ROWS_KEPT * (int)sizeof(SeqRows);
};
// place of a feature in a partial O: rows of O^T in the order of the lanes that hold them
template <int DH>
__device__ __forceinline__ int feature_at(int place) { return (DH / 8) * ((place & 15) >> 1) + 2 * (place >> 4) + (place & 1); }

// units of row tile qt of a sequence for one key / value head: its steps and a constant (so rows without a token are written too)
template <int R>
__device__ __forceinline__ int tile_units(const SeqRows& s, int group, int qt) {
  const int total = s.n * group, last = (min((qt + 1) * R, total) - 1) / group;
  return ((max(s.len - s.n + last + 1, 0) + 31) >> 5) + rows_group_units(R / 8);
}
// A CTA's place in the work (in shared memory: nothing of it is held in registers through the loop over tokens).
struct Place {
  int b, qt, hk, len;            // the group; tokens of its sequence
  int n, total, units;           // rows of its sequence, the same times the group size, the group's units
  int ctas;                      // CTAs with a share
  long long r0;                  // first row
  long long first;               // units before the group
  long long unit, end, all;      // next unit and end of this CTA's share, units of the call
  template <int R>
  __device__ __forceinline__ void enter(const SeqRows& s, int group) {
    len = s.len; n = s.n; r0 = s.r0; total = s.n * group;
    units = tile_units<R>(s, group, qt);
  }
};
struct __align__(16) JoinRecord { int parts, share, group, pad; };   // a group cut into `parts`, from share `share` on; parts 0: not cut

template <int R>
__device__ __forceinline__ long long seq_units(const BlockView& c, int group, const SeqRows& s) {
  const int tiles = (s.n * group + R - 1) / R;
  long long u = 0;
  for (int qt = 0; qt < tiles; ++qt) u += tile_units<R>(s, group, qt);
  return u * c.nkv;
}

template <int DH, int NT, bool BF, bool F8>
__global__ void __launch_bounds__(ROWS_WARPS * 32, rows_ctas(NT)) block_attn_rows_kernel(const __grid_constant__ CUtensorMap tm_k,
                                                                             const __grid_constant__ CUtensorMap tm_v,
                                                                             const __grid_constant__ BlockAttnParams p) {
  using Smem = RowsSmem<DH, NT>;
  constexpr int STAGES = Smem::STAGES;
  constexpr int R = 8 * NT;                      // rows of a tile: (row of the sequence, query head of the group) pairs
  constexpr int KC = DH / 64;                    // 64-feature pieces of a key
  constexpr int VW = DH / 32;                    // words of a lane's value slice
  constexpr int MT = DH / 16;                    // M tiles of O^T
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  float* sm = reinterpret_cast<float*>(smem + Smem::OFF_ML);               // [warps][R] maxima
  float* sl = sm + ROWS_WARPS * R;                                         // [warps][R] sums
  float* refs = sl + ROWS_WARPS * R;                                       // [warps] largest value scales
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  uint64_t* full_bar = reinterpret_cast<uint64_t*>(smem + Smem::OFF_BARS) + warp * STAGES;
  float2* scales = reinterpret_cast<float2*>(smem + Smem::OFF_SCALES) + warp * STAGES * 2;
  if (lane == 0) {
#pragma unroll
    for (int i = 0; i < STAGES; ++i) ptx::mbar_init(&full_bar[i], 2);      // one arrival for each half
    ptx::fence_mbar_init();
  }
  __syncwarp();
  ptx::pdl_launch_dependents();
  ptx::pdl_wait();
  const BlockView& c = p.c;

  // ---- this CTA's share of the units and the group it begins in
  SeqRows* const kept = reinterpret_cast<SeqRows*>(smem + Smem::OFF_SEQ);
  auto sequence = [&](int b) { return b < ROWS_KEPT ? kept[b] : seq_rows(c, b); };
  Place& at = *reinterpret_cast<Place*>(smem + Smem::OFF_PLACE);
  static_assert(sizeof(Place) <= 80, "");
  if (p.direct) {
    const int b = blockIdx.x / c.nkv / p.tiles, qt = blockIdx.x / c.nkv % p.tiles;
    const SeqRows s = seq_rows(c, b);
    if (qt * R >= s.n * p.group) return;
    if (threadIdx.x == 0) {
      at.b = b; at.qt = qt; at.hk = blockIdx.x % c.nkv;
      at.enter<R>(s, p.group);
      at.first = at.unit = 0;
      at.end = at.units;
    }
  } else {
    long long* sums = reinterpret_cast<long long*>(smem + Smem::OFF_PLACE + 80);
    const int chunk = (p.B + ROWS_WARPS * 32 - 1) / (ROWS_WARPS * 32), b0 = min((int)threadIdx.x * chunk, p.B), b1 = min(b0 + chunk, p.B);
    long long own = 0, all = 0;
    for (int b = b0; b < b1; ++b) {
      const SeqRows s = seq_rows(c, b);
      if (b < ROWS_KEPT) kept[b] = s;
      own += seq_units<R>(c, p.group, s);
    }
    long long incl = own;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long x = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += x;
    }
    if (lane == 31) sums[warp] = incl;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < ROWS_WARPS; ++w) { if (w < warp) incl += sums[w]; all += sums[w]; }
    // (the lengths may be far below the host's bound: no share is empty and none is much below ROWS_MIN_UNITS)
    const long long ctas = min((long long)gridDim.x, max(all / ROWS_MIN_UNITS, 1ll));
    const long long unit = all * blockIdx.x / ctas, end = all * (blockIdx.x + 1) / ctas;
    if (blockIdx.x >= ctas || all == 0) {
      if (threadIdx.x == 0 && !p.by_group) p.records[blockIdx.x].parts = 0;
      return;
    }
    if (incl - own <= unit && unit < incl) {     // one thread: the sequence, then the row tile and head
      long long first = incl - own;
      int b = b0;
      for (;; ++b) {
        const long long n = seq_units<R>(c, p.group, sequence(b));
        if (unit < first + n) break;
        first += n;
      }
      const SeqRows s = sequence(b);
      at.b = b; at.unit = unit; at.end = end; at.all = all; at.ctas = (int)ctas;
      for (at.qt = 0;; ++at.qt) {
        at.enter<R>(s, p.group);
        if (unit < first + (long long)at.units * c.nkv) break;
        first += (long long)at.units * c.nkv;
      }
      at.hk = (int)((unit - first) / at.units);
      at.first = first + (long long)at.hk * at.units;
    }
  }
  __syncthreads();

  CopyRing<STAGES> ring;                         // its position and parity go on from group to group
  for (;;) {
    const int b = at.b, hk = at.hk, total = at.total, rb = at.qt * R;
    const int last = (min(rb + R, total) - 1) / p.group, base = at.len - at.n;
    const int L = max(base + last + 1, 0);       // keys of the tile's last row
    const int open = base + rb / p.group + 1;    // keys of its first row: steps below need no mask
    const int k0 = (int)min((long long)L, 32 * (at.unit - at.first)), k1 = (int)min((long long)L, 32 * (at.end - at.first));
    const int steps = (k1 - k0 + 31) >> 5, mine = ring.steps_of(steps > warp ? (steps - warp + ROWS_WARPS - 1) / ROWS_WARPS : 0);

    // lane i looks after half i % 2 of the warp's step i / 2 of every batch of 16: page id, scales, requests
    int my_token = 0, my_id = -1;
    float2 my_scales;
    auto load_pages = [&](int n0) {                // steps n0 .. n0 + 15 of the warp
      const int tok = k0 + 32 * (warp + ROWS_WARPS * (n0 + (lane >> 1))) + 16 * (lane & 1);
      my_id = -1;
      my_token = tok & (c.page - 1);
      my_scales = make_float2(0.f, 0.f);
      if (tok < k1) {
        my_id = page_for_read(c, b, tok >> c.page_shift);
        const long long sc = (long long)my_id * c.nkv + hk;
        my_scales = make_float2(written(c.ks + sc), written(c.vs + sc));
      }
    };
    const uint32_t ring_a = ptx::smem_u32(smem + warp * Smem::WARP);
    auto request = [&](int n, int stage) {         // step n of the warp into a stage
      if (n >= mine) return;
      if (n && (n & 15) == 0) load_pages(n);
      if ((lane >> 1) == (n & 15)) {
        const int h = lane & 1;
        if (my_id >= 0) {
          // (the copies are asked for before the scales have arrived; the bytes may be counted down before they are expected, the
          // phase cannot end without this lane's arrival, which also releases the scales)
          const uint32_t bar = ptx::smem_u32(&full_bar[stage]), dst = ring_a + stage * Smem::STAGE + h * Smem::HALF;
          load_half(dst, &tm_k, my_token, hk, my_id, bar);
          load_half(dst + 2 * Smem::HALF, &tm_v, my_token, hk, my_id, bar);
          scales[2 * stage + h] = my_scales;
          ptx::mbar_expect_tx(&full_bar[stage], 2 * Smem::HALF);
        } else {
          scales[2 * stage + h] = make_float2(0.f, 0.f);
          ptx::mbar_arrive(&full_bar[stage]);
        }
      }
    };
    load_pages(0);
    ring.open(request);

    // query fragments: lane (g, t) holds features 64 c + 16 t .. + 15 of row g of each N tile, scaled by a power of two
    uint32_t qf[NT][KC * 8];
    float f[NT][2], u[NT][2], l[NT][2], acc[NT][MT][4];
    int lim[NT][2];                                // per lane: rows 2 t and 2 t + 1 of each N tile (the columns of S^T and O^T it holds)
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int rr = min(rb + 8 * n + g, total - 1);
      const uint16_t* q = p.q + (at.r0 + rr / p.group) * p.ld_q + ((long long)hk * p.group + rr % p.group) * DH + 16 * t;
      uint32_t raw[KC * 8], top = 0;
#pragma unroll
      for (int k = 0; k < KC; ++k) {
        const uint4 x = written(reinterpret_cast<const uint4*>(q + 64 * k)), y = written(reinterpret_cast<const uint4*>(q + 64 * k + 8));
        raw[8 * k] = x.x; raw[8 * k + 1] = x.y; raw[8 * k + 2] = x.z; raw[8 * k + 3] = x.w;
        raw[8 * k + 4] = y.x; raw[8 * k + 5] = y.y; raw[8 * k + 6] = y.z; raw[8 * k + 7] = y.w;
      }
#pragma unroll
      for (int i = 0; i < KC * 8; ++i) top = __vmaxu2(top, raw[i] & 0x7fff7fffu);
      top = max(top & 0xffffu, top >> 16);
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const float amax = fp16ish_to_f32x2<BF>(top).x;
      const float up = query_factor(amax), down = p.c2 / up;
#pragma unroll
      for (int i = 0; i < KC * 8; ++i) {
        const float2 x = fp16ish_to_f32x2<BF>(raw[i]);
        qf[n][i] = pack_f16(x.x * up, x.y * up);
      }
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        f[n][r] = __shfl_sync(0xffffffffu, down, 4 * (2 * t + r));
        lim[n][r] = base + min(rb + 8 * n + 2 * t + r, total - 1) / p.group + 1;
        u[n][r] = 0.f; l[n][r] = 0.f;              // u = P_SHIFT - running maximum
      }
#pragma unroll
      for (int j = 0; j < MT; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[n][j][i] = 0.f;
    }
    float vref = 0.f, inv_vref = 0.f;
    // byte offsets of the lane's pieces within a half, under the swizzle (128-byte rows: 16-byte piece ^ row % 8; 64-byte rows:
    // piece ^ row / 2 % 4); rows g + 8 and 2 t + 8 lie 8 rows further with the same pattern
    uint32_t k_off[KC], v_off[2];
    if constexpr (DH == 128) {
#pragma unroll
      for (int q = 0; q < KC; ++q) k_off[q] = g * 128 + (((4 * q + t) ^ g) << 4);
#pragma unroll
      for (int r = 0; r < 2; ++r) v_off[r] = (2 * t + r) * 128 + ((g ^ (2 * t + r)) << 4);
    } else {
      k_off[0] = g * 64 + ((t ^ ((g >> 1) & 3)) << 4);
#pragma unroll
      for (int r = 0; r < 2; ++r) v_off[r] = (2 * t + r) * 64 + (((g >> 1) ^ t) << 4) + (g & 1) * 8;
    }

    auto wait = [&](bool go, int stage, uint32_t phase) {
      return __all_sync(0xffffffffu, go && ptx::mbar_wait(&full_bar[stage], phase, c.err, 0x7000 | stage)) != 0;
    };
    for (int n = 0; n < mine && ring.arrive(n, mine, wait); ++n) {
      const int stage = ring.stage, tb = k0 + 32 * (warp + ROWS_WARPS * n);
      const uint8_t* tile = smem + warp * Smem::WARP + stage * Smem::STAGE;
      const float4 sv = *reinterpret_cast<const float4*>(&scales[2 * stage]);   // key and value scale of either half
      // ---- scores, one chain of products per half and 64 features
      float sc[2][NT][4];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float part[KC][NT][4];
#pragma unroll
        for (int q = 0; q < KC; ++q) {
          const uint4 x = *reinterpret_cast<const uint4*>(tile + h * Smem::HALF + k_off[q]);
          const uint4 y = *reinterpret_cast<const uint4*>(tile + h * Smem::HALF + k_off[q] + 8 * DH);
          const uint32_t w0[4] = {x.x, x.y, x.z, x.w}, w1[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
          for (int r = 0; r < NT; ++r) part[q][r][0] = part[q][r][1] = part[q][r][2] = part[q][r][3] = 0.f;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t a0, a1, a2, a3;
            codes4_to_f16<F8>(w0[i], a0, a2);
            codes4_to_f16<F8>(w1[i], a1, a3);
#pragma unroll
            for (int r = 0; r < NT; ++r) mma_f16(part[q][r], a0, a1, a2, a3, qf[r][8 * q + 2 * i], qf[r][8 * q + 2 * i + 1]);
          }
        }
#pragma unroll
        for (int r = 0; r < NT; ++r)
#pragma unroll
          for (int i = 0; i < 4; ++i) sc[h][r][i] = KC == 2 ? part[0][r][i] + part[KC - 1][r][i] : part[0][r][i];
      }
      // ---- probabilities
      if (fmaxf(sv.y, sv.w) > vref) {              // uniform over the warp
        // (a normal number, so that its reciprocal is finite: BF16 values of 1e-37 have scales of 1e-39)
        const float now = fmaxf(fmaxf(sv.y, sv.w), 0x1p-126f), up = vref / now;
#pragma unroll
        for (int r = 0; r < NT; ++r)
#pragma unroll
          for (int k = 0; k < MT; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[r][k][i] *= up;
        vref = now;
        inv_vref = 1.0f / now;
      }
      const float rv[2] = {sv.y * inv_vref, sv.w * inv_vref};
      uint32_t pb[2][NT][2];
#pragma unroll
      for (int r = 0; r < NT; ++r) {
        float x[2][4];                             // score - maximum + P_SHIFT, base 2
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float f0 = f[r][0] * (h ? sv.z : sv.x), f1 = f[r][1] * (h ? sv.z : sv.x);
          x[h][0] = fmaf(sc[h][r][0], f0, u[r][0]); x[h][1] = fmaf(sc[h][r][1], f1, u[r][1]);
          x[h][2] = fmaf(sc[h][r][2], f0, u[r][0]); x[h][3] = fmaf(sc[h][r][3], f1, u[r][1]);
        }
        if (tb + 32 > open) {
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (tb + 16 * h + g + 8 * (i >> 1) >= lim[r][i & 1]) x[h][i] = -INFINITY;
        }
        float mx0 = fmaxf(fmaxf(x[0][0], x[0][2]), fmaxf(x[1][0], x[1][2])), mx1 = fmaxf(fmaxf(x[0][1], x[0][3]), fmaxf(x[1][1], x[1][3]));
        if (n == 0 || __any_sync(0xffffffffu, fmaxf(mx0, mx1) > P_SHIFT + MAX_SLACK)) {
#pragma unroll
          for (int o = 4; o < 32; o <<= 1) {
            mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, o));
            mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, o));
          }
          // the maximum moves by mx - P_SHIFT: up, except in the first step (and not at all where every token is masked)
          float d0 = mx0 - P_SHIFT, d1 = mx1 - P_SHIFT;
          if (n != 0) { d0 = fmaxf(d0, 0.f); d1 = fmaxf(d1, 0.f); }
          if (mx0 == -INFINITY) d0 = 0.f;
          if (mx1 == -INFINITY) d1 = 0.f;
          u[r][0] -= d0; u[r][1] -= d1;
          if (n != 0) {
            const float a0 = ex2(-d0), a1 = ex2(-d1);
            l[r][0] *= a0; l[r][1] *= a1;
#pragma unroll
            for (int k = 0; k < MT; ++k) { acc[r][k][0] *= a0; acc[r][k][2] *= a0; acc[r][k][1] *= a1; acc[r][k][3] *= a1; }
          }
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              // (a maximum beyond 2^26 is itself rounded by more than 4: without the bound a score of 2^27 left P at 2^16, beyond FP16)
              const float moved = x[h][i] - ((i & 1) ? d1 : d0);
              x[h][i] = moved > P_SHIFT + MAX_SLACK ? P_SHIFT + MAX_SLACK : moved;
            }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
          for (int i = 0; i < 4; ++i) x[h][i] = ex2(x[h][i]);
          l[r][0] += x[h][0] + x[h][2]; l[r][1] += x[h][1] + x[h][3];
          pb[h][r][0] = transpose8x8(pack_f16(x[h][0] * rv[h], x[h][1] * rv[h]));
          pb[h][r][1] = transpose8x8(pack_f16(x[h][2] * rv[h], x[h][3] * rv[h]));
        }
      }
      // ---- values; e4m3 slots behind the end may hold NaN, which a zero probability does not silence
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t vr[4][VW];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const uint8_t* at = tile + (2 + h) * Smem::HALF + v_off[r & 1] + (r >> 1) * 8 * DH;
          if constexpr (VW == 4) {
            const uint4 x = *reinterpret_cast<const uint4*>(at);
            vr[r][0] = x.x; vr[r][1] = x.y; vr[r][2] = x.z; vr[r][3] = x.w;
          } else {
            const uint2 x = *reinterpret_cast<const uint2*>(at);
            vr[r][0] = x.x; vr[r][1] = x.y;
          }
          if (F8 && tb + 32 > k1 && tb + 16 * h + 2 * t + (r & 1) + 8 * (r >> 1) >= k1) {
#pragma unroll
            for (int w = 0; w < VW; ++w) vr[r][w] = 0;
          }
        }
#pragma unroll
        for (int w = 0; w < VW; ++w) {
          uint32_t ab[4], cd[4];                   // feature i of the word: tokens (2t, 2t + 1) and (2t + 8, 2t + 9)
          codes4_to_f16<F8>(__byte_perm(vr[0][w], vr[1][w], 0x5140), ab[0], ab[1]);
          codes4_to_f16<F8>(__byte_perm(vr[0][w], vr[1][w], 0x7362), ab[2], ab[3]);
          codes4_to_f16<F8>(__byte_perm(vr[2][w], vr[3][w], 0x5140), cd[0], cd[1]);
          codes4_to_f16<F8>(__byte_perm(vr[2][w], vr[3][w], 0x7362), cd[2], cd[3]);
#pragma unroll
          for (int r = 0; r < NT; ++r) {
            mma_f16(acc[r][2 * w], ab[0], ab[1], cd[0], cd[1], pb[h][r][0], pb[h][r][1]);
            mma_f16(acc[r][2 * w + 1], ab[2], ab[3], cd[2], cd[3], pb[h][r][0], pb[h][r][1]);
          }
        }
      }
      __syncwarp();                                // every lane has read the stage
      ring.leave(n, request);
    }

    // ---- join the warps of the CTA; a warp's partial O takes the place of its ring (every copy it asked for has been waited for)
    float* my_o = reinterpret_cast<float*>(smem + warp * Smem::WARP);
    __syncwarp();
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int r = 0; r < 2; ++r) {
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) l[n][r] += __shfl_xor_sync(0xffffffffu, l[n][r], o);
        const int row = 8 * n + 2 * t + r;
        if (g == 0) { sm[warp * R + row] = l[n][r] != 0.f ? P_SHIFT - u[n][r] : -INFINITY; sl[warp * R + row] = l[n][r]; }
#pragma unroll
        for (int k = 0; k < MT; ++k)
          *reinterpret_cast<float2*>(my_o + row * Smem::OROW + 16 * k + 2 * g) = make_float2(acc[n][k][r], acc[n][k][2 + r]);
      }
    }
    if (lane == 0) refs[warp] = vref;
    const bool complete = __syncthreads_and(ring.ok);     // (a warp whose copies did not arrive, which is reported, has summed some keys only)
    const long long group_end = at.first + at.units;
    const bool head = at.unit == at.first, tail = group_end <= at.end, whole = head && tail;   // the group begins / ends in this share
    const long long slot = 2ll * blockIdx.x + (head ? 1 : 0);            // of a partial result: the group goes on / came in
    // Sums of P V are divided by the row's sum before the value scale enters: P carries up to 2^15 a key, so near the largest BF16 value FP32
    // holds the quotient alone, and near the smallest a scale divided by the row's sum would lose its bits.  The warps' weights carry
    // their scale relative to the largest.
    float ref = refs[0];
#pragma unroll
    for (int w = 1; w < ROWS_WARPS; ++w) ref = fmaxf(ref, refs[w]);
    if (threadIdx.x < R) {                       // one thread per row: the warps' weights, the tile's maximum and sum
      const int row = threadIdx.x;
      float mt = sm[row], lt = 0.f, e[ROWS_WARPS];
#pragma unroll
      for (int w = 1; w < ROWS_WARPS; ++w) mt = fmaxf(mt, sm[w * R + row]);
#pragma unroll
      for (int w = 0; w < ROWS_WARPS; ++w) {
        const float mw = sm[w * R + row];
        e[w] = mw > -INFINITY ? ex2(mw - mt) : 0.f;
        lt = fmaf(e[w], sl[w * R + row], lt);
      }
      const float inv = lt != 0.f ? 1.0f / lt : 0.f, inv_ref = ref > 0.f ? 1.0f / ref : 0.f;
#pragma unroll
      for (int w = 0; w < ROWS_WARPS; ++w) sm[w * R + row] = e[w] * inv * (refs[w] * inv_ref);
      // (a part that is not complete makes its rows NaN, a group that is not leaves them as they were)
      if (!whole && at.qt * R + row < at.total) p.part_ml[slot * R + row] = make_float2(part_maximum(complete, lt != 0.f, mt), lt);
    }
    __syncthreads();
    for (int i = complete ? threadIdx.x : R * DH; i < R * DH; i += ROWS_WARPS * 32) {
      const int row = i / DH, place = i % DH, rr = at.qt * R + row;
      if (rr >= at.total) break;                 // (rows ascend with i)
      float y = 0.f;
#pragma unroll
      for (int w = 0; w < ROWS_WARPS; ++w) y = fmaf(sm[w * R + row], reinterpret_cast<const float*>(smem + w * Smem::WARP)[row * Smem::OROW + place], y);
      y *= ref;
      if (whole) store_out(p, at.r0 + rr / p.group, (at.hk * p.group + rr % p.group) * DH + feature_at<DH>(place), y);
      else p.part_o[slot * (R * DH) + i] = y;
    }
    const bool done = group_end >= at.end;
    __syncthreads();                             // everybody has read the partial O and the place
    if (threadIdx.x == 0) {
      if (!p.direct && (p.by_group ? head : done)) {
        // the CTA that the group's last unit belongs to: shares are [all c / ctas, all (c + 1) / ctas)
        const int parts = head && !tail ? (int)((group_end * at.ctas - 1) / at.all) - (int)blockIdx.x + 1 : 0;
        const int group = (at.b * p.tiles + at.qt) * c.nkv + at.hk;
        p.records[p.by_group ? group : (int)blockIdx.x] = JoinRecord{parts, (int)blockIdx.x, group, 0};
      }
      if (!done) {
        at.unit = at.first = group_end;          // the next group: head, row tile, sequence
        if (++at.hk == c.nkv) {
          at.hk = 0;
          SeqRows s = SeqRows{at.len, at.n, at.r0};
          if (++at.qt * R >= at.total) {
            at.qt = 0;
            do s = sequence(++at.b); while (s.n == 0);   // (a unit is left, so a sequence with rows is)
          }
          at.enter<R>(s, p.group);
        }
      }
    }
    if (done) break;
    ptx::fence_proxy_async_smem();               // the partial O was written where copies will be
    __syncthreads();
  }
}

// joins the partial results of a group that was cut.  CTA (x, row) takes one row of the tile of group x, or, where there are more
// groups than shares, of the group that began in share x and went on.  What it costs is its chain of loads, so there are two links:
// the record beside the sequence's rows, then maxima, sums and values of all parts at once (dealt out to the warps, merged with a
// running maximum).
constexpr int JOIN_WARPS = 8, JOIN_MAX_PARTS = 1024;
template <int DH, int NT>
__global__ void __launch_bounds__(JOIN_WARPS * 32) block_attn_join_kernel(const __grid_constant__ BlockAttnParams p) {
  constexpr int R = 8 * NT, E = DH / 32;
  __shared__ float part[JOIN_WARPS][DH], ms[JOIN_WARPS], ls[JOIN_WARPS];
  // (not first thing, as elsewhere: CTAs of the next kernel that took up the SMs of this one's predecessor cost 64 against 54 us on two
  // sequences of 131072 tokens, step after step)
  ptx::pdl_wait();
  ptx::pdl_launch_dependents();
  JoinRecord rec;
  *reinterpret_cast<int4*>(&rec) = *reinterpret_cast<const int4*>(&p.records[blockIdx.x]);
  int b, qt, hk;
  if (p.by_group) {
    hk = blockIdx.x % p.c.nkv; qt = blockIdx.x / p.c.nkv % p.tiles; b = blockIdx.x / p.c.nkv / p.tiles;
  } else {
    if (rec.parts == 0) return;
    const int rest = rec.group / p.c.nkv;
    hk = rec.group % p.c.nkv; qt = rest % p.tiles; b = rest / p.tiles;
  }
  const SeqRows s = seq_rows(p.c, b);
  const int row = blockIdx.y, rr = qt * R + row, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (rr >= s.n * p.group || rec.parts == 0) return;               // (a record of rows that are not there was never written)
  float m = -INFINITY, l = 0.f, y[E];
#pragma unroll
  for (int e = 0; e < E; ++e) y[e] = 0.f;
  for (int q0 = warp; q0 < rec.parts; q0 += 8 * JOIN_WARPS) {
    float2 ml[8];
    float x[8][E];
#pragma unroll
    for (int k = 0; k < 8; ++k) {                // eight parts in flight per warp (behind the last one: that one again, without weight)
      const int q = min(q0 + k * JOIN_WARPS, rec.parts - 1);
      // the first part lies in the second slot of its CTA, the others in the first slots of the CTAs behind it
      const long long at = (2ll * (rec.share + q) + (q == 0 ? 1 : 0)) * R + row;
      ml[k] = written(p.part_ml + at);
      if constexpr (E == 4) {
        const float4 v = written(reinterpret_cast<const float4*>(p.part_o + at * DH) + lane);
        x[k][0] = v.x; x[k][1] = v.y; x[k][2] = v.z; x[k][3] = v.w;
      } else {
        const float2 v = written(reinterpret_cast<const float2*>(p.part_o + at * DH) + lane);
        x[k][0] = v.x; x[k][1] = v.y;
      }
    }
    float top = m;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (q0 + k * JOIN_WARPS >= rec.parts) ml[k] = make_float2(-INFINITY, 0.f);
      top = fmaxf(top, ml[k].x);
    }
    // (a part is divided by its own sum, so what is merged is their mean under weights that add up to one)
    const float base = top == -INFINITY ? 0.f : top;               // (parts without a key have no maximum)
    l *= ex2(m - base);
    m = top;
    float sum = l;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      ml[k].y *= ex2(ml[k].x - base);
      sum += ml[k].y;
    }
    const float inv = sum != 0.f ? __fdividef(1.0f, sum) : 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) y[e] *= l * inv;
    l = sum;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float f = ml[k].y * inv;
#pragma unroll
      for (int e = 0; e < E; ++e) y[e] = fmaf(f, x[k][e], y[e]);
    }
  }
#pragma unroll
  for (int e = 0; e < E; ++e) part[warp][lane * E + e] = y[e];
  if (lane == 0) { ms[warp] = m; ls[warp] = l; }
  __syncthreads();
  if (threadIdx.x < DH) {
    float mt = ms[0], o = 0.f, lt = 0.f, f[JOIN_WARPS];
#pragma unroll
    for (int w = 1; w < JOIN_WARPS; ++w) mt = fmaxf(mt, ms[w]);
    if (mt == -INFINITY) mt = 0.f;
#pragma unroll
    for (int w = 0; w < JOIN_WARPS; ++w) {
      f[w] = ex2(ms[w] - mt) * ls[w];
      lt += f[w];
    }
    const float inv = lt != 0.f ? __fdividef(1.0f, lt) : 0.f;
#pragma unroll
    for (int w = 0; w < JOIN_WARPS; ++w) o = fmaf(f[w] * inv, part[w][threadIdx.x], o);
    store_out(p, s.r0 + rr / p.group, (hk * p.group + rr % p.group) * DH + feature_at<DH>(threadIdx.x), o);
  }
}

// How a call is dealt out; the host knows upper bounds of lengths and rows only.
struct RowsPlan { int nt, tiles, ctas, records; bool direct, prompt, by_group; size_t bytes; };
static hero_status plan_rows(const hero_handle* h, const hero_block_cache* cc, int nq, int max_rows, RowsPlan* out) {
  const long long rows = (long long)max_rows * (nq / cc->nkv);
  RowsPlan r;
  // Up to 32 rows per key / value head this kernel, more the one for many.  us for 16 sequences of 6000 tokens (heads 32 / 8 of 128) here and
  // there: 24 rows 78 and 114, 32 rows 100 and 120, 36 rows 138 and 121, 64 rows 179 and 120; for 2 sequences of 32768: 32 rows 63 and 103,
  // 36 rows 85 and 104, 64 rows 109 and 104; 16 x 16 heads of 64 on 6000: 32 rows 120 and 189, 64 rows 204 and 186.
  r.prompt = rows > 32;
  if (r.prompt) {
    hero_status st = prompt_workspace_bytes(h, cc, nq, max_rows, &r.bytes);
    *out = r;
    return st;
  }
  // rows of a tile: 8, 16 or 24.  us on the same 16 sequences: 24 rows in one tile 78, in two of 16 97; 28 rows in two of 16 99, of 24 125
  r.nt = rows <= 8 ? 1 : rows > 16 && rows <= 24 ? 3 : 2;
  const long long tiles = (rows + 8 * r.nt - 1) / (8 * r.nt), groups = tiles * cc->nkv * cc->B, steps = ((long long)cc->max_len + 31) / 32;
  HERO_REQUIRE(groups <= (1ll << 30), HERO_ERR_UNSUPPORTED, "B=%d nkv=%d max_rows=%d: too many", cc->B, cc->nkv, max_rows);
  r.tiles = (int)tiles;
  r.direct = steps <= ROWS_DIRECT_STEPS;
  const long long slots = (long long)h->sm_count * rows_ctas(r.nt), full = slots < JOIN_MAX_PARTS ? slots : JOIN_MAX_PARTS, useful = (groups * (steps + rows_group_units(r.nt)) + ROWS_MIN_UNITS - 1) / ROWS_MIN_UNITS;
  r.ctas = (int)(r.direct ? groups : (full < useful ? full : useful));
  r.by_group = groups <= r.ctas;                 // the shorter list of candidates for a join
  r.records = r.by_group ? (int)groups : r.ctas;
  r.bytes = r.direct ? 0 : (size_t)r.ctas * 2 * 8 * r.nt * (cc->dh * 4 + 8) + (size_t)r.records * sizeof(JoinRecord);
  *out = r;
  return HERO_OK;
}

template <int DH, int NT>
static hero_status launch_rows(hero_handle* h, const hero_block_cache* cc, const BlockAttnParams& p, bool bf, int ctas, int records, cudaStream_t stream) {
  auto kern = bf ? (p.c.f8 ? block_attn_rows_kernel<DH, NT, true, true> : block_attn_rows_kernel<DH, NT, true, false>)
                 : (p.c.f8 ? block_attn_rows_kernel<DH, NT, false, true> : block_attn_rows_kernel<DH, NT, false, false>);
  constexpr int BYTES = RowsSmem<DH, NT>::BYTES;
  static PerDeviceOnce configured[4];            // per instantiation of the kernel
  PerDeviceOnce& once = configured[(bf ? 2 : 0) + (p.c.f8 ? 1 : 0)];
  if (!once.done(h->device)) {
    HERO_CUDA(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, BYTES));
    once.set(h->device);
  }
  CUtensorMap tm_k, tm_v;
  hero_status st;
  if ((st = make_tmap_pages(h, &tm_k, cc->k, cc, 16)) != HERO_OK || (st = make_tmap_pages(h, &tm_v, cc->v, cc, 16)) != HERO_OK) return st;
  {
    LaunchScope scope(h, stream, KERNEL_ATTN);
    HERO_CUDA(launch_dependent(kern, dim3((unsigned)ctas), dim3(ROWS_WARPS * 32), BYTES, stream, tm_k, tm_v, p));
  }
  if (!p.direct) {
    LaunchScope scope(h, stream, KERNEL_ATTN);
    HERO_CUDA(launch_dependent(block_attn_join_kernel<DH, NT>, dim3((unsigned)records, 8 * NT), dim3(JOIN_WARPS * 32), 0, stream, p));
  }
  return HERO_OK;
}

static hero_status attn_check(hero_handle* h, const hero_block_cache* cc, int32_t nq, int64_t rows, int32_t max_rows) {
  HERO_REQUIRE(h && cc, HERO_ERR_INVALID_ARG, "hero_block_attention: NULL handle or cache");
  HERO_REQUIRE(cc->nkv >= 1 && nq >= cc->nkv && nq % cc->nkv == 0 && nq <= 65535, HERO_ERR_INVALID_ARG, "nq=%d must be a multiple of nkv=%d", nq, cc->nkv);
  HERO_REQUIRE(rows >= 0 && max_rows >= 1, HERO_ERR_INVALID_ARG, "rows=%lld max_rows=%d", (long long)rows, max_rows);
  // (rows of a key / value head are numbered in 32 bits, up to a row tile behind the last one)
  HERO_REQUIRE((long long)max_rows * (nq / cc->nkv) <= (1ll << 30), HERO_ERR_UNSUPPORTED, "max_rows=%d with %d query heads each: more than 2^30 rows",
               max_rows, nq / cc->nkv);
  return HERO_OK;
}

}  // namespace hero

extern "C" hero_status hero_block_attention_workspace_bytes(hero_handle* h, const hero_block_cache* cc, int32_t nq, int64_t rows, int32_t max_rows,
                                                            size_t* bytes) {
  using namespace hero;
  HERO_REQUIRE(bytes != nullptr, HERO_ERR_INVALID_ARG, "hero_block_attention_workspace_bytes: bytes is NULL");
  *bytes = 0;
  hero_status st = attn_check(h, cc, nq, rows, max_rows);
  if (st != HERO_OK) return st;
  HERO_REQUIRE(cc->B >= 0 && cc->max_len >= 1 && (cc->dh == 64 || cc->dh == 128), HERO_ERR_UNSUPPORTED, "B=%d max_len=%d dh=%d", cc->B, cc->max_len, cc->dh);
  if (cc->B == 0) return HERO_OK;
  RowsPlan plan;
  if ((st = plan_rows(h, cc, nq, max_rows, &plan)) != HERO_OK) return st;
  // a call with a smaller row bound may be dealt out differently and need more: the answer serves it too
  size_t most = plan.bytes;
  for (int m = 1; m < max_rows && (long long)m * (nq / cc->nkv) <= 32; ++m) {
    RowsPlan fewer;                              // (a row bound that is refused needs nothing)
    if (plan_rows(h, cc, nq, m, &fewer) == HERO_OK && fewer.bytes > most) most = fewer.bytes;
  }
  if (plan.prompt) {
    const size_t fewer = prompt_workspace_most(h, cc, nq, max_rows);
    most = fewer > most ? fewer : most;
  }
  *bytes = most;
  return HERO_OK;
}

extern "C" hero_status hero_block_attention(hero_handle* h, const hero_block_cache* cc, const hero_block_attn_args* a, void* stream) {
  using namespace hero;
  HERO_REQUIRE(h && cc && a, HERO_ERR_INVALID_ARG, "hero_block_attention: NULL handle, cache or args");
  hero_status st = attn_check(h, cc, a->nq, a->q.rows, a->max_rows);
  if (st != HERO_OK) return st;
  BlockAttnParams p;
  if ((st = block_view(h, cc, a->row_start, a->q.rows, a->max_rows, &p.c)) != HERO_OK) return st;
  if ((st = check_matrix(a->q, "q")) != HERO_OK || (st = check_matrix(a->out, "out")) != HERO_OK) return st;
  const int64_t cols = (int64_t)a->nq * cc->dh;
  HERO_REQUIRE(is_fp16ish(a->q.dtype), HERO_ERR_UNSUPPORTED, "q: dtype %d: F16 or BF16", a->q.dtype);
  HERO_REQUIRE(a->q.cols == cols && a->out.cols == cols && a->out.rows == a->q.rows, HERO_ERR_INVALID_ARG, "q and out must be [rows, nq*dh = %lld]",
               (long long)cols);
  HERO_REQUIRE(is_fp16ish(a->out.dtype) || is_q8(a->out.dtype), HERO_ERR_UNSUPPORTED, "out: dtype %d: F16, BF16, I8 or F8", a->out.dtype);
  if (is_q8(a->out.dtype))
    HERO_REQUIRE((a->out.gran == HERO_GRAN_FWQ || a->out.gran == HERO_GRAN_SQ) && a->out.scale, HERO_ERR_INVALID_ARG,
                 "an 8-bit output carries a feature-wise or static scale");
  HERO_REQUIRE(std::isfinite(a->scale), HERO_ERR_INVALID_ARG, "scale must be finite");
  if (cc->B == 0 || a->q.rows == 0) return HERO_OK;
  if ((st = check_device(h)) != HERO_OK) return st;
  p.q = static_cast<const uint16_t*>(a->q.data); p.ld_q = a->q.ld;
  p.out = a->out.data; p.ld_out = a->out.ld; p.out_dt = a->out.dtype;
  p.out_scale = is_q8(a->out.dtype) ? a->out.scale : nullptr;
  p.out_scale_stride = a->out.gran == HERO_GRAN_FWQ ? 1 : 0;
  p.group = a->nq / cc->nkv;
  p.c2 = (float)((a->scale != 0.f ? (double)a->scale : 1.0 / std::sqrt((double)cc->dh)) * 1.4426950408889634);
  p.nq = a->nq;
  const bool bf = a->q.dtype == HERO_BF16;
  RowsPlan plan;
  if ((st = plan_rows(h, cc, a->nq, a->max_rows, &plan)) != HERO_OK) return st;
  HERO_REQUIRE(plan.bytes == 0 || (a->workspace && a->workspace_bytes >= plan.bytes), HERO_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed",
               a->workspace_bytes, plan.bytes);
  HERO_REQUIRE(plan.bytes == 0 || aligned16(a->workspace), HERO_ERR_ALIGNMENT, "the workspace must be 16-byte aligned");
  if (plan.prompt) return launch_prompt(h, cc, p, bf, a->workspace, static_cast<cudaStream_t>(stream));
  p.B = cc->B; p.tiles = plan.tiles; p.direct = plan.direct; p.by_group = plan.by_group;
  p.part_o = static_cast<float*>(a->workspace);
  p.part_ml = reinterpret_cast<float2*>(p.part_o + (size_t)plan.ctas * 2 * 8 * plan.nt * cc->dh);
  p.records = reinterpret_cast<JoinRecord*>(p.part_ml + (size_t)plan.ctas * 2 * 8 * plan.nt);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (cc->dh == 64)
    return plan.nt == 1 ? launch_rows<64, 1>(h, cc, p, bf, plan.ctas, plan.records, s) : plan.nt == 2 ? launch_rows<64, 2>(h, cc, p, bf, plan.ctas, plan.records, s)
                                                                         : launch_rows<64, 3>(h, cc, p, bf, plan.ctas, plan.records, s);
  return plan.nt == 1 ? launch_rows<128, 1>(h, cc, p, bf, plan.ctas, plan.records, s) : plan.nt == 2 ? launch_rows<128, 2>(h, cc, p, bf, plan.ctas, plan.records, s)
                                                                        : launch_rows<128, 3>(h, cc, p, bf, plan.ctas, plan.records, s);
}
