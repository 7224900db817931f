// Products grouped by expert (hero_moe_linear): GeMM^quant (Eq. 14, 28-30, 32) of each expert's rows with that expert's weights, over groups whose
// sizes only the device knows.
//
// The operands change sides on the tensor core: 128 output features (rows of W) are the M side of a product and the rows of an
// expert its N side, which an instruction may have in any multiple of 16 (of a CTA pair: 32).  A group of 17 rows then costs 32 columns and
// not a tile of 128 or 256 rows, and the accumulator's lane is a feature, so that the scale, bias and output factor of a thread are three
// registers and the row factors are broadcasts.
//
// A CTA (or a pair of them, tcgen05 cta_group::2, 128 features each) is persistent over tiles of (expert, rows of the expert, features).  The
// rows of an expert are dealt evenly to as few tiles as they need.
//   epilogue warps      (single CTAs 4, pairs 8, pairs with A in order 16)  tensor memory -> registers -> scales, activation, rounding -> shared memory
//                       (turned) -> whole row segments out.  A word holds four (two) rows of a feature: shared memory is what the products' operands
//                       fill already, and a byte at a time costs it four times the cycles
//   row warps           (pairs 8, single CTAs 2)  rows of A picked by token: TMA gathers of four rows.  One warp starts one every 80 cycles or so, a k-block of a pair takes
//                       64, 32 in each CTA, in 512 cycles: eight warps, with the gated products no longer exchanged between lanes, took the gated prompt (8192 tokens,
//                       top 8 of 64, 2048 x 2048) from 259 us to 227
//   load warp           W tiles, and A where its rows are in order (TMA)
//   vector warp         row factors, scales, biases and output factors of the next tile, to shared memory (two loads that depend on one another
//                       and a search for the tile: 2000 cycles that each epilogue warp would spend once a tile)
//   product warp        products (one elected lane); owns the tensor memory
// Rows that warps copy themselves (cp.async) need a hand-off from those warps to the tensor core, whose chain is longer than five stages hide: 1850
// cycles a k-block.  The accumulator is double-buffered.  Every wait is bounded; on expiry the CTA records a code and unwinds.
//
// Gated products (act(gate) * up): a tile's 128 rows of W are eight rows of the gate's half and eight of the other in turn (one tensor map does
// that).  Read in the shape of 16 lanes x 256 bits, tensor memory then gives a thread both products of a feature for the same two rows.
#include "gemm_common.cuh"
#include "moe_deal.cuh"

namespace hero {

constexpr int MOE_MAX_E = 512;
constexpr int MOE_CHUNK = 32;                 // rows that an epilogue group turns at a time

struct MoeLinearParams {
  int R, a_rows, E, N, n_out;
  int num_kb, num_nt;                         // 128-byte steps of K, feature tiles of an expert
  const int* offset; const int* token;
  const float* rs; const float* cs; const float* bias; const float* post;
  void* out; long long out_ld; int out_dt;
  int act, f8;                                // f8: e4m3 operands
  uint32_t idesc;                             // without the N field
  int kelems;                                 // elements of 128 bytes
  float* obs;
  int* err;
};

template <bool PAIR, bool GATHER>
struct MoeCfg {
  static constexpr int MT = MoeRows<PAIR>::MT, ROWS = MoeRows<PAIR>::ROWS, STEP = MoeRows<PAIR>::STEP;
  static constexpr int FEAT = 128;                        // features of this CTA
  static constexpr int W_BYTES = FEAT * GEMM_BK_BYTES, X_BYTES = ROWS * GEMM_BK_BYTES, STAGE_BYTES = W_BYTES + X_BYTES;
  static constexpr int STAGES = PAIR ? 5 : 4;
  static constexpr int EPI_WARPS = !PAIR ? 4 : !GATHER ? 16 : 8, EPI_GROUPS = EPI_WARPS / 4;
  static constexpr int ROW_WARPS = GATHER ? MoeRows<PAIR>::WARPS : 0;
  static constexpr int ROW_WARP = EPI_WARPS, LOAD_WARP = ROW_WARP + ROW_WARPS, MMA_WARP = LOAD_WARP + 1, VEC_WARP = MMA_WARP + 1,
                       THREADS = (VEC_WARP + 1) * 32;
  static constexpr int BOX = MoeRows<PAIR>::BOX;
  static constexpr int TURN_BUFS = EPI_GROUPS <= 2 ? 2 : 1;
  static constexpr int TURN_BYTES = TURN_BUFS * 16 * 128 * 4;             // per epilogue group: buffers of 32 rows of 16-bit outputs, in words of two rows
  static constexpr int TMEM_COLS = 2 * MT;
  static constexpr int TURN_AT = STAGES * STAGE_BYTES;
  static constexpr int VEC_FLOATS = MT + 3 * FEAT + 8;    // of a tile: row factors, scales, biases, output factors, {row0, rows + part and split, expert, feature tile}
  static constexpr int VEC_AT = TURN_AT + EPI_GROUPS * TURN_BYTES;                 // [2]
  static constexpr int TABLE_AT = VEC_AT + 2 * VEC_FLOATS * 4;            // first row [E + 1] and first tile [E + 1] of each expert
  static constexpr int BARS_AT = TABLE_AT + 2 * (MOE_MAX_E + 4) * 4;
  static constexpr int SMEM_BYTES = 1024 + BARS_AT + 256;
  static constexpr int PER_SM = PAIR ? 1 : 2;             // CTAs of an SM
  static_assert(PER_SM * (SMEM_BYTES + 1024) <= 228 * 1024, "shared memory");
};

// v / (1 + 2^x), given x - 15 (ACT_SHIFT): v 2^-15 / (2^-15 + 2^(x - 15)).  Neither the power nor the quotient, whose instructions know no subnormal numbers,
// leaves FP32's normal range up to x = 141, where the result (|v| < 100 there) is below half of the smallest BF16; from there on it is 0.  (Without the shift
// every result below 2^-119 or so was.)  The shift rounds the exponent to 2^-21 for 0 < x < 31, 3e-7 of the result.
constexpr float ACT_SHIFT = 15.0f, ACT_ONE = 1.0f / 32768.0f;
__device__ __forceinline__ float over_one_plus_exp2(float v, float x15) {
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(x15));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(ACT_ONE + e));
  return v * (r * ACT_ONE);
}
// SiLU: v / (1 + e^-v).  GELU(tanh): 0.5 v (1 + tanh(u)) = v / (1 + e^-2u), u = sqrt(2 / pi) (v + 0.044715 v^3); both with log2 e in the constants
__device__ __forceinline__ float silu_f(float v) { return over_one_plus_exp2(v, fmaf(v, -1.44269504088896340736f, -ACT_SHIFT)); }
__device__ __forceinline__ float gelu_tanh_quotient(float v) {
  return over_one_plus_exp2(v, fmaf(v, fmaf(v * v, -0.10294324f, -2.30220819f), -ACT_SHIFT));
}
template <int ACT>
__device__ __forceinline__ float moe_act(float v) {
  if constexpr (ACT == HERO_ACT_GELU_ERF) return gelu_erf_f(v);
  if constexpr (ACT == HERO_ACT_GELU_TANH) return gelu_tanh_quotient(v);
  if constexpr (ACT == HERO_ACT_SILU) return silu_f(v);
  return v;
}

template <bool INT8>
__device__ __forceinline__ float2 moe_acc2(uint32_t a, uint32_t b) {
  return INT8 ? make_float2((float)(int)a, (float)(int)b) : make_float2(__uint_as_float(a), __uint_as_float(b));
}

// What a thread knows of its features: one (its lane), or two gated ones (lane / 4 of each half of 16 lanes).
template <bool GATED>
struct MoeFeature {
  float cs[GATED ? 4 : 1], bias[GATED ? 4 : 1], post[GATED ? 2 : 1];      // gated: gate and up of the first, of the second
};

// Four (8-bit outputs) or two (16-bit) rows of a feature, rounded, in one word.
template <bool INT8, int OUTK>
__device__ __forceinline__ uint32_t moe_word4(float2 a, float2 b) {
  if constexpr (OUTK == OUT_F8) {
    return ptx::f32x4_to_e4m3x4(a.x, a.y, b.x, b.y);       // saturating, round to nearest even
  } else {
    const float2 mg = make_float2(ROUND_MAGIC, ROUND_MAGIC);
    a = __fadd2_rn(a, mg); b = __fadd2_rn(b, mg);          // the adder rounds, ties to even: 1.5 * 2^23 + k has k in its low byte
    const float hi = ptx::max3(ptx::max3(a.x, a.y, b.x), b.y, b.y), lo = ptx::min3(ptx::min3(a.x, a.y, b.x), b.y, b.y);
    // (INT8 operands give no NaN; others are always clipped, which makes a NaN -127)
    if (!INT8 || hi > ROUND_MAGIC + 127.0f || lo < ROUND_MAGIC - 127.0f) {
      a.x = fminf(fmaxf(a.x, ROUND_MAGIC - 127.0f), ROUND_MAGIC + 127.0f); a.y = fminf(fmaxf(a.y, ROUND_MAGIC - 127.0f), ROUND_MAGIC + 127.0f);
      b.x = fminf(fmaxf(b.x, ROUND_MAGIC - 127.0f), ROUND_MAGIC + 127.0f); b.y = fminf(fmaxf(b.y, ROUND_MAGIC - 127.0f), ROUND_MAGIC + 127.0f);
    }
    return __byte_perm(__byte_perm(__float_as_uint(a.x), __float_as_uint(a.y), 0x0040), __byte_perm(__float_as_uint(b.x), __float_as_uint(b.y), 0x0040), 0x5410);
  }
}
__device__ __forceinline__ uint32_t moe_word2(float2 a, int dt) {
  if (dt == HERO_F16) {
    const __half2 h = __floats2half2_rn(a.x, a.y);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  const __nv_bfloat162 h = __floats2bfloat162_rn(a.x, a.y);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// the larger magnitude (16-bit pattern) of the word's rows that exist
__device__ __forceinline__ uint32_t moe_most(uint32_t most, uint32_t w, bool first, bool second) {
  return max(most, max(first ? w & 0x7fffu : 0u, second ? (w >> 16) & 0x7fffu : 0u));
}

template <int ACT>
__device__ __forceinline__ float2 moe_act2(float2 v) {
  if constexpr (ACT == HERO_ACT_GELU_ERF) return gelu_erf_f2(v);
  else return make_float2(moe_act<ACT>(v.x), moe_act<ACT>(v.y));
}

// A turned chunk is words of four (two) rows of a feature: [groups of rows][features].  Ungated, a group is rows that follow one another; gated, a
// thread has rows in pairs, eight apart, and a word of four takes two such pairs.  Gated rows of words are 8 longer, so that the four
// groups of a warp's store lie on banks of their own.
template <bool GATED>
constexpr int MOE_WORD_PITCH = GATED ? 64 + 8 : 128;

// A chunk of 32 rows: products, activation, rounding, to the turned chunk.  `rs`: the chunk's row factors; count: rows that exist (observer)
template <bool INT8, bool GATED, int ACT, int OUTK>
__device__ __forceinline__ void moe_chunk(const MoeLinearParams& p, const uint32_t (&r)[32], const float* rs, const MoeFeature<GATED>& l, uint32_t* buf, int lane,
                                          int count, uint32_t (&most)[2]) {
  constexpr int PITCH = MOE_WORD_PITCH<GATED>;
  if constexpr (GATED) {
    uint32_t* at = buf + (lane & 3) * PITCH + (lane >> 2);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      float2 y[4];
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const float2 f = *reinterpret_cast<const float2*>(rs + 8 * b + 2 * (lane & 3));
        const uint32_t* q = &r[half * 16 + b * 4];
        const float2 g = __ffma2_rn(__fmul2_rn(moe_acc2<INT8>(q[0], q[1]), f), make_float2(l.cs[2 * half], l.cs[2 * half]), make_float2(l.bias[2 * half], l.bias[2 * half]));
        const float2 u = __ffma2_rn(__fmul2_rn(moe_acc2<INT8>(q[2], q[3]), f), make_float2(l.cs[2 * half + 1], l.cs[2 * half + 1]), make_float2(l.bias[2 * half + 1], l.bias[2 * half + 1]));
        y[b] = __fmul2_rn(__fmul2_rn(moe_act2<ACT>(g), u), make_float2(l.post[half], l.post[half]));
      }
      if constexpr (OUTK == OUT_FP) {
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          const uint32_t w = moe_word2(y[b], p.out_dt);
          at[4 * b * PITCH + half * 8] = w;
          if (p.obs) most[half] = moe_most(most[half], w, 8 * b + 2 * (lane & 3) < count, 8 * b + 2 * (lane & 3) + 1 < count);
        }
      } else {
        at[half * 8] = moe_word4<INT8, OUTK>(y[0], y[1]);
        at[4 * PITCH + half * 8] = moe_word4<INT8, OUTK>(y[2], y[3]);
      }
    }
  } else {
    uint32_t* at = buf + lane;
#pragma unroll
    for (int j = 0; j < 32; j += 4) {
      const float4 f = *reinterpret_cast<const float4*>(rs + j);
      float2 y[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        // (without an activation cs and bias carry the output factor)
        y[i] = __ffma2_rn(__fmul2_rn(moe_acc2<INT8>(r[j + 2 * i], r[j + 2 * i + 1]), i ? make_float2(f.z, f.w) : make_float2(f.x, f.y)),
                          make_float2(l.cs[0], l.cs[0]), make_float2(l.bias[0], l.bias[0]));
        if constexpr (ACT != HERO_ACT_NONE) y[i] = __fmul2_rn(moe_act2<ACT>(y[i]), make_float2(l.post[0], l.post[0]));
      }
      if constexpr (OUTK == OUT_FP) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32_t w = moe_word2(y[i], p.out_dt);
          at[(j / 2 + i) * PITCH] = w;
          if (p.obs) most[0] = moe_most(most[0], w, j + 2 * i < count, j + 2 * i + 1 < count);
        }
      } else {
        at[j / 4 * PITCH] = moe_word4<INT8, OUTK>(y[0], y[1]);
      }
    }
  }
}

// A turned chunk to the output: a thread takes four features of a group of rows (16 bytes) and writes them row by row; the warps of a group (quarter 0 .. 3)
// take the groups of rows in turn.  `out`: the chunk's first row at the CTA's first column; lo, hi: the columns that are this
// CTA's to write.
template <bool GATED, int OUTK>
__device__ __forceinline__ void moe_store(const uint32_t* buf, uint8_t* out, long long pitch, int rows, int lo, int hi, int quarter, int lane) {
  constexpr int PITCH = MOE_WORD_PITCH<GATED>, PER = GATED ? 16 : 32, AT_ONCE = 32 / PER;       // threads per group of rows, groups per warp and step
  constexpr int GROUPS = OUTK == OUT_FP ? 16 : 8, ES = OUTK == OUT_FP ? 2 : 1;
  const int col = (lane % PER) * 4;
  if (col < lo || col >= hi) return;
#pragma unroll
  for (int s = 0; s < GROUPS / (4 * AT_ONCE); ++s) {
    const int g = (quarter + 4 * s) * AT_ONCE + lane / PER;
    const uint4 w = *reinterpret_cast<const uint4*>(buf + g * PITCH + col);
    if constexpr (OUTK == OUT_FP) {
      uint8_t* at = out + 2 * g * pitch + col * ES;
      if (2 * g < rows) *reinterpret_cast<uint2*>(at) = make_uint2(__byte_perm(w.x, w.y, 0x5410), __byte_perm(w.z, w.w, 0x5410));
      if (2 * g + 1 < rows) *reinterpret_cast<uint2*>(at + pitch) = make_uint2(__byte_perm(w.x, w.y, 0x7632), __byte_perm(w.z, w.w, 0x7632));
    } else {
      const int row = GATED ? 16 * (g >> 2) + 2 * (g & 3) : 4 * g, skip = GATED ? 8 : 2;          // rows row, row + 1, row + skip, row + skip + 1
      const uint32_t a = __byte_perm(w.x, w.y, 0x5140), b = __byte_perm(w.z, w.w, 0x5140), c = __byte_perm(w.x, w.y, 0x7362), d = __byte_perm(w.z, w.w, 0x7362);
      uint8_t* at = out + row * pitch + col;
      if (row < rows) *reinterpret_cast<uint32_t*>(at) = __byte_perm(a, b, 0x5410);
      if (row + 1 < rows) *reinterpret_cast<uint32_t*>(at + pitch) = __byte_perm(a, b, 0x7632);
      if (row + skip < rows) *reinterpret_cast<uint32_t*>(at + skip * pitch) = __byte_perm(c, d, 0x5410);
      if (row + skip + 1 < rows) *reinterpret_cast<uint32_t*>(at + (skip + 1) * pitch) = __byte_perm(c, d, 0x7632);
    }
  }
}

// 32 columns of this warp's 32 lanes; gated: in two halves of 16 lanes, a thread having lanes l / 4 and l / 4 + 8, columns 2 (l % 4) and one more, of
// each eight columns
template <bool GATED>
__device__ __forceinline__ void moe_tmem_ld(uint32_t taddr, uint32_t (&r)[32]) {
  if constexpr (GATED) {
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      uint32_t* q = &r[16 * half];
      asm volatile(
          "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
          : "=r"(q[0]), "=r"(q[1]), "=r"(q[2]), "=r"(q[3]), "=r"(q[4]), "=r"(q[5]), "=r"(q[6]), "=r"(q[7]), "=r"(q[8]), "=r"(q[9]), "=r"(q[10]),
            "=r"(q[11]), "=r"(q[12]), "=r"(q[13]), "=r"(q[14]), "=r"(q[15])
          : "r"(taddr + ((uint32_t)(16 * half) << 16)) : "memory");
    }
  } else {
    ptx::tmem_ld32(taddr, r);
  }
}

// four rows of A, 128 bytes of each
template <bool PAIR>
__device__ __forceinline__ void load_rows(uint32_t dst, const CUtensorMap* m, int x, const int (&r)[4], uint32_t bar) {
  if constexpr (PAIR)
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile::gather4.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3, %4, %5, %6}], [%7];"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(m)), "r"(x), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(bar) : "memory");
  else
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile::gather4.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(m)), "r"(x), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(bar) : "memory");
}
// a box of rows of A that lie behind one another, 128 bytes of each
template <bool PAIR>
__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap* m, int x, int y, uint32_t bar) {
  if constexpr (PAIR)
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(m)), "r"(x), "r"(y), "r"(bar) : "memory");
  else
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(m)), "r"(x), "r"(y), "r"(bar) : "memory");
}
// a box of one expert's W (pair: 128 rows, else 32): row r0, or (gated) the r0-th group of eight rows of each half
template <bool GATED, bool PAIR>
__device__ __forceinline__ void load_w(uint32_t dst, const CUtensorMap* m, int x, int r0, int e, uint32_t bar) {
  const uint64_t map = reinterpret_cast<uint64_t>(m);
  if constexpr (GATED) {
    if constexpr (PAIR)
      asm volatile("cp.async.bulk.tensor.5d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %3, %4, %5}], [%6];"
                   ::"r"(dst), "l"(map), "r"(x), "r"(0), "r"(r0), "r"(e), "r"(bar) : "memory");
    else
      asm volatile("cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %3, %4, %5}], [%6];"
                   ::"r"(dst), "l"(map), "r"(x), "r"(0), "r"(r0), "r"(e), "r"(bar) : "memory");
  } else {
    if constexpr (PAIR)
      asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                   ::"r"(dst), "l"(map), "r"(x), "r"(r0), "r"(e), "r"(bar) : "memory");
    else
      asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                   ::"r"(dst), "l"(map), "r"(x), "r"(r0), "r"(e), "r"(bar) : "memory");
  }
}

// The vector warp: what the epilogue needs of each tile, one tile ahead.
template <bool GATED, bool PAIR, bool GATHER>
__device__ __forceinline__ void moe_vectors(const MoeLinearParams& p, uint8_t* smem, const MoeDeal& deal, uint64_t* vec_full, uint64_t* vec_empty,
                                            int first_unit, int stride, int rank) {
  using Cfg = MoeCfg<PAIR, GATHER>;
  constexpr int MT = Cfg::MT, COLS = GATED ? 64 : 128;
  const int lane = threadIdx.x & 31;
  int it = 0;
  for (int t = first_unit; t < deal.units; t += stride) {
    const MoeTile w = deal.at<PAIR>(t, lane);
    if (w.rows <= 0) continue;
    float rs[MT / 32], cs[4], bias[4], post[4];
#pragma unroll
    for (int k = 0; k < MT / 32; ++k) {
      const int r = 32 * k + lane;
      rs[k] = 1.0f;
      if (p.rs && r < w.rows) {
        int at = w.row0 + r;
        if constexpr (GATHER) at = min(max(p.token[at], 0), p.a_rows - 1);
        rs[k] = p.rs[at];
      }
    }
    const int c0 = (w.nt * (PAIR ? 2 : 1) + rank) * COLS;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int l = 32 * k + lane;                                  // row of the W tile; gated: eight of the gate, eight of the other
      const int col = c0 + (GATED ? (l >> 4) * 8 + (l & 7) : l), out = c0 + l;
      const long long at = (long long)w.e * p.N + col + (GATED && (l & 8) ? p.n_out : 0);
      cs[k] = col < p.n_out && p.cs ? __ldg(p.cs + at) : 1.0f;
      bias[k] = col < p.n_out && p.bias ? __ldg(p.bias + at) : 0.0f;
      post[k] = l < COLS && out < p.n_out && p.post ? __ldg(p.post + (long long)w.e * p.n_out + out) : 1.0f;
    }
    if (!ptx::mbar_wait(&vec_empty[it & 1], ((it >> 1) & 1) ^ 1, p.err, 0xF80 | (it & 1))) break;
    float* v = reinterpret_cast<float*>(smem + Cfg::VEC_AT) + (it & 1) * Cfg::VEC_FLOATS;
#pragma unroll
    for (int k = 0; k < MT / 32; ++k) v[32 * k + lane] = rs[k];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[MT + 32 * k + lane] = cs[k];
      v[MT + 128 + 32 * k + lane] = bias[k];
      v[MT + 256 + 32 * k + lane] = post[k];
    }
    if (lane == 0) *reinterpret_cast<int4*>(v + MT + 384) = make_int4(w.row0, w.rows | (w.part << 16) | (w.split << 24), w.e, w.nt);
    __syncwarp();
    if (lane == 0) ptx::mbar_arrive(&vec_full[it & 1]);
    ++it;
  }
  // the walk's end: a tile without rows
  if (ptx::mbar_wait(&vec_empty[it & 1], ((it >> 1) & 1) ^ 1, p.err, 0xF82 | (it & 1)) && lane == 0) {
    float* v = reinterpret_cast<float*>(smem + Cfg::VEC_AT) + (it & 1) * Cfg::VEC_FLOATS;
    *reinterpret_cast<int4*>(v + MT + 384) = make_int4(0, 0, 0, 0);
    ptx::mbar_arrive(&vec_full[it & 1]);
  }
}

// Whether all four warps of an epilogue group say so (they meet on the group's barrier): what one warp's wait did not bring ends the walk of all, none of
// them is left at a barrier.
__device__ __forceinline__ bool group_all(bool ok, int id) {
  uint32_t r;
  __syncwarp();
  asm volatile(
      "{\n"
      ".reg .pred p, q;\n"
      "setp.ne.u32 p, %1, 0;\n"
      "bar.red.and.pred q, %2, 128, p;\n"
      "selp.u32 %0, 1, 0, q;\n"
      "}\n" : "=r"(r) : "r"(ok ? 1u : 0u), "r"(id) : "memory");
  return r != 0;
}

// The epilogue warps, tile after tile as the vector warp names them.
template <bool INT8, bool GATED, bool PAIR, bool GATHER, int ACT, int OUTK>
__device__ __forceinline__ void moe_epilogue(const MoeLinearParams& p, uint8_t* smem, uint64_t* acc_full, uint64_t* acc_empty, uint64_t* vec_full,
                                             uint64_t* vec_empty, uint32_t tmem_base, int rank) {
  using Cfg = MoeCfg<PAIR, GATHER>;
  constexpr int MT = Cfg::MT, COLS = GATED ? 64 : 128, ES = OUTK == OUT_FP ? 2 : 1;    // COLS: output columns of this CTA
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int quarter = warp & 3, group = warp >> 2;
  uint32_t* turn = reinterpret_cast<uint32_t*>(smem + Cfg::TURN_AT + group * Cfg::TURN_BYTES);
  const int warp_col = quarter * (GATED ? 16 : 32);                                    // first output column of this warp in the CTA's
  int turned = 0;
  for (int it = 0;; ++it) {
    const int as = it & 1;
    const uint32_t aphase = (it >> 1) & 1;
    bool ok = ptx::mbar_wait(&vec_full[as], aphase, p.err, 0xF84 | as);
    const float* vec = reinterpret_cast<const float*>(smem + Cfg::VEC_AT) + as * Cfg::VEC_FLOATS;
    const int4 tile = *reinterpret_cast<const int4*>(vec + MT + 384);
    const MoeTile w{tile.z, tile.x, tile.y & 0xffff, tile.w, (tile.y >> 16) & 0xff, tile.y >> 24};
    const int c0 = (w.nt * (PAIR ? 2 : 1) + rank) * COLS;
    MoeFeature<GATED> l;
    if constexpr (GATED) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float* at = vec + MT + quarter * 32 + i * 16 + (lane >> 2);
        l.cs[2 * i] = at[0]; l.cs[2 * i + 1] = at[8];
        l.bias[2 * i] = at[128]; l.bias[2 * i + 1] = at[128 + 8];
        l.post[i] = vec[MT + 256 + warp_col + i * 8 + (lane >> 2)];
      }
    } else {
      const float* at = vec + MT + warp_col + lane;
      l.cs[0] = at[0]; l.bias[0] = at[128]; l.post[0] = at[256];
      if (ACT == HERO_ACT_NONE) { l.cs[0] *= l.post[0]; l.bias[0] *= l.post[0]; }     // (acc rs cs + b) post = acc rs (cs post) + b post
    }
    if (ok && w.rows != 0) ok = ptx::mbar_wait(&acc_full[as], aphase, p.err, 0xF00 | as);
    // (a wait that gave up has recorded its code: the group leaves together, and writes nothing of a tile of which any of it is missing)
    if (!group_all(ok, 1 + group) || w.rows == 0) break;
    ptx::tc_fence_after();
    const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + as * MT;
    uint32_t most[2] = {0u, 0u};
    // a part of the features is whole quarters of the lanes
    const int quarters = 4 >> w.split, q0 = w.part * quarters;
    const bool mine = PAIR || (quarter >= q0 && quarter < q0 + quarters);
    const int col_lo = PAIR ? 0 : q0 * (COLS / 4), col_hi = PAIR ? p.n_out - c0 : min(p.n_out - c0, (q0 + quarters) * (COLS / 4));
    const int chunks = (w.rows + MOE_CHUNK - 1) / MOE_CHUNK;
    uint32_t r[32];
    constexpr int GROUPS = Cfg::EPI_GROUPS;
    if (group < chunks) moe_tmem_ld<GATED>(taddr + group * MOE_CHUNK, r);
    for (int c = group; c < chunks; c += GROUPS) {
      ptx::tmem_ld_wait();
      uint32_t* buf = turn;
      if constexpr (Cfg::TURN_BUFS == 2) buf += (turned++ & 1) * (Cfg::TURN_BYTES / 8);
      else asm volatile("bar.sync %0, 128;" ::"r"(1 + group) : "memory");          // the group is through with the chunk before
      const int rows = min(MOE_CHUNK, w.rows - c * MOE_CHUNK);
      if (mine) moe_chunk<INT8, GATED, ACT, OUTK>(p, r, vec + c * MOE_CHUNK, l, buf + warp_col, lane, rows, most);
      if (c + GROUPS < chunks) moe_tmem_ld<GATED>(taddr + (c + GROUPS) * MOE_CHUNK, r);       // on its way while this chunk is stored
      // the group's four warps have written the chunk (of two buffers, the one of two chunks ago is free too)
      asm volatile("bar.sync %0, 128;" ::"r"(1 + group) : "memory");
      moe_store<GATED, OUTK>(buf, static_cast<uint8_t*>(p.out) + ((long long)(w.row0 + c * MOE_CHUNK) * p.out_ld + c0) * ES, p.out_ld * ES, rows, col_lo, col_hi, quarter, lane);
      __syncwarp();
    }
    if (p.obs) {
#pragma unroll
      for (int i = 0; i < (GATED ? 2 : 1); ++i) {
        const int col = c0 + warp_col + (GATED ? i * 8 + (lane >> 2) : lane);
        const float m = p.out_dt == HERO_F16 ? __half2float(__ushort_as_half((unsigned short)most[i])) : __uint_as_float(most[i] << 16);
        if (col < p.n_out && most[i]) atomicMax(reinterpret_cast<unsigned int*>(p.obs) + (long long)w.e * p.n_out + col, __float_as_uint(m));
      }
    }
    // hand the accumulator and the vectors back
    ptx::tc_fence_before();
    __syncwarp();
    if (lane == 0) {
      ptx::mbar_arrive(&vec_empty[as]);
      if constexpr (PAIR) ptx::mbar_arrive_cluster_relaxed(ptx::mapa(ptx::smem_u32(&acc_empty[as]), 0));
      else ptx::mbar_arrive(&acc_empty[as]);
    }
  }
}

template <bool INT8, bool GATED, bool PAIR, bool GATHER>
__device__ __forceinline__ void moe_linear_body(const CUtensorMap& tmW, const CUtensorMap& tmA, const MoeLinearParams& p) {
  using Cfg = MoeCfg<PAIR, GATHER>;
  constexpr int MT = Cfg::MT, STAGES = Cfg::STAGES;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  int* first = reinterpret_cast<int*>(smem + Cfg::TABLE_AT);        // [E + 1]
  int* tiles = first + MOE_MAX_E + 4;                               // [E + 1]
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + Cfg::BARS_AT);   // [STAGES] operands there (of a pair: the leader's)
  uint64_t* empty = full + STAGES;                                  // [STAGES] operands read
  uint64_t* acc_full = empty + STAGES;                              // [2]
  uint64_t* acc_empty = acc_full + 2;                               // [2] (of a pair: the leader's)
  uint64_t* vec_full = acc_empty + 2;                               // [2] vectors of a tile there
  uint64_t* vec_empty = vec_full + 2;                               // [2]
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(vec_empty + 2);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = PAIR ? ptx::cluster_ctarank() : 0u;
  const int group_id = PAIR ? blockIdx.x >> 1 : blockIdx.x, groups = PAIR ? gridDim.x >> 1 : gridDim.x;

  if (threadIdx.x == 0) {
    for (int i = 0; i < STAGES; ++i) { ptx::mbar_init(&full[i], 1); ptx::mbar_init(&empty[i], 1); }
    for (int i = 0; i < 2; ++i) { ptx::mbar_init(&acc_full[i], 1); ptx::mbar_init(&acc_empty[i], Cfg::EPI_WARPS * (PAIR ? 2 : 1)); }
    for (int i = 0; i < 2; ++i) { ptx::mbar_init(&vec_full[i], 1); ptx::mbar_init(&vec_empty[i], Cfg::EPI_WARPS); }
    ptx::fence_mbar_init();
  }
  if (warp == Cfg::MMA_WARP) {
    if constexpr (PAIR) { ptx::tmem_alloc_pair(tmem_slot, Cfg::TMEM_COLS); ptx::tmem_relinquish_pair(); }
    else { ptx::tmem_alloc(tmem_slot, Cfg::TMEM_COLS); ptx::tmem_relinquish(); }
  }
  if (warp == Cfg::LOAD_WARP && lane == 0) { ptx::prefetch_tmap(&tmW); ptx::prefetch_tmap(&tmA); }
  ptx::pdl_launch_dependents();
  ptx::pdl_wait();                                                  // the router's offsets (and all else) are there from here on

  // ---- the experts' first rows and first tiles
  if (warp == 0) {
    int run = 0;
    for (int e0 = 0; e0 < p.E; e0 += 32) {
      const int e = e0 + lane;
      int k = 0;
      if (e < p.E) {
        const int lo = p.offset[e], hi = p.offset[e + 1];
        first[e] = lo;
        if (e == p.E - 1) first[p.E] = hi;
        k = moe_tiles<PAIR>(lo, hi, p.R);
        if (k < 0) { atomicExch(p.err, ERR_BAD_EXPERT); k = 0; }
      }
      int s = k;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += u;
      }
      if (e < p.E) tiles[e] = run + s - k;
      run += __shfl_sync(0xffffffffu, s, 31);
    }
    if (lane == 0) tiles[p.E] = run;
  }
  ptx::tc_fence_before();
  __syncthreads();
  if constexpr (PAIR) ptx::cluster_sync();                          // both CTAs' barriers exist before any remote arrive
  ptx::tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  MoeDeal deal;
  deal.init(p.E, p.num_nt, first, tiles, groups);
  const int num_tiles = deal.units;
  auto tile_at = [&](int t) { return deal.at<PAIR>(t, lane); };

  if (warp == Cfg::LOAD_WARP) {
    // ------------------------------------------------------------------ weights
    const bool issue = ptx::elect_one();
    const uint32_t dst0 = PAIR ? ptx::mapa(ptx::smem_u32(smem), rank) : ptx::smem_u32(smem);
    const uint32_t bar0 = PAIR ? ptx::mapa(ptx::smem_u32(full), 0) : ptx::smem_u32(full);
    int stage = 0; uint32_t phase = 0; bool ok = true;
    for (int t = group_id; t < num_tiles && ok; t += groups) {
      const MoeTile w = tile_at(t);
      if (w.rows <= 0) continue;
      const int r0 = (w.nt * (PAIR ? 2 : 1) + (int)rank) * (GATED ? 8 : 128);
      const int box0 = w.part * (4 >> w.split), box1 = box0 + (4 >> w.split);        // single CTAs: boxes of 32 features
      // what both CTAs' copies of a k-block bring: whole groups of four rows, or whole boxes of rows in order
      const MoeShare s0 = moe_share<PAIR>(w, 0), s1 = moe_share<PAIR>(w, 1), sh = rank ? s1 : s0;
      auto rows_in = [&](const MoeShare& s) { return GATHER ? 4 * s.fours : max(0, (s.n + Cfg::BOX - 1) / Cfg::BOX) * Cfg::BOX; };
      const uint32_t bytes = (PAIR ? 2 * Cfg::W_BYTES : Cfg::W_BYTES >> w.split) + (uint32_t)(rows_in(s0) + (PAIR ? rows_in(s1) : 0)) * GEMM_BK_BYTES;
      const int in_order = GATHER ? 0 : sh.n;
      for (int kb = 0; kb < p.num_kb; ++kb) {
        if (!ptx::mbar_wait(&empty[stage], phase ^ 1, p.err, 0xC00 | stage)) { ok = false; break; }
        if (issue) {
          if (rank == 0) ptx::mbar_expect_tx(&full[stage], bytes);
          if constexpr (PAIR) {
            load_w<GATED, PAIR>(dst0 + stage * Cfg::STAGE_BYTES, &tmW, kb * p.kelems, r0, w.e, bar0 + 8 * stage);
          } else {
#pragma unroll
            for (int b = 0; b < 4; ++b)
              if (b >= box0 && b < box1)
                load_w<GATED, PAIR>(dst0 + stage * Cfg::STAGE_BYTES + b * (Cfg::W_BYTES / 4), &tmW, kb * p.kelems, r0 + b * (GATED ? 2 : 32), w.e, bar0 + 8 * stage);
          }
#pragma unroll
          for (int r = 0; r < Cfg::ROWS; r += Cfg::BOX)
            if (r < in_order)
              load_box<PAIR>(dst0 + stage * Cfg::STAGE_BYTES + Cfg::W_BYTES + r * GEMM_BK_BYTES, &tmA, kb * p.kelems, w.row0 + sh.lo + r, bar0 + 8 * stage);
        }
        if (++stage == STAGES) { stage = 0; phase ^= 1; }
      }
    }
    for (int i = 0; i < STAGES; ++i) {                              // every copy started here has been consumed
      if (!ptx::mbar_wait(&empty[stage], phase ^ 1, p.err, 0xC80 | stage)) break;
      if (++stage == STAGES) { stage = 0; phase ^= 1; }
    }
    __syncwarp();
  } else if (GATHER && warp >= Cfg::ROW_WARP && warp < Cfg::LOAD_WARP) {
    if constexpr (GATHER) {
    // ------------------------------------------------------------------ rows of A
    // warp ww has the groups ww, ww + ROW_WARPS, ..
    constexpr int ROW_WARPS = Cfg::ROW_WARPS, PER = (Cfg::ROWS / 4 + ROW_WARPS - 1) / ROW_WARPS;
    const int ww = warp - Cfg::ROW_WARP;
    const bool issue = ptx::elect_one();
    const uint32_t dst0 = (PAIR ? ptx::mapa(ptx::smem_u32(smem), rank) : ptx::smem_u32(smem)) + Cfg::W_BYTES + ww * (4 * GEMM_BK_BYTES);
    const uint32_t bar0 = PAIR ? ptx::mapa(ptx::smem_u32(full), 0) : ptx::smem_u32(full);
    int stage = 0; uint32_t phase = 0; bool ok = true;
    int fours = 0, mine = 0;                                        // this warp's groups in the tile asked for (-1: no tile), this lane's row of A
    auto ask = [&](int t) {
      const MoeTile w = tile_at(t);
      fours = -1;
      if (w.rows <= 0) return;
      const MoeShare sh = moe_share<PAIR>(w, (int)rank);
      fours = (sh.fours - ww + ROW_WARPS - 1) / ROW_WARPS;
      // (a group that is not full ends with other rows of the tile)
      const int at = w.row0 + min(sh.lo + 4 * (ww + ROW_WARPS * (lane >> 2)) + (lane & 3), w.rows - 1);
      mine = 0;
      if (lane < 4 * fours) {
        mine = p.token[at];
        if ((unsigned)mine >= (unsigned)p.a_rows) {
          atomicExch(p.err, ERR_BAD_EXPERT);
          mine = mine < 0 ? 0 : p.a_rows - 1;
        }
      }
    };
    if (group_id < num_tiles) ask(group_id);
    for (int t = group_id; t < num_tiles && ok; t += groups) {
      const int n4 = fours;
      // (a reduction leaves its result in a uniform register, where a copy's coordinates have to be)
      int r[PER][4];
#pragma unroll
      for (int s = 0; s < PER; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i) r[s][i] = (int)__reduce_max_sync(0xffffffffu, lane == 4 * s + i ? (uint32_t)mine : 0u);
      if (t + groups < num_tiles) ask(t + groups);                  // the next tile's rows, while this one's are copied
      if (n4 < 0) continue;
      for (int kb = 0; kb < p.num_kb; ++kb) {
        if (!ptx::mbar_wait(&empty[stage], phase ^ 1, p.err, 0xD00 | stage)) { ok = false; break; }
        if (issue) {
#pragma unroll
          for (int s = 0; s < PER; ++s)
            if (s < n4) load_rows<PAIR>(dst0 + stage * Cfg::STAGE_BYTES + s * (4 * GEMM_BK_BYTES * ROW_WARPS), &tmA, kb * p.kelems, r[s], bar0 + 8 * stage);
        }
        if (++stage == STAGES) { stage = 0; phase ^= 1; }
      }
    }
    __syncwarp();
    }
  } else if (warp == Cfg::MMA_WARP) {
    // ------------------------------------------------------------------ products (of a pair: the leader's)
    if (rank == 0) {
      const bool issue = ptx::elect_one();
      constexpr uint64_t desc_base = ptx::smem_desc_base(16, 1024, ptx::SWZ_128B);
      const uint64_t ad0 = ptx::smem_desc(desc_base, ptx::smem_u32(smem));
      const uint64_t bd0 = ptx::smem_desc(desc_base, ptx::smem_u32(smem) + Cfg::W_BYTES);
      int stage = 0; uint32_t phase = 0; bool ok = true;
      int it = 0;
      for (int t = group_id; t < num_tiles && ok; t += groups) {
        const MoeTile w = tile_at(t);
        if (w.rows <= 0) continue;
        const uint32_t idesc = p.idesc | ((uint32_t)((w.rows + Cfg::STEP - 1) / Cfg::STEP * (Cfg::STEP / 8)) << 17);
        const int as = it & 1;
        const uint32_t aphase = (it >> 1) & 1;
        ++it;
        if (!ptx::mbar_wait(&acc_empty[as], aphase ^ 1, p.err, 0xE00 | as)) { ok = false; break; }
        ptx::tc_fence_after();
        const uint32_t d_tmem = tmem_base + as * MT;
        for (int kb = 0; kb < p.num_kb; ++kb) {
          if (!ptx::mbar_wait(&full[stage], phase, p.err, 0xE80 | stage)) { ok = false; break; }
          ptx::tc_fence_after();
          if (issue) {
            const uint32_t so = (uint32_t)(stage * Cfg::STAGE_BYTES) >> 4;
#pragma unroll
            for (int k = 0; k < GEMM_BK_BYTES / 32; ++k) {
              const uint64_t ad = ad0 + (so + 2 * k), bd = bd0 + (so + 2 * k);
              const uint32_t acc = (kb | k) != 0 ? 1u : 0u;
              if constexpr (PAIR) {
                if constexpr (INT8) ptx::umma_i8_pair(d_tmem, ad, bd, idesc, acc);
                else if (p.f8) ptx::umma_f8_pair(d_tmem, ad, bd, idesc, acc);
                else ptx::umma_f16_pair(d_tmem, ad, bd, idesc, acc);
              } else {
                if constexpr (INT8) ptx::umma_i8(d_tmem, ad, bd, idesc, acc);
                else if (p.f8) ptx::umma_f8(d_tmem, ad, bd, idesc, acc);
                else ptx::umma_f16(d_tmem, ad, bd, idesc, acc);
              }
            }
            if constexpr (PAIR) ptx::umma_commit_pair(&empty[stage], 3);
            else ptx::umma_commit(&empty[stage]);
          }
          if (++stage == STAGES) { stage = 0; phase ^= 1; }
        }
        if (ok && issue) {
          if constexpr (PAIR) ptx::umma_commit_pair(&acc_full[as], 3);
          else ptx::umma_commit(&acc_full[as]);
        }
      }
    }
    __syncwarp();
  } else if (warp == Cfg::VEC_WARP) {
    moe_vectors<GATED, PAIR, GATHER>(p, smem, deal, vec_full, vec_empty, group_id, groups, (int)rank);
    __syncwarp();
  } else {
    // ------------------------------------------------------------------ epilogue
#define MOE_EPILOGUE(ACT, OUTK) \
  moe_epilogue<INT8, GATED, PAIR, GATHER, ACT, OUTK>(p, smem, acc_full, acc_empty, vec_full, vec_empty, tmem_base, (int)rank)
#define MOE_EPILOGUE_OUT(ACT)                                        \
  do {                                                               \
    if (p.out_dt == HERO_I8) MOE_EPILOGUE(ACT, OUT_I8);              \
    else if (p.out_dt != HERO_F8) MOE_EPILOGUE(ACT, OUT_FP);         \
    else if constexpr (!INT8) MOE_EPILOGUE(ACT, OUT_F8);             \
  } while (0)
    switch (p.act) {
      case HERO_ACT_GELU_ERF: MOE_EPILOGUE_OUT(HERO_ACT_GELU_ERF); break;
      case HERO_ACT_GELU_TANH: MOE_EPILOGUE_OUT(HERO_ACT_GELU_TANH); break;
      case HERO_ACT_SILU: MOE_EPILOGUE_OUT(HERO_ACT_SILU); break;
      default: MOE_EPILOGUE_OUT(HERO_ACT_NONE); break;
    }
#undef MOE_EPILOGUE_OUT
#undef MOE_EPILOGUE
  }

  ptx::tc_fence_before();
  __syncthreads();
  if constexpr (PAIR) ptx::cluster_sync();                          // the peer may still be reading this CTA's shared memory / barriers
  if (warp == Cfg::MMA_WARP) {
    if constexpr (PAIR) ptx::tmem_dealloc_pair(tmem_base, Cfg::TMEM_COLS);
    else ptx::tmem_dealloc(tmem_base, Cfg::TMEM_COLS);
  }
}

template <bool INT8, bool GATED, bool GATHER>
__global__ void __launch_bounds__(MoeCfg<false, GATHER>::THREADS, MoeCfg<false, GATHER>::PER_SM)
moe_linear_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmA, const __grid_constant__ MoeLinearParams p) {
  moe_linear_body<INT8, GATED, false, GATHER>(tmW, tmA, p);
}
template <bool INT8, bool GATED, bool GATHER>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(MoeCfg<true, GATHER>::THREADS, 1)
moe_linear_pair_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmA, const __grid_constant__ MoeLinearParams p) {
  moe_linear_body<INT8, GATED, true, GATHER>(tmW, tmA, p);
}

template <bool INT8, bool GATED, bool GATHER>
static hero_status launch_moe_linear(hero_handle* h, const CUtensorMap& tmW, const CUtensorMap& tmA, MoeLinearParams& p, bool pair, cudaStream_t s) {
  using One = MoeCfg<false, GATHER>;
  using Two = MoeCfg<true, GATHER>;
  const int feat = (pair ? 256 : 128) / (GATED ? 2 : 1);
  p.num_nt = (p.n_out + feat - 1) / feat;
  // a launch never needs more CTAs than an even deal of all rows over all experts could make tiles of
  const long long most = ((long long)p.R / (pair ? Two::MT : One::MT) + (p.E < p.R ? p.E : p.R)) * p.num_nt;
  const long long room = pair ? h->sm_count / 2 : One::PER_SM * h->sm_count;
  const unsigned groups = (unsigned)(4 * most < room ? 4 * most : room);   // (a tile may be cut in four)
  LaunchScope scope(h, s, KERNEL_GEMM);
  if (pair) {
    auto kern = moe_linear_pair_kernel<INT8, GATED, GATHER>;
    HERO_SMEM_OPT_IN(h, kern, Two::SMEM_BYTES);
    HERO_CUDA(launch_dependent(kern, dim3(2 * groups), dim3(Two::THREADS), Two::SMEM_BYTES, s, tmW, tmA, p));
  } else {
    auto kern = moe_linear_kernel<INT8, GATED, GATHER>;
    HERO_SMEM_OPT_IN(h, kern, One::SMEM_BYTES);
    HERO_CUDA(launch_dependent(kern, dim3(groups), dim3(One::THREADS), One::SMEM_BYTES, s, tmW, tmA, p));
  }
  return HERO_OK;
}

}  // namespace hero

extern "C" hero_status hero_moe_linear(hero_handle* h, const hero_moe_linear_args* a, void* stream) {
  using namespace hero;
  HERO_REQUIRE(h && a, HERO_ERR_INVALID_ARG, "hero_moe_linear: NULL handle or args");
  hero_status st;
  if ((st = check_matrix(a->A, "A")) != HERO_OK) return st;
  if ((st = check_matrix(a->out, "out")) != HERO_OK) return st;
  const bool int8 = a->A.dtype == HERO_I8, f8 = a->A.dtype == HERO_F8, q8 = int8 || f8;
  HERO_REQUIRE(q8 || is_fp16ish(a->A.dtype), HERO_ERR_UNSUPPORTED, "A dtype %d: INT8, e4m3, F16 or BF16 expected", a->A.dtype);
  const int eb = q8 ? 1 : 2;
  const int64_t K = a->A.cols, N = a->N, E = a->n_experts, R = a->out.rows;
  HERO_REQUIRE(E >= 1 && E <= MOE_MAX_E, HERO_ERR_UNSUPPORTED, "n_experts=%lld: 1 to %d", (long long)E, MOE_MAX_E);
  HERO_REQUIRE(a->gated == 0 || a->gated == 1, HERO_ERR_INVALID_ARG, "gated=%d", a->gated);
  HERO_REQUIRE(N > 0 && N % (a->gated ? 32 : 16) == 0, HERO_ERR_UNSUPPORTED, "N=%lld must be a positive multiple of %d", (long long)N, a->gated ? 32 : 16);
  HERO_REQUIRE((K * eb) % 16 == 0, HERO_ERR_UNSUPPORTED, "K=%lld: K * element size must be a multiple of 16 bytes", (long long)K);
  HERO_REQUIRE(a->W != nullptr && aligned16(a->W), a->W ? HERO_ERR_ALIGNMENT : HERO_ERR_INVALID_ARG, "W must be a 16-byte aligned device pointer");
  HERO_REQUIRE(K < (1ll << 30) && N < (1ll << 30) && R < (1ll << 31) && a->A.rows < (1ll << 31), HERO_ERR_UNSUPPORTED, "dimension too large");
  HERO_REQUIRE(a->ldw >= K && (a->ldw * eb) % 16 == 0, HERO_ERR_ALIGNMENT, "ldw=%lld invalid", (long long)a->ldw);
  HERO_REQUIRE(E == 1 || (a->expert_stride >= K && (a->expert_stride * eb) % 16 == 0), HERO_ERR_ALIGNMENT, "expert_stride=%lld invalid",
               (long long)a->expert_stride);
  HERO_REQUIRE(a->ldw < (1ll << 38) / N && a->expert_stride < (1ll << 38), HERO_ERR_UNSUPPORTED, "weights too far apart");
  const int64_t n_out = a->gated ? N / 2 : N;
  HERO_REQUIRE(a->out.cols == n_out, HERO_ERR_INVALID_ARG, "out has %lld columns, %lld expected", (long long)a->out.cols, (long long)n_out);
  HERO_REQUIRE(a->token || a->A.rows == R, HERO_ERR_INVALID_ARG, "without token A and out have the same rows (%lld, %lld)", (long long)a->A.rows, (long long)R);
  HERO_REQUIRE(is_q8(a->out.dtype) || is_fp16ish(a->out.dtype), HERO_ERR_UNSUPPORTED, "out dtype %d", a->out.dtype);
  HERO_REQUIRE(a->out.dtype != HERO_F8 || !int8, HERO_ERR_UNSUPPORTED, "an e4m3 output needs e4m3 or FP operands");
  HERO_REQUIRE(a->out.dtype != HERO_I8 || !f8, HERO_ERR_UNSUPPORTED, "an INT8 output needs INT8 or FP operands");
  HERO_REQUIRE(!(is_q8(a->out.dtype) && a->out.gran == HERO_GRAN_TWQ), HERO_ERR_UNSUPPORTED,
               "a token-wise (TWQ) output needs a row reduction, which is kept out of GEMM epilogues (Sec. 2.1)");
  HERO_REQUIRE(!q8 || a->w_scale, HERO_ERR_INVALID_ARG, "w_scale is required");
  HERO_REQUIRE(a->act >= HERO_ACT_NONE && a->act <= HERO_ACT_SILU, HERO_ERR_INVALID_ARG, "unknown activation %d", a->act);
  HERO_REQUIRE(a->out_col_absmax == nullptr || is_fp16ish(a->out.dtype), HERO_ERR_UNSUPPORTED, "out_col_absmax observes an F16 / BF16 output");
  HERO_REQUIRE(a->offset, HERO_ERR_INVALID_ARG, "offset is required");
  if (R == 0) return HERO_OK;
  HERO_REQUIRE(a->A.rows > 0, HERO_ERR_INVALID_ARG, "A has no rows");
  if ((st = check_device(h)) != HERO_OK) return st;

  MoeLinearParams p;
  memset(&p, 0, sizeof(p));
  p.R = (int)R; p.a_rows = (int)a->A.rows; p.E = (int)E; p.N = (int)N; p.n_out = (int)n_out;
  p.num_kb = (int)((K * eb + GEMM_BK_BYTES - 1) / GEMM_BK_BYTES);
  p.offset = a->offset; p.token = a->token;
  p.rs = q8 && a->A.gran == HERO_GRAN_TWQ ? a->A.scale : nullptr;
  p.cs = q8 ? a->w_scale : nullptr;
  p.bias = a->bias; p.post = a->post_scale;
  p.out = a->out.data; p.out_ld = a->out.ld; p.out_dt = a->out.dtype;
  p.act = a->act; p.f8 = f8 ? 1 : 0;
  p.kelems = GEMM_BK_BYTES / eb;
  p.obs = a->out_col_absmax;
  p.err = h->d_error;
  // Rows of an expert on average decide.  Few: single CTAs with tiles of 32 rows, two on an SM, so that one streams weights while the other starts or
  // ends (a chain of router, FC1, FC2 and combine, 16 tokens, 64 experts, top 8, 2048 x 1024: 81 us; one CTA an SM, 64 rows: 91).  Many: pairs.
  // Both sides, us, FC1 / FC2 of 64 experts, 2048 x 1024: 24 rows 50.4 / 26.9 single, 52.4 / 28.7 pairs; 32 rows 54.0 / 28.4 and 53.4 / 29.4;
  // 16 experts, 4096 x 2048: 24 rows 47.2 / 27.3 and 52.9 / 30.1; 32 rows 52.0 / 29.8 and 53.3 / 30.2.  Beyond, a second tile of an expert costs singles
  // the weights again.
  const bool pair = R > 32 * E;
  const uint32_t bf = a->A.dtype == HERO_BF16 ? 1 : 0;
  const int m = pair ? 256 : 128;
  p.idesc = int8 ? ptx::make_idesc(2, 1, 1, 0, 0, m, 0) : f8 ? ptx::make_idesc(1, 0, 0, 0, 0, m, 0) : ptx::make_idesc(1, bf, bf, 0, 0, m, 0);
  CUtensorMap tmW, tmA;
  st = make_tmap_experts(h, &tmW, a->W, a->A.dtype, a->gated != 0, pair ? 128 : 32, N, K, E, a->ldw, E == 1 ? N * a->ldw : a->expert_stride);
  if (st != HERO_OK) return st;
  st = make_tmap_2d(h, &tmA, a->A.data, eb, a->A.dtype == HERO_F16, a->A.dtype == HERO_BF16, (uint64_t)a->A.rows, (uint64_t)K, (uint64_t)a->A.ld * eb,
                    GEMM_BK_BYTES / eb, a->token ? 1 : pair ? MoeCfg<true, false>::BOX : MoeCfg<false, false>::BOX, 128);
  if (st != HERO_OK) return st;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
#define MOE_LAUNCH(INT8, GATED) (a->token ? launch_moe_linear<INT8, GATED, true>(h, tmW, tmA, p, pair, s) : launch_moe_linear<INT8, GATED, false>(h, tmW, tmA, p, pair, s))
  if (int8) return a->gated ? MOE_LAUNCH(true, true) : MOE_LAUNCH(true, false);
  return a->gated ? MOE_LAUNCH(false, true) : MOE_LAUNCH(false, false);
#undef MOE_LAUNCH
}
