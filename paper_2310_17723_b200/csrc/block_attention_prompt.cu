// hero_block_attention for many rows per key / value head (pieces of a prompt, long drafts): tensor-core bound, so the products run
// on tcgen05 (kind::f16, FP32 accumulators in tensor memory) and everything else is arranged around keeping them fed.
//
// One CTA takes 256 rows ((row of the sequence, query head of the group) pairs, two tiles of 128) of one (sequence, key / value head)
// and walks its keys, or one of several equal parts of them where CTAs are few, in tiles of 128.  Keys and values have to become FP16 operands in shared memory on the way: done once per CTA,
// for both row tiles.  Roles:
//   warps 0-3, 4-7   softmax of row tile 0 / 1, one row per thread: no reduction across threads.  A tile of keys is two halves of 64
//                    with a score buffer each, so the softmax of one half runs beside the products of the other.  Scores are read
//                    from tensor memory once (again only when the maximum moves); P goes back as FP16 into the columns of
//                    the scores and is the A operand of P V from there.  These warps bound the kernel: two on each scheduler, whose
//                    exponentials take 40 % of the cycles and whose waits and instructions the rest, so they have one barrier to
//                    wait for per half, the scores'
//   warps 8-15       codes -> FP16: 16-byte loads one tile ahead in registers, exact conversion, stores in the 128-byte swizzled
//                    operand layout
//   warps 16, 17     issue the products of row tile 0 / 1
//   warp 18          publishes what the softmax needs of each 16 tokens: key scale, value scale relative to the largest so far.  It
//                    arrives on the barrier of the keys, which the scores wait for (a barrier of their own cost 319 against 291 us,
//                    2048 rows on 6000 tokens, heads 32 / 8 of 128)
// The value scale of a page is folded into the exponent, e' = 2^(x + log2 rv), so that it costs nothing per element; the row sum
// undoes it per 16 tokens (rv is kept above 2^-40, where P is zero anyway).  As in the kernel for few rows, queries are scaled into
// FP16 by a power of two and P is rounded to FP16 (the products take 16 bits on both sides): half a step, and 2^-33 of the largest
// value scale met where a probability times its page's relative scale is below 2^-22.  No maximum is taken per tile: P is formed with the maximum so far, and only if 16 probabilities
// sum to more than FP16 holds (or in the first half) is the half read again for its maximum, O rescaled in tensor memory.
#include "block_attention.cuh"
#include "block_ring.cuh"
#include <cmath>
#include <type_traits>

namespace hero {

constexpr int PR_SM_WARPS = 8, PR_CV_WARPS = 8;
constexpr int PR_MMA_WARP = PR_SM_WARPS + PR_CV_WARPS;         // and the next one
constexpr int PR_SCRIBE_WARP = PR_MMA_WARP + 2;
constexpr int PR_THREADS = (PR_MMA_WARP + 4) * 32;             // whole warpgroups: the register file is dealt out to them
// 640 threads are launched with 96 registers each; 256 x 136 + 256 x 72 + 128 x 56 = 60416 of those 61440
constexpr int PR_SM_REGS = 136, PR_CV_REGS = 72, PR_MMA_REGS = 56;
constexpr int PR_ROWS = 256, PR_KEYS = 128;
constexpr int PR_PART = 4;                                     // tiles of keys of a part, at least, where a group's keys are split
constexpr int PR_INFO = 4;                                     // ring of scale records
constexpr float PR_SHIFT = 8.0f;                               // P carries a factor 2^8 when the maximum has just moved
constexpr float PR_MOST = 65504.0f;                            // and 16 of them sum to no more than this, so none overflows FP16
constexpr float PR_HIGH = 11.9f;                               // 16 x 2^PR_HIGH stays below that
constexpr float PR_COARSE = 524288.0f;                         // 2^19: maxima up to here are rounded by less than 2^-4
constexpr float PR_MIN_RV = 9.094947e-13f;                     // 2^-40


__device__ __forceinline__ float min_or_nan(float a, float b) {
  float y;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}

template <int DH>
struct PromptCfg {
  static constexpr int SUB = 128 * 128;                        // one [128 rows x 64 features] FP16 sub-tile, 128-byte rows
  static constexpr int TILE = SUB * (DH / 64);
  static constexpr int OFF_K = 2 * TILE, OFF_V = OFF_K + 2 * TILE;
  static constexpr int OFF_INFO = OFF_V + 2 * TILE;            // float4 [PR_INFO][8], of 16 tokens each: key scale, log2 and reciprocal of the relative value scale
  static constexpr int OFF_REF = OFF_INFO + PR_INFO * 8 * 16;  // float2 [PR_INFO]: largest value scale so far, its old / new ratio
  static constexpr int OFF_BARS = OFF_REF + PR_INFO * 8;
  static constexpr int NBARS = 2 + 4 + 4 + 12;
  static constexpr int BYTES = 1024 + OFF_BARS + NBARS * 8 + 16;
  static constexpr int S_COL = 0, O_COL = 256;                 // scores (then P) 2 x 128 columns, O 2 x DH columns
};

// sequence, head and row tile of a group: late rows, which see many keys, of all sequences first
__device__ __forceinline__ void prompt_group(const BlockAttnParams& p, int group, int& b, int& hk, int& qt) {
  const int bh = group % (p.c.nkv * p.B);
  hk = bh % p.c.nkv; b = bh / p.c.nkv; qt = p.tiles - 1 - group / (p.c.nkv * p.B);
}

template <int DH, bool BF, bool F8>
__global__ void __launch_bounds__(PR_THREADS, 1) block_attn_prompt_kernel(const __grid_constant__ BlockAttnParams p, const uint32_t idesc_qk,
                                                                          const uint32_t idesc_pv) {
  using Cfg = PromptCfg<DH>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + Cfg::OFF_BARS);
  uint64_t* q_full = bars;                       // [2] softmax warps of a tile -> its issuer
  uint64_t* k_full = q_full + 2;                 // [2] converters and scribe -> issuers
  uint64_t* k_empty = k_full + 2;                // [2] issuers -> converters
  uint64_t* v_full = k_empty + 2;                // [2]
  uint64_t* v_empty = v_full + 2;                // [2]
  uint64_t* s_full = v_empty + 2;                // [tile][half] scores are complete
  uint64_t* p_full = s_full + 4;                 // [tile][half] P is in place (and O rescaled)
  uint64_t* o_full = p_full + 4;                 // [tile] P V of a half is complete
  uint64_t* o_last = o_full + 2;                 // [tile] the last one is
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(o_last + 2);
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;   // (uniform: addresses by warp stay in uniform registers)

  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      ptx::mbar_init(&q_full[i], 4);
      ptx::mbar_init(&k_full[i], PR_CV_WARPS + 1); ptx::mbar_init(&k_empty[i], 2);
      ptx::mbar_init(&v_full[i], PR_CV_WARPS); ptx::mbar_init(&v_empty[i], 2);
      ptx::mbar_init(&o_full[i], 1); ptx::mbar_init(&o_last[i], 1);
    }
    for (int i = 0; i < 4; ++i) { ptx::mbar_init(&s_full[i], 1); ptx::mbar_init(&p_full[i], 4); }
    ptx::fence_mbar_init();
  }
  if (warp == PR_MMA_WARP) { ptx::tmem_alloc(tmem_slot, 512); ptx::tmem_relinquish(); }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  ptx::pdl_launch_dependents();
  ptx::pdl_wait();

  const BlockView& c = p.c;
  int b, hk, qt;
  prompt_group(p, blockIdx.x / p.splits, b, hk, qt);
  const SeqRows s = seq_rows(c, b);
  const int total = s.n * p.group, rb = qt * PR_ROWS, base = s.len - s.n;
  // keys of a row tile's last row, and its tiles of keys
  auto keys_of = [&](int t) {
    const int first = rb + 128 * t;
    return first >= total ? 0 : max(base + (min(first + 128, total) - 1) / p.group + 1, 0);
  };
  const int L = max(keys_of(0), keys_of(1));
  // of its tiles of keys this CTA has one part: n_all tiles from key0 on
  const int n_group = (L + PR_KEYS - 1) / PR_KEYS, part = blockIdx.x % p.splits;
  const int per = p.splits == 1 ? n_group : max((n_group + p.splits - 1) / p.splits, PR_PART);
  const int j0 = min(part * per, n_group), n_all = min(per, n_group - j0), key0 = j0 * PR_KEYS;
  auto tiles_of = [&](int t) { return min(max((keys_of(t) + PR_KEYS - 1) / PR_KEYS - j0, 0), n_all); };

  if (rb >= total) {
    // nothing of this sequence here
  } else if (warp < PR_SM_WARPS) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(PR_SM_REGS));
    // ------------------------------------------------------------------ softmax of one row tile
    const int t = warp >> 2, quarter = warp & 3, r = quarter * 32 + lane;
    const int n = tiles_of(t);
    const int rr = rb + 128 * t + r;
    const bool row_ok = rr < total;
    const int lim = row_ok ? base + rr / p.group + 1 - key0 : 0;
    const long long row_g = s.r0 + (row_ok ? rr / p.group : 0);
    const int hq = hk * p.group + (row_ok ? rr % p.group : 0);
    float f = 0.f;
    if (n > 0) {
      // the row as FP16, scaled by a power of two (and by the sign of the score factor), in the swizzled operand layout
      uint32_t w[DH / 2], top = 0;
      const uint4* q = reinterpret_cast<const uint4*>(p.q + row_g * p.ld_q + (long long)hq * DH);
#pragma unroll
      for (int i = 0; i < DH / 8; ++i) {
        const uint4 x = row_ok ? written(q + i) : make_uint4(0, 0, 0, 0);
        w[4 * i] = x.x; w[4 * i + 1] = x.y; w[4 * i + 2] = x.z; w[4 * i + 3] = x.w;
      }
#pragma unroll
      for (int i = 0; i < DH / 2; ++i) top = __vmaxu2(top, w[i] & 0x7fff7fffu);
      const float amax = fp16ish_to_f32x2<BF>(max(top & 0xffffu, top >> 16)).x;
      const float up = query_factor(amax);
      f = fabsf(p.c2) / up;
      const float up_s = p.c2 < 0.f ? -up : up;
      uint8_t* row = smem + t * Cfg::TILE + (r >> 3) * 1024 + (r & 7) * 128;
#pragma unroll
      for (int i = 0; i < DH / 8; ++i) {
        uint32_t h[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 x = fp16ish_to_f32x2<BF>(w[4 * i + j]);
          h[j] = pack_f16(x.x * up_s, x.y * up_s);
        }
        *reinterpret_cast<uint4*>(row + (i >> 3) * Cfg::SUB + (((i & 7) ^ (r & 7)) << 4)) = make_uint4(h[0], h[1], h[2], h[3]);
      }
      ptx::fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(&q_full[t]);
    }
    const uint32_t t_lane = tmem_base + ((uint32_t)(quarter * 32) << 16);
    const uint32_t s_col = t_lane + Cfg::S_COL + t * 128, o_col = t_lane + Cfg::O_COL + t * DH;
    float u = 0.f, l = 0.f, vref = 0.f;            // u = PR_SHIFT - running maximum
    bool ok = true;
    // The first 32 scores of the next half can be read beside the second half's work on this one: 452 -> 403 us with 64 features (2 x 16
    // heads, 4096 rows on 4096 tokens); with 128 the products of the two row tiles keep tensor memory busier, and it cost 1 %.
    constexpr bool AHEAD = DH == 64;
    bool ahead = false;
    uint32_t x[2][32];
    for (int j = 0; j < n && ok; ++j) {
      const int slot = j % PR_INFO;
#pragma unroll 1
      for (int h = 0; h < 2; ++h) {
        if (!AHEAD || !ahead) {
          ok = __all_sync(0xffffffffu, ok && ptx::mbar_wait(&s_full[2 * t + h], j & 1, c.err, 0x8100 | t));
          if (!ok) break;
          ptx::tc_fence_after();
          if (AHEAD) ptx::tmem_ld32(s_col + 64 * h, x[0]);
        }
        // (the record was there before the tile's keys were announced, so before its scores)
        const float2 ref = reinterpret_cast<const float2*>(smem + Cfg::OFF_REF)[slot];
        vref = ref.x;
        const uint32_t s_half = s_col + 64 * h;
        const float4* info = reinterpret_cast<const float4*>(smem + Cfg::OFF_INFO) + slot * 8 + 4 * h;
        const int valid = lim - j * PR_KEYS - 64 * h;                      // keys of this half that the row sees
        const bool whole = __all_sync(0xffffffffu, valid >= 64), first = (j | h) == 0, turn = h == 0 && ref.y != 1.0f;
        // e' = 2^(score - maximum + 8 + log2 rv) and the row sum in one reading; false, with nothing changed, if a sum outgrows FP16.
        // (Compiled for each case by itself: chosen at every 16 keys it took 291 against 285 us, 2048 rows on 6000 tokens.)
        auto one_reading = [&](auto masked) {
          float4 gi[4];                            // of 16 keys each: key scale, log2 rv, 1 / rv
#pragma unroll
          for (int g = 0; g < 4; ++g) gi[g] = info[g];
          uint32_t w[32];
          if (!AHEAD) ptx::tmem_ld32(s_half, x[0]);
          ptx::tmem_ld_wait();
          ptx::tmem_ld32(s_half + 32, x[1]);
          float l_new = l, most = 0.f;
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            if (g == 2) {
              ptx::tmem_ld_wait();
              if (AHEAD) {
                const bool more = h == 0 || j + 1 < n;
                ahead = __all_sync(0xffffffffu, more && ptx::mbar_test(&s_full[2 * t + (h ^ 1)], (j + h) & 1));
                if (ahead) {
                  ptx::tc_fence_after();
                  ptx::tmem_ld32(s_col + 64 * (h ^ 1), x[0]);
                }
              }
            }
            const uint32_t* y = &x[g >> 1][16 * (g & 1)];
            const float fk = f * gi[g].x, ug = u + gi[g].y;
            float2 sum = make_float2(0.f, 0.f);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float2 a = __ffma2_rn(make_float2(__uint_as_float(y[2 * i]), __uint_as_float(y[2 * i + 1])), make_float2(fk, fk), make_float2(ug, ug));
              float2 e = make_float2(ex2(a.x), ex2(a.y));
              if constexpr (decltype(masked)::value) {
                if (16 * g + 2 * i >= valid) e.x = 0.f;
                if (16 * g + 2 * i + 1 >= valid) e.y = 0.f;
              }
              sum = __fadd2_rn(sum, e);
              w[8 * g + i] = pack_f16(e.x, e.y);
            }
            const float both = sum.x + sum.y;
            most = fmaxf(most, both);
            l_new = fmaf(both, gi[g].z, l_new);
          }
          const bool fits = !__any_sync(0xffffffffu, most > PR_MOST);
          if (AHEAD) ptx::tmem_ld_wait();
          if (fits) {
            l = l_new;
            // P over the scores' columns
#pragma unroll
            for (int k = 0; k < 2; ++k) ptx::tmem_st16(s_half + 16 * k, *reinterpret_cast<const uint32_t(*)[16]>(&w[16 * k]));
          }
          return fits;
        };
        if (first || turn || !(whole ? one_reading(std::false_type()) : one_reading(std::true_type()))) {
          if (AHEAD) { ahead = false; ptx::tmem_ld_wait(); }
          // ---- the first keys, a larger value scale, or probabilities that outgrow FP16: the half's maximum first
          float mx = -INFINITY;
#pragma unroll 1
          for (int g = 0; g < 4; ++g) {
            uint32_t z[16];
            ptx::tmem_ld16(s_half + 16 * g, z);
            ptx::tmem_ld_wait();
            float m = -INFINITY;
#pragma unroll
            for (int i = 0; i < 16; ++i) m = fmaxf(m, 16 * g + i < valid ? __uint_as_float(z[i]) : -INFINITY);
            if (m > -INFINITY) mx = fmaxf(mx, fmaf(m, f * info[g].x, u));
          }
          // where it calls for it, it moves the row's, O and the sum follow, and O the value reference
          // (A maximum beyond 2^PR_COARSE is itself rounded by more than the places above the largest probability can take.  Such a row's
          // reference is put eight of its roundings too low, so that no rounding leaves the largest key without weight, keys up
          // there count alike (the bound on e0, e1 below), and the maximum moves for a key above all of them only.)
          const float slack = fabsf(u) > PR_COARSE ? fabsf(u) * 0x1p-20f : 0.f;
          if (__any_sync(0xffffffffu, first || mx > PR_HIGH + slack) || turn) {
            float d = mx - PR_SHIFT;
            if (!first) d = fmaxf(d, 0.f);
            if (mx == -INFINITY) d = 0.f;
            if (fabsf(u - d) > PR_COARSE) {
              if (!first && slack != 0.f && mx <= PR_HIGH + slack) d = 0.f;
              if (d != 0.f) d = u - fmaf(fabsf(u - d), 0x1p-21f, u - d);
            }
            u -= d;
            if (!first) {
              ok = __all_sync(0xffffffffu, ok && ptx::mbar_wait(&o_full[t], (h + 1) & 1, c.err, 0x8180 | t));   // the previous half's P V
              ptx::tc_fence_after();
              const float a = ex2(-d);
              l *= a;
              const float ao = turn ? a * ref.y : a;
#pragma unroll 1
              for (int k = 0; k < DH / 16; ++k) {
                uint32_t z[16];
                ptx::tmem_ld16(o_col + 16 * k, z);
                ptx::tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < 16; ++i) z[i] = __float_as_uint(__uint_as_float(z[i]) * ao);
                ptx::tmem_st16(o_col + 16 * k, z);
              }
            }
          }
          // P of 16 keys takes the place of scores that have been read: columns 8 g .. 8 g + 7, after 16 g .. 16 g + 15
#pragma unroll 1
          for (int g = 0; g < 4; ++g) {
            const float4 gi = info[g];
            const float fk = f * gi.x, ug = u + gi.y;
            uint32_t z[16], w[8];
            ptx::tmem_ld16(s_half + 16 * g, z);
            ptx::tmem_ld_wait();
            float2 sum = make_float2(0.f, 0.f);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const int key = 16 * g + 2 * i;
              const float x0 = fmaf(__uint_as_float(z[2 * i]), fk, ug), x1 = fmaf(__uint_as_float(z[2 * i + 1]), fk, ug);
              const float e0 = key < valid ? ex2(min_or_nan(x0, PR_HIGH)) : 0.f;
              const float e1 = key + 1 < valid ? ex2(min_or_nan(x1, PR_HIGH)) : 0.f;
              sum.x += e0; sum.y += e1;
              w[i] = pack_f16(e0, e1);
            }
            l = fmaf(sum.x + sum.y, gi.z, l);
            ptx::tmem_st8(s_half + 8 * g, w);
          }
        }
        ptx::tmem_st_wait();
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&p_full[2 * t + h]);
      }
    }
    // ---- output, or the part's sums
    // (O is divided by the row's sum before the value scale enters: near the ends of BF16's range neither O times the scale nor the scale
    // over the sum is a number that FP32 holds)
    float scale_o = 0.f;
    const bool tiny = vref < 0x1p-60f;
    if (n > 0) {
      ok = __all_sync(0xffffffffu, ok && ptx::mbar_wait(&o_last[t], 0, c.err, 0x8200 | t));
      ptx::tc_fence_after();
      scale_o = l != 0.f ? (tiny ? 1.0f : vref) / l : 0.f;
    }
    const long long own = (long long)blockIdx.x * PR_ROWS + 128 * t + r;   // the row's place among the parts
    const bool seen = n > 0 && l != 0.f;
    if (p.splits > 1 && row_ok) p.part_ml[own] = make_float2(part_maximum(ok, seen, -u), l);
#pragma unroll
    for (int k = 0; k < DH / 32; ++k) {
      uint32_t x[32];
      if (n > 0) {
        ptx::tmem_ld32(o_col + 32 * k, x);
        ptx::tmem_ld_wait();
      }
      float y[32];
#pragma unroll
      for (int i = 0; i < 32; ++i) y[i] = seen ? __uint_as_float(x[i]) * scale_o : 0.f;
      if (tiny) {
#pragma unroll
        for (int i = 0; i < 32; ++i) y[i] *= vref;
      }
      if (p.splits > 1) {
        if (seen && row_ok && ok) {
          float4* dst = reinterpret_cast<float4*>(p.part_o + own * DH + 32 * k);
#pragma unroll
          for (int i = 0; i < 8; ++i) dst[i] = make_float4(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
        }
      } else if (row_ok && ok) {
        const int col = hq * DH + 32 * k;
        const long long at = row_g * p.ld_out + col;
        if (p.out_dt == HERO_F16 || p.out_dt == HERO_BF16) {
          uint4* dst = reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.out) + at);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t o[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
              o[e] = p.out_dt == HERO_F16 ? f32x2_to_fp16ish<false>(y[8 * i + 2 * e], y[8 * i + 2 * e + 1]) : f32x2_to_fp16ish<true>(y[8 * i + 2 * e], y[8 * i + 2 * e + 1]);
            dst[i] = make_uint4(o[0], o[1], o[2], o[3]);
          }
        } else {
          uint4* dst = reinterpret_cast<uint4*>(static_cast<uint8_t*>(p.out) + at);
#pragma unroll
          for (int i = 0; i < 32; ++i) y[i] /= __ldg(p.out_scale + (long long)(col + i) * p.out_scale_stride);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            uint32_t o[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float* z = y + 16 * i + 4 * e;
              o[e] = p.out_dt == HERO_F8 ? f32_to_codes4<true>(z[0], z[1], z[2], z[3]) : f32_to_codes4<false>(z[0], z[1], z[2], z[3]);
            }
            dst[i] = make_uint4(o[0], o[1], o[2], o[3]);
          }
        }
      }
    }
  } else if (warp < PR_MMA_WARP) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(PR_CV_REGS));
    // ------------------------------------------------------------------ codes -> FP16 operands
    constexpr int NP = DH / 32;                    // 16-code pieces of a tile per thread
    constexpr int NSUB = DH / 64;
    // four lanes take 64 features of a row, eight lanes two rows: whole sectors from memory, no bank conflicts in the operand tile
    const int ct = threadIdx.x - PR_SM_WARPS * 32, piece = ct & 3, r0 = ct >> 2;       // rows r0 + 64 i
    const long long mine = (long long)hk * c.head_stride + (long long)(r0 & 15) * c.ld + piece * 16;
    uint8_t* const to0 = smem + (r0 >> 3) * 1024 + (r0 & 7) * 128 + (((2 * piece) ^ (r0 & 7)) << 4);
    uint8_t* const to1 = smem + (r0 >> 3) * 1024 + (r0 & 7) * 128 + (((2 * piece + 1) ^ (r0 & 7)) << 4);
    auto page_of = [&](int j) {                    // lane g < 8: page of tokens key0 + 128 j + 16 g ..
      const int tok = key0 + j * PR_KEYS + 16 * lane;
      return lane < 8 && tok < L ? page_for_read(c, b, tok >> c.page_shift) : -1;
    };
    long long at[2];                               // where the thread's two rows begin in the pool
    auto locate = [&](int j, int id) {
      const long long off = (long long)id * c.page_stride + (long long)((j * PR_KEYS + 16 * lane) & (c.page - 1)) * c.ld;
#pragma unroll
      for (int i = 0; i < 2; ++i) at[i] = mine + __shfl_sync(0xffffffffu, off, 4 * i + (r0 >> 4));
    };
    auto load = [&](const uint8_t* pool, int j, uint4 (&raw)[NP]) {
      if (key0 + (j + 1) * PR_KEYS <= L) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int h = 0; h < NSUB; ++h) raw[i * NSUB + h] = written(reinterpret_cast<const uint4*>(pool + at[i] + 64 * h));
      } else {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int h = 0; h < NSUB; ++h) {
            raw[i * NSUB + h] = make_uint4(0, 0, 0, 0);        // slots behind the end may hold anything (e4m3: NaN)
            if (key0 + j * PR_KEYS + r0 + 64 * i < L) raw[i * NSUB + h] = written(reinterpret_cast<const uint4*>(pool + at[i] + 64 * h));
          }
      }
    };
    auto store = [&](uint32_t tile, const uint4 (&raw)[NP]) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int h = 0; h < NSUB; ++h) {
          const uint4 x = raw[i * NSUB + h];
          uint32_t y[8];
          codes4_to_f16<F8>(x.x, y[0], y[1]);
          codes4_to_f16<F8>(x.y, y[2], y[3]);
          codes4_to_f16<F8>(x.z, y[4], y[5]);
          codes4_to_f16<F8>(x.w, y[6], y[7]);
          *reinterpret_cast<uint4*>(to0 + tile + h * Cfg::SUB + i * 8192) = make_uint4(y[0], y[1], y[2], y[3]);
          *reinterpret_cast<uint4*>(to1 + tile + h * Cfg::SUB + i * 8192) = make_uint4(y[4], y[5], y[6], y[7]);
        }
      ptx::fence_proxy_async_smem();
      __syncwarp();
    };
    uint4 kr[NP], vr[NP];
    bool ok = true;
    int ids_next = page_of(1);
    if (n_all > 0) { locate(0, page_of(0)); load(c.k, 0, kr); load(c.v, 0, vr); }
    for (int j = 0; j < n_all; ++j) {
      const int st = j & 1;
      const uint32_t par = ((j >> 1) & 1) ^ 1;
      locate(j + 1, ids_next);
      ids_next = page_of(j + 2);
      ok = ok && ptx::mbar_wait(&k_empty[st], par, c.err, 0x8400 | st);
      store(Cfg::OFF_K + st * Cfg::TILE, kr);
      if (lane == 0) ptx::mbar_arrive(&k_full[st]);
      if (j + 1 < n_all) load(c.k, j + 1, kr);
      ok = ok && ptx::mbar_wait(&v_empty[st], par, c.err, 0x8500 | st);
      store(Cfg::OFF_V + st * Cfg::TILE, vr);
      if (lane == 0) ptx::mbar_arrive(&v_full[st]);
      if (j + 1 < n_all) load(c.v, j + 1, vr);
      if (!__all_sync(0xffffffffu, ok)) break;
    }
  } else {
   asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(PR_MMA_REGS));
   if (warp == PR_SCRIBE_WARP) {
    // ------------------------------------------------------------------ scale records
    auto page_of = [&](int j) {                    // lane g < 8: page of tokens key0 + 128 j + 16 g ..
      const int tok = key0 + j * PR_KEYS + 16 * lane;
      return lane < 8 && tok < L ? page_for_read(c, b, tok >> c.page_shift) : -1;
    };
    auto scales = [&](int i) { return i >= 0 ? make_float2(written(c.ks + (long long)i * c.nkv + hk), written(c.vs + (long long)i * c.nkv + hk)) : make_float2(0.f, 0.f); };
    int ids_next = page_of(1);
    float2 sc = scales(page_of(0));
    float vref = 0.f;
    for (int j = 0; j < n_all; ++j) {
      const int slot = j % PR_INFO;
      const float2 now_sc = sc;
      sc = scales(ids_next);
      ids_next = page_of(j + 2);
      float top = now_sc.y;
#pragma unroll
      for (int o = 4; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      const float now = fmaxf(vref, __shfl_sync(0xffffffffu, top, 0));
      const float rv = fmaxf(now > 0.f ? now_sc.y / now : 1.f, PR_MIN_RV);
      // the keys' place is free: the scores two tiles back are complete, so nobody reads records four tiles back any more
      if (!__all_sync(0xffffffffu, ptx::mbar_wait(&k_empty[j & 1], ((j >> 1) & 1) ^ 1, c.err, 0x8300 | slot))) break;
      if (lane < 8) *reinterpret_cast<float4*>(smem + Cfg::OFF_INFO + (slot * 8 + lane) * 16) = make_float4(now_sc.x, __log2f(rv), 1.0f / rv, 0.f);
      if (lane == 0) reinterpret_cast<float2*>(smem + Cfg::OFF_REF)[slot] = make_float2(now, now > vref ? vref / now : 1.0f);
      vref = now;
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(&k_full[j & 1]);
    }
   } else if (warp < PR_SCRIBE_WARP) {
    // ------------------------------------------------------------------ issuer of one row tile
    const int t = warp - PR_MMA_WARP, n = tiles_of(t);
    const bool issue = ptx::elect_one();
    constexpr uint64_t kmaj = ptx::smem_desc_base(16, 1024, ptx::SWZ_128B);            // Q, K: K-major, 128-byte rows
    constexpr uint64_t vmaj = ptx::smem_desc_base(Cfg::SUB, 1024, ptx::SWZ_128B);      // V: MN-major; 64-feature chunks SUB apart
    const uint64_t qd = ptx::smem_desc(kmaj, ptx::smem_u32(smem + t * Cfg::TILE));
    const uint64_t kd0 = ptx::smem_desc(kmaj, ptx::smem_u32(smem + Cfg::OFF_K)), vd0 = ptx::smem_desc(vmaj, ptx::smem_u32(smem + Cfg::OFF_V));
    const uint32_t s_tmem = tmem_base + Cfg::S_COL + t * 128, o_tmem = tmem_base + Cfg::O_COL + t * DH;
    auto scores = [&](int j, int h) {              // of 64 keys, into buffer h
      if (issue) {
        const uint64_t kd = kd0 + (uint32_t)(((j & 1) * Cfg::TILE + h * 8192) >> 4);
#pragma unroll
        for (int k = 0; k < DH / 16; ++k) {
          const uint32_t o = (uint32_t)(((k >> 2) * Cfg::SUB + (k & 3) * 32) >> 4);
          ptx::umma_f16(s_tmem + 64 * h, qd + o, kd + o, idesc_qk, k != 0);
        }
        ptx::umma_commit(&s_full[2 * t + h]);
        if (h == 1) ptx::umma_commit(&k_empty[j & 1]);
      }
    };
    auto keys_ready = [&](int j) {
      const bool r = ptx::mbar_wait(&k_full[j & 1], (j >> 1) & 1, c.err, 0x8600 | (j & 1));
      ptx::tc_fence_after();
      return r;
    };
    bool ok = true;
    if (n > 0) {
      ok = ptx::mbar_wait(&q_full[t], 0, c.err, 0x8700 | t) && keys_ready(0);
      if (ok) { scores(0, 0); scores(0, 1); }
    }
    for (int j = 0; j < n && ok; ++j) {
      const int st = j & 1;
      ok = ptx::mbar_wait(&v_full[st], (j >> 1) & 1, c.err, 0x8800 | st);
#pragma unroll 1
      for (int h = 0; h < 2 && ok; ++h) {
        ok = ptx::mbar_wait(&p_full[2 * t + h], j & 1, c.err, 0x8900 | t);
        if (!ok) break;
        ptx::tc_fence_after();
        if (issue) {
          const uint64_t vd = vd0 + (uint32_t)((st * Cfg::TILE + h * 8192) >> 4);
#pragma unroll
          for (int k = 0; k < 4; ++k)              // 16 keys: 8 columns of P, 2 eight-key groups of V
            ptx::umma_f16_ta(o_tmem, s_tmem + 64 * h + 8 * k, vd + (uint32_t)((k * 2048) >> 4), idesc_pv, (j | h | k) != 0);
          if (h == 1) ptx::umma_commit(&v_empty[st]);
          ptx::umma_commit(&o_full[t]);
          if (h == 1 && j + 1 == n) ptx::umma_commit(&o_last[t]);
        }
        if (j + 1 < n) {
          // the next tile's scores of this half take the place of its P: P V has to be complete
          ok = (h == 1 || keys_ready(j + 1)) && ptx::mbar_wait(&o_full[t], h, c.err, 0x8A00 | t);
          if (ok) scores(j + 1, h);
        }
      }
    }
    // keys that only the other row tile needs
    for (int j = n; j < n_all && ok; ++j) {
      const int st = j & 1;
      ok = ptx::mbar_wait(&k_full[st], (j >> 1) & 1, c.err, 0x8B00 | st);
      if (ok && lane == 0) ptx::mbar_arrive(&k_empty[st]);
      ok = ok && ptx::mbar_wait(&v_full[st], (j >> 1) & 1, c.err, 0x8C00 | st);
      if (ok && lane == 0) ptx::mbar_arrive(&v_empty[st]);
    }
    __syncwarp();
   }
  }
  ptx::tc_fence_before();
  __syncthreads();
  if (warp == PR_MMA_WARP) ptx::tmem_dealloc(tmem_base, 512);
}

// joins the parts of a group whose keys were split: CTA (x, y) takes 32 rows of group x, a warp four of them, side by side
constexpr int PJ_WARPS = 8, PJ_EACH = 4, PJ_ROWS = PJ_WARPS * PJ_EACH;
template <int DH>
__global__ void __launch_bounds__(PJ_WARPS * 32) block_attn_prompt_join_kernel(const __grid_constant__ BlockAttnParams p) {
  constexpr int E = DH / 32;
  ptx::pdl_wait();
  ptx::pdl_launch_dependents();
  int b, hk, qt;
  prompt_group(p, blockIdx.x, b, hk, qt);
  const SeqRows s = seq_rows(p.c, b);
  const int total = s.n * p.group, lane = threadIdx.x & 31, row0 = blockIdx.y * PJ_ROWS + (threadIdx.x >> 5) * PJ_EACH;
  float m[PJ_EACH], l[PJ_EACH], y[PJ_EACH][E];
#pragma unroll
  for (int i = 0; i < PJ_EACH; ++i) {
    m[i] = -INFINITY; l[i] = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) y[i][e] = 0.f;
  }
#pragma unroll 2
  for (int q = 0; q < p.splits; ++q) {
#pragma unroll
    for (int i = 0; i < PJ_EACH; ++i) {
      if (qt * PR_ROWS + row0 + i >= total) continue;              // rows that are not there were not written
      const long long at = ((long long)blockIdx.x * p.splits + q) * PR_ROWS + row0 + i;
      const float2 ml = written(p.part_ml + at);
      if (ml.x == -INFINITY) continue;                             // nor were sums of no keys
      // (a part is divided by its own sum: their mean, under weights that add up to one)
      const float now = fmaxf(m[i], ml.x), old = l[i] * ex2(m[i] - now), w = ex2(ml.x - now) * ml.y, inv = 1.0f / (old + w);
      m[i] = now;
      l[i] = old + w;
#pragma unroll
      for (int e = 0; e < E; ++e) y[i][e] = fmaf(y[i][e], old * inv, w * inv * written(p.part_o + at * DH + 32 * e + lane));
    }
  }
#pragma unroll
  for (int i = 0; i < PJ_EACH; ++i) {
    const int rr = qt * PR_ROWS + row0 + i;
    if (rr >= total) break;
#pragma unroll
    for (int e = 0; e < E; ++e) store_out(p, s.r0 + rr / p.group, (hk * p.group + rr % p.group) * DH + 32 * e + lane, y[i][e]);
  }
}

// Where there are fewer groups than half the SMs, each group's keys are split over as many CTAs as fit, and a second kernel joins them:
// 592 -> 104 us for 64 rows of one sequence on 32768 tokens (heads 32 / 8 of 128; 8 groups, 18 parts), 605 -> 329 for 512 rows (64 groups, 2
// parts), 66 -> 52 for 4 x 128 rows on 4096 tokens (64 groups of 64 features).
struct PromptPlan { long long tiles, groups; int splits; size_t bytes; };
static PromptPlan plan_tiles(const hero_handle* h, const hero_block_cache* cc, long long tiles) {
  PromptPlan r;
  r.tiles = tiles;
  r.groups = r.tiles * cc->nkv * cc->B;
  const long long fit = h->sm_count / r.groups, steps = ((long long)cc->max_len + PR_KEYS - 1) / PR_KEYS, useful = steps / PR_PART;
  const long long splits = fit < useful ? fit : useful;
  r.splits = splits > 1 ? (int)splits : 1;
  r.bytes = r.splits > 1 ? (size_t)r.groups * r.splits * PR_ROWS * (cc->dh * 4 + 8) : 0;
  return r;
}
static long long tiles_of(const hero_block_cache* cc, int nq, int max_rows) { return ((long long)max_rows * (nq / cc->nkv) + PR_ROWS - 1) / PR_ROWS; }
static hero_status plan_prompt(const hero_handle* h, const hero_block_cache* cc, int nq, int max_rows, PromptPlan* out) {
  const long long groups = tiles_of(cc, nq, max_rows) * cc->nkv * cc->B;
  HERO_REQUIRE(groups < (1ll << 31), HERO_ERR_UNSUPPORTED, "max_rows=%d nkv=%d B=%d: too many", max_rows, cc->nkv, cc->B);
  *out = plan_tiles(h, cc, tiles_of(cc, nq, max_rows));
  return HERO_OK;
}
hero_status prompt_workspace_bytes(const hero_handle* h, const hero_block_cache* cc, int nq, int max_rows, size_t* bytes) {
  PromptPlan plan;
  hero_status st = plan_prompt(h, cc, nq, max_rows, &plan);
  if (st == HERO_OK) *bytes = plan.bytes;
  return st;
}
// the most that any row bound up to max_rows needs here (keys are split up to half the SMs' groups only, so there are few to look at)
size_t prompt_workspace_most(const hero_handle* h, const hero_block_cache* cc, int nq, int max_rows) {
  const long long last = tiles_of(cc, nq, max_rows), split = h->sm_count / 2 / ((long long)cc->nkv * cc->B);
  size_t most = 0;
  for (long long t = 1; t <= last && t <= split; ++t) {
    const size_t bytes = plan_tiles(h, cc, t).bytes;
    most = bytes > most ? bytes : most;
  }
  return most;
}

template <int DH>
static hero_status launch(hero_handle* h, const PromptPlan& plan, const BlockAttnParams& p, bool bf, cudaStream_t stream) {
  auto kern = bf ? (p.c.f8 ? block_attn_prompt_kernel<DH, true, true> : block_attn_prompt_kernel<DH, true, false>)
                 : (p.c.f8 ? block_attn_prompt_kernel<DH, false, true> : block_attn_prompt_kernel<DH, false, false>);
  constexpr int BYTES = PromptCfg<DH>::BYTES;
  static PerDeviceOnce configured[4];              // per instantiation of the kernel
  PerDeviceOnce& once = configured[(bf ? 2 : 0) + (p.c.f8 ? 1 : 0)];
  if (!once.done(h->device)) {
    HERO_CUDA(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, BYTES));
    once.set(h->device);
  }
  const uint32_t idesc_qk = ptx::make_idesc(1, 0, 0, 0, 0, 128, 64), idesc_pv = ptx::make_idesc(1, 0, 0, 0, 1, 128, DH);
  {
    LaunchScope scope(h, stream, KERNEL_ATTN);
    HERO_CUDA(launch_dependent(kern, dim3((unsigned)(plan.groups * plan.splits)), dim3(PR_THREADS), BYTES, stream, p, idesc_qk, idesc_pv));
  }
  if (plan.splits > 1) {
    LaunchScope scope(h, stream, KERNEL_ATTN);
    HERO_CUDA(launch_dependent(block_attn_prompt_join_kernel<DH>, dim3((unsigned)plan.groups, PR_ROWS / PJ_ROWS), dim3(PJ_WARPS * 32), 0, stream, p));
  }
  return HERO_OK;
}

hero_status launch_prompt(hero_handle* h, const hero_block_cache* cc, const BlockAttnParams& p_, bool bf, void* workspace, cudaStream_t stream) {
  BlockAttnParams p = p_;
  PromptPlan plan;
  hero_status st = plan_prompt(h, cc, p.nq, p.c.max_rows, &plan);
  if (st != HERO_OK) return st;
  p.tiles = (int)plan.tiles; p.B = cc->B; p.splits = plan.splits;
  p.part_o = static_cast<float*>(workspace);
  p.part_ml = reinterpret_cast<float2*>(p.part_o + (size_t)plan.groups * plan.splits * PR_ROWS * cc->dh);
  return cc->dh == 64 ? launch<64>(h, plan, p, bf, stream) : launch<128>(h, plan, p, bf, stream);
}

}  // namespace hero
