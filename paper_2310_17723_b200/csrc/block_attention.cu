// Attention over the 8-bit block cache (hero_block_attention): o = softmax(scale q K^T) V, causal in a sequence's new rows.
#include "block_cache.cuh"
#include <cmath>
#include <cstdlib>
#include <cstdio>

namespace hero {

struct BlockAttnParams {
  BlockView c;
  const uint16_t* q; long long ld_q;
  void* out; long long ld_out; int out_dt;
  const float* out_scale; int out_scale_stride;
  int nq, group;
  float c2;                      // scale * log2(e)
  int cluster, outer;            // CTAs that share the tokens of a (sequence, head, row tile): of a cluster, clusters
  float* part_o; float2* part_ml; // partial results [row][query head][cluster]: sum of P V [DH], (maximum, sum of P)
};

__device__ __forceinline__ void store_out(const BlockAttnParams& p, long long row, int col, float y) {
  const long long at = row * p.ld_out + col;
  if (p.out_dt == HERO_F16) static_cast<__half*>(p.out)[at] = __float2half_rn(y);
  else if (p.out_dt == HERO_BF16) static_cast<__nv_bfloat16*>(p.out)[at] = __float2bfloat16_rn(y);
  else {
    const float z = y / __ldg(p.out_scale + (long long)col * p.out_scale_stride);
    static_cast<uint8_t*>(p.out)[at] = (uint8_t)(p.out_dt == HERO_F8 ? f32_to_codes4<true>(z, 0.f, 0.f, 0.f) : f32_to_codes4<false>(z, 0.f, 0.f, 0.f));
  }
}

// ------------------------------------------------------------------------------------------------------------------
// Few rows per key / value head (decode steps, drafts).  Every cached byte is read once and meets at most 16 query rows, so
// the kernel is bound by HBM and is built to keep loads in flight.  Each warp walks tiles of 16 tokens of its own through a ring of
// asynchronous copies in which every lane fetches exactly the 16 bytes that it will hold in the matrix instruction's fragments: no
// barrier in the loop, no bank conflicts, no transposition.  That works because the contraction's index may be permuted at will as
// long as both operands agree:
//   S^T [16 tokens x 8 rows] = K Q^T: lane (g, t) of mma.m16n8k16 loads features 64 c + 16 t .. + 15 of tokens g and g + 8; the four
//       k slots it holds in step (c, j) stand for features 64 c + 16 t + 4 j .. + 3, for K and Q alike.
//   O^T [features x 8 rows] = V^T P^T: lane (g, t) loads DH / 8 consecutive features of tokens 2t, 2t + 1, 2t + 8, 2t + 9; row g / g + 8
//       of M tile j stands for feature (DH / 8) g + 2 j / + 1.
// Rows are the N dimension (8, the smallest there is), so a single query row does not pad a tile to 16.  Codes become FP16
// exactly (INT8: byte permute into 1024 + u, subtract; e4m3: conversion instruction).  A query row is scaled by a power of two
// into FP16 (exact for F16, for BF16 down to 2^-39 of the row's maximum).  The page's key scale multiplies the scores; the value
// scale enters P relative to the largest one the warp has met (P <= 2^15: P is formed with a factor 2^11 so that pages whose scale
// is 2^-25 of the largest still meet FP16's normal range).  The running maximum is moved only when a score exceeds it by more than
// 4 in the exponent, so that most tiles need no reduction over tokens at all.
// Tokens are split over the warps of a CTA, the CTAs of a cluster (joined through distributed shared memory) and, where that does
// not fill the GPU, over clusters (partial results in the workspace, joined by a second kernel).
constexpr int ROWS_WARPS = 4;
constexpr int ROWS_MAX_CLUSTER = 8;
constexpr int ROWS_STAGES = 3;                  // ring depth in tiles of 16 tokens (keys and values: 32 DH bytes)
constexpr float P_SHIFT = 11.0f, MAX_SLACK = 4.0f;

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// four codes of one word -> f16x2 of codes (0, 1) and (2, 3)
template <bool F8>
__device__ __forceinline__ void codes4_to_f16(uint32_t w, uint32_t& lo, uint32_t& hi) {
  if constexpr (F8) {
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(lo) : "h"((uint16_t)(w & 0xffffu)));
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(hi) : "h"((uint16_t)(w >> 16)));
  } else {
    const uint32_t u = w ^ 0x80808080u;
    const __half2 off = __floats2half2_rn(1152.f, 1152.f);               // 1024 + 128
    uint32_t a = __byte_perm(u, 0x64646464u, 0x4140), b = __byte_perm(u, 0x64646464u, 0x4342);
    const __half2 x = __hsub2(*reinterpret_cast<__half2*>(&a), off), y = __hsub2(*reinterpret_cast<__half2*>(&b), off);
    lo = *reinterpret_cast<const uint32_t*>(&x); hi = *reinterpret_cast<const uint32_t*>(&y);
  }
}
__device__ __forceinline__ float ld_cluster_f32(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return __uint_as_float(v);
}

__device__ __forceinline__ void copy16(uint32_t dst, const void* src) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory"); }
__device__ __forceinline__ void copy8(uint32_t dst, const void* src) { asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(src) : "memory"); }
__device__ __forceinline__ void copy4(uint32_t dst, const void* src) { asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory"); }
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

template <int DH, int NT>
struct RowsSmem {
  static constexpr int STAGE = 32 * DH;                                     // bytes of a tile's keys and values
  static constexpr int RING = ROWS_STAGES * STAGE;                          // per warp; afterwards its partial O [8 NT][DH]
  static constexpr int PARTIAL = 8 * NT * DH * 4;
  static constexpr int WARP = RING > PARTIAL ? RING : PARTIAL;
  static constexpr int OFF_SCALES = ROWS_WARPS * WARP;                      // float [warps][stages][2]
  static constexpr int OFF_ML = OFF_SCALES + ROWS_WARPS * ROWS_STAGES * 8;  // float [2][warps][8 NT], then the CTA's [2][8 NT]
  static constexpr int BYTES = OFF_ML + (ROWS_WARPS + 1) * 8 * NT * 8;
};

struct SplitPlan { int cluster, outer; };       // CTAs per cluster, clusters per (sequence, head, row tile)

template <int DH, int NT, bool BF, bool F8>
__global__ void __launch_bounds__(ROWS_WARPS * 32, NT == 1 ? 4 : 3) block_attn_rows_kernel(const BlockAttnParams p) {
  constexpr int R = 8 * NT;                      // rows of a tile: (row of the sequence, query head of the group) pairs
  constexpr int KC = DH / 64;                    // 64-feature pieces of a key
  constexpr int VW = DH / 32;                    // words of a lane's value slice
  constexpr int MT = DH / 16;                    // M tiles of O^T
  using Smem = RowsSmem<DH, NT>;
  extern __shared__ __align__(16) uint8_t smem[];
  float* sm = reinterpret_cast<float*>(smem + Smem::OFF_ML);               // [warps][R] maxima
  float* sl = sm + ROWS_WARPS * R;                                         // [warps][R] sums
  float* cm = sl + ROWS_WARPS * R;                                         // [R] the CTA's
  float* cl = cm + R;
  ptx::pdl_launch_dependents();
  ptx::pdl_wait();
  const BlockView& c = p.c;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int b = blockIdx.z, hk = blockIdx.y % c.nkv, qt = blockIdx.y / c.nkv;
  const int splits = gridDim.x, cs = p.cluster;
  const SeqRows s = seq_rows(c, b);
  const int total = s.n * p.group, rb = qt * R;
  if (rb >= total) return;                       // uniform over the cluster
  const int last = (min(rb + R, total) - 1) / p.group, base = s.len - s.n;
  const int L = max(base + last + 1, 0);         // keys of the tile's last row
  const int full = base + rb / p.group + 1;      // keys of its first row: tiles below need no mask
  const int per = ((L + splits - 1) / splits + 15) & ~15;
  const int k0 = min((int)blockIdx.x * per, L), k1 = min(k0 + per, L);
  const int nt = (k1 - k0 + 15) >> 4;

  // page ids of the warp's next 32 tiles, one per lane
  int my_id = 0;
  auto load_pages = [&](int j0) {                // tiles j0, j0 + warps, ...
    const int j = j0 + ROWS_WARPS * lane;
    if (j < nt) my_id = page_for_read(c, b, (k0 + 16 * j) >> c.page_shift);
  };
  load_pages(warp);
  const uint8_t* kbase = c.k + (long long)hk * c.head_stride + (long long)g * c.ld + 16 * t;
  const uint8_t* vbase = c.v + (long long)hk * c.head_stride + (long long)(2 * t) * c.ld + (DH / 8) * g;
  const uint8_t* ring = smem + warp * Smem::WARP;
  const uint32_t ring_a = ptx::smem_u32(ring), scales_a = ptx::smem_u32(smem + Smem::OFF_SCALES) + warp * ROWS_STAGES * 8;
  int jp = warp, slot = 0;                       // next tile to be requested, lane that holds its page
  // requests tile jp into a stage: the lane's key pieces at [r * KC + q][lane], its value slices behind them, the two scales
  auto request = [&](int stage) {
    if (jp < nt) {
      const int id = __shfl_sync(0xffffffffu, my_id, slot);
      const long long at = (long long)id * c.page_stride + (long long)((k0 + 16 * jp) & (c.page - 1)) * c.ld;
      const uint32_t dst = ring_a + stage * Smem::STAGE;
#pragma unroll
      for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int q = 0; q < KC; ++q) copy16(dst + ((r * KC + q) * 32 + lane) * 16, kbase + at + (long long)(8 * r) * c.ld + 64 * q);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const uint8_t* src = vbase + at + (long long)((r & 1) + 8 * (r >> 1)) * c.ld;
        if constexpr (VW == 4) copy16(dst + 16 * DH + (r * 32 + lane) * 16, src);
        else copy8(dst + 16 * DH + (r * 32 + lane) * 8, src);
      }
      if (lane < 2) copy4(scales_a + stage * 8 + lane * 4, (lane ? c.vs : c.ks) + (long long)id * c.nkv + hk);
      jp += ROWS_WARPS;
      if (++slot == 32) { slot = 0; load_pages(jp); }
    }
    copy_commit();                               // (an empty group keeps the count)
  };
#pragma unroll
  for (int i = 0; i < ROWS_STAGES - 1; ++i) request(i);

  // query fragments: lane (g, t) holds features 64 c + 16 t .. + 15 of row g of each N tile, scaled by a power of two
  uint32_t qf[NT][KC * 8];
  float qs[NT];                                  // what undoes that scaling, for row g
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int rr = min(rb + 8 * n + g, total - 1);
    const uint16_t* q = p.q + (s.r0 + rr / p.group) * p.ld_q + ((long long)hk * p.group + rr % p.group) * DH + 16 * t;
    uint32_t raw[KC * 8], top = 0;
#pragma unroll
    for (int k = 0; k < KC; ++k) {
      const uint4 x = __ldg(reinterpret_cast<const uint4*>(q + 64 * k)), y = __ldg(reinterpret_cast<const uint4*>(q + 64 * k + 8));
      raw[8 * k] = x.x; raw[8 * k + 1] = x.y; raw[8 * k + 2] = x.z; raw[8 * k + 3] = x.w;
      raw[8 * k + 4] = y.x; raw[8 * k + 5] = y.y; raw[8 * k + 6] = y.z; raw[8 * k + 7] = y.w;
    }
#pragma unroll
    for (int i = 0; i < KC * 8; ++i) top = __vmaxu2(top, raw[i] & 0x7fff7fffu);
    top = max(top & 0xffffu, top >> 16);
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const float amax = fp16ish_to_f32x2<BF>(top).x;
    // 2^(14 - exponent of the maximum); zero, infinite and NaN rows are left as they are
    const int e = (int)(__float_as_uint(amax) >> 23);
    const bool odd = e == 0 || e == 255;
    const float up = odd ? 1.0f : __uint_as_float((uint32_t)min(max(127 + 14 + 127 - e, 1), 254) << 23);
    qs[n] = 1.0f / up;                           // a power of two within the normal range: exact
#pragma unroll
    for (int i = 0; i < KC * 8; ++i) {
      const float2 f = fp16ish_to_f32x2<BF>(raw[i]);
      qf[n][i] = pack_f16(f.x * up, f.y * up);
    }
  }
  // per lane: rows 2 t and 2 t + 1 of each N tile (the columns of S^T and O^T it holds)
  float f[NT][2], m[NT][2], l[NT][2], acc[NT][MT][4];
  int lim[NT][2];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      f[n][r] = p.c2 * __shfl_sync(0xffffffffu, qs[n], 4 * (2 * t + r));
      lim[n][r] = base + min(rb + 8 * n + 2 * t + r, total - 1) / p.group + 1;
      m[n][r] = -INFINITY; l[n][r] = 0.f;
    }
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int j = 0; j < MT; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[n][j][i] = 0.f;
  float vref = 0.f;

  int stage = 0;
  for (int j = warp; j < nt; j += ROWS_WARPS) {
    copy_wait<ROWS_STAGES - 2>();
    __syncwarp();                                // the scales come from other lanes' copies; and every lane is done with the stage requested next
    request(stage == 0 ? ROWS_STAGES - 1 : stage - 1);
    const uint8_t* tile = ring + stage * Smem::STAGE;
    const float2 scales = *reinterpret_cast<const float2*>(smem + Smem::OFF_SCALES + (warp * ROWS_STAGES + stage) * 8);
    const float ks = scales.x, vs = scales.y;
    if (++stage == ROWS_STAGES) stage = 0;
    const int tb = k0 + 16 * j;
    // ---- scores
    float sc[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n) sc[n][0] = sc[n][1] = sc[n][2] = sc[n][3] = 0.f;
#pragma unroll
    for (int q = 0; q < KC; ++q) {
      const uint4 x = reinterpret_cast<const uint4*>(tile)[q * 32 + lane], y = reinterpret_cast<const uint4*>(tile)[(KC + q) * 32 + lane];
      const uint32_t w0[4] = {x.x, x.y, x.z, x.w}, w1[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t a0, a1, a2, a3;
        codes4_to_f16<F8>(w0[i], a0, a2);
        codes4_to_f16<F8>(w1[i], a1, a3);
#pragma unroll
        for (int n = 0; n < NT; ++n) mma_f16(sc[n], a0, a1, a2, a3, qf[n][8 * q + 2 * i], qf[n][8 * q + 2 * i + 1]);
      }
    }
    // ---- probabilities
    if (vs > vref) {                             // uniform over the warp
      const float up = vref / vs;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int k = 0; k < MT; ++k)
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[n][k][i] *= up;
      vref = vs;
    }
    const float rv = vref > 0.f ? vs / vref : 0.f;
    uint32_t pb[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const float f0 = f[n][0] * ks, f1 = f[n][1] * ks;
      float x0 = sc[n][0] * f0, x1 = sc[n][1] * f1, x2 = sc[n][2] * f0, x3 = sc[n][3] * f1;
      if (tb + 16 > full) {
        if (tb + g >= lim[n][0]) x0 = -INFINITY;
        if (tb + g >= lim[n][1]) x1 = -INFINITY;
        if (tb + g + 8 >= lim[n][0]) x2 = -INFINITY;
        if (tb + g + 8 >= lim[n][1]) x3 = -INFINITY;
      }
      float mx0 = fmaxf(x0, x2), mx1 = fmaxf(x1, x3);
      if (__any_sync(0xffffffffu, mx0 > m[n][0] + MAX_SLACK || mx1 > m[n][1] + MAX_SLACK)) {
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) {
          mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, o));
          mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, o));
        }
        mx0 = fmaxf(mx0, m[n][0]); mx1 = fmaxf(mx1, m[n][1]);
        const float a0 = mx0 > -INFINITY ? ex2(m[n][0] - mx0) : 1.f, a1 = mx1 > -INFINITY ? ex2(m[n][1] - mx1) : 1.f;
        m[n][0] = mx0; m[n][1] = mx1;
        l[n][0] *= a0; l[n][1] *= a1;
#pragma unroll
        for (int k = 0; k < MT; ++k) { acc[n][k][0] *= a0; acc[n][k][2] *= a0; acc[n][k][1] *= a1; acc[n][k][3] *= a1; }
      }
      const float u0 = m[n][0] > -INFINITY ? P_SHIFT - m[n][0] : 0.f, u1 = m[n][1] > -INFINITY ? P_SHIFT - m[n][1] : 0.f;
      x0 = ex2(x0 + u0); x1 = ex2(x1 + u1); x2 = ex2(x2 + u0); x3 = ex2(x3 + u1);
      l[n][0] += x0 + x2; l[n][1] += x1 + x3;
      pb[n][0] = transpose8x8(pack_f16(x0 * rv, x1 * rv));
      pb[n][1] = transpose8x8(pack_f16(x2 * rv, x3 * rv));
    }
    uint32_t vr[4][VW];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      if constexpr (VW == 4) {
        const uint4 x = reinterpret_cast<const uint4*>(tile + 16 * DH)[r * 32 + lane];
        vr[r][0] = x.x; vr[r][1] = x.y; vr[r][2] = x.z; vr[r][3] = x.w;
      } else {
        const uint2 x = reinterpret_cast<const uint2*>(tile + 16 * DH)[r * 32 + lane];
        vr[r][0] = x.x; vr[r][1] = x.y;
      }
    }
    // ---- values; e4m3 slots behind the end may hold NaN, which a zero probability does not silence
    if (F8 && tb + 16 > k1) {
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (tb + 2 * t + (r & 1) + 8 * (r >> 1) >= k1) {
#pragma unroll
          for (int w = 0; w < VW; ++w) vr[r][w] = 0;
        }
    }
#pragma unroll
    for (int w = 0; w < VW; ++w) {
      uint32_t ab[4], cd[4];                     // feature i of the word: tokens (2t, 2t + 1) and (2t + 8, 2t + 9)
      codes4_to_f16<F8>(__byte_perm(vr[0][w], vr[1][w], 0x5140), ab[0], ab[1]);
      codes4_to_f16<F8>(__byte_perm(vr[0][w], vr[1][w], 0x7362), ab[2], ab[3]);
      codes4_to_f16<F8>(__byte_perm(vr[2][w], vr[3][w], 0x5140), cd[0], cd[1]);
      codes4_to_f16<F8>(__byte_perm(vr[2][w], vr[3][w], 0x7362), cd[2], cd[3]);
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        mma_f16(acc[n][2 * w], ab[0], ab[1], cd[0], cd[1], pb[n][0], pb[n][1]);
        mma_f16(acc[n][2 * w + 1], ab[2], ab[3], cd[2], cd[3], pb[n][0], pb[n][1]);
      }
    }
  }

  // ---- join the warps of the CTA; a warp's partial O takes the place of its ring (all its copies have been waited for)
  copy_wait<0>();
  __syncwarp();
  float* my_o = reinterpret_cast<float*>(smem + warp * Smem::WARP);
#pragma unroll
  for (int n = 0; n < NT; ++n) {
#pragma unroll
    for (int r = 0; r < 2; ++r) {
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) l[n][r] += __shfl_xor_sync(0xffffffffu, l[n][r], o);
      if (g == 0) { sm[warp * R + 8 * n + 2 * t + r] = m[n][r]; sl[warp * R + 8 * n + 2 * t + r] = l[n][r]; }
#pragma unroll
      for (int k = 0; k < MT; ++k)
        *reinterpret_cast<float2*>(my_o + (8 * n + 2 * t + r) * DH + (DH / 8) * g + 2 * k) = make_float2(acc[n][k][r] * vref, acc[n][k][2 + r] * vref);
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < R * DH; i += ROWS_WARPS * 32) {
    const int row = i / DH, d = i % DH;
    float mt = sm[row];
#pragma unroll
    for (int w = 1; w < ROWS_WARPS; ++w) mt = fmaxf(mt, sm[w * R + row]);
    float y = 0.f, lt = 0.f;
#pragma unroll
    for (int w = 0; w < ROWS_WARPS; ++w) {
      const float mw = sm[w * R + row], e = mw > -INFINITY ? ex2(mw - mt) : 0.f;
      y = fmaf(e, reinterpret_cast<const float*>(smem + w * Smem::WARP)[i], y); lt = fmaf(e, sl[w * R + row], lt);
    }
    reinterpret_cast<float*>(smem)[i] = y;
    if (d == 0) { cm[row] = mt; cl[row] = lt; }
  }
  // ---- join the CTAs of the cluster: each finishes its share of the tile
  if (cs > 1) ptx::cluster_sync(); else __syncthreads();
  const int rank = cs > 1 ? (int)ptx::cluster_ctarank() : 0, share = R * DH / cs;
  const uint32_t am = ptx::smem_u32(cm), al = ptx::smem_u32(cl), ao = ptx::smem_u32(smem);
  for (int i = rank * share + threadIdx.x; i < (rank + 1) * share; i += ROWS_WARPS * 32) {
    const int row = i / DH, d = i % DH, rr = rb + row;
    if (rr >= total) continue;
    float mt = cm[row], lt = cl[row], y = reinterpret_cast<const float*>(smem)[i];
    if (cs > 1) {
      float mq[ROWS_MAX_CLUSTER];
      mt = -INFINITY;
#pragma unroll
      for (int q = 0; q < ROWS_MAX_CLUSTER; ++q) {
        mq[q] = q < cs ? ld_cluster_f32(ptx::mapa(am + 4 * row, q)) : -INFINITY;
        mt = fmaxf(mt, mq[q]);
      }
      lt = 0.f; y = 0.f;
#pragma unroll
      for (int q = 0; q < ROWS_MAX_CLUSTER; ++q)
        if (q < cs) {
          const float e = mq[q] > -INFINITY ? ex2(mq[q] - mt) : 0.f;
          lt = fmaf(e, ld_cluster_f32(ptx::mapa(al + 4 * row, q)), lt);
          y = fmaf(e, ld_cluster_f32(ptx::mapa(ao + 4 * i, q)), y);
        }
    }
    const long long row_g = s.r0 + rr / p.group;
    const int hq = hk * p.group + rr % p.group;
    if (p.outer == 1) {
      store_out(p, row_g, hq * DH + d, lt > 0.f ? y / lt : 0.f);
    } else {
      const long long at = (row_g * p.nq + hq) * p.outer + blockIdx.x / cs;
      p.part_o[at * DH + d] = y;
      if (d == 0) p.part_ml[at] = make_float2(mt, lt);
    }
  }
  if (cs > 1) ptx::cluster_sync();               // nobody leaves while a peer may still read its shared memory
}

// joins the partial results of the clusters of one (row, query head): a warp each
template <int DH>
__global__ void __launch_bounds__(128) block_attn_join_kernel(const BlockAttnParams p) {
  ptx::pdl_launch_dependents();
  ptx::pdl_wait();
  const SeqRows s = seq_rows(p.c, blockIdx.y);
  const long long w = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
  const int i = (int)(w / p.nq), hq = (int)(w % p.nq), lane = threadIdx.x & 31;
  if (i >= s.n) return;
  const long long at = ((s.r0 + i) * p.nq + hq) * p.outer;
  float mt = -INFINITY;
  for (int q = lane; q < p.outer; q += 32) mt = fmaxf(mt, p.part_ml[at + q].x);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) mt = fmaxf(mt, __shfl_xor_sync(0xffffffffu, mt, o));
  constexpr int E = DH / 32;
  float lt = 0.f, y[E];
#pragma unroll
  for (int e = 0; e < E; ++e) y[e] = 0.f;
#pragma unroll 4
  for (int q = 0; q < p.outer; ++q) {
    const float2 ml = p.part_ml[at + q];
    const float f = ml.x > -INFINITY ? ex2(ml.x - mt) : 0.f;
    lt = fmaf(f, ml.y, lt);
#pragma unroll
    for (int e = 0; e < E; ++e) y[e] = fmaf(f, p.part_o[(at + q) * DH + 32 * e + lane], y[e]);
  }
#pragma unroll
  for (int e = 0; e < E; ++e) store_out(p, s.r0 + i, hq * DH + 32 * e + lane, lt > 0.f ? y[e] / lt : 0.f);
}

// How the tokens of a (sequence, key / value head, row tile) are split: the host knows an upper bound of the lengths only.
static SplitPlan plan_rows(const hero_handle* h, const hero_block_cache* cc, int nq, int max_rows, int nt) {
  const long long tiles = ((long long)max_rows * (nq / cc->nkv) + 8 * nt - 1) / (8 * nt);
  const long long groups = tiles * cc->nkv * cc->B;
  const long long slots = (long long)h->sm_count * (nt == 1 ? 4 : 3);
  long long want = (2 * slots + groups - 1) / groups;             // CTAs for two rounds of the GPU
  const long long most = (cc->max_len + 255) / 256;               // of at least 256 tokens each
  if (want > most) want = most;
  SplitPlan s = {1, 1};
  if (getenv("DEV_SPLIT")) { sscanf(getenv("DEV_SPLIT"), "%d,%d", &s.cluster, &s.outer); return s; }
  while (s.cluster < ROWS_MAX_CLUSTER && s.cluster < want) s.cluster *= 2;
  if (want > ROWS_MAX_CLUSTER) s.outer = (int)((want + ROWS_MAX_CLUSTER - 1) / ROWS_MAX_CLUSTER);
  return s;
}
static int rows_nt(const hero_block_cache* cc, int nq, int max_rows) { return (long long)max_rows * (nq / cc->nkv) <= 8 ? 1 : 2; }
static size_t part_bytes(const SplitPlan& s, long long rows, int nq, int dh) {
  return s.outer == 1 ? 0 : (size_t)rows * nq * s.outer * (dh * 4 + 8);
}

template <int DH, int NT>
static hero_status launch_rows(hero_handle* h, const BlockAttnParams& p, bool bf, int B, int tiles, cudaStream_t stream) {
  auto kern = bf ? (p.c.f8 ? block_attn_rows_kernel<DH, NT, true, true> : block_attn_rows_kernel<DH, NT, true, false>)
                 : (p.c.f8 ? block_attn_rows_kernel<DH, NT, false, true> : block_attn_rows_kernel<DH, NT, false, false>);
  static PerDeviceOnce configured[4];            // per instantiation of the kernel
  PerDeviceOnce& once = configured[(bf ? 2 : 0) + (p.c.f8 ? 1 : 0)];
  if (RowsSmem<DH, NT>::BYTES > 48 * 1024 && !once.done(h->device)) {
    HERO_CUDA(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, RowsSmem<DH, NT>::BYTES));
    once.set(h->device);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(p.cluster * p.outer), (unsigned)(p.c.nkv * tiles), (unsigned)B);
  cfg.blockDim = dim3(ROWS_WARPS * 32);
  cfg.dynamicSmemBytes = RowsSmem<DH, NT>::BYTES;
  cfg.stream = stream;
  cudaLaunchAttribute at[2];
  int n = 0;
  if (p.cluster > 1) {
    at[n].id = cudaLaunchAttributeClusterDimension;
    at[n].val.clusterDim.x = (unsigned)p.cluster; at[n].val.clusterDim.y = 1; at[n].val.clusterDim.z = 1;
    ++n;
  }
  if (!pdl_take_fence(stream)) {                 // a fenced stream: ordinary serialisation
    at[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[n].val.programmaticStreamSerializationAllowed = 1;
    ++n;
  }
  cfg.attrs = at; cfg.numAttrs = n;
  {
    LaunchScope scope(h, stream, KERNEL_ATTN);
    HERO_CUDA(cudaLaunchKernelEx(&cfg, kern, p));
  }
  if (p.outer > 1) {
    LaunchScope scope(h, stream, KERNEL_ATTN);
    HERO_CUDA(launch_dependent(block_attn_join_kernel<DH>, dim3((unsigned)(((long long)p.c.max_rows * p.nq + 3) / 4), (unsigned)B), dim3(128), 0, stream, p));
  }
  return HERO_OK;
}

static hero_status attn_check(hero_handle* h, const hero_block_cache* cc, int32_t nq, int64_t rows, int32_t max_rows) {
  HERO_REQUIRE(h && cc, HERO_ERR_INVALID_ARG, "hero_block_attention: NULL handle or cache");
  HERO_REQUIRE(cc->nkv >= 1 && nq >= cc->nkv && nq % cc->nkv == 0 && nq <= 65535, HERO_ERR_INVALID_ARG, "nq=%d must be a multiple of nkv=%d", nq, cc->nkv);
  HERO_REQUIRE(rows >= 0 && max_rows >= 1, HERO_ERR_INVALID_ARG, "rows=%lld max_rows=%d", (long long)rows, max_rows);
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
  *bytes = part_bytes(plan_rows(h, cc, nq, max_rows, rows_nt(cc, nq, max_rows)), rows, nq, cc->dh);
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
  const int nt = rows_nt(cc, a->nq, a->max_rows);
  const SplitPlan plan = plan_rows(h, cc, a->nq, a->max_rows, nt);
  const size_t need = part_bytes(plan, a->q.rows, a->nq, cc->dh);
  HERO_REQUIRE(need == 0 || (a->workspace && a->workspace_bytes >= need), HERO_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", a->workspace_bytes, need);
  HERO_REQUIRE(need == 0 || aligned16(a->workspace), HERO_ERR_ALIGNMENT, "the workspace must be 16-byte aligned");
  p.cluster = plan.cluster; p.outer = plan.outer;
  p.part_o = static_cast<float*>(a->workspace);
  p.part_ml = reinterpret_cast<float2*>(p.part_o + (size_t)a->q.rows * a->nq * plan.outer * cc->dh);
  const long long tiles = ((long long)a->max_rows * p.group + 8 * nt - 1) / (8 * nt);
  HERO_REQUIRE(tiles * cc->nkv <= 65535, HERO_ERR_UNSUPPORTED, "max_rows=%d", a->max_rows);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (cc->dh == 64)
    return nt == 1 ? launch_rows<64, 1>(h, p, bf, cc->B, (int)tiles, s) : launch_rows<64, 2>(h, p, bf, cc->B, (int)tiles, s);
  return nt == 1 ? launch_rows<128, 1>(h, p, bf, cc->B, (int)tiles, s) : launch_rows<128, 2>(h, p, bf, cc->B, (int)tiles, s);
}
