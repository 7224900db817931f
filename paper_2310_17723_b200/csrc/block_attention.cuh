// Shared by the kernels of hero_block_attention: parameters, output stage, conversions of codes.
#pragma once
#include "block_cache.cuh"

namespace hero {

struct BlockAttnParams {
  BlockView c;
  const uint16_t* q; long long ld_q;
  void* out; long long ld_out; int out_dt;
  const float* out_scale; int out_scale_stride;
  int nq, group;
  float c2;                      // scale * log2(e)
  int B, tiles, direct;          // direct: CTA index = (sequence, row tile, head); else equal shares of all units
  int by_group;                  // records of cut groups are listed by group, else by share
  struct JoinRecord* records;
  int splits;                    // many rows: parts of a group's keys, a CTA each
  float* part_o; float2* part_ml; // partial results ([CTA][2]; many rows: [CTA]): output of the part's keys alone [rows][DH], (maximum, sum of P) [rows]
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

// Few rows: P is formed with a factor 2^P_SHIFT; the running maximum moves when a score exceeds it by more than MAX_SLACK in the exponent
// of two, so P stays below 2^15 and a probability 2^-25 of the largest is still a normal FP16 number.
constexpr float P_SHIFT = 11.0f, MAX_SLACK = 4.0f;

// Factor that brings a query row of this largest magnitude into FP16: 2^(14 - its exponent), at most 2^126 (which BF16's subnormal rows
// need, and which leaves the score factor divided by it within three bits of FP32's subnormal numbers); infinite and NaN rows are left alone.
__device__ __forceinline__ float query_factor(float amax) {
  const int e = (int)(__float_as_uint(amax) >> 23);
  return e == 255 ? 1.0f : __uint_as_float((uint32_t)min(127 + 14 + 127 - e, 253) << 23);
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

// many rows per key / value head (block_attention_prompt.cu)
hero_status prompt_workspace_bytes(const hero_handle* h, const hero_block_cache* cc, int nq, int max_rows, size_t* bytes);
size_t prompt_workspace_most(const hero_handle* h, const hero_block_cache* cc, int nq, int max_rows);
hero_status launch_prompt(hero_handle* h, const hero_block_cache* cc, const BlockAttnParams& p, bool bf, void* workspace, cudaStream_t stream);

}  // namespace hero
