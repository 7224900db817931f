// Shared by the kernels of the 8-bit block cache: the device view of a cache and of a call's rows, the bounds that the
// host cannot check, conversions between codes, FP32 and the 16-bit types.
#pragma once
#include "common.cuh"
#include "ptx.cuh"
#include <cuda_fp16.h>
#include <cuda_bf16.h>

namespace hero {

struct BlockView {
  uint8_t* k; uint8_t* v;
  float* ks; float* vs;
  int f8;                       // e4m3 codes, else INT8
  int page, page_shift;
  int n_pages;
  long long page_stride, head_stride, ld;
  const int* table; long long ld_table;
  const int* len;
  int max_len, nkv;
  // the call's rows
  const int* row_start;         // NULL: row b for sequence b
  long long rows;
  int max_rows;
  int* err;
};

// checks shared by every entry point of the cache; `rows` / `max_rows` describe the call's matrices
hero_status block_view(hero_handle* h, const hero_block_cache* c, const int32_t* row_start, int64_t rows, int32_t max_rows, BlockView* out);

// A load of what an earlier call of the stream may have written: codes, scales, tables, lengths, rows, partial results.  These kernels may be
// resident while the one before them still runs, so such data is not read-only for their whole life, which a non-coherent load
// (__ldg) takes for granted: it may be moved ahead of the wait for that kernel.
template <typename T>
__device__ __forceinline__ T written(const T* p) { return *p; }

struct SeqRows {
  int len, n;                   // tokens held, rows of the call
  long long r0;                 // first row
};
__device__ __forceinline__ SeqRows seq_rows(const BlockView& v, int b) {
  SeqRows s;
  s.len = min(max(written(v.len + b), 0), v.max_len);
  if (v.row_start == nullptr) {
    s.r0 = b; s.n = 1;
    return s;
  }
  long long r0 = written(v.row_start + b), r1 = written(v.row_start + b + 1);
  if (r0 < 0 || r1 < r0 || r1 > v.rows || r1 - r0 > v.max_rows) {
    atomicExch(v.err, ERR_BAD_ROWS);
    r0 = min(max(r0, 0ll), v.rows);
    r1 = min(max(r1, r0), v.rows);
  }
  s.r0 = r0;
  s.n = (int)min(r1 - r0, (long long)v.max_rows);
  return s;
}
// page id of the sequence's page `pi`, clamped into the pool (and reported) for reading
__device__ __forceinline__ int page_for_read(const BlockView& v, int b, int pi) {
  int id = __ldcg(v.table + (long long)b * v.ld_table + pi);   // (as `written`; past the first-level cache it costs fewer registers: drafts 57.0 -> 56.3 us)
  if ((unsigned)id >= (unsigned)v.n_pages) {
    atomicExch(v.err, ERR_BAD_PAGE);
    id = id < 0 ? 0 : v.n_pages - 1;
  }
  return id;
}

// ---- 16-bit <-> FP32
template <bool BF>
__device__ __forceinline__ float2 fp16ish_to_f32x2(uint32_t w) {
  if constexpr (BF) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
  else return __half22float2(*reinterpret_cast<const __half2*>(&w));
}
template <bool BF>
__device__ __forceinline__ uint32_t f32x2_to_fp16ish(float a, float b) {
  if constexpr (BF) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  } else {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
}
// ---- four codes -> FP32.  INT8: the byte, offset to unsigned, becomes the low mantissa byte of 2^23 (exact), no conversion unit
template <bool F8>
__device__ __forceinline__ void codes4_to_f32(uint32_t w, float (&y)[4]) {
  if constexpr (F8) {
    const float2 a = ptx::e4m3x2_to_f32x2(w & 0xffffu), b = ptx::e4m3x2_to_f32x2(w >> 16);
    y[0] = a.x; y[1] = a.y; y[2] = b.x; y[3] = b.y;
  } else {
    const uint32_t u = w ^ 0x80808080u;
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = __uint_as_float(__byte_perm(u, 0x4B000000u, 0x7440 + i)) - 8388736.0f;
  }
}
// ---- FP32 (already divided by the scale) -> four codes, saturating, round to nearest even
template <bool F8>
__device__ __forceinline__ uint32_t f32_to_codes4(float a, float b, float c, float d) {
  if constexpr (F8) {
    return ptx::f32x4_to_e4m3x4(a, b, c, d);
  } else {
    constexpr float MAGIC = 12582912.0f;         // 1.5 * 2^23: the adder rounds to the nearest integer, ties to even
    const uint32_t x = __float_as_uint(fminf(fmaxf(a, -127.f), 127.f) + MAGIC), y = __float_as_uint(fminf(fmaxf(b, -127.f), 127.f) + MAGIC);
    const uint32_t z = __float_as_uint(fminf(fmaxf(c, -127.f), 127.f) + MAGIC), w = __float_as_uint(fminf(fmaxf(d, -127.f), 127.f) + MAGIC);
    return __byte_perm(__byte_perm(x, y, 0x0040), __byte_perm(z, w, 0x0040), 0x5410);
  }
}
// the same for quotients that are known to lie within the codes' range (|x| <= 127 s (1 + 2^-23)): no clamping
template <bool F8>
__device__ __forceinline__ uint32_t f32_to_codes4_inside(float2 a, float2 b) {
  if constexpr (F8) {
    return ptx::f32x4_to_e4m3x4(a.x, a.y, b.x, b.y);
  } else {
    const float2 magic = make_float2(12582912.0f, 12582912.0f), x = __fadd2_rn(a, magic), y = __fadd2_rn(b, magic);
    return __byte_perm(__byte_perm(__float_as_uint(x.x), __float_as_uint(x.y), 0x0040), __byte_perm(__float_as_uint(y.x), __float_as_uint(y.y), 0x0040), 0x5410);
  }
}
// x / s rounded to nearest, for many x and one s: with r the correctly rounded reciprocal of s, q = x r is within one unit of the
// quotient and q + r (x - s q), the remainder formed exactly by a fused multiply-add, is the correctly rounded quotient
// (P. Markstein, "Computation of elementary functions on the IBM RISC System/6000 processor", 1990).  Scales so small or
// large that a remainder could leave the normal range take the division itself.
struct Divider {
  float s, r;
  bool fast;
  __device__ __forceinline__ explicit Divider(float s_) : s(s_), r(s_ > 0.f ? 1.0f / s_ : 0.f), fast(s_ > 7.8886e-31f && s_ < 1.2676e30f) {}
  // two quotients at once; `fast` only
  __device__ __forceinline__ float2 pair(float2 x) const {
    const float2 r2 = make_float2(r, r), q = __fmul2_rn(x, r2);
    return __ffma2_rn(__ffma2_rn(make_float2(-s, -s), q, x), r2, q);
  }
  __device__ __forceinline__ float operator()(float x) const {
    if (!fast) return s > 0.f ? x / s : 0.f;
    const float q = x * r;
    return fmaf(fmaf(-s, q, x), r, q);
  }
};

}  // namespace hero
