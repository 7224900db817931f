// Attention over the 8-bit block cache (hero_block_attention): o = softmax(scale q K^T) V, causal in a sequence's new rows.
#include "block_cache.cuh"
#include <cmath>

namespace hero {

struct BlockAttnParams {
  BlockView c;
  const uint16_t* q; long long ld_q;
  void* out; long long ld_out; int out_dt;
  const float* out_scale; int out_scale_stride;
  int group;
  float c2;                      // scale * log2(e)
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

// One CTA per (row, query head): four warps share the keys, a lane holds DH / 32 features, running maximum and sum per warp.
template <int DH, bool BF, bool F8>
__global__ void __launch_bounds__(128) block_attn_simple_kernel(const BlockAttnParams p) {
  constexpr int E = DH / 32;
  __shared__ float sm[4], sl[4], so[4][DH];
  ptx::pdl_launch_dependents();
  ptx::pdl_wait();
  const BlockView& c = p.c;
  const int b = blockIdx.z, hq = blockIdx.y, g = hq / p.group, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const SeqRows s = seq_rows(c, b);
  const int i = blockIdx.x;
  if (i >= s.n) return;
  const int keys = s.len - s.n + i + 1;
  const uint16_t* q = p.q + (s.r0 + i) * p.ld_q + hq * DH + lane * E;
  float qf[E], acc[E];
#pragma unroll
  for (int e = 0; e < E; e += 2) {
    const float2 f = fp16ish_to_f32x2<BF>(*reinterpret_cast<const uint32_t*>(q + e));
    qf[e] = f.x * p.c2; qf[e + 1] = f.y * p.c2;
    acc[e] = acc[e + 1] = 0.f;
  }
  float m = -INFINITY, l = 0.f;
  for (int t = warp; t < keys; t += 4) {
    const int id = page_for_read(c, b, t >> c.page_shift);
    const long long at = (long long)id * c.page_stride + (long long)g * c.head_stride + (long long)(t & (c.page - 1)) * c.ld + lane * E;
    float kf[4], vf[4];
    codes4_to_f32<F8>(E == 4 ? *reinterpret_cast<const uint32_t*>(c.k + at) : *reinterpret_cast<const uint16_t*>(c.k + at), kf);
    codes4_to_f32<F8>(E == 4 ? *reinterpret_cast<const uint32_t*>(c.v + at) : *reinterpret_cast<const uint16_t*>(c.v + at), vf);
    float d = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) d = fmaf(qf[e], kf[e], d);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) d += __shfl_xor_sync(0xffffffffu, d, o);
    d *= c.ks[(long long)id * c.nkv + g];
    const float mn = fmaxf(m, d), f = exp2f(m - mn), pr = exp2f(d - mn), sv = c.vs[(long long)id * c.nkv + g];
    m = mn;
    l = l * f + pr;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = fmaf(acc[e], f, pr * sv * vf[e]);
  }
#pragma unroll
  for (int e = 0; e < E; ++e) so[warp][lane * E + e] = acc[e];
  if (lane == 0) { sm[warp] = m; sl[warp] = l; }
  __syncthreads();
  if (threadIdx.x < DH) {
    float mt = fmaxf(fmaxf(sm[0], sm[1]), fmaxf(sm[2], sm[3])), lt = 0.f, y = 0.f;
    for (int w = 0; w < 4; ++w) {
      const float f = sm[w] > -INFINITY ? exp2f(sm[w] - mt) : 0.f;
      lt += f * sl[w]; y += f * so[w][threadIdx.x];
    }
    store_out(p, s.r0 + i, hq * DH + threadIdx.x, lt > 0.f ? y / lt : 0.f);
  }
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
  return attn_check(h, cc, nq, rows, max_rows);
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
  const bool bf = a->q.dtype == HERO_BF16;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  auto kern = cc->dh == 64 ? (bf ? (p.c.f8 ? block_attn_simple_kernel<64, true, true> : block_attn_simple_kernel<64, true, false>)
                                 : (p.c.f8 ? block_attn_simple_kernel<64, false, true> : block_attn_simple_kernel<64, false, false>))
                           : (bf ? (p.c.f8 ? block_attn_simple_kernel<128, true, true> : block_attn_simple_kernel<128, true, false>)
                                 : (p.c.f8 ? block_attn_simple_kernel<128, false, true> : block_attn_simple_kernel<128, false, false>));
  cudaError_t e;
  {
    LaunchScope scope(h, s, KERNEL_ATTN);
    e = launch_dependent(kern, dim3((unsigned)a->max_rows, (unsigned)a->nq, (unsigned)cc->B), dim3(128), 0, s, p);
  }
  HERO_CUDA(e);
  return HERO_OK;
}
