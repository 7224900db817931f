// Norm and rotation of query and key heads in one pass (hero_qk_norm_rope): every element is read and written once, so the
// kernel is bound by HBM for many rows and by its latency for few.  A head vector is held by LPH lanes of a warp (8 features,
// 16 bytes each; LPH is the power of two that covers dh), the sum of squares is log2(LPH) shuffles, a rotation partner in
// the other half of the head is one shuffle per feature and a neighbouring one is the lane's own.  A warp takes ITERS * 32 / LPH
// heads of ONE row, so that cos and sin of the row's position are loaded once for all of them.  What a feature and its partner are
// multiplied with (gamma cos, +-gamma sin) is formed once per row too: per head there remain the sum of squares, two products a feature
// and the norm factor.
#include "block_cache.cuh"

namespace hero {

struct RopeParams {
  const uint16_t* x[2]; long long ld_x[2];       // q, k
  void* y[2]; long long ld_y[2];
  const float* gamma[2];
  const float* out_scale[2];                     // I8 outputs: one value each; NULL for a 16-bit output
  int heads[2], chunks[2];                       // chunks: warps per row
  int dh, rot, adjacent;
  float eps, inv_dh;
  const int* pos; const float* cos; const float* sin;
  long long n_pos, rows;
  int* err;
};

constexpr int ROPE_WARPS = 4;

template <int LPH, int ITERS, bool BF>
__global__ void __launch_bounds__(ROPE_WARPS * 32, ITERS == 8 ? 5 : 8) qk_rope_kernel(const __grid_constant__ RopeParams p) {
  constexpr int HPI = 32 / LPH;                  // heads per iteration
  ptx::pdl_launch_dependents();
  ptx::pdl_wait();
  const unsigned per_row = p.chunks[0] + p.chunks[1], unit = blockIdx.x * ROPE_WARPS + (threadIdx.x >> 5);
  const long long row = unit / per_row;
  if (row >= p.rows) return;
  const int this_pos = p.rot > 0 ? __ldg(p.pos + row) : 0;
  int ch = (int)(unit - (unsigned)row * per_row);
  const int side = ch >= p.chunks[0];            // 0: queries, 1: keys
  if (side) ch -= p.chunks[0];
  const int lane = threadIdx.x & 31, sub = lane % LPH, f0 = sub * 8;
  const bool live = f0 < p.dh;
  const int first = ch * (HPI * ITERS), h0 = first + lane / LPH, heads = p.heads[side];
  const uint16_t* x0 = p.x[side] + row * p.ld_x[side] + f0;
  uint4 raw[ITERS];
#pragma unroll
  for (int i = 0; i < ITERS; ++i) {
    const int hd = h0 + i * HPI;
    raw[i] = make_uint4(0, 0, 0, 0);
    if (live && hd < heads) raw[i] = *reinterpret_cast<const uint4*>(x0 + (long long)hd * p.dh);
  }
  // what a feature and its partner are multiplied with before the norm factor: gamma cos and +-gamma(partner) sin
  float2 own[4], mate[4];
  const bool norm = p.gamma[side] != nullptr, turns = f0 < p.rot;
  const int half = p.rot >> 1;
  {
    const bool second = !p.adjacent && f0 >= half;
    const int pf = p.adjacent || !turns ? f0 : second ? f0 - half : f0 + half;       // the partner features (adjacent: the lane's own)
    float g[8], gp[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) g[e] = gp[e] = 1.f;
    if (norm && live) {
      const float* gm = p.gamma[side];
#pragma unroll
      for (int e = 0; e < 8; ++e) { g[e] = __ldg(gm + f0 + e); gp[e] = __ldg(gm + pf + e); }
    }
    float cs[8], sn[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) { cs[e] = 1.f; sn[e] = 0.f; }
    if (p.rot > 0) {
      long long t = this_pos;
      if (t < 0 || t >= p.n_pos) {
        if (lane == 0) atomicExch(p.err, ERR_BAD_POS);
        t = t < 0 ? 0 : p.n_pos - 1;
      }
      if (turns) {
        const float* ct = p.cos + t * half;
        const float* st = p.sin + t * half;
        if (p.adjacent) {
          const float4 x = __ldg(reinterpret_cast<const float4*>(ct + f0 / 2)), y = __ldg(reinterpret_cast<const float4*>(st + f0 / 2));
          cs[0] = cs[1] = x.x; cs[2] = cs[3] = x.y; cs[4] = cs[5] = x.z; cs[6] = cs[7] = x.w;
          sn[0] = -y.x; sn[1] = y.x; sn[2] = -y.y; sn[3] = y.y; sn[4] = -y.z; sn[5] = y.z; sn[6] = -y.w; sn[7] = y.w;
        } else {
          const int j = second ? f0 - half : f0;
          const float4 x0 = __ldg(reinterpret_cast<const float4*>(ct + j)), x1 = __ldg(reinterpret_cast<const float4*>(ct + j + 4));
          const float4 y0 = __ldg(reinterpret_cast<const float4*>(st + j)), y1 = __ldg(reinterpret_cast<const float4*>(st + j + 4));
          cs[0] = x0.x; cs[1] = x0.y; cs[2] = x0.z; cs[3] = x0.w; cs[4] = x1.x; cs[5] = x1.y; cs[6] = x1.z; cs[7] = x1.w;
          sn[0] = y0.x; sn[1] = y0.y; sn[2] = y0.z; sn[3] = y0.w; sn[4] = y1.x; sn[5] = y1.y; sn[6] = y1.z; sn[7] = y1.w;
          if (!second) {
#pragma unroll
            for (int e = 0; e < 8; ++e) sn[e] = -sn[e];
          }
        }
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      own[e] = make_float2(g[2 * e] * cs[2 * e], g[2 * e + 1] * cs[2 * e + 1]);
      mate[e] = p.adjacent ? make_float2(gp[2 * e + 1] * sn[2 * e], gp[2 * e] * sn[2 * e + 1]) : make_float2(gp[2 * e] * sn[2 * e], gp[2 * e + 1] * sn[2 * e + 1]);
    }
  }
  float inv_s = 0.f;
  const bool to_i8 = p.out_scale[side] != nullptr;
  if (to_i8) inv_s = __ldg(p.out_scale[side]);
  const Divider div(inv_s);
  // the lane that holds the partner features under HERO_PAIR_HALVES
  const int r2 = p.rot >> 4;
  const int mate_lane = (lane - sub) + (turns ? (sub < r2 ? sub + r2 : sub - r2) : sub);

#pragma unroll
  for (int i = 0; i < ITERS; ++i) {
    if (first + i * HPI >= heads) break;         // (uniform)
    const int hd = h0 + i * HPI;
    const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
    float2 x[4], y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = fp16ish_to_f32x2<BF>(w[e]);
    float r = 1.f;
    if (norm) {
      float2 ss = __fmul2_rn(x[0], x[0]);
#pragma unroll
      for (int e = 1; e < 4; ++e) ss = __ffma2_rn(x[e], x[e], ss);
      float sum = ss.x + ss.y;
#pragma unroll
      for (int o = LPH / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      r = rsqrtf(fmaf(sum, p.inv_dh, p.eps));
    }
    if (p.adjacent) {
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = __ffma2_rn(make_float2(x[e].y, x[e].x), mate[e], __fmul2_rn(x[e], own[e]));
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)                // (the 16-bit pairs travel, not the FP32 values)
        y[e] = __ffma2_rn(fp16ish_to_f32x2<BF>(__shfl_sync(0xffffffffu, w[e], mate_lane)), mate[e], __fmul2_rn(x[e], own[e]));
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = __fmul2_rn(y[e], make_float2(r, r));
    if (live && hd < heads) {
      const long long at = row * p.ld_y[side] + (long long)hd * p.dh + f0;
      if (to_i8) {
        uint2 code;
        code.x = f32_to_codes4<false>(div(y[0].x), div(y[0].y), div(y[1].x), div(y[1].y));
        code.y = f32_to_codes4<false>(div(y[2].x), div(y[2].y), div(y[3].x), div(y[3].y));
        *reinterpret_cast<uint2*>(static_cast<uint8_t*>(p.y[side]) + at) = code;
      } else {
        *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.y[side]) + at) =
            make_uint4(f32x2_to_fp16ish<BF>(y[0].x, y[0].y), f32x2_to_fp16ish<BF>(y[1].x, y[1].y), f32x2_to_fp16ish<BF>(y[2].x, y[2].y), f32x2_to_fp16ish<BF>(y[3].x, y[3].y));
      }
    }
  }
}

template <int LPH, int ITERS>
static cudaError_t launch_rope_steps(RopeParams& p, bool bf, cudaStream_t s) {
  for (int i = 0; i < 2; ++i) p.chunks[i] = (p.heads[i] + (32 / LPH) * ITERS - 1) / ((32 / LPH) * ITERS);
  const long long warps = p.rows * (p.chunks[0] + p.chunks[1]);
  return launch_dependent(bf ? qk_rope_kernel<LPH, ITERS, true> : qk_rope_kernel<LPH, ITERS, false>, dim3((unsigned)((warps + ROPE_WARPS - 1) / ROPE_WARPS)),
                          dim3(ROPE_WARPS * 32), 0, s, p);
}
// many rows: eight steps a warp, so that what is formed once per row is shared by many heads; few rows: two, more warps
template <int LPH>
static cudaError_t launch_rope(const hero_handle* h, RopeParams& p, bool bf, cudaStream_t s) {
  const bool many = p.rows * (p.heads[0] + p.heads[1]) >= (long long)h->sm_count * 16 * 8 * (32 / LPH);   // 16 warps of eight steps per SM
  return many ? launch_rope_steps<LPH, 8>(p, bf, s) : launch_rope_steps<LPH, 2>(p, bf, s);
}

static hero_status check_head_matrix(const hero_tensor& t, const char* name, int64_t rows, int64_t cols) {
  hero_status st = check_matrix(t, name);
  if (st != HERO_OK) return st;
  HERO_REQUIRE(t.rows == rows && t.cols == cols, HERO_ERR_INVALID_ARG, "%s: [%lld, %lld], expected [%lld, %lld]", name, (long long)t.rows,
               (long long)t.cols, (long long)rows, (long long)cols);
  return HERO_OK;
}

}  // namespace hero

extern "C" hero_status hero_qk_norm_rope(hero_handle* h, const hero_qk_norm_rope_args* a, void* stream) {
  using namespace hero;
  HERO_REQUIRE(h && a, HERO_ERR_INVALID_ARG, "hero_qk_norm_rope: NULL handle or args");
  HERO_REQUIRE(a->dh >= 16 && a->dh <= 256 && a->dh % 16 == 0, HERO_ERR_UNSUPPORTED, "dh=%d: a multiple of 16 up to 256", a->dh);
  HERO_REQUIRE(a->nq >= 1 && a->nkv >= 0 && a->nq <= 65536 && a->nkv <= 65536, HERO_ERR_UNSUPPORTED, "nq=%d nkv=%d", a->nq, a->nkv);
  HERO_REQUIRE(a->rot >= 0 && a->rot <= a->dh && a->rot % 16 == 0, HERO_ERR_UNSUPPORTED, "rot=%d: a multiple of 16 up to dh=%d", a->rot, a->dh);
  HERO_REQUIRE(a->pairing == HERO_PAIR_HALVES || a->pairing == HERO_PAIR_ADJACENT, HERO_ERR_INVALID_ARG, "pairing %d", a->pairing);
  const int64_t rows = a->q.rows;
  RopeParams p;
  memset(&p, 0, sizeof(p));
  const hero_tensor* in[2] = {&a->q, &a->k};
  const hero_tensor* out[2] = {&a->q_out, &a->k_out};
  const float* gamma[2] = {a->q_gamma, a->k_gamma};
  const int heads[2] = {a->nq, a->nkv};
  const char* names[2][2] = {{"q", "q_out"}, {"k", "k_out"}};
  for (int i = 0; i < 2; ++i) {
    if (heads[i] == 0) {
      HERO_REQUIRE(in[i]->data == nullptr && out[i]->data == nullptr, HERO_ERR_INVALID_ARG, "nkv = 0 with keys given");
      continue;
    }
    hero_status st;
    const int64_t cols = (int64_t)heads[i] * a->dh;
    if ((st = check_head_matrix(*in[i], names[i][0], rows, cols)) != HERO_OK || (st = check_head_matrix(*out[i], names[i][1], rows, cols)) != HERO_OK) return st;
    HERO_REQUIRE(is_fp16ish(in[i]->dtype) && in[i]->dtype == a->q.dtype, HERO_ERR_UNSUPPORTED, "%s: dtype %d: q and k are F16 or BF16, both alike",
                 names[i][0], in[i]->dtype);
    HERO_REQUIRE(out[i]->dtype == in[i]->dtype || (out[i]->dtype == HERO_I8 && out[i]->gran == HERO_GRAN_SQ), HERO_ERR_UNSUPPORTED,
                 "%s: dtype %d gran %d: the input's type, or I8 with a static scale", names[i][1], out[i]->dtype, out[i]->gran);
    HERO_REQUIRE(out[i]->data != in[i]->data || rows == 0 || (out[i]->dtype == in[i]->dtype && out[i]->ld == in[i]->ld), HERO_ERR_INVALID_ARG,
                 "%s: in place only with the input's type and ld", names[i][1]);
    p.x[i] = static_cast<const uint16_t*>(in[i]->data); p.ld_x[i] = in[i]->ld;
    p.y[i] = out[i]->data; p.ld_y[i] = out[i]->ld;
    p.gamma[i] = gamma[i];
    p.out_scale[i] = out[i]->dtype == HERO_I8 ? out[i]->scale : nullptr;
    p.heads[i] = heads[i];
  }
  if (a->rot > 0 && rows > 0) {
    HERO_REQUIRE(a->pos && a->cos && a->sin && a->n_pos >= 1, HERO_ERR_INVALID_ARG, "a rotation needs pos, cos, sin and n_pos >= 1");
    HERO_REQUIRE(aligned16(a->cos) && aligned16(a->sin), HERO_ERR_ALIGNMENT, "cos and sin must be 16-byte aligned");
  }
  HERO_REQUIRE(rows * ((long long)a->nq + a->nkv) < (1ll << 31), HERO_ERR_UNSUPPORTED, "rows * heads = %lld: below 2^31",
               (long long)(rows * ((long long)a->nq + a->nkv)));
  if (rows == 0) return HERO_OK;
  hero_status st = check_device(h);
  if (st != HERO_OK) return st;
  p.dh = a->dh; p.rot = a->rot; p.adjacent = a->pairing == HERO_PAIR_ADJACENT;
  p.eps = a->eps; p.inv_dh = 1.0f / (float)a->dh;
  p.pos = a->pos; p.cos = a->cos; p.sin = a->sin; p.n_pos = a->n_pos; p.rows = rows;
  p.err = h->d_error;
  const bool bf = a->q.dtype == HERO_BF16;
  const int lph = a->dh <= 16 ? 2 : a->dh <= 32 ? 4 : a->dh <= 64 ? 8 : a->dh <= 128 ? 16 : 32;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  {
    LaunchScope scope(h, s, KERNEL_CACHE);
    e = lph == 2 ? launch_rope<2>(h, p, bf, s) : lph == 4 ? launch_rope<4>(h, p, bf, s) : lph == 8 ? launch_rope<8>(h, p, bf, s)
      : lph == 16 ? launch_rope<16>(h, p, bf, s) : launch_rope<32>(h, p, bf, s);
  }
  HERO_CUDA(e);
  return HERO_OK;
}
