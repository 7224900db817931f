// Norm and rotation of query and key heads in one pass (hero_qk_norm_rope): every element is read and written once, so the
// kernel is bound by HBM for many rows and by its latency for few.  A head vector is held by LPH lanes of a warp (8 features,
// 16 bytes each; LPH is the power of two that covers dh), the sum of squares is log2(LPH) shuffles, a rotation partner in
// the other half of the head is one shuffle per feature and a neighbouring one is the lane's own.  A warp takes ITERS * 32 / LPH
// heads of ONE row, so that cos and sin of the row's position are loaded once for all of them.
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
__global__ void __launch_bounds__(ROPE_WARPS * 32) qk_rope_kernel(const RopeParams p) {
  constexpr int HPI = 32 / LPH;                  // heads per iteration
  ptx::pdl_launch_dependents();
  ptx::pdl_wait();
  const int per_row = p.chunks[0] + p.chunks[1];
  const long long w = (long long)blockIdx.x * ROPE_WARPS + (threadIdx.x >> 5);
  const long long row = w / per_row;
  if (row >= p.rows) return;
  int ch = (int)(w - row * per_row);
  const int side = ch >= p.chunks[0];            // 0: queries, 1: keys
  if (side) ch -= p.chunks[0];
  const int lane = threadIdx.x & 31, sub = lane % LPH, f0 = sub * 8;
  const bool live = f0 < p.dh;
  const int h0 = ch * (HPI * ITERS) + lane / LPH, heads = p.heads[side];
  const uint16_t* x = p.x[side] + row * p.ld_x[side] + f0;

  uint4 raw[ITERS];
#pragma unroll
  for (int i = 0; i < ITERS; ++i) {
    const int hd = h0 + i * HPI;
    raw[i] = make_uint4(0, 0, 0, 0);
    if (live && hd < heads) raw[i] = *reinterpret_cast<const uint4*>(x + (long long)hd * p.dh);
  }
  // cos and sin of the lane's features: sn carries the sign with which the partner enters
  float cs[8], sn[8];
  const bool turns = f0 < p.rot;
  const int half = p.rot >> 1;
  if (p.rot > 0) {
    long long t = __ldg(p.pos + row);
    if (t < 0 || t >= p.n_pos) {
      if (lane == 0) atomicExch(p.err, ERR_BAD_POS);
      t = t < 0 ? 0 : p.n_pos - 1;
    }
    const float* ct = p.cos + t * half;
    const float* st = p.sin + t * half;
    if (turns) {
      if (p.adjacent) {
        const float4 c = __ldg(reinterpret_cast<const float4*>(ct + f0 / 2)), s = __ldg(reinterpret_cast<const float4*>(st + f0 / 2));
        cs[0] = cs[1] = c.x; cs[2] = cs[3] = c.y; cs[4] = cs[5] = c.z; cs[6] = cs[7] = c.w;
        sn[0] = -s.x; sn[1] = s.x; sn[2] = -s.y; sn[3] = s.y; sn[4] = -s.z; sn[5] = s.z; sn[6] = -s.w; sn[7] = s.w;
      } else {
        const bool second = f0 >= half;
        const int j = second ? f0 - half : f0;
        const float4 c0 = __ldg(reinterpret_cast<const float4*>(ct + j)), c1 = __ldg(reinterpret_cast<const float4*>(ct + j + 4));
        const float4 s0 = __ldg(reinterpret_cast<const float4*>(st + j)), s1 = __ldg(reinterpret_cast<const float4*>(st + j + 4));
        cs[0] = c0.x; cs[1] = c0.y; cs[2] = c0.z; cs[3] = c0.w; cs[4] = c1.x; cs[5] = c1.y; cs[6] = c1.z; cs[7] = c1.w;
        sn[0] = s0.x; sn[1] = s0.y; sn[2] = s0.z; sn[3] = s0.w; sn[4] = s1.x; sn[5] = s1.y; sn[6] = s1.z; sn[7] = s1.w;
        if (!second) {
#pragma unroll
          for (int e = 0; e < 8; ++e) sn[e] = -sn[e];
        }
      }
    }
  }
  float g[8];
  const bool norm = p.gamma[side] != nullptr;
  if (norm && live) {
#pragma unroll
    for (int e = 0; e < 8; ++e) g[e] = __ldg(p.gamma[side] + f0 + e);
  }
  float inv_s = 0.f;
  const bool to_i8 = p.out_scale[side] != nullptr;
  if (to_i8) inv_s = __ldg(p.out_scale[side]);
  const Divider div(inv_s);
  // the lane that holds the partner features under HERO_PAIR_HALVES
  const int r2 = p.rot >> 4;
  const int mate = (lane - sub) + (turns ? (sub < r2 ? sub + r2 : sub - r2) : sub);

#pragma unroll
  for (int i = 0; i < ITERS; ++i) {
    const int hd = h0 + i * HPI;
    float y[8];
    {
      const float2 a = fp16ish_to_f32x2<BF>(raw[i].x), b = fp16ish_to_f32x2<BF>(raw[i].y);
      const float2 c = fp16ish_to_f32x2<BF>(raw[i].z), d = fp16ish_to_f32x2<BF>(raw[i].w);
      y[0] = a.x; y[1] = a.y; y[2] = b.x; y[3] = b.y; y[4] = c.x; y[5] = c.y; y[6] = d.x; y[7] = d.y;
    }
    if (norm) {
      float ss = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) ss = fmaf(y[e], y[e], ss);
#pragma unroll
      for (int o = LPH / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
      const float r = rsqrtf(fmaf(ss, p.inv_dh, p.eps));
      if (live) {
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = y[e] * r * g[e];
      }
    }
    if (p.rot > 0) {
      float z[8];
      if (p.adjacent) {
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = y[e ^ 1];
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = __shfl_sync(0xffffffffu, y[e], mate);
      }
      if (turns) {
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = fmaf(z[e], sn[e], y[e] * cs[e]);
      }
    }
    if (live && hd < heads) {
      const long long at = row * p.ld_y[side] + (long long)hd * p.dh + f0;
      if (to_i8) {
        uint2 code;
        code.x = f32_to_codes4<false>(div(y[0]), div(y[1]), div(y[2]), div(y[3]));
        code.y = f32_to_codes4<false>(div(y[4]), div(y[5]), div(y[6]), div(y[7]));
        *reinterpret_cast<uint2*>(static_cast<uint8_t*>(p.y[side]) + at) = code;
      } else {
        *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.y[side]) + at) =
            make_uint4(f32x2_to_fp16ish<BF>(y[0], y[1]), f32x2_to_fp16ish<BF>(y[2], y[3]), f32x2_to_fp16ish<BF>(y[4], y[5]), f32x2_to_fp16ish<BF>(y[6], y[7]));
      }
    }
  }
}

template <int LPH, int ITERS>
static cudaError_t launch_rope(RopeParams& p, bool bf, cudaStream_t s) {
  for (int i = 0; i < 2; ++i) p.chunks[i] = (p.heads[i] + (32 / LPH) * ITERS - 1) / ((32 / LPH) * ITERS);
  const long long warps = p.rows * (p.chunks[0] + p.chunks[1]);
  const unsigned grid = (unsigned)((warps + ROPE_WARPS - 1) / ROPE_WARPS);
  return launch_dependent(bf ? qk_rope_kernel<LPH, ITERS, true> : qk_rope_kernel<LPH, ITERS, false>, dim3(grid), dim3(ROPE_WARPS * 32), 0, s, p);
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
    e = lph == 2 ? launch_rope<2, 4>(p, bf, s) : lph == 4 ? launch_rope<4, 4>(p, bf, s) : lph == 8 ? launch_rope<8, 4>(p, bf, s)
      : lph == 16 ? launch_rope<16, 4>(p, bf, s) : launch_rope<32, 4>(p, bf, s);
  }
  HERO_CUDA(e);
  return HERO_OK;
}
