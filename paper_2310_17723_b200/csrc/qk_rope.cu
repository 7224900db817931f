// Norm and rotation of query and key heads in one pass (hero_qk_norm_rope): every element is read and written once, so the
// kernel is bound by HBM for many rows and by its latency for few.  A head vector is held by LPH lanes of a warp (8 features,
// 16 bytes each; LPH is the power of two that covers dh), the sum of squares is log2(LPH) shuffles, a rotation partner in
// the other half of the head is a shuffle of the 16-bit pairs and a neighbouring one is the lane's own.  One CTA takes one row: what a
// feature and its partner are multiplied with (gamma cos, +-gamma sin) is formed once per row in shared memory, and per head there
// remain the sum of squares, two products a feature and the norm factor.  (Forming it in every warp cost as many instructions
// as the heads themselves: 60 against 55 us on 16383 rows of 64 heads of 64.)
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

constexpr int ROPE_MAX_WARPS = 8, ROPE_ITERS = 4, ROPE_MAX_DH = 256;

template <int LPH, bool BF, bool ADJ>
__global__ void __launch_bounds__(ROPE_MAX_WARPS * 32, 4) qk_rope_kernel(const __grid_constant__ RopeParams p) {
  constexpr int HPI = 32 / LPH;                  // heads per step of a warp
  __shared__ __align__(16) float own[2][ROPE_MAX_DH], mate[2][ROPE_MAX_DH];
  ptx::pdl_launch_dependents();
  ptx::pdl_wait();
  const long long row = blockIdx.x;
  const int per_row = p.chunks[0] + p.chunks[1], warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = lane % LPH, f0 = sub * 8;
  const bool live = f0 < p.dh;
  const long long t0 = p.rot > 0 ? written(p.pos + row) : 0;
  uint4 raw[ROPE_ITERS];
  int side = 0, first = 0, heads = 0;
  auto request = [&](int unit) {
    side = unit >= p.chunks[0];                  // 0: queries, 1: keys
    first = (unit - (side ? p.chunks[0] : 0)) * (HPI * ROPE_ITERS);
    heads = p.heads[side];
    const uint16_t* x = p.x[side] + row * p.ld_x[side] + f0;
#pragma unroll
    for (int i = 0; i < ROPE_ITERS; ++i) {
      const int hd = first + lane / LPH + i * HPI;
      raw[i] = make_uint4(0, 0, 0, 0);
      if (live && hd < heads) raw[i] = *reinterpret_cast<const uint4*>(x + (long long)hd * p.dh);
    }
  };
  if (warp < per_row) request(warp);
  // ---- the row's factors
  {
    long long t = t0;
    if (t < 0 || (p.rot > 0 && t >= p.n_pos)) {
      if (threadIdx.x == 0) atomicExch(p.err, ERR_BAD_POS);
      t = t < 0 ? 0 : p.n_pos - 1;
    }
    const int half = p.rot >> 1;
    for (int f = threadIdx.x; f < p.dh; f += blockDim.x) {
      float c = 1.f, sn = 0.f;
      int pf = f;                                // partner
      if (f < p.rot) {
        const bool second = ADJ ? (f & 1) : f >= half;
        const int j = ADJ ? f >> 1 : second ? f - half : f;
        pf = ADJ ? f ^ 1 : second ? f - half : f + half;
        c = __ldg(p.cos + t * half + j);
        sn = __ldg(p.sin + t * half + j);
        if (!second) sn = -sn;
      }
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const float* gm = p.gamma[q];
        own[q][f] = gm ? __ldg(gm + f) * c : c;
        mate[q][f] = gm ? __ldg(gm + pf) * sn : sn;
      }
    }
  }
  __syncthreads();
  // the lane that holds the partner features under HERO_PAIR_HALVES (all eight features of a lane turn, or none)
  const bool turned = f0 < p.rot;
  const int r2 = p.rot >> 4, mate_lane = (lane - sub) + (turned ? (sub < r2 ? sub + r2 : sub - r2) : sub);
  for (int unit = warp; unit < per_row;) {
    const bool norm = p.gamma[side] != nullptr;
    float2 o[4], m[4];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const float4 x = live ? *reinterpret_cast<const float4*>(&own[side][f0 + 4 * e]) : make_float4(0.f, 0.f, 0.f, 0.f);
      const float4 y = live ? *reinterpret_cast<const float4*>(&mate[side][f0 + 4 * e]) : make_float4(0.f, 0.f, 0.f, 0.f);
      o[2 * e] = make_float2(x.x, x.y); o[2 * e + 1] = make_float2(x.z, x.w);
      m[2 * e] = make_float2(y.x, y.y); m[2 * e + 1] = make_float2(y.z, y.w);
    }
    const bool to_i8 = p.out_scale[side] != nullptr;
    const float i8_scale = to_i8 ? __ldg(p.out_scale[side]) : 0.f;
    const long long at0 = row * p.ld_y[side] + (long long)(first + lane / LPH) * p.dh + f0;
#pragma unroll
    for (int i = 0; i < ROPE_ITERS; ++i) {
      if (first + i * HPI >= heads) break;       // (uniform)
      const int hd = first + lane / LPH + i * HPI;
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
        for (int k = LPH / 2; k > 0; k >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, k);
        r = rsqrtf(fmaf(sum, p.inv_dh, p.eps));
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[e] = __fmul2_rn(x[e], make_float2(r, r));              // first: a norm factor of 0 (squares beyond FP32) meets no infinite product
        y[e] = __fmul2_rn(x[e], o[e]);
        // (what does not turn has no partner: a factor of zero would let an infinite or NaN neighbour in)
        if constexpr (ADJ) {
          if (turned) {
            y[e].x = fmaf(x[e].y, m[e].x, y[e].x);
            y[e].y = fmaf(x[e].x, m[e].y, y[e].y);
          }
        } else {
          const uint32_t partner = __shfl_sync(0xffffffffu, w[e], mate_lane);
          if (turned) y[e] = __ffma2_rn(__fmul2_rn(fp16ish_to_f32x2<BF>(partner), make_float2(r, r)), m[e], y[e]);
        }
      }
      if (live && hd < heads) {
        const long long at = at0 + i * HPI * p.dh;
        if (to_i8) {
          const Divider div(i8_scale);
          // (bounded before the division: a quotient beyond FP32, an infinity's too, would leave a remainder that is NaN; and then the codes
          // need no bound of their own)
          const float most = 127.f * i8_scale;
          float2 b[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) b[e] = make_float2(fminf(fmaxf(y[e].x, -most), most), fminf(fmaxf(y[e].y, -most), most));
          uint2 code;
          if (div.fast) {
            code.x = f32_to_codes4_inside<false>(div.pair(b[0]), div.pair(b[1]));
            code.y = f32_to_codes4_inside<false>(div.pair(b[2]), div.pair(b[3]));
          } else {
            code.x = f32_to_codes4<false>(div(b[0].x), div(b[0].y), div(b[1].x), div(b[1].y));
            code.y = f32_to_codes4<false>(div(b[2].x), div(b[2].y), div(b[3].x), div(b[3].y));
          }
          *reinterpret_cast<uint2*>(static_cast<uint8_t*>(p.y[side]) + at) = code;
        } else {
          *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.y[side]) + at) =
              make_uint4(f32x2_to_fp16ish<BF>(y[0].x, y[0].y), f32x2_to_fp16ish<BF>(y[1].x, y[1].y), f32x2_to_fp16ish<BF>(y[2].x, y[2].y), f32x2_to_fp16ish<BF>(y[3].x, y[3].y));
        }
      }
    }
    unit += blockDim.x >> 5;
    if (unit < per_row) request(unit);
  }
}

template <int LPH>
static cudaError_t launch_rope(RopeParams& p, bool bf, cudaStream_t s) {
  for (int i = 0; i < 2; ++i) p.chunks[i] = (p.heads[i] + (32 / LPH) * ROPE_ITERS - 1) / ((32 / LPH) * ROPE_ITERS);
  auto kern = bf ? (p.adjacent ? qk_rope_kernel<LPH, true, true> : qk_rope_kernel<LPH, true, false>)
                 : (p.adjacent ? qk_rope_kernel<LPH, false, true> : qk_rope_kernel<LPH, false, false>);
  const int units = p.chunks[0] + p.chunks[1], rounds = (units + ROPE_MAX_WARPS - 1) / ROPE_MAX_WARPS;   // equal rounds for all warps
  return launch_dependent(kern, dim3((unsigned)p.rows), dim3((unsigned)((units + rounds - 1) / rounds) * 32), 0, s, p);
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
    e = lph == 2 ? launch_rope<2>(p, bf, s) : lph == 4 ? launch_rope<4>(p, bf, s) : lph == 8 ? launch_rope<8>(p, bf, s)
      : lph == 16 ? launch_rope<16>(p, bf, s) : launch_rope<32>(p, bf, s);
  }
  HERO_CUDA(e);
  return HERO_OK;
}
