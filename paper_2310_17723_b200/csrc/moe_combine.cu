// The end of a mixture of experts (hero_moe_combine): residual + weighted sum of each token's expert rows, LN^quant of the result.
// One CTA per token; a thread holds eight features (NCH times), sums the token's rows in FP32 in the order of its choices and
// keeps the sum in registers through the statistics (mean, then centred variance, then the largest magnitude of a token-wise output),
// so that every byte is read and written once.  Bound by HBM: the k rows are asked for together.
#include "block_cache.cuh"

namespace hero {

constexpr int COMBINE_MAX_K = 16;

struct CombineSide {
  const void* data; int dt; long long ld;
  const float* row_scale;       // TWQ
  const float* col_scale;       // FWQ (stride 1) or SQ (stride 0)
  int col_stride;
};
struct CombineParams {
  CombineSide y, res, shared;   // y: FWQ scales are [E][H]
  const int* row; const float* weight; const int* expert;
  int k, E; long long R;
  const float* gamma; const float* beta; float eps;
  void* out; int out_dt; long long out_ld; int out_gran; float* out_scale;
  void* fp_out; int fp_dt; long long fp_ld;
  int H;
  int* err;
};

struct Raw8 { uint32_t w[4]; };
__device__ __forceinline__ Raw8 load8(const void* p, int dt, long long at) {      // (written by an earlier call: a coherent load)
  Raw8 r = {{0u, 0u, 0u, 0u}};
  if (is_q8(dt)) {
    const uint2 v = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(p) + at);
    r.w[0] = v.x; r.w[1] = v.y;
  } else {
    const uint4 v = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + at);
    r.w[0] = v.x; r.w[1] = v.y; r.w[2] = v.z; r.w[3] = v.w;
  }
  return r;
}
__device__ __forceinline__ void values8(const Raw8& r, int dt, float (&v)[8]) {
  if (dt == HERO_I8 || dt == HERO_F8) {
    float a[4], b[4];
    if (dt == HERO_I8) { codes4_to_f32<false>(r.w[0], a); codes4_to_f32<false>(r.w[1], b); }
    else { codes4_to_f32<true>(r.w[0], a); codes4_to_f32<true>(r.w[1], b); }
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = dt == HERO_BF16 ? fp16ish_to_f32x2<true>(r.w[i]) : fp16ish_to_f32x2<false>(r.w[i]);
      v[2 * i] = f.x; v[2 * i + 1] = f.y;
    }
  }
}
__device__ __forceinline__ void scales8(const CombineSide& s, long long at, float (&f)[8]) {
  if (s.col_stride) {
    const float4 a = __ldg(reinterpret_cast<const float4*>(s.col_scale + at)), b = __ldg(reinterpret_cast<const float4*>(s.col_scale + at + 4));
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  } else {
    const float one = s.col_scale ? __ldg(s.col_scale) : 1.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = one;
  }
}
__device__ __forceinline__ void add_side(const CombineSide& s, long long t, int f0, float (&sum)[8]) {
  if (!s.data) return;
  float v[8], f[8];
  values8(load8(s.data, s.dt, t * s.ld + f0), s.dt, v);
  scales8(s, f0, f);
  const float rs = s.row_scale ? s.row_scale[t] : 1.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) sum[i] = fmaf(v[i] * rs, f[i], sum[i]);
}

// sum (or maximum) over the CTA; `part`: shared float[32] that no other reduction in flight uses
template <bool MAX>
__device__ __forceinline__ float block_reduce(float v, float* part) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float u = __shfl_xor_sync(0xffffffffu, v, o);
    v = MAX ? fmaxf(v, u) : v + u;
  }
  const int warps = blockDim.x >> 5;
  if (warps == 1) return v;
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
  __syncthreads();
  float a = part[0];
  for (int w = 1; w < warps; ++w) a = MAX ? fmaxf(a, part[w]) : a + part[w];
  return a;
}

__device__ __forceinline__ void store16(void* p, int dt, long long at, float (&v)[8], bool reread) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = dt == HERO_BF16 ? f32x2_to_fp16ish<true>(v[2 * i], v[2 * i + 1]) : f32x2_to_fp16ish<false>(v[2 * i], v[2 * i + 1]);
  *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p) + at) = make_uint4(w[0], w[1], w[2], w[3]);
  if (reread) values8(Raw8{{w[0], w[1], w[2], w[3]}}, dt, v);
}

template <int NCH>
__global__ void __launch_bounds__(512) moe_combine_kernel(const __grid_constant__ CombineParams p) {
  __shared__ float part[3][32];
  __shared__ int at_row[COMBINE_MAX_K], at_expert[COMBINE_MAX_K];
  __shared__ float at_weight[COMBINE_MAX_K];
  ptx::pdl_launch_dependents();
  ptx::pdl_wait();
  const long long t = blockIdx.x;
  if (threadIdx.x < p.k) {
    int r = p.row[t * p.k + threadIdx.x], e = 0;
    if (r >= 0 && p.y.col_stride) e = p.expert[t * p.k + threadIdx.x];
    if (r >= p.R || r < -1 || e < 0 || e >= p.E) { atomicExch(p.err, ERR_BAD_EXPERT); r = -1; }
    at_row[threadIdx.x] = r;
    at_expert[threadIdx.x] = e;
    at_weight[threadIdx.x] = p.weight[t * p.k + threadIdx.x];
  }
  __syncthreads();
  float v[NCH][8];
  float sum = 0.f;
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    const int f0 = (threadIdx.x + c * blockDim.x) * 8;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[c][i] = 0.f;
    if (f0 >= p.H) continue;
    add_side(p.res, t, f0, v[c]);
    add_side(p.shared, t, f0, v[c]);
    constexpr int AHEAD = 8;                               // rows asked for together
    for (int j0 = 0; j0 < p.k; j0 += AHEAD) {
      Raw8 raw[AHEAD];
#pragma unroll
      for (int j = 0; j < AHEAD; ++j)
        if (j0 + j < p.k && at_row[j0 + j] >= 0) raw[j] = load8(p.y.data, p.y.dt, at_row[j0 + j] * p.y.ld + f0);
#pragma unroll
      for (int j = 0; j < AHEAD; ++j) {
        if (j0 + j < p.k && at_row[j0 + j] >= 0) {
          float x[8], f[8];
          values8(raw[j], p.y.dt, x);
          scales8(p.y, (long long)at_expert[j0 + j] * p.H + f0, f);
          const float w = at_weight[j0 + j];
#pragma unroll
          for (int i = 0; i < 8; ++i) v[c][i] = fmaf(x[i] * f[i], w, v[c][i]);
        }
      }
    }
    if (p.fp_out) store16(p.fp_out, p.fp_dt, t * p.fp_ld + f0, v[c], p.out != nullptr);
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += v[c][i];
  }
  if (!p.out) return;
  const float inv = 1.f / (float)p.H;
  const float mean = block_reduce<false>(sum, part[0]) * inv;
  float sq = 0.f;
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    if ((threadIdx.x + c * blockDim.x) * 8 >= p.H) continue;
#pragma unroll
    for (int i = 0; i < 8; ++i) { v[c][i] -= mean; sq = fmaf(v[c][i], v[c][i], sq); }
  }
  const float rstd = 1.f / sqrtf(block_reduce<false>(sq, part[1]) * inv + p.eps);
  float most = 0.f;
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    const int f0 = (threadIdx.x + c * blockDim.x) * 8;
    if (f0 >= p.H) continue;
#pragma unroll
    for (int i = 0; i < 8; i += 4) {
      const float4 g = __ldg(reinterpret_cast<const float4*>(p.gamma + f0 + i)), b = __ldg(reinterpret_cast<const float4*>(p.beta + f0 + i));
      v[c][i] = fmaf(v[c][i], rstd * g.x, b.x); v[c][i + 1] = fmaf(v[c][i + 1], rstd * g.y, b.y);
      v[c][i + 2] = fmaf(v[c][i + 2], rstd * g.z, b.z); v[c][i + 3] = fmaf(v[c][i + 3], rstd * g.w, b.w);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(v[c][i]));
  }
  const bool q8 = is_q8(p.out_dt), f8 = p.out_dt == HERO_F8;
  float s = 1.f;
  if (q8 && p.out_gran == HERO_GRAN_TWQ) {
    most = block_reduce<true>(most, part[2]);
    s = most > 0.f ? most / (f8 ? 448.f : 127.f) : 1.f;
    if (threadIdx.x == 0) p.out_scale[t] = s;
  } else if (q8 && p.out_gran == HERO_GRAN_SQ) {
    s = __ldg(p.out_scale);
  }
  const Divider div(s);
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    const int f0 = (threadIdx.x + c * blockDim.x) * 8;
    if (f0 >= p.H) continue;
    if (!q8) {
      store16(p.out, p.out_dt, t * p.out_ld + f0, v[c], false);
      continue;
    }
    if (p.out_gran == HERO_GRAN_FWQ) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[c][i] = v[c][i] / __ldg(p.out_scale + f0 + i);
    } else if (p.out_gran != HERO_GRAN_NONE) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[c][i] = div(v[c][i]);
    }
    uint2 code;
    if (f8) {
      code.x = f32_to_codes4<true>(v[c][0], v[c][1], v[c][2], v[c][3]);
      code.y = f32_to_codes4<true>(v[c][4], v[c][5], v[c][6], v[c][7]);
    } else {
      code.x = f32_to_codes4<false>(v[c][0], v[c][1], v[c][2], v[c][3]);
      code.y = f32_to_codes4<false>(v[c][4], v[c][5], v[c][6], v[c][7]);
    }
    *reinterpret_cast<uint2*>(static_cast<uint8_t*>(p.out) + t * p.out_ld + f0) = code;
  }
}

static hero_status combine_side(const hero_tensor& t, const char* name, int64_t rows, int64_t H, CombineSide* s) {
  memset(s, 0, sizeof(*s));
  if (!t.data && t.cols == 0) return HERO_OK;
  hero_status st = check_matrix(t, name);
  if (st != HERO_OK) return st;
  HERO_REQUIRE(t.rows == rows && t.cols == H, HERO_ERR_INVALID_ARG, "%s: [%lld, %lld], expected [%lld, %lld]", name, (long long)t.rows,
               (long long)t.cols, (long long)rows, (long long)H);
  HERO_REQUIRE(is_q8(t.dtype) || is_fp16ish(t.dtype), HERO_ERR_UNSUPPORTED, "%s: dtype %d: I8, F8, F16 or BF16", name, t.dtype);
  s->data = t.data; s->dt = t.dtype; s->ld = t.ld;
  if (is_q8(t.dtype)) {
    if (t.gran == HERO_GRAN_TWQ) s->row_scale = t.scale;
    if (t.gran == HERO_GRAN_FWQ) {
      HERO_REQUIRE(aligned16(t.scale), HERO_ERR_ALIGNMENT, "%s: a feature-wise scale must be 16-byte aligned", name);
      s->col_scale = t.scale; s->col_stride = 1;
    }
    if (t.gran == HERO_GRAN_SQ) s->col_scale = t.scale;
  }
  return HERO_OK;
}

}  // namespace hero

extern "C" hero_status hero_moe_combine(hero_handle* h, const hero_moe_combine_args* a, void* stream) {
  using namespace hero;
  HERO_REQUIRE(h && a, HERO_ERR_INVALID_ARG, "hero_moe_combine: NULL handle or args");
  const bool norm = a->out.cols != 0, fp = a->fp_out.cols != 0;       // (an absent tensor has no columns)
  HERO_REQUIRE(norm || fp, HERO_ERR_INVALID_ARG, "out or fp_out is required");
  const hero_tensor& like = norm ? a->out : a->fp_out;
  const int64_t T = like.rows, H = like.cols;
  HERO_REQUIRE(H >= 16 && H % 16 == 0 && H <= 16384, HERO_ERR_UNSUPPORTED, "H=%lld: a multiple of 16 up to 16384", (long long)H);
  HERO_REQUIRE(a->top_k >= 1 && a->top_k <= COMBINE_MAX_K, HERO_ERR_UNSUPPORTED, "top_k=%d: 1 to %d", a->top_k, COMBINE_MAX_K);
  HERO_REQUIRE(T < (1ll << 31) / a->top_k, HERO_ERR_UNSUPPORTED, "tokens=%lld with top_k=%d: below 2^31 pairs", (long long)T, a->top_k);
  CombineParams p;
  memset(&p, 0, sizeof(p));
  hero_status st;
  if (norm) {
    if ((st = check_matrix(a->out, "out")) != HERO_OK) return st;
    HERO_REQUIRE(is_q8(a->out.dtype) || is_fp16ish(a->out.dtype), HERO_ERR_UNSUPPORTED, "out: dtype %d", a->out.dtype);
    HERO_REQUIRE(!is_q8(a->out.dtype) || a->out.gran != HERO_GRAN_NONE, HERO_ERR_UNSUPPORTED, "an 8-bit out needs a granularity");
    HERO_REQUIRE(a->gamma && a->beta, HERO_ERR_INVALID_ARG, "gamma and beta are required with out");
    HERO_REQUIRE(aligned16(a->gamma) && aligned16(a->beta), HERO_ERR_ALIGNMENT, "gamma and beta must be 16-byte aligned");
  }
  if (fp) {
    if ((st = check_matrix(a->fp_out, "fp_out")) != HERO_OK) return st;
    HERO_REQUIRE(is_fp16ish(a->fp_out.dtype), HERO_ERR_UNSUPPORTED, "fp_out: dtype %d: F16 or BF16", a->fp_out.dtype);
    HERO_REQUIRE(a->fp_out.rows == T && a->fp_out.cols == H, HERO_ERR_INVALID_ARG, "fp_out: [%lld, %lld], expected [%lld, %lld]",
                 (long long)a->fp_out.rows, (long long)a->fp_out.cols, (long long)T, (long long)H);
  }
  if ((st = combine_side(a->residual, "residual", T, H, &p.res)) != HERO_OK || (st = combine_side(a->shared, "shared", T, H, &p.shared)) != HERO_OK) return st;
  if (T == 0) return HERO_OK;
  HERO_REQUIRE(a->y.rows < (1ll << 31) && a->y.data, HERO_ERR_INVALID_ARG, "y: data is NULL or too many rows");
  if ((st = combine_side(a->y, "y", a->y.rows, H, &p.y)) != HERO_OK) return st;
  HERO_REQUIRE(!is_q8(a->y.dtype) || a->y.gran != HERO_GRAN_TWQ, HERO_ERR_UNSUPPORTED, "y: FWQ (one scale per expert and feature), SQ or none");
  HERO_REQUIRE(a->row && a->weight, HERO_ERR_INVALID_ARG, "row and weight are required");
  HERO_REQUIRE(!p.y.col_stride || (a->expert && a->n_experts >= 1), HERO_ERR_INVALID_ARG, "a feature-wise y needs expert and n_experts");
  if ((st = check_device(h)) != HERO_OK) return st;
  p.row = a->row; p.weight = a->weight; p.expert = a->expert;
  p.k = a->top_k; p.E = p.y.col_stride ? a->n_experts : 1; p.R = a->y.rows;
  p.gamma = a->gamma; p.beta = a->beta; p.eps = a->eps;
  if (norm) { p.out = a->out.data; p.out_dt = a->out.dtype; p.out_ld = a->out.ld; p.out_gran = a->out.gran; p.out_scale = a->out.scale; }
  if (fp) { p.fp_out = a->fp_out.data; p.fp_dt = a->fp_out.dtype; p.fp_ld = a->fp_out.ld; }
  p.H = (int)H;
  p.err = h->d_error;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const int chunks = (int)(H / 8);
  const int nch = chunks <= 512 ? 1 : chunks <= 1024 ? 2 : 4;
  const unsigned threads = (unsigned)(((chunks + nch - 1) / nch + 31) / 32 * 32);
  LaunchScope scope(h, s, KERNEL_LN);
  auto kern = nch == 1 ? moe_combine_kernel<1> : nch == 2 ? moe_combine_kernel<2> : moe_combine_kernel<4>;
  HERO_CUDA(launch_dependent(kern, dim3((unsigned)T), dim3(threads), 0, s, p));
  return HERO_OK;
}
