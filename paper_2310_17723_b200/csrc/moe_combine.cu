// The end of a mixture of experts (hero_moe_combine): residual + weighted sum of each token's expert rows, LN^quant of the result.
// A token belongs to a few warps; a lane holds NCH times eight features, sums the token's rows in FP32 in the order of its choices and keeps
// the sums in registers through the statistics (mean, then centred variance, then the largest magnitude of a token-wise output), so that every
// byte is read and written once.  Bound by HBM, which wants many bytes in flight.  Two kernels:
//
//   moe_combine_kernel       a token to 1, 2, 4 or 8 warps that load its rows into registers, eight rows at a time.  For few tokens, wide rows.
//   moe_combine_ring_kernel  many tokens: persistent, four warps copy whole rows (cp.async.bulk) into a ring of stages of one token each, two
//                            or six groups of four warps take the tokens in turn
//
// 8192 tokens, top 8, 2048 features of BF16, LN^quant: the ring 69 us (0.78 of copy bandwidth; two copying warps 76, three groups 94), registers 87, a CTA a token
// 147.  INT8 rows with a scale for each expert and feature: 92 us (4 bytes of scale for each code, through L2: the ring leaves the first-level cache nothing).
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
  int k, E; long long R, T;
  int warps;                    // of a token: 1, 2, 4 or 8
  int stages;                   // of the ring
  const float* gamma; const float* beta; float eps;
  void* out; int out_dt; long long out_ld; int out_gran; float* out_scale;
  void* fp_out; int fp_dt; long long fp_ld;
  int H;
  int* err;
};

constexpr int Y_BF16 = 0, Y_F16 = 1, Y_I8 = 2, Y_F8 = 3;
constexpr int COMBINE_THREADS = 256, COMBINE_MAX_WARPS = 8;

struct Raw8 { uint32_t w[4]; };               // eight values of 8 or 16 bits
template <bool Q8>
__device__ __forceinline__ Raw8 load8(const void* p, long long at) {              // (written by an earlier call: a coherent load)
  Raw8 r = {{0u, 0u, 0u, 0u}};
  if constexpr (Q8) {
    const uint2 v = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(p) + at);
    r.w[0] = v.x; r.w[1] = v.y;
  } else {
    const uint4 v = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + at);
    r.w[0] = v.x; r.w[1] = v.y; r.w[2] = v.z; r.w[3] = v.w;
  }
  return r;
}
template <int KIND>
__device__ __forceinline__ void values8(const Raw8& r, float2 (&v)[4]) {
  if constexpr (KIND == Y_I8 || KIND == Y_F8) {
    float a[4], b[4];
    codes4_to_f32<KIND == Y_F8>(r.w[0], a);
    codes4_to_f32<KIND == Y_F8>(r.w[1], b);
    v[0] = make_float2(a[0], a[1]); v[1] = make_float2(a[2], a[3]);
    v[2] = make_float2(b[0], b[1]); v[3] = make_float2(b[2], b[3]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = fp16ish_to_f32x2<KIND == Y_BF16>(r.w[i]);
  }
}
__device__ __forceinline__ void scales8(const float* p, float2 (&f)[4]) {
  const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p + 4));
  f[0] = make_float2(a.x, a.y); f[1] = make_float2(a.z, a.w); f[2] = make_float2(b.x, b.y); f[3] = make_float2(b.z, b.w);
}
// sum += the eight values of an addend of row t
__device__ __forceinline__ void add_side(const CombineSide& s, long long t, int f0, float2 (&sum)[4]) {
  if (!s.data) return;
  float2 v[4], f[4];
  const long long at = t * s.ld + f0;
  if (s.dt == HERO_BF16) values8<Y_BF16>(load8<false>(s.data, at), v);
  else if (s.dt == HERO_F16) values8<Y_F16>(load8<false>(s.data, at), v);
  else if (s.dt == HERO_I8) values8<Y_I8>(load8<true>(s.data, at), v);
  else values8<Y_F8>(load8<true>(s.data, at), v);
  const float one = (s.row_scale ? s.row_scale[t] : 1.f) * (s.col_scale && !s.col_stride ? __ldg(s.col_scale) : 1.f);
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = make_float2(1.f, 1.f);
  if (s.col_stride) scales8(s.col_scale + f0, f);
#pragma unroll
  for (int i = 0; i < 4; ++i) sum[i] = __ffma2_rn(__fmul2_rn(v[i], make_float2(one, one)), f[i], sum[i]);
}
// sum += weight * the eight values of a row of y; scale: of the row's expert and these features (YCOL), one: the factor of all else
template <int KIND, bool YCOL>
__device__ __forceinline__ void add_row(const Raw8& raw, const float* scale, float one, float weight, float2 (&sum)[4]) {
  float2 x[4];
  values8<KIND>(raw, x);
  if constexpr (YCOL) {
    float2 f[4];
    scales8(scale, f);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __fmul2_rn(x[i], f[i]);
  } else if constexpr (KIND == Y_I8 || KIND == Y_F8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __fmul2_rn(x[i], make_float2(one, one));
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) sum[i] = __ffma2_rn(x[i], make_float2(weight, weight), sum[i]);
}

// The warps of a token: `warps` of them on named barrier `id`; part: shared float[3][warps].
struct TokenTeam { int warps, id, w; float* part; };
// sum (or maximum) over the token's lanes; k: which of the three statistics
template <bool MAX>
__device__ __forceinline__ float token_reduce(float v, const TokenTeam& team, int k) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float u = __shfl_xor_sync(0xffffffffu, v, o);
    v = MAX ? fmaxf(v, u) : v + u;
  }
  if (team.warps == 1) return v;
  float* part = team.part + k * team.warps;
  if ((threadIdx.x & 31) == 0) part[team.w] = v;
  asm volatile("bar.sync %0, %1;" ::"r"(team.id), "r"(team.warps * 32) : "memory");
  float a = part[0];
  for (int w = 1; w < team.warps; ++w) a = MAX ? fmaxf(a, part[w]) : a + part[w];
  return a;
}

__device__ __forceinline__ void store16(void* p, int dt, long long at, float2 (&v)[4], bool reread) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = dt == HERO_BF16 ? f32x2_to_fp16ish<true>(v[i].x, v[i].y) : f32x2_to_fp16ish<false>(v[i].x, v[i].y);
  *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p) + at) = make_uint4(w[0], w[1], w[2], w[3]);
  if (!reread) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = dt == HERO_BF16 ? fp16ish_to_f32x2<true>(w[i]) : fp16ish_to_f32x2<false>(w[i]);
}
template <bool F8>
__device__ __forceinline__ void store_codes(void* p, long long at, const float2 (&v)[4]) {
  *reinterpret_cast<uint2*>(static_cast<uint8_t*>(p) + at) =
      make_uint2(f32_to_codes4<F8>(v[0].x, v[0].y, v[1].x, v[1].y), f32_to_codes4<F8>(v[2].x, v[2].y, v[3].x, v[3].y));
}

// What follows the sums v of token t: fp_out, the statistics, out.  This lane has features first + c * stride .. + 7, c < NCH.
template <int NCH>
__device__ __forceinline__ void finish_token(const CombineParams& p, long long t, int first, int stride, float2 (&v)[NCH][4], const TokenTeam& team) {
  float sum = 0.f;
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    const int f0 = first + c * stride;
    if (f0 >= p.H) continue;
    if (p.fp_out) store16(p.fp_out, p.fp_dt, t * p.fp_ld + f0, v[c], p.out != nullptr);
#pragma unroll
    for (int i = 0; i < 4; ++i) sum += v[c][i].x + v[c][i].y;
  }
  if (!p.out) return;
  const float inv = 1.f / (float)p.H;
  const float mean = token_reduce<false>(sum, team, 0) * inv;
  float sq = 0.f;
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    if (first + c * stride >= p.H) continue;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[c][i] = __fadd2_rn(v[c][i], make_float2(-mean, -mean));
      sq = fmaf(v[c][i].x, v[c][i].x, sq);
      sq = fmaf(v[c][i].y, v[c][i].y, sq);
    }
  }
  const float rstd = 1.f / sqrtf(token_reduce<false>(sq, team, 1) * inv + p.eps);
  float most = 0.f;
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    const int f0 = first + c * stride;
    if (f0 >= p.H) continue;
    float2 g[4], b[4];
    scales8(p.gamma + f0, g);
    scales8(p.beta + f0, b);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[c][i] = __ffma2_rn(v[c][i], __fmul2_rn(g[i], make_float2(rstd, rstd)), b[i]);
      most = ptx::max3(most, fabsf(v[c][i].x), fabsf(v[c][i].y));
    }
  }
  const bool q8 = is_q8(p.out_dt), f8 = p.out_dt == HERO_F8;
  float s = 1.f;
  if (q8 && p.out_gran == HERO_GRAN_TWQ) {
    most = token_reduce<true>(most, team, 2);
    s = most > 0.f ? most / (f8 ? 448.f : 127.f) : 1.f;
    if (team.w == 0 && (threadIdx.x & 31) == 0) p.out_scale[t] = s;
  } else if (q8 && p.out_gran == HERO_GRAN_SQ) {
    s = __ldg(p.out_scale);
  }
  const Divider div(s);
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    const int f0 = first + c * stride;
    if (f0 >= p.H) continue;
    const long long at = t * p.out_ld + f0;
    if (!q8) {
      store16(p.out, p.out_dt, at, v[c], false);
      continue;
    }
    if (p.out_gran == HERO_GRAN_FWQ) {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[c][i] = make_float2(v[c][i].x / __ldg(p.out_scale + f0 + 2 * i), v[c][i].y / __ldg(p.out_scale + f0 + 2 * i + 1));
    } else if (div.fast) {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[c][i] = div.pair(v[c][i]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[c][i] = make_float2(div(v[c][i].x), div(v[c][i].y));
    }
    if (f8) store_codes<true>(p.out, at, v[c]);
    else store_codes<false>(p.out, at, v[c]);
  }
}

// Place j of a token, by lane j: row of y (-1: none), expert, weight.
struct Place { int row, expert; float weight; };
template <bool YCOL>
__device__ __forceinline__ Place load_place(const CombineParams& p, long long t, int lane) {
  Place a{-1, 0, 0.f};
  if (lane < p.k && t < p.T) {
    a.row = p.row[t * p.k + lane];
    if (YCOL) a.expert = p.expert[t * p.k + lane];
    a.weight = p.weight[t * p.k + lane];
  }
  return a;
}
// (apart from the loads, so that they can be on their way for a while)
__device__ __forceinline__ void check_place(const CombineParams& p, Place& a) {
  if (a.row == -1) a.expert = 0;
  if (a.row >= p.R || a.row < -1 || (unsigned)a.expert >= (unsigned)p.E) { atomicExch(p.err, ERR_BAD_EXPERT); a.row = -1; a.expert = 0; }
}

template <int KIND, bool YCOL, int NCH>
__global__ void __launch_bounds__(COMBINE_THREADS, NCH <= 2 ? 4 : 1) moe_combine_kernel(const __grid_constant__ CombineParams p) {
  __shared__ float part[3 * COMBINE_MAX_WARPS];
  constexpr bool Q8 = KIND == Y_I8 || KIND == Y_F8;
  ptx::pdl_launch_dependents();
  ptx::pdl_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, id = warp / p.warps;
  const TokenTeam team{p.warps, 1 + id, warp - id * p.warps, part + 3 * id * p.warps};
  const long long t = (long long)blockIdx.x * (COMBINE_MAX_WARPS / p.warps) + id;
  if (t >= p.T) return;                                    // (all warps of a token together)
  const int stride = p.warps * 256;                        // features from one chunk of a lane to the next
  const int first = (team.w * 32 + lane) * 8;
  Place place = load_place<YCOL>(p, t, lane);
  check_place(p, place);
  const int row = place.row, expert = place.expert;
  const float weight = place.weight;
  const float one = !YCOL && p.y.col_scale ? __ldg(p.y.col_scale) : 1.f;
  float2 v[NCH][4];
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    const int f0 = first + c * stride;
    const bool in = f0 < p.H;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[c][i] = make_float2(0.f, 0.f);
    if (in) {
      add_side(p.res, t, f0, v[c]);
      add_side(p.shared, t, f0, v[c]);
    }
    constexpr int AHEAD = 8;                               // rows asked for together
    for (int j0 = 0; j0 < p.k; j0 += AHEAD) {
      Raw8 raw[AHEAD];
#pragma unroll
      for (int j = 0; j < AHEAD; ++j) {
        const int r = __shfl_sync(0xffffffffu, row, j0 + j);                      // (j0 + j < 32; places from k on hold -1)
        if (in && r >= 0) raw[j] = load8<Q8>(p.y.data, r * p.y.ld + f0);
      }
#pragma unroll
      for (int j = 0; j < AHEAD; ++j) {
        const int r = __shfl_sync(0xffffffffu, row, j0 + j), e = YCOL ? __shfl_sync(0xffffffffu, expert, j0 + j) : 0;
        const float wj = __shfl_sync(0xffffffffu, weight, j0 + j);
        if (in && r >= 0) add_row<KIND, YCOL>(raw[j], p.y.col_scale + (long long)e * p.H + f0, one, wj, v[c]);
      }
    }
  }
  finish_token<NCH>(p, t, first, stride, v, team);
}

// ---- many tokens
constexpr int RING_GROUP_WARPS = 4, RING_COPY_WARPS = 4, RING_MAX_STAGES = 12, RING_BYTES = 216 * 1024;
// groups of warps that the registers allow (the sums of a lane are 8 NCH)
template <int NCH>
constexpr int RING_GROUPS = NCH <= 2 ? 6 : 2;
struct RingPlace { int row[COMBINE_MAX_K]; int expert[COMBINE_MAX_K]; float weight[COMBINE_MAX_K]; int all; };

template <int KIND, bool YCOL, int NCH>
__global__ void __launch_bounds__((RING_GROUPS<NCH> * RING_GROUP_WARPS + RING_COPY_WARPS) * 32, 1) moe_combine_ring_kernel(const __grid_constant__ CombineParams p) {
  constexpr int GROUPS = RING_GROUPS<NCH>;
  constexpr bool Q8 = KIND == Y_I8 || KIND == Y_F8;
  extern __shared__ __align__(128) uint8_t rows[];         // [stages][k][H]
  __shared__ __align__(8) uint64_t full[RING_MAX_STAGES], empty[RING_MAX_STAGES];
  __shared__ RingPlace places[RING_MAX_STAGES];
  __shared__ float part[GROUPS][3 * RING_GROUP_WARPS];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (threadIdx.x == 0) {
    for (int i = 0; i < p.stages; ++i) { ptx::mbar_init(&full[i], RING_COPY_WARPS); ptx::mbar_init(&empty[i], RING_GROUP_WARPS); }
    ptx::fence_mbar_init();
  }
  __syncthreads();
  ptx::pdl_launch_dependents();
  ptx::pdl_wait();
  const uint32_t row_bytes = (uint32_t)p.H * (Q8 ? 1 : 2);
  int stage = 0; uint32_t phase = 0;
  if (warp >= GROUPS * RING_GROUP_WARPS) {
    // ------------------------------------------------------------------ copies: warp q has the places q, q + RING_COPY_WARPS, .. of every token
    const int q = warp - GROUPS * RING_GROUP_WARPS;
    long long t = blockIdx.x;
    Place now = load_place<YCOL>(p, t, lane), next = load_place<YCOL>(p, t + gridDim.x, lane);
    for (; t < p.T; t += gridDim.x) {
      const Place later = load_place<YCOL>(p, t + 2 * (long long)gridDim.x, lane);
      check_place(p, now);
      if (!__all_sync(0xffffffffu, ptx::mbar_wait(&empty[stage], phase ^ 1, p.err, 0x1000 | stage))) break;
      const uint32_t some = __ballot_sync(0xffffffffu, now.row >= 0);
      const bool mine = now.row >= 0 && lane % RING_COPY_WARPS == q;
      const uint32_t ours = __ballot_sync(0xffffffffu, mine);
      if (q == 0) {
        if (lane < COMBINE_MAX_K) { places[stage].row[lane] = now.row; places[stage].expert[lane] = now.expert; places[stage].weight[lane] = now.weight; }
        if (lane == 0) places[stage].all = __popc(some) == p.k;
      }
      __syncwarp();
      if (lane == 0) ptx::mbar_expect_tx(&full[stage], __popc(ours) * row_bytes);         // (an arrival that tells of the places too)
      __syncwarp();
      if (mine)
        asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                     ::"r"(ptx::smem_u32(rows + ((size_t)stage * p.k + lane) * row_bytes)),
                     "l"(static_cast<const uint8_t*>(p.y.data) + now.row * p.y.ld * (Q8 ? 1 : 2)), "r"(row_bytes), "r"(ptx::smem_u32(&full[stage])) : "memory");
      now = next; next = later;
      if (++stage == p.stages) { stage = 0; phase ^= 1; }
    }
    // every copy started here has landed before the CTA leaves
    for (int i = 0; i < p.stages; ++i) {
      if (!ptx::mbar_wait(&empty[stage], phase ^ 1, p.err, 0x1080 | stage)) break;
      if (++stage == p.stages) { stage = 0; phase ^= 1; }
    }
  } else {
    // ------------------------------------------------------------------ sums: group g has the CTA's tokens g, g + GROUPS, ..
    // (the number of stages is a multiple of the groups: a stage is always the same group's, which so never waits for a use of it before the use before)
    const int g = warp / RING_GROUP_WARPS;
    const TokenTeam team{RING_GROUP_WARPS, 1 + g, warp % RING_GROUP_WARPS, part[g]};
    constexpr int STRIDE = RING_GROUP_WARPS * 256;
    const int first = (team.w * 32 + lane) * 8;
    const float one = !YCOL && p.y.col_scale ? __ldg(p.y.col_scale) : 1.f;
    auto forward = [&]() { if (++stage == p.stages) { stage = 0; phase ^= 1; } };
    for (int i = 0; i < g; ++i) forward();
    bool ok = true;
    for (long long t = blockIdx.x + (long long)g * gridDim.x; t < p.T; t += (long long)GROUPS * gridDim.x) {
      float2 v[NCH][4];
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[c][i] = make_float2(0.f, 0.f);
        if (first + c * STRIDE < p.H) {
          add_side(p.res, t, first + c * STRIDE, v[c]);
          add_side(p.shared, t, first + c * STRIDE, v[c]);
        }
      }
      // (a wait that gave up has recorded its code: the warp runs on without waiting, so that none is left at a barrier, and its tokens become NaN)
      ok = ok && __all_sync(0xffffffffu, ptx::mbar_wait(&full[stage], phase, p.err, 0x1100 | stage));
      const RingPlace& at = places[stage];
      const uint8_t* base = rows + (size_t)stage * p.k * row_bytes;
      auto add = [&](int j) {
        const float* scale = p.y.col_scale + (long long)at.expert[j] * p.H + first;
        const float wj = at.weight[j];
#pragma unroll
        for (int c = 0; c < NCH; ++c)
          if (first + c * STRIDE < p.H)
            add_row<KIND, YCOL>(load8<Q8>(base + j * row_bytes, first + c * STRIDE), scale + c * STRIDE, one, wj, v[c]);
      };
      int j = ok ? 0 : p.k;
      for (; at.all && j + 4 <= p.k; j += 4) {             // no place is empty: four rows at a time, without a question between their loads
        add(j); add(j + 1); add(j + 2); add(j + 3);
      }
      for (; j < p.k; ++j)
        if (at.row[j] >= 0) add(j);
      if (!ok) {
#pragma unroll
        for (int c = 0; c < NCH; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) v[c][i] = make_float2(NAN, NAN);
      }
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(&empty[stage]);
      finish_token<NCH>(p, t, first, STRIDE, v, team);
      for (int i = 0; i < GROUPS; ++i) forward();
    }
  }
}

template <int KIND, bool YCOL>
static cudaError_t launch_combine(const CombineParams& p, int nch, unsigned ctas, cudaStream_t s) {
  auto kern = nch == 1 ? moe_combine_kernel<KIND, YCOL, 1> : nch == 2 ? moe_combine_kernel<KIND, YCOL, 2> : nch <= 4 ? moe_combine_kernel<KIND, YCOL, 4>
                                                                                                        : moe_combine_kernel<KIND, YCOL, 8>;
  return launch_dependent(kern, dim3(ctas), dim3(COMBINE_THREADS), 0, s, p);
}
template <int KIND, bool YCOL, int NCH>
static hero_status launch_ring_of(hero_handle* h, const CombineParams& p, cudaStream_t s) {
  auto kern = moe_combine_ring_kernel<KIND, YCOL, NCH>;
  HERO_SMEM_OPT_IN(h, kern, RING_BYTES);
  const size_t bytes = (size_t)p.stages * p.k * p.H * (KIND == Y_I8 || KIND == Y_F8 ? 1 : 2);
  LaunchScope scope(h, s, KERNEL_LN);
  HERO_CUDA(launch_dependent(kern, dim3((unsigned)h->sm_count), dim3((RING_GROUPS<NCH> * RING_GROUP_WARPS + RING_COPY_WARPS) * 32), bytes, s, p));
  return HERO_OK;
}
static int ring_chunks(int64_t H) { return (int)((H + RING_GROUP_WARPS * 256 - 1) / (RING_GROUP_WARPS * 256)); }
template <int KIND, bool YCOL>
static hero_status launch_ring(hero_handle* h, const CombineParams& p, cudaStream_t s) {
  const int nch = ring_chunks(p.H);
  return nch == 1 ? launch_ring_of<KIND, YCOL, 1>(h, p, s) : nch == 2 ? launch_ring_of<KIND, YCOL, 2>(h, p, s) : launch_ring_of<KIND, YCOL, 4>(h, p, s);
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
  p.H = (int)H; p.T = T;
  p.err = h->d_error;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool col = p.y.col_stride != 0;
  // The ring wants a few tokens for each SM and room for one of each group
  const long long token_bytes = (long long)p.k * H * dtype_size(a->y.dtype);
  p.stages = (int)(RING_BYTES / token_bytes < RING_MAX_STAGES ? RING_BYTES / token_bytes : RING_MAX_STAGES);
  const int groups = ring_chunks(H) <= 2 ? RING_GROUPS<2> : RING_GROUPS<4>;
  p.stages = p.stages / groups * groups;
  if (T >= 4ll * h->sm_count && p.stages > 0 && H <= RING_GROUP_WARPS * 256 * 4) {
    switch (a->y.dtype) {
      case HERO_BF16: return launch_ring<Y_BF16, false>(h, p, s);
      case HERO_F16: return launch_ring<Y_F16, false>(h, p, s);
      case HERO_I8: return col ? launch_ring<Y_I8, true>(h, p, s) : launch_ring<Y_I8, false>(h, p, s);
      default: return col ? launch_ring<Y_F8, true>(h, p, s) : launch_ring<Y_F8, false>(h, p, s);
    }
  }
  // Two chunks of 256 features a warp (more where eight warps are not enough); one where there are too few tokens to fill the SMs
  const int chunks = (int)((H + 255) / 256);
  p.warps = 1;
  while (p.warps < COMBINE_MAX_WARPS && (chunks + p.warps - 1) / p.warps > 2) p.warps *= 2;
  while (p.warps < COMBINE_MAX_WARPS && p.warps < chunks && T * p.warps < 8ll * h->sm_count) p.warps *= 2;
  const int nch = (chunks + p.warps - 1) / p.warps, tokens = COMBINE_MAX_WARPS / p.warps;
  const unsigned ctas = (unsigned)((T + tokens - 1) / tokens);
  LaunchScope scope(h, s, KERNEL_LN);
  const cudaError_t e = a->y.dtype == HERO_BF16 ? launch_combine<Y_BF16, false>(p, nch, ctas, s)
                        : a->y.dtype == HERO_F16 ? launch_combine<Y_F16, false>(p, nch, ctas, s)
                        : a->y.dtype == HERO_I8 ? (col ? launch_combine<Y_I8, true>(p, nch, ctas, s) : launch_combine<Y_I8, false>(p, nch, ctas, s))
                                                : (col ? launch_combine<Y_F8, true>(p, nch, ctas, s) : launch_combine<Y_F8, false>(p, nch, ctas, s));
  HERO_CUDA(e);
  return HERO_OK;
}
