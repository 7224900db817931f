// The router of a mixture of experts (hero_moe_route): top k of every token's logits, their weights, and the order of the (token, expert)
// pairs by expert.
//
// Choice: one warp per token, expert lane + 32 r in the lane's register r.  Every logit becomes an unsigned key whose order is the logits'
// (0: does not take part); a round is the lane's own maximum, a warp maximum (redux), and the winner's lane taking it out.  16-bit
// logits carry the inverted expert in the key's low half, so that one reduction finds the lowest of equal ones; 32-bit keys take a
// second reduction over the index.  With a selection bias the keys are FP32 scores plus bias: where two neighbours of the k + 1 largest
// are nearer than FP32 can tell apart, the token is chosen again from FP64 keys.
//
// Order: a bit per (expert, token) in shared memory.  The rank of a pair within its expert is the number of bits before its own, whatever
// the order in which warps set them, so that the result does not depend on timing and no global atomics are needed.  Few tokens: one
// CTA does everything.  More: each CTA of a first kernel counts its own tokens' experts, and each CTA of a second one adds up the
// counts of those before it (and of all, for the experts' first rows) and places its pairs.
//
// The bytes are few (2 to 4 per logit); what bounds it is the chain of k rounds per token, about 40 instructions each.
#include "common.cuh"
#include "ptx.cuh"
#include <cuda_fp16.h>
#include <cuda_bf16.h>

namespace hero {

constexpr int ROUTE_MAX_E = 512, ROUTE_MAX_K = 16;
constexpr int ROUTE_THREADS = 1024;
constexpr int ROUTE_ONE_CTA = 96;        // tokens that one CTA takes alone
constexpr int ROUTE_MAX_CHUNK = 1024;    // tokens per CTA of the two-kernel form (bit words: E * chunk / 32)

struct RouteParams {
  const void* logits; long long ld;
  const int* n_tokens;
  const float* bias;
  int T, E, k, score, renorm;
  float scale;
  int* expert; float* weight; int* offset; int* token; int* row;
  int* counts;                           // [CTAs][E] (two-kernel form)
  int chunk, words;                      // tokens per CTA (a multiple of 32), chunk / 32
};

__device__ __forceinline__ uint32_t order32(float x) {     // larger float <=> larger key; -inf and NaN: 0
  if (!(x > -INFINITY)) return 0u;
  const uint32_t b = x == 0.f ? 0u : __float_as_uint(x);   // (-0 and +0 are equal)
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ unsigned long long order64(double x) {
  if (!(x > -INFINITY)) return 0ull;
  const unsigned long long b = x == 0.0 ? 0ull : (unsigned long long)__double_as_longlong(x);
  return (b >> 63) ? ~b : (b | 0x8000000000000000ull);
}
template <typename F>
__device__ __forceinline__ F warp_sum(F v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
// e^(x - m) where m is the largest of the x: several of +inf count alike, -inf (and NaN) not at all
__device__ __forceinline__ float exp_below(float x, float m) { return !(x > -INFINITY) ? 0.f : x == m ? 1.f : expf(x - m); }
__device__ __forceinline__ double exp_below(double x, double m) { return !(x > -INFINITY) ? 0. : x == m ? 1. : exp(x - m); }

template <int DT>
__device__ __forceinline__ float load_logit(const void* p, long long i) {
  if constexpr (DT == HERO_F32) return *(static_cast<const float*>(p) + i);
  else if constexpr (DT == HERO_F16) return __half2float(*(static_cast<const __half*>(p) + i));
  else return __bfloat162float(*(static_cast<const __nv_bfloat16*>(p) + i));
}

// The k largest of x + bias' keys in FP64 (rarely needed: keys that FP32 cannot order).  Lane j < k returns its choice.
template <int R>
__device__ __noinline__ int choose_exactly(const RouteParams& p, const float (&x)[R], float m, int lane) {
  double key[R];
  double sum = 0.0;
  if (p.score == HERO_SCORE_SOFTMAX) {
#pragma unroll
    for (int r = 0; r < R; ++r) sum += key[r] = exp_below((double)x[r], (double)m);
    sum = warp_sum(sum);
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int e = lane + 32 * r;
    const double s = p.score == HERO_SCORE_SOFTMAX ? key[r] / sum : 1.0 / (1.0 + exp(-(double)x[r]));
    key[r] = e < p.E && x[r] > -INFINITY ? s + (double)p.bias[e] : -INFINITY;
  }
  int mine = -1;
  for (int j = 0; j < p.k; ++j) {
    unsigned long long best = 0;
    int at = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const unsigned long long o = order64(key[r]);
      if (o > best) { best = o; at = r; }
    }
    const uint32_t hi = __reduce_max_sync(0xffffffffu, (uint32_t)(best >> 32));
    const uint32_t lo = __reduce_max_sync(0xffffffffu, (uint32_t)(best >> 32) == hi ? (uint32_t)best : 0u);
    if ((hi | lo) == 0u) break;
    const bool cand = best == (((unsigned long long)hi << 32) | lo);
    const int e = (int)__reduce_min_sync(0xffffffffu, cand ? (uint32_t)(lane + 32 * at) : 0xffffffffu);
    if (lane == j) mine = e;
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (e == lane + 32 * r) key[r] = -INFINITY;
  }
  return mine;
}

// One token by one warp: experts and weights written, lane j < k returns the expert of place j (-1: none).
template <int R, int DT>
__device__ __forceinline__ int route_token(const RouteParams& p, int t, int tokens, int lane) {
  int mine = -1;                                           // lane j: the expert of place j
  float mine_x = -INFINITY;                                // ... and its logit
  if (t < tokens) {
    float x[R];
    const long long at0 = (long long)t * p.ld;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int e = lane + 32 * r;
      x[r] = e < p.E ? load_logit<DT>(p.logits, at0 + e) : -INFINITY;
    }
    const bool biased = p.bias != nullptr;
    float bias[R];
    if (biased) {
#pragma unroll
      for (int r = 0; r < R; ++r) {
        bias[r] = lane + 32 * r < p.E ? __ldg(p.bias + lane + 32 * r) : -INFINITY;
        if (!(bias[r] > -INFINITY)) x[r] = -INFINITY;      // such an expert does not take part at all
      }
    }
    float m = -INFINITY, sum = 0.f;
    const bool softmax_all = p.score == HERO_SCORE_SOFTMAX && (biased || !p.renorm);
    if (softmax_all) {
#pragma unroll
      for (int r = 0; r < R; ++r) m = fmaxf(m, x[r]);      // (fmaxf passes over NaN)
      m = warp_max(m);
#pragma unroll
      for (int r = 0; r < R; ++r) sum += exp_below(x[r], m);
      sum = warp_sum(sum);
    }
    if constexpr (DT != HERO_F32) {
      if (!biased) {
        uint32_t key[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
          // the 16-bit value is the upper half of its own ordered FP32 pattern for BF16; FP16 has an order of its own
          uint32_t o;
          if constexpr (DT == HERO_BF16) o = order32(x[r]) >> 16;
          else {
            const uint32_t b = x[r] == 0.f ? 0u : (uint32_t)__half_as_ushort(__float2half_rn(x[r]));
            o = !(x[r] > -INFINITY) ? 0u : (b & 0x8000u) ? (~b & 0xffffu) : (b | 0x8000u);
          }
          key[r] = o ? (o << 16) | (0xffffu - (uint32_t)(lane + 32 * r)) : 0u;
        }
        for (int j = 0; j < p.k; ++j) {
          uint32_t best = key[0];
#pragma unroll
          for (int r = 1; r < R; ++r) best = max(best, key[r]);
          const uint32_t top = __reduce_max_sync(0xffffffffu, best);
          if (top == 0u) break;
          if (lane == j) {
            const uint32_t o = top >> 16;
            mine = (int)(0xffffu - (top & 0xffffu));
            const uint32_t b = (o & 0x8000u) ? (o & 0x7fffu) : (~o & 0xffffu);
            mine_x = DT == HERO_BF16 ? __uint_as_float(b << 16) : __half2float(__ushort_as_half((unsigned short)b));
          }
#pragma unroll
          for (int r = 0; r < R; ++r) key[r] = key[r] == top ? 0u : key[r];
        }
      }
    }
    if (DT == HERO_F32 || biased) {
      uint32_t key[R];
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float v = x[r];
        if (biased && v > -INFINITY) v = (p.score == HERO_SCORE_SOFTMAX ? exp_below(v, m) / sum : 1.f / (1.f + expf(-v))) + bias[r];
        key[r] = order32(v);
      }
      // one round beyond k: the border to what is not chosen
      float last = INFINITY;
      bool near = false;
      for (int j = 0; j < p.k + (biased ? 1 : 0); ++j) {
        uint32_t best = key[0];
        int at = 0;
#pragma unroll
        for (int r = 1; r < R; ++r)
          if (key[r] > best) { best = key[r]; at = r; }
        const uint32_t top = __reduce_max_sync(0xffffffffu, best);
        if (top == 0u) break;
        const int e = (int)__reduce_min_sync(0xffffffffu, best == top ? (uint32_t)(lane + 32 * at) : 0xffffffffu);
        if (biased) {
          // FP32 keys are off by a few units of 2^-24 of the score (at most 1) and half a unit of the key
          const float v = __uint_as_float((top & 0x80000000u) ? (top & 0x7fffffffu) : ~top);
          near = near || last - v < 4e-6f * (1.f + fabsf(v)) || v == last;
          last = v;
        }
        if (lane == j && j < p.k) mine = e;
#pragma unroll
        for (int r = 0; r < R; ++r)
          if (e == lane + 32 * r) key[r] = 0u;
      }
      if (near) mine = choose_exactly<R>(p, x, m, lane);
      if (mine >= 0) mine_x = load_logit<DT>(p.logits, at0 + mine);
    }
    // ---- weights
    float w = 0.f;
    if (p.score == HERO_SCORE_SOFTMAX) {
      if (p.renorm) {
        const float top = warp_max(mine_x);
        w = exp_below(mine_x, top);
        const float all = warp_sum(w);
        w = mine >= 0 ? w / all : 0.f;
      } else if (mine >= 0) {
        w = exp_below(mine_x, m) / sum;
      }
    } else if (p.renorm) {
      // sigmoid(x) = e^min(x, 0) / (1 + e^-|x|); the first factor relative to its largest, so that logits far below 0 keep their ratios
      const float low = mine >= 0 ? fminf(mine_x, 0.f) : -INFINITY, top = warp_max(low);
      w = mine >= 0 ? exp_below(low, top) / (1.f + expf(-fabsf(mine_x))) : 0.f;
      const float all = warp_sum(w);
      w = mine >= 0 ? w / all : 0.f;
    } else if (mine >= 0) {
      w = 1.f / (1.f + expf(-mine_x));
    }
    if (lane < p.k) p.weight[(long long)t * p.k + lane] = w * p.scale;
  } else if (lane < p.k) {
    p.weight[(long long)t * p.k + lane] = 0.f;
  }
  if (lane < p.k) p.expert[(long long)t * p.k + lane] = mine;
  return mine;
}

__device__ __forceinline__ int token_count(const RouteParams& p) { return p.n_tokens ? min(max(*p.n_tokens, 0), p.T) : p.T; }

// bits of expert e before token i of the chunk
__device__ __forceinline__ int rank_before(const uint32_t* bits, int words, int e, int i) {
  const uint32_t* b = bits + e * words;
  int n = 0;
  for (int w = 0; w < (i >> 5); ++w) n += __popc(b[w]);
  return n + __popc(b[i >> 5] & ((1u << (i & 31)) - 1u));
}
__device__ __forceinline__ int bits_of(const uint32_t* bits, int words, int e) {
  int n = 0;
  for (int w = 0; w < words; ++w) n += __popc(bits[e * words + w]);
  return n;
}
// exclusive sums of v over threads 0 .. ROUTE_MAX_E - 1 (the others pass 0); `warps`: shared int[32].  All threads call.
__device__ __forceinline__ int exclusive_sum(int v, int* warps) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int s = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, s, o);
    if (lane >= o) s += u;
  }
  if (lane == 31) warps[warp] = s;
  __syncthreads();
  int before = 0;
  for (int w = 0; w < warp; ++w) before += warps[w];
  return before + s - v;
}

// Few tokens: all of it in one CTA.
template <int R, int DT>
__global__ void __launch_bounds__(ROUTE_THREADS, 1) route_one_kernel(const __grid_constant__ RouteParams p) {
  extern __shared__ uint32_t bits[];                       // [E][words]
  __shared__ int first[ROUTE_MAX_E], warps[32];
  ptx::pdl_launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nw = blockDim.x >> 5;
  for (int i = threadIdx.x; i < p.E * p.words; i += blockDim.x) bits[i] = 0u;
  ptx::pdl_wait();
  const int tokens = token_count(p);
  __syncthreads();
  constexpr int PER_WARP = (ROUTE_ONE_CTA + 31) / 32;      // (a launch has a warp for every token up to 32)
  int mine[PER_WARP];
#pragma unroll
  for (int i = 0; i < PER_WARP; ++i) {
    const int t = warp + i * nw;
    mine[i] = -1;
    if (t < p.T) {
      mine[i] = route_token<R, DT>(p, t, tokens, lane);
      if (mine[i] >= 0) atomicOr(&bits[mine[i] * p.words + (t >> 5)], 1u << (t & 31));
    }
  }
  __syncthreads();
  const int e = threadIdx.x;
  int n[(ROUTE_MAX_E + 31) / 32] = {};
  // (a block may have fewer threads than experts: each takes E / threads of them, in order)
  const int per = (p.E + blockDim.x - 1) / blockDim.x;
  int own = 0;
#pragma unroll
  for (int i = 0; i < (ROUTE_MAX_E + 31) / 32; ++i) {
    if (i >= per) break;
    const int ee = e * per + i;
    n[i] = ee < p.E ? bits_of(bits, p.words, ee) : 0;
    own += n[i];
  }
  int at = exclusive_sum(own, warps);
#pragma unroll
  for (int i = 0; i < (ROUTE_MAX_E + 31) / 32; ++i) {
    if (i >= per) break;
    const int ee = e * per + i;
    if (ee < p.E) {
      first[ee] = at;
      p.offset[ee] = at;
      if (ee == p.E - 1) p.offset[p.E] = at + n[i];
    }
    at += n[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < PER_WARP; ++i) {
    const int t = warp + i * nw;
    if (t < p.T && lane < p.k) {
      int r = -1;
      if (mine[i] >= 0) {
        r = first[mine[i]] + rank_before(bits, p.words, mine[i], t);
        p.token[r] = t;
      }
      p.row[(long long)t * p.k + lane] = r;
    }
  }
}

// Two-kernel form, first: choose, and count the chunk's pairs of every expert.
template <int R, int DT>
__global__ void __launch_bounds__(ROUTE_THREADS, 1) route_choose_kernel(const __grid_constant__ RouteParams p) {
  __shared__ int count[ROUTE_MAX_E];
  ptx::pdl_launch_dependents();
  for (int e = threadIdx.x; e < p.E; e += blockDim.x) count[e] = 0;
  ptx::pdl_wait();
  const int tokens = token_count(p), lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nw = blockDim.x >> 5;
  __syncthreads();
  const long long t0 = (long long)blockIdx.x * p.chunk;
  const int n = (int)min((long long)p.chunk, p.T - t0);
  for (int i = warp; i < n; i += nw) {
    const int e = route_token<R, DT>(p, (int)(t0 + i), tokens, lane);
    if (e >= 0) atomicAdd(&count[e], 1);                   // (shared memory, whole numbers: any order gives the same)
  }
  __syncthreads();
  for (int e = threadIdx.x; e < p.E; e += blockDim.x) p.counts[(long long)blockIdx.x * p.E + e] = count[e];
}

// Two-kernel form, second: the first row of every expert for this chunk, and the place of each of its pairs.
__global__ void __launch_bounds__(ROUTE_THREADS, 1) route_place_kernel(const __grid_constant__ RouteParams p) {
  extern __shared__ uint32_t bits[];                       // [E][words]
  __shared__ int before[ROUTE_MAX_E], total[ROUTE_MAX_E], warps[32];
  ptx::pdl_launch_dependents();
  for (int i = threadIdx.x; i < p.E * p.words; i += blockDim.x) bits[i] = 0u;
  for (int e = threadIdx.x; e < p.E; e += blockDim.x) before[e] = total[e] = 0;
  ptx::pdl_wait();
  __syncthreads();
  // counts of all chunks: as many threads of an expert as fit, each a share of the chunks
  int pe = 32;
  while (pe < p.E) pe <<= 1;
  {
    const int e = threadIdx.x & (pe - 1), g = threadIdx.x / pe, groups = blockDim.x / pe;
    if (e < p.E) {
      int b = 0, a = 0;
#pragma unroll 8
      for (int c = g; c < (int)gridDim.x; c += groups) {
        const int v = p.counts[(long long)c * p.E + e];
        a += v;
        b += c < (int)blockIdx.x ? v : 0;
      }
      if (a) atomicAdd(&total[e], a);
      if (b) atomicAdd(&before[e], b);
    }
  }
  const long long t0 = (long long)blockIdx.x * p.chunk;
  const int n = (int)min((long long)p.chunk, p.T - t0);
  const int pairs = n * p.k;
  const int* expert = p.expert + t0 * p.k;
  for (int i = threadIdx.x; i < pairs; i += blockDim.x) {
    const int e = expert[i], t = i / p.k;
    if (e >= 0) atomicOr(&bits[e * p.words + (t >> 5)], 1u << (t & 31));
  }
  __syncthreads();
  const int e = threadIdx.x;
  const int all = e < p.E ? total[e] : 0;
  const int at = exclusive_sum(all, warps);
  if (e < p.E) {
    before[e] += at;
    if (blockIdx.x == 0) {
      p.offset[e] = at;
      if (e == p.E - 1) p.offset[p.E] = at + all;
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < pairs; i += blockDim.x) {
    const int e = expert[i], t = i / p.k;
    int r = -1;
    if (e >= 0) {
      r = before[e] + rank_before(bits, p.words, e, t);
      p.token[r] = (int)t0 + t;
    }
    p.row[t0 * p.k + i] = r;
  }
}

__global__ void route_none_kernel(int* offset, int E) {    // no tokens at all
  ptx::pdl_launch_dependents();
  ptx::pdl_wait();
  for (int e = threadIdx.x; e <= E; e += blockDim.x) offset[e] = 0;
}

static int route_chunk(const hero_handle* h, long long T) {
  long long c = ((T + h->sm_count - 1) / h->sm_count + 31) / 32 * 32;
  return (int)(c > ROUTE_MAX_CHUNK ? ROUTE_MAX_CHUNK : c);
}

template <int R, int DT>
static hero_status launch_route(hero_handle* h, RouteParams& p, cudaStream_t s) {
  if (p.T <= ROUTE_ONE_CTA) {
    p.words = (p.T + 31) / 32;
    const int warps = p.T < 32 ? p.T : 32;
    LaunchScope scope(h, s, KERNEL_ROUTE);
    HERO_CUDA(launch_dependent(route_one_kernel<R, DT>, dim3(1), dim3(32 * warps), (size_t)p.E * p.words * 4, s, p));
    return HERO_OK;
  }
  const unsigned ctas = (unsigned)((p.T + p.chunk - 1) / p.chunk);
  {
    LaunchScope scope(h, s, KERNEL_ROUTE);
    HERO_CUDA(launch_dependent(route_choose_kernel<R, DT>, dim3(ctas), dim3(ROUTE_THREADS), 0, s, p));
  }
  HERO_SMEM_OPT_IN(h, route_place_kernel, ROUTE_MAX_E * (ROUTE_MAX_CHUNK / 32) * 4);
  {
    LaunchScope scope(h, s, KERNEL_ROUTE);
    HERO_CUDA(launch_dependent(route_place_kernel, dim3(ctas), dim3(ROUTE_THREADS), (size_t)p.E * p.words * 4, s, p));
  }
  return HERO_OK;
}

template <int DT>
static hero_status route_for(hero_handle* h, RouteParams& p, cudaStream_t s) {
  if (p.E <= 32) return launch_route<1, DT>(h, p, s);
  if (p.E <= 64) return launch_route<2, DT>(h, p, s);
  if (p.E <= 128) return launch_route<4, DT>(h, p, s);
  if (p.E <= 256) return launch_route<8, DT>(h, p, s);
  return launch_route<16, DT>(h, p, s);
}

static hero_status route_sizes(int64_t T, int32_t E, int32_t k) {
  HERO_REQUIRE(E >= 1 && E <= ROUTE_MAX_E, HERO_ERR_UNSUPPORTED, "n_experts=%d: 1 to %d", E, ROUTE_MAX_E);
  HERO_REQUIRE(k >= 1 && k <= ROUTE_MAX_K && k <= E, HERO_ERR_UNSUPPORTED, "top_k=%d: 1 to %d and at most n_experts=%d", k, ROUTE_MAX_K, E);
  HERO_REQUIRE(T >= 0 && T < (1ll << 31) / k, HERO_ERR_UNSUPPORTED, "tokens=%lld with top_k=%d: below 2^31 pairs", (long long)T, k);
  return HERO_OK;
}
static size_t route_workspace(const hero_handle* h, int64_t T, int32_t E) {
  // the most chunks that any smaller number of tokens takes: one per SM, or T / ROUTE_MAX_CHUNK
  const int64_t ctas = (T + ROUTE_MAX_CHUNK - 1) / ROUTE_MAX_CHUNK;
  const int64_t few = (T + 31) / 32 < h->sm_count ? (T + 31) / 32 : h->sm_count;
  return T <= ROUTE_ONE_CTA ? 0 : (size_t)(ctas > few ? ctas : few) * (size_t)E * 4;
}

}  // namespace hero

extern "C" hero_status hero_moe_route_workspace_bytes(hero_handle* h, int64_t n_tokens, int32_t n_experts, int32_t top_k, size_t* bytes) {
  using namespace hero;
  HERO_REQUIRE(h && bytes, HERO_ERR_INVALID_ARG, "hero_moe_route_workspace_bytes: NULL handle or result");
  const hero_status st = route_sizes(n_tokens, n_experts, top_k);
  if (st != HERO_OK) return st;
  *bytes = route_workspace(h, n_tokens, n_experts);
  return HERO_OK;
}

extern "C" hero_status hero_moe_route(hero_handle* h, const hero_moe_route_args* a, void* stream) {
  using namespace hero;
  HERO_REQUIRE(h && a, HERO_ERR_INVALID_ARG, "hero_moe_route: NULL handle or args");
  const hero_tensor& x = a->logits;
  HERO_REQUIRE(x.dtype == HERO_F32 || is_fp16ish(x.dtype), HERO_ERR_UNSUPPORTED, "logits: dtype %d: F16, BF16 or F32", x.dtype);
  const uintptr_t es = dtype_size(x.dtype);
  HERO_REQUIRE(x.rows >= 0 && x.cols >= 1 && x.ld >= x.cols && (x.data || x.rows == 0), HERO_ERR_INVALID_ARG, "logits: rows=%lld cols=%lld ld=%lld",
               (long long)x.rows, (long long)x.cols, (long long)x.ld);
  HERO_REQUIRE(reinterpret_cast<uintptr_t>(x.data) % es == 0, HERO_ERR_ALIGNMENT, "logits: not aligned to an element");
  HERO_REQUIRE(x.cols <= ROUTE_MAX_E, HERO_ERR_UNSUPPORTED, "n_experts=%lld: at most %d", (long long)x.cols, ROUTE_MAX_E);
  hero_status st = route_sizes(x.rows, (int32_t)x.cols, a->top_k);
  if (st != HERO_OK) return st;
  HERO_REQUIRE(a->score == HERO_SCORE_SOFTMAX || a->score == HERO_SCORE_SIGMOID, HERO_ERR_INVALID_ARG, "score %d", a->score);
  HERO_REQUIRE(a->offset && (x.rows == 0 || (a->expert && a->weight && a->token && a->row)), HERO_ERR_INVALID_ARG,
               "expert, weight, offset, token and row are required");
  const size_t need = route_workspace(h, x.rows, (int32_t)x.cols);
  HERO_REQUIRE(need == 0 || (a->workspace && a->workspace_bytes >= need), HERO_ERR_WORKSPACE, "workspace of %zu bytes, %zu are needed",
               a->workspace ? a->workspace_bytes : (size_t)0, need);
  HERO_REQUIRE(need == 0 || aligned16(a->workspace), HERO_ERR_ALIGNMENT, "the workspace must be 16-byte aligned");
  if ((st = check_device(h)) != HERO_OK) return st;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (x.rows == 0) {
    LaunchScope scope(h, s, KERNEL_ROUTE);
    HERO_CUDA(launch_dependent(route_none_kernel, dim3(1), dim3(256), 0, s, a->offset, (int)x.cols));
    return HERO_OK;
  }
  RouteParams p;
  memset(&p, 0, sizeof(p));
  p.logits = x.data; p.ld = x.ld;
  p.n_tokens = a->n_tokens; p.bias = a->select_bias;
  p.T = (int)x.rows; p.E = (int)x.cols; p.k = a->top_k; p.score = a->score; p.renorm = a->renorm;
  p.scale = a->scale;
  p.expert = a->expert; p.weight = a->weight; p.offset = a->offset; p.token = a->token; p.row = a->row;
  p.counts = static_cast<int*>(a->workspace);
  p.chunk = route_chunk(h, p.T);
  p.words = p.chunk / 32;
  return x.dtype == HERO_F32 ? route_for<HERO_F32>(h, p, s) : x.dtype == HERO_F16 ? route_for<HERO_F16>(h, p, s) : route_for<HERO_BF16>(h, p, s);
}
