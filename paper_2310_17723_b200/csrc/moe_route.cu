// The router of a mixture of experts (hero_moe_route): top k of every token's logits, their weights, and the order of the (token, expert)
// pairs by expert.
//
// Choice: every logit becomes an unsigned key whose order is the logits' (0: does not take part).
//   few tokens   one warp per token, expert lane + 32 r in the lane's register r.  A round is the lane's own maximum, a warp maximum (redux), and the
//                winner's lane taking it out: about 500 instructions a token at 128 experts, 1300 with a bias at 256.
//   more tokens  eight lanes per token go through an eighth of its keys each, out of shared memory, and keep the largest in a sorted list in
//                registers (a maximum and a minimum for each place); three exchanges between lanes merge the eight lists.  A key's low bits are the
//                inverted expert, so that one comparison orders equal logits too: below the 16 bits of a 16-bit logit, in the last 5 to 9 bits of
//                all other keys, whose k + 1 places are put in order by the whole keys afterwards.  (Whole keys in 64 bits: 36 us against
//                27 on 5000 tokens of 256 experts, the rest alike.)  Where what the low bits hid could change the choice, the token is chosen again.
// With a selection bias the keys are FP32 scores plus bias.  Where two neighbours of the k + 1 largest are nearer than FP32 can tell apart, the
// token is chosen again from FP64 keys: of the experts that are near enough to matter, one a lane, or (more than 32 of them, a softmax) of all.
//
// Order: a bit per (expert, token) in shared memory.  The rank of a pair within its expert is the number of bits before its own, whatever
// the order in which warps set them, so that the result does not depend on timing and no global atomics are needed.  Few tokens: one
// CTA does everything.  More: each CTA of a first kernel counts its own tokens' experts, and each CTA of a second one adds up the
// counts of those before it (and of all, for the experts' first rows) and places its pairs.  Where there are more CTAs than SMs (each has the most
// tokens that it can have then), a kernel between the two adds the counts up, one CTA for each expert: for every CTA to add up all of them
// would grow with the square of the tokens (8 experts, top 1: 24.5 ms instead of 8.6 for 2^25 tokens, a minute for 2^31).
//
// The bytes are few (2 to 4 per logit); what bounds it is the instructions of the choice and the latency of two launches: 16383 tokens of 128 experts, top 8,
// 15 us with BF16 logits (18.5 with a warp a token) and 24 with FP32 ones, 5000 tokens of 256 experts with sigmoid and bias 22.4 (29.6); 16 tokens of 64
// experts 4.2 in a graph.
#include "common.cuh"
#include "ptx.cuh"
#include <cuda_fp16.h>
#include <cuda_bf16.h>
#include <type_traits>

namespace hero {

constexpr int ROUTE_MAX_E = 512, ROUTE_MAX_K = 16;
constexpr int ROUTE_THREADS = 1024;
constexpr int ROUTE_ONE_CTA = 96;        // tokens that one CTA takes alone
constexpr int ROUTE_LANES = 8, ROUTE_TOKENS = 32 / ROUTE_LANES;   // lanes of a token, tokens of a warp (many tokens)
constexpr uint32_t ROUTE_TEAM = (1u << ROUTE_LANES) - 1u;
constexpr int ROUTE_KEY_BYTES = 192 * 1024;   // shared memory for keys
constexpr int ROUTE_MAX_CHUNK = 1024;    // tokens per CTA of the two-kernel form (bit words: E * chunk / 32)

struct RouteParams {
  const void* logits; long long ld;
  const int* n_tokens;
  const float* bias;
  int T, E, k, score, renorm;
  float scale;
  int* expert; float* weight; int* offset; int* token; int* row;
  int* counts;                           // [CTAs][E] (two-kernel form); summed: of the CTAs before, and [E] of all behind them
  int summed;
  int chunk, words;                      // tokens per CTA, their 32-bit words
  uint32_t low;                          // bits of a key that hold the expert (more tokens, FP32 keys)
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

// Weights of a token by one warp: lane j < k has place j's expert and logit; m, sum: of the softmax over all experts, where it is needed.
__device__ __forceinline__ void route_weights(const RouteParams& p, int t, int lane, int mine, float mine_x, float m, float sum) {
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
    route_weights(p, t, lane, mine, mine_x, m, sum);
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
__device__ __forceinline__ float from_order32(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? (k & 0x7fffffffu) : ~k); }
// list (falling) takes v in, at place `from` or behind
template <int KM>
__device__ __forceinline__ void insert(uint32_t (&list)[KM], uint32_t v, int from) {
#pragma unroll
  for (int i = 0; i < KM; ++i) {
    if (i < from) continue;                                // (from is a constant wherever this is unrolled)
    const uint32_t m = max(list[i], v);
    v = min(list[i], v);
    list[i] = m;
  }
}
// How near two FP32 keys with a bias may be and still have their order.  Sigmoid: a score at most 1 with an exponential within 2 + 1.2 |x| units (which
// score (1 - score) multiplies) and a quotient within 2, half a unit of the sum: below 5e-7 (1 + |v|) each.  Softmax: a sum of up to 512 on top.
__device__ __forceinline__ float key_error(const RouteParams& p, float v) { return (p.score == HERO_SCORE_SOFTMAX ? 4e-6f : 1e-6f) * (1.f + fabsf(v)); }

// A token without a bias or with sigmoid scores, by one warp: from FP64 keys of the experts whose FP32 keys (row, shared memory) are not clearly below `least`,
// which the k largest are not below.  list: shared int[64] of the warp.  False: there are more than 32 of them, nothing is written.
template <int DT>
__device__ __noinline__ bool route_near(const RouteParams& p, int t, const uint32_t* row, float least, float2 st, int* list, int lane, int& mine) {
  const uint32_t border = order32(p.bias ? least - 4.f * key_error(p, least) : least);
  int n = 0;
  for (int e0 = 0; e0 < p.E; e0 += 32) {
    const int e = e0 + lane;
    const bool in = e < p.E && row[e] != 0u && row[e] >= border;
    const uint32_t some = __ballot_sync(0xffffffffu, in);
    const int at = n + __popc(some & ((1u << lane) - 1u));
    if (in && at < 32) list[at] = e;
    n += __popc(some);
  }
  __syncwarp();
  if (n > 32) return false;
  const int e = lane < n ? list[lane] : -1;
  const float x = e >= 0 ? load_logit<DT>(p.logits, (long long)t * p.ld + e) : -INFINITY;
  const double key = e < 0 ? 0.0 : p.bias ? 1.0 / (1.0 + exp(-(double)x)) + (double)p.bias[e] : (double)x;
  int rank = 0;
  for (int c = 0; c < n; ++c) {                            // (experts rise with the lane: of equal keys the lower one is first)
    const double other = __shfl_sync(0xffffffffu, key, c);
    rank += other > key || (other == key && c < lane) ? 1 : 0;
  }
  if (e >= 0) list[32 + rank] = lane;
  __syncwarp();
  const int from = lane < n ? list[32 + lane] : 0;
  const int place = __shfl_sync(0xffffffffu, e, from);
  const float place_x = __shfl_sync(0xffffffffu, x, from);
  mine = lane < n && lane < p.k ? place : -1;
  route_weights(p, t, lane, mine, mine >= 0 ? place_x : -INFINITY, st.x, st.y);
  if (lane < p.k) p.expert[(long long)t * p.k + lane] = mine;
  __syncwarp();
  return true;
}
__device__ __forceinline__ int route_pitch(int E) { return (E + 31) / 32 * 32 + ROUTE_LANES; }    // (tokens on banks of their own)

// (keys in 32 bits that are put in order afterwards take more than 64 registers)
template <bool PACK16>
constexpr int ROUTE_CHOOSE_THREADS = PACK16 ? 1024 : 512;

// KM: places of a lane's list, at least k (PACK16: 16-bit logits without a bias) or k + 1
template <int KM, int DT, bool PACK16>
__global__ void __launch_bounds__(ROUTE_CHOOSE_THREADS<PACK16>, 1) route_choose_kernel(const __grid_constant__ RouteParams p) {
  extern __shared__ uint32_t keys_of[];                    // [warps][tokens][pitch]
  __shared__ int count[ROUTE_MAX_E];
  __shared__ float bias[PACK16 ? 1 : ROUTE_MAX_E];
  __shared__ int near_list[PACK16 ? 1 : ROUTE_CHOOSE_THREADS<PACK16> / 32][64];
  __shared__ float2 stats[ROUTE_CHOOSE_THREADS<PACK16> / 32][ROUTE_TOKENS];          // of a token's softmax over all experts: maximum, sum
  ptx::pdl_launch_dependents();
  for (int e = threadIdx.x; e < p.E; e += blockDim.x) count[e] = 0;
  ptx::pdl_wait();
  const int tokens = token_count(p), lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nw = blockDim.x >> 5;
  const int pitch = route_pitch(p.E), wide = pitch - ROUTE_LANES;
  uint32_t* keys = keys_of + warp * ROUTE_TOKENS * pitch;
  const bool softmax = p.score == HERO_SCORE_SOFTMAX, biased = !PACK16 && p.bias != nullptr, whole = softmax && (biased || !p.renorm);
  if (biased)
    for (int e = threadIdx.x; e < wide; e += blockDim.x) bias[e] = e < p.E ? p.bias[e] : -INFINITY;
  __syncthreads();
  const long long t0 = (long long)blockIdx.x * p.chunk;
  const int n = (int)min((long long)p.chunk, p.T - t0);
  for (int base = warp * ROUTE_TOKENS; base < n; base += nw * ROUTE_TOKENS) {
    // ---- keys of the warp's tokens, 16 loads at a time
    const int here = (int)min((long long)min(ROUTE_TOKENS, n - base), max(0ll, tokens - (t0 + base)));       // tokens among them
    {
      constexpr int AT_ONCE = 16;
      int i = 0, e0 = 0, ci = 0, c0 = 0;                   // token and first expert of the step that is loaded, that is converted
      const int steps = here * (wide >> 5);
      for (int s0 = 0; s0 < steps; s0 += AT_ONCE) {
        float x[AT_ONCE];
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {                // (indexes kept inside, so that no load waits for a condition)
          x[u] = load_logit<DT>(p.logits, (t0 + base + min(i, here - 1)) * p.ld + min(e0 + lane, p.E - 1));
          e0 += 32;
          if (e0 == wide) { e0 = 0; ++i; }
        }
        // (no branch between the steps: their chains overlap)
        auto convert = [&](auto sigmoid_key) {
#pragma unroll
          for (int u = 0; u < AT_ONCE; ++u) {
            const int e = c0 + lane;
            float v = x[u];
            if constexpr (!PACK16) {
              if (biased) {                                // (an expert whose bias is -inf or NaN does not take part at all)
                const float b = bias[e];
                if constexpr (decltype(sigmoid_key)::value) v = v > -INFINITY && b > -INFINITY ? __fdividef(1.f, 1.f + __expf(-v)) + b : -INFINITY;
                else v = b > -INFINITY ? v : -INFINITY;
              }
            }
            uint32_t k;
            if constexpr (PACK16) {
              uint32_t o;
              if constexpr (DT == HERO_BF16) o = order32(v) >> 16;
              else {
                const uint32_t h = v == 0.f ? 0u : (uint32_t)__half_as_ushort(__float2half_rn(v));
                o = !(v > -INFINITY) ? 0u : (h & 0x8000u) ? (~h & 0xffffu) : (h | 0x8000u);
              }
              k = o ? (o << 16) | (0xffffu - (uint32_t)e) : 0u;
            } else {
              k = order32(v);
            }
            if (s0 + u < steps) keys[ci * pitch + e] = e < p.E ? k : 0u;
            c0 += 32;
            if (c0 == wide) { c0 = 0; ++ci; }
          }
        };
        if (biased && !softmax) convert(std::true_type{});
        else convert(std::false_type{});
      }
    }
    if (whole) {
      for (int i = 0; i < here; ++i) {
        uint32_t* row = keys + i * pitch;
        const long long t = t0 + base + i;
        auto logit = [&](int e) {
          if constexpr (PACK16) return load_logit<DT>(p.logits, t * p.ld + e);
          else return row[e] ? from_order32(row[e]) : -INFINITY;
        };
        float m = -INFINITY;
        for (int e = lane; e < p.E; e += 32) m = fmaxf(m, logit(e));
        m = warp_max(m);
        float sum = 0.f;
        for (int e = lane; e < p.E; e += 32) sum += exp_below(logit(e), m);
        sum = warp_sum(sum);
        if (lane == 0) stats[warp][i] = make_float2(m, sum);
        if (biased)
          for (int e = lane; e < p.E; e += 32)
            if (row[e]) row[e] = order32(exp_below(from_order32(row[e]), m) / sum + bias[e]);
      }
    }
    __syncwarp();
    // ---- ROUTE_LANES lanes a token
    const int i = lane / ROUTE_LANES, q = lane % ROUTE_LANES, t = (int)(t0 + base) + i;
    const bool live = base + i < n, real = live && t < tokens;
    const uint32_t* row = keys + i * pitch;
    uint32_t list[KM];
#pragma unroll
    for (int j = 0; j < KM; ++j) list[j] = 0u;
    if (real) {
#pragma unroll 4
      for (int e = q; e < wide; e += ROUTE_LANES) {
        uint32_t v = row[e];
        if (!PACK16 && v) v = (v & ~p.low) | (p.low - (uint32_t)e);
        insert<KM>(list, v, 0);
      }
    }
#pragma unroll
    for (int o = 1; o < ROUTE_LANES; o <<= 1) {
      uint32_t other[KM];
#pragma unroll
      for (int j = 0; j < KM; ++j) other[j] = __shfl_xor_sync(0xffffffffu, list[j], o);
#pragma unroll
      for (int j = 0; j < KM; ++j) insert<KM>(list, other[j], j);      // (what is j-th there has j larger ones before it)
    }
    // ---- this lane's entries: q, q + ROUTE_LANES, ..: their places, experts (-1: none, or not among the k largest) and logits
    constexpr int MINE = (KM + ROUTE_LANES - 1) / ROUTE_LANES;
    int place[MINE], expert[MINE];
    float x[MINE];
    float top = -INFINITY;
    bool near = false;
    uint32_t whole_key[PACK16 ? 1 : KM];
    float least = -INFINITY;                               // the k largest are not below it
    if constexpr (!PACK16) {
      uint32_t kth = 0u, behind = 0u;                      // k-th and k + 1-th entry
#pragma unroll
      for (int j = 0; j < KM; ++j) {
        whole_key[j] = list[j] ? row[p.low - (list[j] & p.low)] : 0u;
        if (j == p.k - 1) kth = list[j];
        if (j == p.k) behind = list[j];
      }
      if (kth) least = from_order32(kth & ~p.low);
      // an expert outside the list may share the bits of the first that is not chosen
      if (behind) {
        const float u = from_order32(behind | p.low);
        near = ((kth ^ behind) & ~p.low) == 0u || (biased && (least - u < key_error(p, u) || !(least > u)));
      }
    }
#pragma unroll
    for (int a = 0; a < MINE; ++a) {
      uint32_t k = 0u, key = 0u;
#pragma unroll
      for (int b = 0; b < ROUTE_LANES; ++b) {
        const int j = ROUTE_LANES * a + b;
        if (j < KM && b == q) {
          k = list[j];
          if constexpr (!PACK16) key = whole_key[j];
        }
      }
      place[a] = ROUTE_LANES * a + q;
      expert[a] = -1;
      x[a] = -INFINITY;
      if (place[a] < KM && k) {
        if constexpr (PACK16) {
          if (place[a] < p.k) {
            expert[a] = (int)(0xffffu - (k & 0xffffu));
            const uint32_t o = k >> 16, b = (o & 0x8000u) ? (o & 0x7fffu) : (~o & 0xffffu);
            x[a] = DT == HERO_BF16 ? __uint_as_float(b << 16) : __half2float(__ushort_as_half((unsigned short)b));
          }
        } else {
          // its place among the k + 1 by the whole key; the largest key behind it
          const int e = (int)(p.low - (k & p.low));
          int rank = 0;
          uint32_t next = 0u;
#pragma unroll
          for (int c = 0; c < KM; ++c) {
            const int ec = (int)(p.low - (list[c] & p.low));
            const bool before = whole_key[c] > key || (whole_key[c] == key && ec < e && list[c] != 0u);
            if (c <= p.k) {
              rank += before ? 1 : 0;
              if (!before && ec != e) next = max(next, whole_key[c]);
            }
          }
          if (place[a] <= p.k && rank < p.k) {
            place[a] = rank;
            expert[a] = e;
            const float v = from_order32(key);
            x[a] = biased ? load_logit<DT>(p.logits, (long long)t * p.ld + e) : v;
            if (biased && next) {
              const float u = from_order32(next);
              near = near || v - u < key_error(p, u) || v == u;
            }
          }
        }
      }
    }
    const uint32_t slow = PACK16 ? 0u : __ballot_sync(0xffffffffu, near);
    const bool given = (slow >> (ROUTE_LANES * i) & ROUTE_TEAM) != 0u;       // this token is chosen again
    // ---- weights
    float w[MINE], all = 0.f;
#pragma unroll
    for (int a = 0; a < MINE; ++a) top = fmaxf(top, softmax ? x[a] : expert[a] >= 0 ? fminf(x[a], 0.f) : -INFINITY);
#pragma unroll
    for (int o = 1; o < ROUTE_LANES; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const float2 st = whole ? stats[warp][i] : make_float2(0.f, 1.f);
#pragma unroll
    for (int a = 0; a < MINE; ++a) {
      w[a] = 0.f;
      if (expert[a] >= 0) {
        if (p.renorm) {
          // softmax: the factor of all experts cancels.  sigmoid(x) = e^min(x, 0) / (1 + e^-|x|), the first factor relative to its largest
          if (softmax) w[a] = exp_below(x[a], top);
          else w[a] = exp_below(fminf(x[a], 0.f), top) / (1.f + expf(-fabsf(x[a])));
        } else {
          w[a] = softmax ? exp_below(x[a], st.x) / st.y : 1.f / (1.f + expf(-x[a]));
        }
      }
      all += w[a];
    }
#pragma unroll
    for (int o = 1; o < ROUTE_LANES; o <<= 1) all += __shfl_xor_sync(0xffffffffu, all, o);
    // (an empty place is one from the number of experts found on: the list is full up to there)
    int found = 0;
#pragma unroll
    for (int j = 0; j < KM; ++j) found += j < p.k && list[j] ? 1 : 0;
    if (live && !given) {
#pragma unroll
      for (int a = 0; a < MINE; ++a) {
        if (expert[a] >= 0) {
          p.expert[(long long)t * p.k + place[a]] = expert[a];
          p.weight[(long long)t * p.k + place[a]] = (p.renorm ? w[a] / all : w[a]) * p.scale;
          atomicAdd(&count[expert[a]], 1);                 // (shared memory, whole numbers: any order gives the same)
        }
        const int j = ROUTE_LANES * a + q;
        if (j >= found && j < p.k) {
          p.expert[(long long)t * p.k + j] = -1;
          p.weight[(long long)t * p.k + j] = 0.f;
        }
      }
    }
    if constexpr (!PACK16) {
      if (slow) {
        for (int s = 0; s < ROUTE_TOKENS; ++s) {
          if (!(slow >> (ROUTE_LANES * s) & ROUTE_TEAM)) continue;
          const float border = __shfl_sync(0xffffffffu, least, ROUTE_LANES * s);
          int e = -1;
          if ((softmax && biased) || !route_near<DT>(p, (int)(t0 + base) + s, keys + s * pitch, border, whole ? stats[warp][s] : make_float2(0.f, 1.f), near_list[warp], lane, e))
            e = route_token<16, DT>(p, (int)(t0 + base) + s, tokens, lane);
          if (e >= 0) atomicAdd(&count[e], 1);
        }
      }
    }
    __syncwarp();                                          // the keys are read
  }
  __syncthreads();
  for (int e = threadIdx.x; e < p.E; e += blockDim.x) p.counts[(long long)blockIdx.x * p.E + e] = count[e];
}

// More CTAs than SMs, between the two kernels: CTA e turns the counts of expert e into sums over the CTAs before, and puts that of all behind them.
__global__ void __launch_bounds__(ROUTE_THREADS, 1) route_sum_kernel(const __grid_constant__ RouteParams p, int ctas) {
  __shared__ int warps[32];
  ptx::pdl_launch_dependents();
  ptx::pdl_wait();
  int run = 0;
  for (int c0 = 0; c0 < ctas; c0 += ROUTE_THREADS) {
    const int c = c0 + threadIdx.x;
    int* at = p.counts + (long long)c * p.E + blockIdx.x;
    const int v = c < ctas ? *at : 0, before = exclusive_sum(v, warps);
    if (c < ctas) *at = run + before;
    for (int w = 0; w < ROUTE_THREADS / 32; ++w) run += warps[w];
    __syncthreads();                                       // the sums of the warps are read
  }
  if (threadIdx.x == 0) p.counts[(long long)ctas * p.E + blockIdx.x] = run;
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
  if (p.summed) {
    for (int e = threadIdx.x; e < p.E; e += blockDim.x) {
      before[e] = p.counts[(long long)blockIdx.x * p.E + e];
      total[e] = p.counts[(long long)gridDim.x * p.E + e];
    }
  } else {
    // counts of all chunks: as many threads of an expert as fit, each a share of the chunks
    int pe = 32;
    while (pe < p.E) pe <<= 1;
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
  // as many chunks as SMs, of whole warps' eights
  long long c = ((T + h->sm_count - 1) / h->sm_count + 7) / 8 * 8;
  return (int)(c > ROUTE_MAX_CHUNK ? ROUTE_MAX_CHUNK : c);
}
static long long route_ctas(long long T, int chunk) { return (T + chunk - 1) / chunk; }    // (in 64 bits: T may be 2^31 - 1)

template <int R, int DT>
static hero_status launch_one(hero_handle* h, RouteParams& p, cudaStream_t s) {
  p.words = (p.T + 31) / 32;
  const int warps = p.T < 32 ? p.T : 32;
  LaunchScope scope(h, s, KERNEL_ROUTE);
  HERO_CUDA(launch_dependent(route_one_kernel<R, DT>, dim3(1), dim3(32 * warps), (size_t)p.E * p.words * 4, s, p));
  return HERO_OK;
}
template <int KM, int DT, bool PACK16>
static hero_status launch_two(hero_handle* h, RouteParams& p, cudaStream_t s) {
  const unsigned ctas = (unsigned)route_ctas(p.T, p.chunk);
  p.summed = ctas > (unsigned)h->sm_count;
  // a warp for every four tokens of the chunk, as many as the shared memory holds the keys of
  const size_t warp_bytes = ROUTE_TOKENS * (size_t)((p.E + 31) / 32 * 32 + ROUTE_LANES) * 4;
  int warps = (p.chunk + ROUTE_TOKENS - 1) / ROUTE_TOKENS;
  if (warps > ROUTE_CHOOSE_THREADS<PACK16> / 32) warps = ROUTE_CHOOSE_THREADS<PACK16> / 32;
  if (warps > (int)(ROUTE_KEY_BYTES / warp_bytes)) warps = (int)(ROUTE_KEY_BYTES / warp_bytes);
  auto choose = route_choose_kernel<KM, DT, PACK16>;
  HERO_SMEM_OPT_IN(h, choose, ROUTE_KEY_BYTES);
  {
    LaunchScope scope(h, s, KERNEL_ROUTE);
    HERO_CUDA(launch_dependent(choose, dim3(ctas), dim3(32 * warps), warps * warp_bytes, s, p));
  }
  if (p.summed) {
    LaunchScope scope(h, s, KERNEL_ROUTE);
    HERO_CUDA(launch_dependent(route_sum_kernel, dim3((unsigned)p.E), dim3(ROUTE_THREADS), 0, s, p, (int)ctas));
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
  if (p.T <= ROUTE_ONE_CTA) {
    if (p.E <= 32) return launch_one<1, DT>(h, p, s);
    if (p.E <= 64) return launch_one<2, DT>(h, p, s);
    if (p.E <= 128) return launch_one<4, DT>(h, p, s);
    if (p.E <= 256) return launch_one<8, DT>(h, p, s);
    return launch_one<16, DT>(h, p, s);
  }
  if constexpr (DT != HERO_F32) {
    if (p.bias == nullptr) {
      if (p.k <= 2) return launch_two<2, DT, true>(h, p, s);
      if (p.k <= 4) return launch_two<4, DT, true>(h, p, s);
      if (p.k <= 8) return launch_two<8, DT, true>(h, p, s);
      return launch_two<16, DT, true>(h, p, s);
    }
  }
  p.low = 31u;
  while (p.low < (uint32_t)p.E - 1) p.low = 2 * p.low + 1;
  const int places = p.k + 1;
  if (places <= 4) return launch_two<4, DT, false>(h, p, s);
  if (places <= 9) return launch_two<9, DT, false>(h, p, s);
  return launch_two<17, DT, false>(h, p, s);
}

static hero_status route_sizes(int64_t T, int32_t E, int32_t k) {
  HERO_REQUIRE(E >= 1 && E <= ROUTE_MAX_E, HERO_ERR_UNSUPPORTED, "n_experts=%d: 1 to %d", E, ROUTE_MAX_E);
  HERO_REQUIRE(k >= 1 && k <= ROUTE_MAX_K && k <= E, HERO_ERR_UNSUPPORTED, "top_k=%d: 1 to %d and at most n_experts=%d", k, ROUTE_MAX_K, E);
  HERO_REQUIRE(T >= 0 && T < (1ll << 31) / k, HERO_ERR_UNSUPPORTED, "tokens=%lld with top_k=%d: below 2^31 pairs", (long long)T, k);
  return HERO_OK;
}
static size_t route_workspace(const hero_handle* h, int64_t T, int32_t E) {
  // the most chunks that any smaller number of tokens takes: one per SM, or T / ROUTE_MAX_CHUNK and a place for the sums of all
  const int64_t ctas = route_ctas(T, ROUTE_MAX_CHUNK) + 1;
  const int64_t few = (T + 7) / 8 < h->sm_count ? (T + 7) / 8 : h->sm_count;
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
  p.words = (p.chunk + 31) / 32;
  return x.dtype == HERO_F32 ? route_for<HERO_F32>(h, p, s) : x.dtype == HERO_F16 ? route_for<HERO_F16>(h, p, s) : route_for<HERO_BF16>(h, p, s);
}
