// The 8-bit block cache: argument checks, quantised append, read-back.
//
// Append.  A page and head has one scale, so its new tokens have to be seen whole before the first code is formed: one CTA
// takes one (page, head, key | value), keeps the page's new tokens in registers between the maximum and the codes, and reads
// and writes each element once (2 bytes in, 1 out).  DH / 8 lanes hold a token, 16 bytes each.  The maximum is taken over the
// 16-bit patterns without their sign, two per instruction: for finite values that is the order of the magnitudes, and a
// maximum at or above the pattern of infinity says that the page holds a non-finite value and takes a slower path.
#include "block_cache.cuh"
#include <climits>

namespace hero {

hero_status block_view(hero_handle* h, const hero_block_cache* c, const int32_t* row_start, int64_t rows, int32_t max_rows, BlockView* out) {
  HERO_REQUIRE(h && c, HERO_ERR_INVALID_ARG, "block cache: NULL handle or cache");
  HERO_REQUIRE(c->B >= 0 && c->B <= 65535, HERO_ERR_UNSUPPORTED, "block cache: B=%d: 0 .. 65535", c->B);
  HERO_REQUIRE(c->dtype == HERO_I8 || c->dtype == HERO_F8, HERO_ERR_UNSUPPORTED, "block cache: dtype %d: I8 or F8", c->dtype);
  HERO_REQUIRE(c->page == 16 || c->page == 32 || c->page == 64 || c->page == 128, HERO_ERR_UNSUPPORTED, "block cache: page=%d: 16, 32, 64 or 128", c->page);
  HERO_REQUIRE(c->dh == 64 || c->dh == 128, HERO_ERR_UNSUPPORTED, "block cache: dh=%d: 64 or 128", c->dh);
  HERO_REQUIRE(c->nkv >= 1 && c->nkv <= 16384, HERO_ERR_UNSUPPORTED, "block cache: nkv=%d: 1 .. 16384", c->nkv);
  HERO_REQUIRE(c->max_len >= 1 && c->max_len <= (1 << 30), HERO_ERR_UNSUPPORTED, "block cache: max_len=%d: 1 .. 2^30", c->max_len);
  HERO_REQUIRE(c->n_pages >= 1 && c->n_pages <= INT_MAX, HERO_ERR_INVALID_ARG, "block cache: n_pages=%lld", (long long)c->n_pages);
  HERO_REQUIRE(c->ld_table >= ((long long)c->max_len + c->page - 1) / c->page, HERO_ERR_INVALID_ARG,
               "block cache: a table row of %lld pages of %d tokens is shorter than max_len=%d", (long long)c->ld_table, c->page, c->max_len);
  HERO_REQUIRE(c->k && c->v && c->k_scale && c->v_scale && ((c->table && c->len) || c->B == 0), HERO_ERR_INVALID_ARG,
               "block cache: k, v, k_scale, v_scale, table and len are required");
  HERO_REQUIRE(aligned16(c->k) && aligned16(c->v) && c->ld % 16 == 0 && c->head_stride % 16 == 0 && c->page_stride % 16 == 0,
               HERO_ERR_ALIGNMENT, "block cache: k, v and their strides must be multiples of 16 bytes");
  HERO_REQUIRE(c->ld >= c->dh && c->head_stride >= c->dh && c->page_stride >= c->dh, HERO_ERR_INVALID_ARG,
               "block cache: strides must be at least dh=%d", c->dh);
  HERO_REQUIRE(rows >= 0 && max_rows >= 1, HERO_ERR_INVALID_ARG, "block cache: rows=%lld max_rows=%d", (long long)rows, max_rows);
  HERO_REQUIRE(row_start != nullptr || (rows >= c->B && max_rows == 1), HERO_ERR_INVALID_ARG,
               "block cache: without row_start every sequence has one row: rows >= B and max_rows = 1");
  out->k = static_cast<uint8_t*>(c->k); out->v = static_cast<uint8_t*>(c->v);
  out->ks = c->k_scale; out->vs = c->v_scale;
  out->f8 = c->dtype == HERO_F8;
  out->page = c->page;
  out->page_shift = c->page == 16 ? 4 : c->page == 32 ? 5 : c->page == 64 ? 6 : 7;
  out->n_pages = (int)c->n_pages;
  out->page_stride = c->page_stride; out->head_stride = c->head_stride; out->ld = c->ld;
  out->table = c->table; out->ld_table = c->ld_table; out->len = c->len;
  out->max_len = c->max_len; out->nkv = c->nkv;
  // a sequence has at most max_len tokens, but a call's rows may reach behind its first one
  out->row_start = row_start; out->rows = rows; out->max_rows = max_rows;
  out->err = h->d_error;
  return HERO_OK;
}

constexpr int APP_THREADS = 128;

struct AppendParams {
  BlockView c;
  const uint16_t* k; long long ld_k;
  const uint16_t* v; long long ld_v;
};

// NP: passes of the CTA over a page (page * DH / 8 lanes over 128 threads), all held in registers
template <int DH, int NP, bool BF, bool F8>
__global__ void __launch_bounds__(APP_THREADS) block_append_kernel(const __grid_constant__ AppendParams p) {
  constexpr int LPT = DH / 8;                    // lanes per token
  constexpr int TPP = APP_THREADS / LPT;         // tokens per pass
  constexpr uint32_t INF2 = BF ? 0x7f80u : 0x7c00u;
  constexpr float TOP = F8 ? 448.0f : 127.0f;
  __shared__ float red[APP_THREADS / 32];
  ptx::pdl_launch_dependents();
  ptx::pdl_wait();
  const BlockView& c = p.c;
  const int b = blockIdx.z, head = blockIdx.y >> 1, is_v = blockIdx.y & 1;
  const SeqRows s = seq_rows(c, b);
  const int begin = s.len - s.n, first = max(begin, 0);      // first new token (rows before token 0 store nothing)
  const int pi = (first >> c.page_shift) + blockIdx.x, p0 = pi << c.page_shift;
  if (s.n <= 0 || p0 >= s.len) return;
  const int id = written(c.table + (long long)b * c.ld_table + pi);
  const int lo = max(first - p0, 0), hi = min(s.len - p0, c.page);   // the page's slots that receive new tokens
  const long long ld_x = is_v ? p.ld_v : p.ld_k;
  const uint16_t* src = (is_v ? p.v : p.k) + (s.r0 + (p0 - begin)) * ld_x + (long long)head * DH;   // row of slot 0
  const int sub = threadIdx.x % LPT, tg = threadIdx.x / LPT;

  // the rows are requested before the page's number has arrived
  uint4 raw[NP];
  uint32_t top2 = 0;
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int t = i * TPP + tg;
    raw[i] = make_uint4(0, 0, 0, 0);
    if (t >= lo && t < hi) raw[i] = written(reinterpret_cast<const uint4*>(src + (long long)t * ld_x + sub * 8));
  }
  if ((unsigned)id >= (unsigned)c.n_pages) {
    if (threadIdx.x == 0) atomicExch(c.err, ERR_BAD_PAGE);
    return;
  }
  uint8_t* dst = (is_v ? c.v : c.k) + (long long)id * c.page_stride + (long long)head * c.head_stride;
  float* scale = (is_v ? c.vs : c.ks) + (long long)id * c.nkv + head;
  const float s_old = lo > 0 ? *scale : 0.f;
#pragma unroll
  for (int i = 0; i < NP; ++i)
    top2 = __vmaxu2(top2, __vmaxu2(__vmaxu2(raw[i].x & 0x7fff7fffu, raw[i].y & 0x7fff7fffu), __vmaxu2(raw[i].z & 0x7fff7fffu, raw[i].w & 0x7fff7fffu)));
  uint32_t bits = max(top2 & 0xffffu, top2 >> 16);
  const bool odd = __syncthreads_or(bits >= INF2);           // a NaN or an infinity somewhere in the page's new tokens
  float amax;
  if (!odd) {
    const float2 f = fp16ish_to_f32x2<BF>(bits);
    amax = f.x;
  } else {
    amax = 0.f;
    const uint32_t* w = reinterpret_cast<const uint32_t*>(raw);
#pragma unroll
    for (int i = 0; i < 4 * NP; ++i) {
      // the largest finite magnitude
      const float2 f = fp16ish_to_f32x2<BF>(w[i]);
      if ((w[i] & 0x7fffu) < INF2) amax = fmaxf(amax, fabsf(f.x));
      if ((w[i] >> 16 & 0x7fffu) < INF2) amax = fmaxf(amax, fabsf(f.y));
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = amax;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < APP_THREADS / 32; ++w) amax = fmaxf(amax, red[w]);
  const float s_new = fmaxf(s_old, amax / TOP);

  Divider div(s_new);
  if (odd) div.fast = false;                                 // (an infinity has no remainder)
  if (div.fast) {
    // no new value exceeds top * s_new, so the codes need no clamping
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int t = i * TPP + tg;
      if (t >= lo && t < hi) {
        uint2 code;
        code.x = f32_to_codes4_inside<F8>(div.pair(fp16ish_to_f32x2<BF>(raw[i].x)), div.pair(fp16ish_to_f32x2<BF>(raw[i].y)));
        code.y = f32_to_codes4_inside<F8>(div.pair(fp16ish_to_f32x2<BF>(raw[i].z)), div.pair(fp16ish_to_f32x2<BF>(raw[i].w)));
        *reinterpret_cast<uint2*>(dst + (long long)t * c.ld + sub * 8) = code;
      }
    }
  } else {
#pragma unroll 1
    for (int i = 0; i < NP; ++i) {
      const int t = i * TPP + tg;
      if (t >= lo && t < hi) {
        // (reads the row again: indexing the registers here would put them all into memory)
        const uint4 x = written(reinterpret_cast<const uint4*>(src + (long long)t * ld_x + sub * 8));
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
        float y[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 f = fp16ish_to_f32x2<BF>(w[e]);
          y[2 * e] = isnan(f.x) ? 0.f : div(f.x);
          y[2 * e + 1] = isnan(f.y) ? 0.f : div(f.y);
        }
        uint2 code;
        code.x = f32_to_codes4<F8>(y[0], y[1], y[2], y[3]);
        code.y = f32_to_codes4<F8>(y[4], y[5], y[6], y[7]);
        *reinterpret_cast<uint2*>(dst + (long long)t * c.ld + sub * 8) = code;
      }
    }
  }
  if (lo > 0 && s_new > s_old) {
    // the scale grew: the page's earlier tokens are quantised again (their codes stay clear of the new tokens' slots)
    for (int t = tg; t < lo; t += TPP) {
      uint2* at = reinterpret_cast<uint2*>(dst + (long long)t * c.ld + sub * 8);
      const uint2 old = *at;
      float x[4], y[4];
      codes4_to_f32<F8>(old.x, x);
      codes4_to_f32<F8>(old.y, y);
      uint2 code;
      code.x = f32_to_codes4<F8>(div(x[0] * s_old), div(x[1] * s_old), div(x[2] * s_old), div(x[3] * s_old));
      code.y = f32_to_codes4<F8>(div(y[0] * s_old), div(y[1] * s_old), div(y[2] * s_old), div(y[3] * s_old));
      *at = code;
    }
  }
  if (threadIdx.x == 0 && (lo == 0 || s_new > s_old)) *scale = s_new;
}

// ---- read-back.  One thread turns 16 codes into 16 values of READ_TOKENS tokens, all of them in flight.  The 32 bytes it writes
// leave in one store where the rows allow it (WIDE: 32-byte aligned); two stores of 16 bytes each are half a sector.
constexpr int READ_THREADS = 256, READ_TOKENS = 4;

struct ReadParams {
  BlockView c;
  uint16_t* k; long long ld_k;
  uint16_t* v; long long ld_v;
  int ppt;                      // 16-code pieces per token: nkv * DH / 16
  int tpp;                      // tokens per pass of the CTA
  int first_v;                  // grid y 0 is the values (no keys wanted)
};

template <int DH, bool BF, bool F8, bool WIDE>
__global__ void __launch_bounds__(READ_THREADS, 4) block_read_kernel(const __grid_constant__ ReadParams p) {
  constexpr int PPH = DH / 16;                   // pieces per head
  ptx::pdl_launch_dependents();
  ptx::pdl_wait();
  const BlockView& c = p.c;
  const int b = blockIdx.z, is_v = blockIdx.y + p.first_v;
  const SeqRows s = seq_rows(c, b);
  const int i0 = blockIdx.x * p.tpp * READ_TOKENS;
  if (i0 >= s.n) return;
  const uint8_t* pool = is_v ? c.v : c.k;
  const float* scales = is_v ? c.vs : c.ks;
  uint16_t* out = is_v ? p.v : p.k;
  const long long ld = is_v ? p.ld_v : p.ld_k;
  const int* table = c.table + (long long)b * c.ld_table;
  const int tok = p.tpp > 1 ? threadIdx.x / p.ppt : 0;
  if (tok >= p.tpp) return;
  for (int piece = threadIdx.x - tok * p.ppt; piece < p.ppt; piece += READ_THREADS) {     // (one pass where a token fits the CTA)
    const int head = piece / PPH;
    const uint8_t* from = pool + (long long)head * c.head_stride + (piece % PPH) * 16;
    uint4 code[READ_TOKENS];
    float sc[READ_TOKENS];
    // (no branch between the look-ups and the loads: the pages of all tokens are fetched together, then all codes)
    int id[READ_TOKENS];
    bool bad = false;
#pragma unroll
    for (int j = 0; j < READ_TOKENS; ++j) {
      const int i = i0 + tok + j * p.tpp, t = s.len - s.n + i;             // row of the sequence, its token
      const int pi = min(max(t, 0), c.max_len - 1) >> c.page_shift;
      const int n = written(table + pi);
      id[j] = min(max(n, 0), c.n_pages - 1);
      bad |= id[j] != n && i < s.n && t >= 0;
    }
#pragma unroll
    for (int j = 0; j < READ_TOKENS; ++j) {
      const int i = i0 + tok + j * p.tpp, t = s.len - s.n + i;
      code[j] = written(reinterpret_cast<const uint4*>(from + (long long)id[j] * c.page_stride + (long long)(t & (c.page - 1)) * c.ld));
      sc[j] = written(scales + (long long)id[j] * c.nkv + head);
      if (i >= s.n || t < 0) { code[j] = make_uint4(0, 0, 0, 0); sc[j] = 0.f; }  // a row without a token
    }
    if (bad) atomicExch(c.err, ERR_BAD_PAGE);
#pragma unroll
    for (int j = 0; j < READ_TOKENS; ++j) {
      const int i = i0 + tok + j * p.tpp;
      if (i >= s.n) break;
      const uint32_t w[4] = {code[j].x, code[j].y, code[j].z, code[j].w};
      uint32_t o[8];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float y[4];
        codes4_to_f32<F8>(w[q], y);
        o[2 * q] = f32x2_to_fp16ish<BF>(y[0] * sc[j], y[1] * sc[j]);
        o[2 * q + 1] = f32x2_to_fp16ish<BF>(y[2] * sc[j], y[3] * sc[j]);
      }
      uint16_t* at = out + (s.r0 + i) * ld + piece * 16;
      if constexpr (WIDE) {
        asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(at), "r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3]), "r"(o[4]), "r"(o[5]),
                     "r"(o[6]), "r"(o[7]) : "memory");
      } else {
        reinterpret_cast<uint4*>(at)[0] = make_uint4(o[0], o[1], o[2], o[3]);
        reinterpret_cast<uint4*>(at)[1] = make_uint4(o[4], o[5], o[6], o[7]);
      }
    }
  }
}

static hero_status check_rows_matrix(const hero_tensor& t, const char* name, const hero_block_cache* c) {
  hero_status st = check_matrix(t, name);
  if (st != HERO_OK) return st;
  HERO_REQUIRE(is_fp16ish(t.dtype), HERO_ERR_UNSUPPORTED, "%s: dtype %d: F16 or BF16", name, t.dtype);
  HERO_REQUIRE(t.cols == (int64_t)c->nkv * c->dh, HERO_ERR_INVALID_ARG, "%s: %lld columns, nkv*dh = %lld", name, (long long)t.cols,
               (long long)c->nkv * c->dh);
  return HERO_OK;
}

typedef void (*read_fn)(const ReadParams);
template <int DH>
static read_fn read_kernel(bool bf, bool f8, bool wide) {
  if (wide)
    return bf ? (f8 ? block_read_kernel<DH, true, true, true> : block_read_kernel<DH, true, false, true>)
              : (f8 ? block_read_kernel<DH, false, true, true> : block_read_kernel<DH, false, false, true>);
  return bf ? (f8 ? block_read_kernel<DH, true, true, false> : block_read_kernel<DH, true, false, false>)
            : (f8 ? block_read_kernel<DH, false, true, false> : block_read_kernel<DH, false, false, false>);
}

template <int DH, int NP>
static cudaError_t launch_append(const AppendParams& p, bool bf, dim3 grid, cudaStream_t s) {
  auto kern = bf ? (p.c.f8 ? block_append_kernel<DH, NP, true, true> : block_append_kernel<DH, NP, true, false>)
                 : (p.c.f8 ? block_append_kernel<DH, NP, false, true> : block_append_kernel<DH, NP, false, false>);
  return launch_dependent(kern, grid, dim3(APP_THREADS), 0, s, p);
}

}  // namespace hero

extern "C" hero_status hero_block_cache_append(hero_handle* h, const hero_block_cache* cc, const hero_block_rows_args* a, void* stream) {
  using namespace hero;
  HERO_REQUIRE(h && cc && a, HERO_ERR_INVALID_ARG, "hero_block_cache_append: NULL handle, cache or args");
  AppendParams p;
  hero_status st = block_view(h, cc, a->row_start, a->k.rows, a->max_rows, &p.c);
  if (st != HERO_OK) return st;
  if ((st = check_rows_matrix(a->k, "k", cc)) != HERO_OK || (st = check_rows_matrix(a->v, "v", cc)) != HERO_OK) return st;
  HERO_REQUIRE(a->k.rows == a->v.rows && a->k.dtype == a->v.dtype, HERO_ERR_INVALID_ARG, "k and v have the same rows and type");
  if (cc->B == 0 || a->k.rows == 0) return HERO_OK;
  if ((st = check_device(h)) != HERO_OK) return st;
  p.k = static_cast<const uint16_t*>(a->k.data); p.ld_k = a->k.ld;
  p.v = static_cast<const uint16_t*>(a->v.data); p.ld_v = a->v.ld;
  // a run of n tokens touches at most (n + page - 2) / page + 1 pages, and no more than the table has
  const long long n = a->max_rows < cc->max_len ? a->max_rows : cc->max_len;
  const long long pages = (n + cc->page - 2) / cc->page + 1;
  const dim3 grid((unsigned)pages, 2u * (unsigned)cc->nkv, (unsigned)cc->B);
  const bool bf = a->k.dtype == HERO_BF16;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  {
    LaunchScope scope(h, s, KERNEL_CACHE);
    const int np = cc->page * cc->dh / 8 / APP_THREADS;
    if (cc->dh == 64)
      e = np == 1 ? launch_append<64, 1>(p, bf, grid, s) : np == 2 ? launch_append<64, 2>(p, bf, grid, s)
        : np == 4 ? launch_append<64, 4>(p, bf, grid, s) : launch_append<64, 8>(p, bf, grid, s);
    else
      e = np == 2 ? launch_append<128, 2>(p, bf, grid, s) : np == 4 ? launch_append<128, 4>(p, bf, grid, s)
        : np == 8 ? launch_append<128, 8>(p, bf, grid, s) : launch_append<128, 16>(p, bf, grid, s);
  }
  HERO_CUDA(e);
  return HERO_OK;
}

extern "C" hero_status hero_block_cache_read(hero_handle* h, const hero_block_cache* cc, const hero_block_rows_args* a, void* stream) {
  using namespace hero;
  HERO_REQUIRE(h && cc && a, HERO_ERR_INVALID_ARG, "hero_block_cache_read: NULL handle, cache or args");
  const bool has_k = a->k.data != nullptr, has_v = a->v.data != nullptr;
  if (!has_k && !has_v) {
    HERO_REQUIRE(a->k.rows == 0 && a->v.rows == 0, HERO_ERR_INVALID_ARG, "hero_block_cache_read: neither k nor v is wanted");
    return HERO_OK;
  }
  const hero_tensor& one = has_k ? a->k : a->v;
  ReadParams p;
  hero_status st = block_view(h, cc, a->row_start, one.rows, a->max_rows, &p.c);
  if (st != HERO_OK) return st;
  if ((has_k && (st = check_rows_matrix(a->k, "k", cc)) != HERO_OK) || (has_v && (st = check_rows_matrix(a->v, "v", cc)) != HERO_OK)) return st;
  HERO_REQUIRE(!(has_k && has_v) || (a->k.rows == a->v.rows && a->k.dtype == a->v.dtype), HERO_ERR_INVALID_ARG, "k and v have the same rows and type");
  if (cc->B == 0 || one.rows == 0) return HERO_OK;
  if ((st = check_device(h)) != HERO_OK) return st;
  p.k = static_cast<uint16_t*>(a->k.data); p.ld_k = a->k.ld;
  p.v = static_cast<uint16_t*>(a->v.data); p.ld_v = a->v.ld;
  p.ppt = cc->nkv * cc->dh / 16;
  p.tpp = p.ppt < READ_THREADS ? READ_THREADS / p.ppt : 1;
  p.first_v = has_k ? 0 : 1;
  const int per_cta = p.tpp * READ_TOKENS;
  const dim3 grid((unsigned)((a->max_rows + (long long)per_cta - 1) / per_cta), has_k && has_v ? 2 : 1, (unsigned)cc->B);
  const bool bf = one.dtype == HERO_BF16;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  auto wide_rows = [](const hero_tensor& t) { return reinterpret_cast<uintptr_t>(t.data) % 32 == 0 && t.ld % 16 == 0; };
  const bool wide = (!has_k || wide_rows(a->k)) && (!has_v || wide_rows(a->v));
  auto kern = cc->dh == 64 ? read_kernel<64>(bf, p.c.f8, wide) : read_kernel<128>(bf, p.c.f8, wide);
  cudaError_t e;
  {
    LaunchScope scope(h, s, KERNEL_CACHE);
    e = launch_dependent(kern, grid, dim3(READ_THREADS), 0, s, p);
  }
  HERO_CUDA(e);
  return HERO_OK;
}
