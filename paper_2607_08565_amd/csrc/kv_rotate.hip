// Norms and rotation of queries and keys, alone or on the way into the paged cache.
//
// Mathematics: per token and head, y = x w / sqrt(mean(x^2) + eps), then the pairs of the
// first rot_dim components turned by the angles of the token's position (smetric_kv.h).
// Two operations per byte at most: the bound is memory, each activation read once and
// written once.
//
// Mapping to gfx950: a head is held by head_dim / 16 neighbouring lanes, each with two
// 8-component (16-byte) pieces that are paired so that a rotation never leaves its lane --
// pieces c and c + rot_dim / 16 for halves, 2c and 2c + 1 for neighbours -- and the mean
// square takes two to four lane exchanges.  Rows (token, head) are dealt to lanes in
// order, so a wavefront reads consecutive heads of one token in one run and the token's
// cosines and sines come from memory once and from the nearest cache for its other heads.
//
// Measured: 8,191 tokens of 40 heads of 128 32.1 us, 5.3 TB/s (a copy of 4 GiB moves 4.8); the
// keys, values and queries of 6,249 tokens appended 38.1 us, 4.1 TB/s (pages in any order, the
// queries kept in the caches for the attention); a token's append 4.4 us, its launch; of 256 5.3.
#include "common.h"
#include "kv_common.h"

namespace smk {
namespace {

constexpr int RT = 256;  // threads per workgroup

struct TurnArgs {
  const void *weight[2];  // queries, keys
  const float *table;
  int64_t n_pos;
  int32_t rot;
  float eps;
  const int32_t *positions;
  int32_t *status;
};
struct BatchArgs {
  const int64_t *q_off;
  const int32_t *kv_len;
  int32_t n_req;
};

// Request of token t: the last r with q_off[r] <= t.  64 lanes bisect together (two rounds
// of one load up to 4,096 requests instead of a chain of twelve) for the wavefront's first
// token; its other tokens are a few steps on.
__device__ __forceinline__ int32_t request_of(const int64_t *__restrict__ q_off, int32_t n_req, int64_t first, int64_t t,
                                              int lane) {
  int32_t lo = 0, hi = n_req;  // the answer is in [lo, hi), if anywhere
  while (hi - lo > 1) {
    const int32_t step = (hi - lo + 63) / 64;
    const int32_t at = lo + lane * step;
    const bool le = at < hi && q_off[at] <= first;
    const int n = __popcll(__ballot(le));
    if (n == 0) break;
    lo += (n - 1) * step;
    hi = lo + step < hi ? lo + step : hi;
  }
  while (lo + 1 < n_req && q_off[lo + 1] <= t) ++lo;
  return lo;
}

template <typename T>
__device__ __forceinline__ void widen(u32x4 v, float *x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = T::lo(v[i]);
    x[2 * i + 1] = T::hi(v[i]);
  }
}
template <typename T>
__device__ __forceinline__ u32x4 narrow(const float *x) {
  u32x4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = T::pack(x[2 * i], x[2 * i + 1]);
  return v;
}
__device__ __forceinline__ float saturate(float x) {  // NaN stays NaN
  return x != x ? x : __builtin_amdgcn_fmed3f(x, -E4M3_MAX, E4M3_MAX);
}
__device__ __forceinline__ u32x2 narrow_e4m3(const float *x, float scale) {
  u32x2 v;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(saturate(x[4 * i] / scale), saturate(x[4 * i + 1] / scale), 0, false);
    v[i] = __builtin_amdgcn_cvt_pk_fp8_f32(saturate(x[4 * i + 2] / scale), saturate(x[4 * i + 3] / scale), w, true);
  }
  return v;
}

// PAGED: k goes to the cache (places from the batch) and v exists; else k goes to k_out and
// positions are given.
template <typename T, int D, bool INTER, bool PAGED, bool KV8>
__global__ __launch_bounds__(RT) void turn_kernel(TurnArgs ta, BatchArgs ba, CacheView cache, HeadsView q, HeadsView q_out,
                                                  HeadsView k, HeadsView k_out, HeadsView v, int64_t n_tokens, int32_t n_q,
                                                  int32_t n_kv) {
  constexpr int LPR = D / 16;  // lanes per row
  const int32_t per_token = n_q + (PAGED ? 2 : 1) * n_kv;
  const int64_t row = (int64_t(blockIdx.x) * RT + threadIdx.x) / LPR;
  const int lane = threadIdx.x & 63, sub = threadIdx.x % LPR;
  const int64_t n_rows = n_tokens * per_token;
  // rows of one workgroup: at most RT / LPR, so 32 bits hold the distance from its first
  const int64_t t0 = (int64_t(blockIdx.x) * RT + (threadIdx.x & ~63)) / LPR / per_token;
  const bool live = row < n_rows;
  const int64_t t = live ? row / per_token : n_tokens - 1;
  const int32_t h = live ? int32_t(row - t * per_token) : 0;
  const int kind = h < n_q ? 0 : h < n_q + n_kv ? 1 : 2;
  const int32_t head = kind == 0 ? h : kind == 1 ? h - n_q : h - n_q - n_kv;

  // this lane's two pieces of 8 components
  const int half = ta.rot / 16;
  int c0 = sub, c1 = sub + LPR;
  if (!INTER) {
    c0 = sub < half ? sub : 2 * sub;
    c1 = sub < half ? sub + half : 2 * sub + 1;
  }
  // (which of the two turn: both or none for halves)
  const bool turns0 = c0 < (INTER ? 2 * half : half) && kind != 2;
  const bool turns1 = INTER ? c1 < 2 * half && kind != 2 : turns0;
  // asked for before the chain of loads that finds the place
  const HeadsView &src = kind == 0 ? q : kind == 1 ? k : v;
  const uint16_t *from = src.data + t * src.token + head * src.head;
  const u32x4 in0 = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(from + 8 * c0));
  const u32x4 in1 = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(from + 8 * c1));

  int32_t place = 0, pos = 0;
  int64_t page_row = 0;
  bool ok = live, bad = false;
  if (PAGED) {
    // In a decoding step token t is request t's: asked for at once; a search of the whole
    // wavefront where that is not so for one of its lanes.
    int32_t r = t < ba.n_req ? int32_t(t) : ba.n_req - 1;
    int64_t a = ba.q_off[r], z = ba.q_off[r + 1];
    int32_t len = ba.kv_len[r];
    if (__any(a > t || z <= t)) {
      r = request_of(ba.q_off, ba.n_req, t0 < n_tokens ? t0 : n_tokens - 1, t, lane);
      a = ba.q_off[r];
      z = ba.q_off[r + 1];
      len = ba.kv_len[r];
    }
    bad = t < a || t >= z || len < 0 || len > MAX_PLACES || int64_t(len) > int64_t(cache.max_pages) * cache.ps.size;
    const int64_t p = int64_t(len) - (z - t);
    ok = ok && !bad && p >= 0;
    place = ok ? int32_t(p) : 0;
    pos = place;
    if (ok) {
      const int32_t page = page_of(cache.ps, place);
      const int32_t id = cache.table[r * cache.table_stride + page];
      const bool fine = uint32_t(id) < uint32_t(cache.n_pages);
      bad = !fine;
      ok = fine;
      const PageSide &s = kind == 2 ? cache.v : cache.k;
      page_row = ok ? id * s.page + head * s.head + (place - page * cache.ps.size) * s.token : 0;
    }
  }
  if (ta.rot > 0) {
    if (ta.positions) pos = ta.positions[t];
    if (pos < 0 || pos >= ta.n_pos) {
      bad = bad || ok;
      ok = false;
    }
  }
  if (live && bad && sub == 0) set_status(ta.status, SMETRIC_EINVAL);

  float x[16];
  widen<T>(ok ? in0 : u32x4{0, 0, 0, 0}, x);
  widen<T>(ok ? in1 : u32x4{0, 0, 0, 0}, x + 8);
  const uint16_t *w = static_cast<const uint16_t *>(kind == 2 ? nullptr : ta.weight[kind]);
  // the exchange is outside the condition: rows with and without a weight share a wavefront
  float ss = 0.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i) ss = fmaf(x[i], x[i], ss);
#pragma unroll
  for (int m = 1; m < LPR; m *= 2) ss += __shfl_xor(ss, m, 64);
  if (w && ok) {  // (zeros stay zeros also where eps is 0)
    const float rstd = 1.0f / sqrtf(ss * (1.0f / D) + ta.eps);
    float g[16];
    widen<T>(*reinterpret_cast<const u32x4 *>(w + 8 * c0), g);
    widen<T>(*reinterpret_cast<const u32x4 *>(w + 8 * c1), g + 8);
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = x[i] * rstd * g[i];
  }
  if (ok && (turns0 || turns1)) {
    // angles: eight in a row for halves; four of each piece for neighbours
    const float *cs = ta.table + int64_t(pos) * ta.rot, *sn = cs + ta.rot / 2;
    const int a0 = INTER ? 4 * c0 : 8 * sub, a1 = INTER ? 4 * c1 : 8 * sub + 4;
    float co[8], si[8];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const bool on = i ? turns1 : turns0;
      const int at = i ? a1 : a0;
      const f32x4 a = on ? *reinterpret_cast<const f32x4 *>(cs + at) : f32x4{1, 1, 1, 1};
      const f32x4 b = on ? *reinterpret_cast<const f32x4 *>(sn + at) : f32x4{0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        co[4 * i + j] = a[j];
        si[4 * i + j] = b[j];
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (INTER && !(i < 4 ? turns0 : turns1)) continue;
      float &a = INTER ? x[2 * i] : x[i], &b = INTER ? x[2 * i + 1] : x[8 + i];
      const float ya = a, yb = b;
      a = ya * co[i] - yb * si[i];
      b = yb * co[i] + ya * si[i];
    }
  }
  if (!live) return;
  if (PAGED && kind != 0) {
    if (!ok) return;
    const PageSide &s = kind == 1 ? cache.k : cache.v;
    char *p = s.base + page_row;
    if (KV8) {
      const float *sc = kind == 1 ? cache.k_scale : cache.v_scale;
      const float scale = sc ? sc[head] : 1.0f;
      *reinterpret_cast<u32x2 *>(p + 8 * c0) = narrow_e4m3(x, scale);
      *reinterpret_cast<u32x2 *>(p + 8 * c1) = narrow_e4m3(x + 8, scale);
    } else {
      *reinterpret_cast<u32x4 *>(p + 16 * c0) = narrow<T>(x);
      *reinterpret_cast<u32x4 *>(p + 16 * c1) = narrow<T>(x + 8);
    }
  } else {
    const HeadsView &dst = kind == 0 ? q_out : k_out;
    uint16_t *p = dst.data + t * dst.token + head * dst.head;
    if (PAGED) {  // attention reads it next
      *reinterpret_cast<u32x4 *>(p + 8 * c0) = narrow<T>(x);
      *reinterpret_cast<u32x4 *>(p + 8 * c1) = narrow<T>(x + 8);
    } else {
      __builtin_nontemporal_store(narrow<T>(x), reinterpret_cast<u32x4 *>(p + 8 * c0));
      __builtin_nontemporal_store(narrow<T>(x + 8), reinterpret_cast<u32x4 *>(p + 8 * c1));
    }
  }
}

struct Launch {
  TurnArgs ta;
  BatchArgs ba;
  CacheView cache;
  HeadsView q, q_out, k, k_out, v;
  int64_t n_tokens;
  int32_t n_q, n_kv;
  bool inter, paged, kv8;
  hipStream_t stream;
};
template <typename T, int D, bool INTER, bool PAGED, bool KV8>
int launch(const Launch &a) {
  const int64_t rows = a.n_tokens * (a.n_q + int64_t(a.paged ? 2 : 1) * a.n_kv), wg = RT / (D / 16);
  const int64_t grid = (rows + wg - 1) / wg;
  if (grid > 0x7FFFFFFF) return SMETRIC_EINVAL;
  turn_kernel<T, D, INTER, PAGED, KV8><<<dim3(uint32_t(grid)), dim3(RT), 0, a.stream>>>(
      a.ta, a.ba, a.cache, a.q, a.q_out, a.k, a.k_out, a.v, a.n_tokens, a.n_q, a.n_kv);
  return hip_status(hipGetLastError());
}
template <typename T, int D>
int launch_td(const Launch &a) {
  if (!a.paged) return a.inter ? launch<T, D, true, false, false>(a) : launch<T, D, false, false, false>(a);
  if (a.kv8) return a.inter ? launch<T, D, true, true, true>(a) : launch<T, D, false, true, true>(a);
  return a.inter ? launch<T, D, true, true, false>(a) : launch<T, D, false, true, false>(a);
}
template <typename T>
int launch_t(const Launch &a, int32_t head_dim) {
  return head_dim == 64 ? launch_td<T, 64>(a) : head_dim == 128 ? launch_td<T, 128>(a) : launch_td<T, 256>(a);
}
int launch_any(const Launch &a, int32_t dtype, int32_t head_dim) {
  return dtype == SMETRIC_BF16 ? launch_t<Bf16>(a, head_dim) : launch_t<F16>(a, head_dim);
}

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
bool dims_ok(int32_t dtype, int32_t head_dim) {
  return (dtype == SMETRIC_BF16 || dtype == SMETRIC_F16) && (head_dim == 64 || head_dim == 128 || head_dim == 256);
}
bool rotary_ok(const smetric_rotary *r, int32_t head_dim) {
  if (r->rot_dim < 0 || r->rot_dim > head_dim || r->rot_dim % 16 || !(r->eps >= 0.0f)) return false;
  if (r->rot_dim > 0 && (!r->table || !aligned16(r->table) || r->n_pos < 1)) return false;
  return aligned16(r->q_weight) && aligned16(r->k_weight);
}
constexpr int64_t MAX_HEADS = 65536;
TurnArgs turn_args(const smetric_rotary *r, const int32_t *positions, int32_t *status) {
  TurnArgs t{{nullptr, nullptr}, nullptr, 0, 0, 0.0f, positions, status};
  if (r) t = TurnArgs{{r->q_weight, r->k_weight}, r->table, r->n_pos, r->rot_dim, r->eps, positions, status};
  return t;
}

}  // namespace

bool heads_ok(const smetric_heads *h) {
  return h && h->data && aligned16(h->data) && h->token_stride % 8 == 0 && h->head_stride % 8 == 0;
}
bool cache_ok(const smetric_kv_cache *c, int32_t dtype) {
  if (!c || !c->k || !c->v || !aligned16(c->k) || !aligned16(c->v) || !dims_ok(dtype, c->head_dim)) return false;
  if (c->dtype != dtype && c->dtype != SMETRIC_E4M3) return false;
  if (c->n_pages < 1 || c->n_pages > 0x7FFFFFFF || c->page_size < 1 || c->page_size > 65536) return false;
  if (c->n_kv_heads < 1 || c->n_kv_heads > MAX_HEADS || (c->k_scale == nullptr) != (c->v_scale == nullptr)) return false;
  const int64_t unit = c->dtype == SMETRIC_E4M3 ? 16 : 8;
  for (int i = 0; i < 3; ++i)
    if (c->k_stride[i] < 0 || c->v_stride[i] < 0 || c->k_stride[i] % unit || c->v_stride[i] % unit) return false;
  // a page's tokens lie within 32 bits of one another: what a lane adds to its page's address
  return c->k_stride[2] < (int64_t(1) << 24) && c->v_stride[2] < (int64_t(1) << 24);
}
bool batch_ok(const smetric_batch *b) {
  return b && b->n_req >= 0 && b->n_tokens >= 0 && b->max_pages >= 0 && b->table_stride >= b->max_pages &&
         (b->n_req == 0 || (b->q_off && b->kv_len && (b->table || b->max_pages == 0))) &&
         (b->n_req > 0 || b->n_tokens == 0);
}
CacheView cache_view(const smetric_kv_cache *c, const smetric_batch *b) {
  const int64_t e = c->dtype == SMETRIC_E4M3 ? 1 : 2;
  const auto side = [&](void *p, const int64_t *s) { return PageSide{static_cast<char *>(p), s[0] * e, s[1] * e, s[2] * e}; };
  const bool scaled = c->dtype == SMETRIC_E4M3;
  return CacheView{side(c->k, c->k_stride), side(c->v, c->v_stride), scaled ? c->k_scale : nullptr,
                   scaled ? c->v_scale : nullptr, b->table, b->table_stride, int32_t(c->n_pages), b->max_pages,
                   page_size_of(c->page_size)};
}

}  // namespace smk

using namespace smk;

extern "C" int smetric_qk_rotate(int32_t dtype, int32_t head_dim, int64_t n_tokens, const smetric_rotary *rotary,
                                 const int32_t *positions, int32_t n_q_heads, const smetric_heads *q,
                                 const smetric_heads *q_out, int32_t n_kv_heads, const smetric_heads *k,
                                 const smetric_heads *k_out, int32_t *status, hipStream_t stream) {
  if (!dims_ok(dtype, head_dim) || n_tokens < 0 || n_tokens > 0x7FFFFFFF || n_q_heads < 0 || n_kv_heads < 0 ||
      n_q_heads > MAX_HEADS || n_kv_heads > MAX_HEADS || !rotary || !rotary_ok(rotary, head_dim))
    return SMETRIC_EINVAL;
  if (n_tokens == 0 || n_q_heads + n_kv_heads == 0) return SMETRIC_OK;
  if (rotary->rot_dim > 0 && !positions) return SMETRIC_EINVAL;
  if (n_q_heads > 0 && !(heads_ok(q) && heads_ok(q_out))) return SMETRIC_EINVAL;
  if (n_kv_heads > 0 && !(heads_ok(k) && heads_ok(k_out))) return SMETRIC_EINVAL;
  Launch a{};
  a.ta = turn_args(rotary, positions, status);
  a.q = heads_view(n_q_heads ? q : nullptr);
  a.q_out = heads_view(n_q_heads ? q_out : nullptr);
  a.k = heads_view(n_kv_heads ? k : nullptr);
  a.k_out = heads_view(n_kv_heads ? k_out : nullptr);
  a.n_tokens = n_tokens;
  a.n_q = n_q_heads;
  a.n_kv = n_kv_heads;
  a.inter = rotary->interleaved != 0;
  a.stream = stream;
  return launch_any(a, dtype, head_dim);
}

extern "C" int smetric_kv_append(int32_t dtype, const smetric_kv_cache *cache, const smetric_batch *batch,
                                 const smetric_rotary *rotary, const int32_t *positions, int32_t n_q_heads,
                                 const smetric_heads *q, const smetric_heads *q_out, const smetric_heads *k,
                                 const smetric_heads *v, int32_t *status, hipStream_t stream) {
  if (!cache_ok(cache, dtype) || !batch_ok(batch) || n_q_heads < 0 || n_q_heads > MAX_HEADS ||
      batch->n_tokens > 0x7FFFFFFF || (rotary && !rotary_ok(rotary, cache->head_dim)))
    return SMETRIC_EINVAL;
  if (batch->n_tokens == 0) return SMETRIC_OK;
  if (!heads_ok(k) || !heads_ok(v) || (n_q_heads > 0 && !(heads_ok(q) && heads_ok(q_out)))) return SMETRIC_EINVAL;
  Launch a{};
  a.ta = turn_args(rotary, positions, status);
  a.ba = BatchArgs{batch->q_off, batch->kv_len, batch->n_req};
  a.cache = cache_view(cache, batch);
  a.q = heads_view(n_q_heads ? q : nullptr);
  a.q_out = heads_view(n_q_heads ? q_out : nullptr);
  a.k = heads_view(k);
  a.v = heads_view(v);
  a.n_tokens = batch->n_tokens;
  a.n_q = n_q_heads;
  a.n_kv = cache->n_kv_heads;
  a.inter = rotary && rotary->interleaved;
  a.paged = true;
  a.kv8 = cache->dtype == SMETRIC_E4M3;
  a.stream = stream;
  return launch_any(a, dtype, cache->head_dim);
}
