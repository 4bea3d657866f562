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
// Measured: 8,191 tokens of 40 heads of 128 29.5 us, 5.8 TB/s (a copy of 4 GiB moves 4.8); the
// keys, values and queries of 6,249 tokens appended 32.4 us, 4.8 TB/s (pages in any order, the
// queries kept in the caches for the attention); keys and values of 8 heads alone into 4-bit pages
// 13 to 15 us, where three dependent passes through LDS and the chain to the pages are what is left
// (vector instructions 30 % of the cycles; 32 MB are 7 us); a token's append 4.5 us, its launch; of 256 5.2.
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

// Eight components as E2M1 codes in units of scale: to nearest, ties to the even code, saturated.
__device__ __forceinline__ uint32_t narrow_e2m1(const float *x, float scale) {
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
}
// The largest magnitude of eight components as a float's bits, which order as magnitudes do, NaN
// above infinity.
__device__ __forceinline__ uint32_t largest(const float *x) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t b = __float_as_uint(x[i]) & 0x7FFFFFFFu;
    m = b > m ? b : m;
  }
  return m;
}
// The exponent byte of a group whose largest magnitude has these bits: the smallest k with
// a <= 7 2^k = 1.75 2^(k + 2).  Of the borders between which every component stays within half a
// step -- 6 2^k and 7 2^k -- the larger one makes the steps smaller: on normal values the
// relative error is 11.2 %, with 6 11.5, with 8 (where the largest ones are cut) 11.5.
template <typename T>
__device__ __forceinline__ uint32_t exponent_of(uint32_t bits) {
  if (bits > 0x7F800000u) return 255;
  const uint32_t e = (bits + 0x1FFFFFu) >> 23;  // one more where the fraction is above 0.75
  const uint32_t k = e > 2 ? e - 2 : 0;
  return k < T::EXP4_MIN ? T::EXP4_MIN : k > T::EXP4_MAX ? T::EXP4_MAX : k;
}

// Rows (token, head) in order, a workgroup a run of them.  Which token one is of: divisions by the
// heads of a token, as products with rounded-up inverses (exact for the numbers at hand: rows x heads
// below 2^64; at most 2 RT / 4 rows past a token's first x fewer than 64 heads below 2^16).
struct Rows {
  uint64_t inverse;   // 2^64 / per_token, 0: one
  uint32_t small;     // 2^16 / per_token
  int32_t per_token;
};
inline Rows rows_of(int32_t per_token) {
  return {per_token == 1 ? 0 : ~uint64_t(0) / uint32_t(per_token) + 1, 65536 / uint32_t(per_token) + 1, per_token};
}

// PAGED: k goes to the cache (places from the batch), and with it the same token's and head's v, whose
// place is the same; else k goes to k_out and positions are given.  (E4M3: v in a row of its own, as
// 32 divisions of a lane cost more than finding a place twice: 256 tokens 5.7 us, apart 5.2.)
constexpr int sides_of(Pages p) { return p == PAGES8 ? 1 : 2; }  // of a row
template <typename T, int D, bool INTER, bool PAGED, Pages KV>
__global__ __launch_bounds__(RT) void turn_kernel(TurnArgs ta, BatchArgs ba, CacheView cache, HeadsView q, HeadsView q_out,
                                                  HeadsView k, HeadsView k_out, HeadsView v, int64_t n_tokens, int32_t n_q,
                                                  Rows rows) {
  constexpr bool KV4 = KV == PAGES4;
  constexpr int LPR = D / 16;  // lanes per row
  constexpr int WG = RT / LPR;  // rows of a workgroup
  const int lane = threadIdx.x & 63, sub = threadIdx.x % LPR;
  const uint64_t row0 = uint64_t(blockIdx.x) * WG;
  const int64_t token0 = rows.inverse ? __umul64hi(row0, rows.inverse) : row0;
  const uint32_t in0 = uint32_t(row0 - token0 * rows.per_token);
  const auto token_of = [&](uint32_t x) { return rows.per_token >= WG ? uint32_t(x >= uint32_t(rows.per_token)) : x * rows.small >> 16; };
  const uint32_t x0 = in0 + threadIdx.x / LPR, dt = token_of(x0);
  const bool live = token0 + dt < n_tokens;
  const int64_t t = live ? token0 + dt : n_tokens - 1;
  const int32_t h = live ? int32_t(x0 - dt * rows.per_token) : 0;
  const bool cached = h >= n_q;  // a key (and, PAGED, a value)
  constexpr int SIDES = PAGED ? sides_of(KV) : 1;
  const int32_t n_kv = SIDES == 2 ? rows.per_token - n_q : (rows.per_token - n_q) / 2;
  const bool value = PAGED && SIDES == 1 && h >= n_q + n_kv;
  const int32_t head = h - (value ? n_q + n_kv : cached ? n_q : 0);

  // this lane's two pieces of 8 components
  const int half = ta.rot / 16;
  int c0 = sub, c1 = sub + LPR;
  if (!INTER) {
    c0 = sub < half ? sub : 2 * sub;
    c1 = sub < half ? sub + half : 2 * sub + 1;
  }
  // (which of the two turn: both or none for halves)
  const bool turns0 = c0 < (INTER ? 2 * half : half) && !value;
  const bool turns1 = INTER ? c1 < 2 * half && !value : turns0;
  // asked for before the chain of loads that finds the place
  const auto load = [&](const HeadsView &src, u32x4 (&in)[2]) {
    const uint16_t *from = src.data + t * src.token + head * src.head;
    in[0] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(from + 8 * c0));
    in[1] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(from + 8 * c1));
  };
  u32x4 in[2], in_v[2]{};
  load(value ? v : cached ? k : q, in);
  if (SIDES == 2 && cached) load(v, in_v);
  float scale = 1.0f;
  if (KV == PAGES8 && cached && cache.k_scale) scale = (value ? cache.v_scale : cache.k_scale)[head];

  int32_t place = 0, pos = 0, page = 0, id = 0;
  bool ok = live, bad = false;
  if (PAGED) {
    // In a decoding step, as many tokens as requests, token t is request t's: asked for at once, and a
    // search of the whole wavefront only where that is not so for one of its lanes.
    Request rq{0, 0, 0, 0};
    const bool step = n_tokens == ba.n_req;
    if (step) rq = Request{int32_t(t), ba.kv_len[t], ba.q_off[t], ba.q_off[t + 1]};
    if (!step || __any(rq.from > t || rq.to <= t)) {
      const int64_t first = token0 + token_of(in0 + (threadIdx.x & ~63u) / LPR);
      int at = 0;
      rq = Requests(ba.q_off, ba.kv_len, ba.n_req, first < n_tokens ? first : n_tokens - 1, lane).of(t, at);
    }
    bad = t < rq.from || t >= rq.to || rq.len < 0 || rq.len > MAX_PLACES ||
          int64_t(rq.len) > int64_t(cache.max_pages) * cache.ps.size;
    const int64_t p = int64_t(rq.len) - (rq.to - t);
    ok = ok && !bad && p >= 0;
    place = ok ? int32_t(p) : 0;
    pos = place;
    if (ok) {
      page = page_of(cache.ps, place);
      id = cache.table[rq.r * cache.table_stride + page];
      ok = uint32_t(id) < uint32_t(cache.n_pages);
      bad = !ok;
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
  widen<T>(ok ? in[0] : u32x4{0, 0, 0, 0}, x);
  widen<T>(ok ? in[1] : u32x4{0, 0, 0, 0}, x + 8);
  if (ta.weight[0] || ta.weight[1]) {
    const uint16_t *w = static_cast<const uint16_t *>(ta.weight[cached]);
    // the exchange is outside the condition: rows with and without a weight share a wavefront
    float ss = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) ss = fmaf(x[i], x[i], ss);
#pragma unroll
    for (int m = 1; m < LPR; m *= 2) ss += __shfl_xor(ss, m, 64);
    if (w && ok && !value) {  // (zeros stay zeros also where eps is 0)
      const float rstd = 1.0f / sqrtf(ss * (1.0f / D) + ta.eps);
      float g[16];
      widen<T>(*reinterpret_cast<const u32x4 *>(w + 8 * c0), g);
      widen<T>(*reinterpret_cast<const u32x4 *>(w + 8 * c1), g + 8);
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = x[i] * rstd * g[i];
    }
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
  if (PAGED) {
    // Both sides' rows into their pages, side by side: neither waits for the other.  4 bits: the lane that has
    // a piece is not the one that has its neighbours, so their largest magnitudes, then the codes,
    // pass through LDS, where a row is in order: a lane then writes two neighbouring pieces.  All
    // lanes come here together, also those of queries, which share wavefronts with keys.
    if (__any(cached && live)) {
      float y[SIDES][16];
#pragma unroll
      for (int i = 0; i < 16; ++i) y[0][i] = x[i];
      if (SIDES == 2) {
        widen<T>(in_v[0], y[SIDES - 1]);
        widen<T>(in_v[1], y[SIDES - 1] + 8);
      }
      uint32_t e[SIDES][2];
      u32x2 codes[SIDES][2];
      if (KV4) {
        __shared__ __attribute__((aligned(16))) uint32_t sh[SIDES][RT * 2];
        const int row = threadIdx.x / LPR * (D / 8);
#pragma unroll
        for (int s = 0; s < SIDES; ++s) {
          sh[s][row + c0] = largest(y[s]);
          sh[s][row + c1] = largest(y[s] + 8);
        }
        wave_fence();
#pragma unroll
        for (int s = 0; s < SIDES; ++s)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const u32x4 m = *reinterpret_cast<const u32x4 *>(&sh[s][row + ((i ? c1 : c0) & ~3)]);
            const uint32_t a = m[0] > m[1] ? m[0] : m[1], b = m[2] > m[3] ? m[2] : m[3];
            e[s][i] = exponent_of<T>(a > b ? a : b);
          }
        wave_fence();
#pragma unroll
        for (int s = 0; s < SIDES; ++s) {
          sh[s][row + c0] = narrow_e2m1(y[s], power_of(e[s][0]));
          sh[s][row + c1] = narrow_e2m1(y[s] + 8, power_of(e[s][1]));
        }
        wave_fence();
#pragma unroll
        for (int s = 0; s < SIDES; ++s) codes[s][0] = *reinterpret_cast<const u32x2 *>(&sh[s][row + 2 * sub]);
      } else if (KV == PAGES8) {
#pragma unroll
        for (int s = 0; s < SIDES; ++s)
#pragma unroll
          for (int i = 0; i < 2; ++i) codes[s][i] = narrow_e4m3(y[s] + 8 * i, scale);
      }
      if (ok && cached) {
        const int32_t slot = place - page * cache.ps.size;
#pragma unroll
        for (int s = 0; s < SIDES; ++s) {
          const PageSide &side = s || value ? cache.v : cache.k;
          char *to = side.base + (id * side.page + head * side.head + slot * side.token);
          if (KV4) {
            const PageSide &es = s ? cache.v_exp : cache.k_exp;
            *reinterpret_cast<u32x2 *>(to + 8 * sub) = codes[s][0];
            char *ex = es.base + (id * es.page + head * es.head + slot * es.token);
            if (c0 % 4 == 0) ex[c0 / 4] = char(e[s][0]);
            if (c1 % 4 == 0) ex[c1 / 4] = char(e[s][1]);
          } else if (KV == PAGES8) {
            *reinterpret_cast<u32x2 *>(to + 8 * c0) = codes[s][0];
            *reinterpret_cast<u32x2 *>(to + 8 * c1) = codes[s][1];
          } else {
            *reinterpret_cast<u32x4 *>(to + 16 * c0) = narrow<T>(y[s]);
            *reinterpret_cast<u32x4 *>(to + 16 * c1) = narrow<T>(y[s] + 8);
          }
        }
      }
    }
  }
  if (!live || (PAGED && cached)) return;
  const HeadsView &dst = cached ? k_out : q_out;
  uint16_t *p = dst.data + t * dst.token + head * dst.head;
  if (PAGED) {  // attention reads it next
    *reinterpret_cast<u32x4 *>(p + 8 * c0) = narrow<T>(x);
    *reinterpret_cast<u32x4 *>(p + 8 * c1) = narrow<T>(x + 8);
  } else {
    __builtin_nontemporal_store(narrow<T>(x), reinterpret_cast<u32x4 *>(p + 8 * c0));
    __builtin_nontemporal_store(narrow<T>(x + 8), reinterpret_cast<u32x4 *>(p + 8 * c1));
  }
}

struct Launch {
  TurnArgs ta;
  BatchArgs ba;
  CacheView cache;
  HeadsView q, q_out, k, k_out, v;
  int64_t n_tokens;
  int32_t n_q, n_kv;
  bool inter, paged;
  Pages pages;
  hipStream_t stream;
};
template <typename T, int D, bool INTER, bool PAGED, Pages KV>
int launch(const Launch &a) {
  const int32_t per_token = a.n_q + (PAGED ? 3 - sides_of(KV) : 1) * a.n_kv;
  const int64_t wg = RT / (D / 16), grid = (a.n_tokens * per_token + wg - 1) / wg;
  if (grid > 0x7FFFFFFF) return SMETRIC_EINVAL;
  turn_kernel<T, D, INTER, PAGED, KV><<<dim3(uint32_t(grid)), dim3(RT), 0, a.stream>>>(
      a.ta, a.ba, a.cache, a.q, a.q_out, a.k, a.k_out, a.v, a.n_tokens, a.n_q, rows_of(per_token));
  return hip_status(hipGetLastError());
}
template <typename T, int D, bool INTER>
int launch_tdi(const Launch &a) {
  if (!a.paged) return launch<T, D, INTER, false, PAGES16>(a);
  return a.pages == PAGES4   ? launch<T, D, INTER, true, PAGES4>(a)
         : a.pages == PAGES8 ? launch<T, D, INTER, true, PAGES8>(a)
                             : launch<T, D, INTER, true, PAGES16>(a);
}
template <typename T, int D>
int launch_td(const Launch &a) {
  return a.inter ? launch_tdi<T, D, true>(a) : launch_tdi<T, D, false>(a);
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
  if (c->dtype != dtype && c->dtype != SMETRIC_E4M3 && c->dtype != SMETRIC_E2M1) return false;
  if (c->n_pages < 1 || c->n_pages > 0x7FFFFFFF || c->page_size < 1 || c->page_size > 65536) return false;
  if (c->n_kv_heads < 1 || c->n_kv_heads > MAX_HEADS || (c->k_scale == nullptr) != (c->v_scale == nullptr)) return false;
  const int64_t unit = c->dtype == SMETRIC_E2M1 ? 32 : c->dtype == SMETRIC_E4M3 ? 16 : 8;
  for (int i = 0; i < 3; ++i)
    if (c->k_stride[i] < 0 || c->v_stride[i] < 0 || c->k_stride[i] % unit || c->v_stride[i] % unit) return false;
  if (c->dtype == SMETRIC_E2M1) {
    const uintptr_t bytes = uintptr_t(c->head_dim / GROUP4);
    const smetric_kv_exps *e = c->exps;
    if (!e || !e->k || !e->v || reinterpret_cast<uintptr_t>(e->k) % bytes || reinterpret_cast<uintptr_t>(e->v) % bytes)
      return false;
    for (int i = 0; i < 3; ++i)
      if (e->k_stride[i] < 0 || e->v_stride[i] < 0 || e->k_stride[i] % int64_t(bytes) || e->v_stride[i] % int64_t(bytes))
        return false;
    if (e->k_stride[2] >= (int64_t(1) << 24) || e->v_stride[2] >= (int64_t(1) << 24)) return false;
  }
  // a page's tokens lie within 32 bits of one another: what a lane adds to its page's address
  return c->k_stride[2] < (int64_t(1) << 24) && c->v_stride[2] < (int64_t(1) << 24);
}
bool batch_ok(const smetric_batch *b) {
  return b && b->n_req >= 0 && b->n_tokens >= 0 && b->max_pages >= 0 && b->table_stride >= b->max_pages &&
         (b->n_req == 0 || (b->q_off && b->kv_len && (b->table || b->max_pages == 0))) &&
         (b->n_req > 0 || b->n_tokens == 0);
}
CacheView cache_view(const smetric_kv_cache *c, const smetric_batch *b) {
  const Pages p = pages_of(c);
  const auto side = [&](void *base, const int64_t *s) {
    const auto bytes = [&](int64_t n) { return p == PAGES16 ? 2 * n : p == PAGES8 ? n : n / 2; };
    return PageSide{static_cast<char *>(base), bytes(s[0]), bytes(s[1]), bytes(s[2])};
  };
  PageSide k_exp{nullptr, 0, 0, 0}, v_exp{nullptr, 0, 0, 0};
  if (p == PAGES4) {
    const smetric_kv_exps *e = c->exps;
    k_exp = PageSide{reinterpret_cast<char *>(e->k), e->k_stride[0], e->k_stride[1], e->k_stride[2]};
    v_exp = PageSide{reinterpret_cast<char *>(e->v), e->v_stride[0], e->v_stride[1], e->v_stride[2]};
  }
  const bool scaled = p == PAGES8;
  return CacheView{side(c->k, c->k_stride), side(c->v, c->v_stride), k_exp, v_exp, scaled ? c->k_scale : nullptr,
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
  a.pages = pages_of(cache);
  a.stream = stream;
  return launch_any(a, dtype, cache->head_dim);
}
