// Cached tokens read back from the paged cache as activations.
//
// Mathematics: a stored x stands for itself (16 bits), for x scale (E4M3, a scale per head) or for
// x 2^(e - 127) (E2M1, an exponent per 32 components): widened in float32, rounded once.
// Bound: memory, each row read once and written once as 16 bits; 8 components, 16 bytes, a lane, stored
// past the caches (24 sessions of 8-bit pages 132 us, so 121; a few tokens that the next kernel reads pay little
// for it: 4,096 read back and added up 16.9 us, 16.2 through the caches, one token 4.8 both).
//
// Measured: a session of 16,384 tokens, 4 heads of 128 in 4 bits (42 MB moved) 9.2 us, 4.6 TB/s; 24
// sessions, 16 heads of 64 of 8 bits (630 MB) 117 us, 5.4 TB/s; 16 of 8,192, 8 heads of 128 of 16 bits
// (1.07 GB) 191 us, 5.6 TB/s; the 4-bit ones of 16,384 (1.36 GB) 307 us, 4.4 TB/s, where the instructions
// that widen and address are what is left.
#include "kv_common.h"

namespace smk {
namespace {

constexpr int ET = 256;  // threads per workgroup
constexpr int EU = 2;    // tokens of a thread

struct ReadArgs {
  const int64_t *q_off;
  const int32_t *kv_len;
  int32_t n_req, n_kv;
  int64_t n_tokens;
  CacheView cache;
  HeadsView out[2];  // keys, values; no memory: left out
  int32_t *status;
  uint32_t per_token, side, inverse;  // pieces of a token; tokens side by side; 2^16 / per_token, rounded up
};

// Eight components from the pieces of a row in memory, rounded to T.
template <typename T, Pages KV>
__device__ __forceinline__ u32x4 widened(u32x4 x, uint32_t e, float scale) {
  if (KV == PAGES16) return x;
  if (KV == PAGES4) return T::eight_e2m1(x.x, power_of(e));
  u32x4 y;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(x[i], false), b = __builtin_amdgcn_cvt_pk_f32_fp8(x[i], true);
    y[2 * i] = T::pack(a.x * scale, a.y * scale);
    y[2 * i + 1] = T::pack(b.x * scale, b.y * scale);
  }
  return y;
}

// A workgroup takes EU tokens side by side, or several times as many: threads are dealt to (which of
// them, head, piece), a thread's EU tokens follow each other.  blockIdx.y: 256 pieces of rows longer
// than that.  A row's address is four products of 64 bits, at a quarter of the rate, for each of its two sides
// and their exponents: it is worked out once, and the next token's is a stride on until its page or its
// request ends (16 sessions of 16,384 tokens, 8 heads of 128 in 4 bits: 340 us, so 307; with four tokens a
// thread 299, but 256 requests' last tokens 11.4 for 8.8).
template <typename T, Pages KV, int D>
__global__ __launch_bounds__(ET) void read_kernel(ReadArgs a) {
  constexpr int PPR = D / 8;  // pieces of a row
  constexpr int PB = page_bytes(KV, 8);
  const uint32_t per_token = a.per_token;
  const int lane = threadIdx.x & 63;
  const auto token_of = [&](uint32_t x) { return per_token < ET ? x * a.inverse >> 16 : 0; };  // x / per_token
  const uint32_t which = token_of(threadIdx.x);
  const uint32_t in = per_token < ET ? threadIdx.x - which * per_token : blockIdx.y * ET + threadIdx.x;
  const int64_t base = int64_t(blockIdx.x) * (a.side * EU), t0 = base + which * EU;
  const int64_t first = base + token_of(threadIdx.x & ~63u) * EU;
  if (first >= a.n_tokens) return;  // the whole wavefront
  const bool live = t0 < a.n_tokens && which < a.side && in < per_token;
  const int32_t head = live ? in / PPR : 0, piece = in % PPR;
  const Requests requests(a.q_off, a.kv_len, a.n_req, first, lane);
  int at_request = 0;
  Request q = requests.of(live ? t0 : first, at_request);

  // page 0 to begin with: rows without a place read what is there, for nothing
  uint64_t at[2], ex[2];
  const PageSide *const sides[2] = {&a.cache.k, &a.cache.v}, *const exps[2] = {&a.cache.k_exp, &a.cache.v_exp};
  const auto start = [&](int32_t id, int32_t slot) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      at[s] = reinterpret_cast<uint64_t>(sides[s]->base) + id * sides[s]->page + head * sides[s]->head + slot * sides[s]->token + piece * PB;
      if (KV == PAGES4)
        ex[s] = reinterpret_cast<uint64_t>(exps[s]->base) + id * exps[s]->page + head * exps[s]->head + slot * exps[s]->token + piece / 4;
    }
  };
  start(0, 0);
  u32x4 x[EU][2];
  uint32_t e[EU][2];
  bool ok[EU], bad = false, before = false;
  int32_t slot = 0, r = -1;
#pragma unroll
  for (int u = 0; u < EU; ++u) {
    const int64_t t = t0 + u;
    const bool mine = live && t < a.n_tokens;
    if (u > 0 && __any(mine && t >= q.to)) q = requests.of(mine ? t : first, at_request);
    const int64_t p = int64_t(q.len) - (q.to - t);
    const bool good = t >= q.from && t < q.to && q.len >= 0 && q.len <= MAX_PLACES &&
                      int64_t(q.len) <= int64_t(a.cache.max_pages) * a.cache.ps.size;
    bad |= mine && !good;
    ok[u] = mine && good && p >= 0;
    const bool on = before && ok[u] && q.r == r && slot + 1 < a.cache.ps.size;
    if (on) {
      ++slot;
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        at[s] += sides[s]->token;
        if (KV == PAGES4) ex[s] += exps[s]->token;
      }
    } else if (ok[u]) {
      const int32_t place = int32_t(p), page = page_of(a.cache.ps, place);
      const int32_t id = a.cache.table[q.r * a.cache.table_stride + page];
      slot = place - page * a.cache.ps.size;
      r = q.r;
      ok[u] = uint32_t(id) < uint32_t(a.cache.n_pages);
      bad |= !ok[u];
      if (ok[u]) start(id, slot);
    }
    before = ok[u];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      if (!a.out[s].data) continue;
      if (KV == PAGES16) x[u][s] = from_memory<u32x4>(at[s]);
      if (KV == PAGES8) {
        const u32x2 y = from_memory<u32x2>(at[s]);
        x[u][s] = u32x4{y.x, y.y, 0, 0};
      }
      if (KV == PAGES4) {
        x[u][s] = u32x4{from_memory<uint32_t>(at[s]), 0, 0, 0};
        e[u][s] = from_memory<uint8_t>(ex[s]);
      }
    }
  }
  if (bad) set_status(a.status, SMETRIC_EINVAL);
  float scale[2] = {1.0f, 1.0f};
  if (KV == PAGES8 && a.cache.k_scale) {
    scale[0] = a.cache.k_scale[head];
    scale[1] = a.cache.v_scale[head];
  }
  if (!live) return;
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    if (!a.out[s].data) continue;
    uint16_t *to = a.out[s].data + t0 * a.out[s].token + head * a.out[s].head + 8 * piece;
#pragma unroll
    for (int u = 0; u < EU; ++u, to += a.out[s].token) {
      if (t0 + u >= a.n_tokens) break;
      const u32x4 y = widened<T, KV>(x[u][s], e[u][s], scale[s]);
      // past the caches, see above
      __builtin_nontemporal_store(ok[u] ? y : u32x4{0, 0, 0, 0}, reinterpret_cast<u32x4 *>(to));
    }
  }
}

template <typename T, Pages KV, int D>
int launch_d(ReadArgs a, hipStream_t stream) {
  const uint32_t per_token = uint32_t(a.n_kv) * (D / 8), side = per_token < ET ? ET / per_token : 1;
  const int64_t grid = (a.n_tokens + side * EU - 1) / (side * EU), wide = per_token < ET ? 1 : (per_token + ET - 1) / ET;
  if (grid > 0x7FFFFFFF || wide > 65535) return SMETRIC_EINVAL;
  a.per_token = per_token;
  a.side = side;
  a.inverse = 65536 / per_token + 1;  // exact below 2^8 / per_token: both are below 2^8
  read_kernel<T, KV, D><<<dim3(uint32_t(grid), uint32_t(wide)), dim3(ET), 0, stream>>>(a);
  return hip_status(hipGetLastError());
}
template <typename T, Pages KV>
int launch_k(const ReadArgs &a, int32_t d, hipStream_t stream) {
  return d == 64 ? launch_d<T, KV, 64>(a, stream) : d == 128 ? launch_d<T, KV, 128>(a, stream) : launch_d<T, KV, 256>(a, stream);
}
template <typename T>
int launch_t(const ReadArgs &a, Pages p, int32_t d, hipStream_t stream) {
  return p == PAGES4   ? launch_k<T, PAGES4>(a, d, stream)
         : p == PAGES8 ? launch_k<T, PAGES8>(a, d, stream)
                       : launch_k<T, PAGES16>(a, d, stream);
}

}  // namespace
}  // namespace smk

using namespace smk;

extern "C" int smetric_kv_read(int32_t dtype, const smetric_kv_cache *cache, const smetric_batch *batch,
                               const smetric_heads *k_out, const smetric_heads *v_out, int32_t *status, hipStream_t stream) {
  if (!cache_ok(cache, dtype) || !batch_ok(batch) || batch->n_tokens > 0x7FFFFFFF) return SMETRIC_EINVAL;
  if (batch->n_tokens == 0 || (!k_out && !v_out)) return SMETRIC_OK;
  if ((k_out && !heads_ok(k_out)) || (v_out && !heads_ok(v_out))) return SMETRIC_EINVAL;
  const ReadArgs a{batch->q_off, batch->kv_len, batch->n_req, cache->n_kv_heads, batch->n_tokens, cache_view(cache, batch),
                   {heads_view(k_out), heads_view(v_out)}, status, 0, 0, 0};
  return dtype == SMETRIC_BF16 ? launch_t<Bf16>(a, pages_of(cache), cache->head_dim, stream)
                               : launch_t<F16>(a, pages_of(cache), cache->head_dim, stream);
}
