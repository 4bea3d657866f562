// Cached tokens read back from the paged cache as activations.
//
// Mathematics: a stored x stands for itself (16 bits), for x scale (E4M3, a scale per head) or for
// x 2^(e - 127) (E2M1, an exponent per 32 components): widened in float32, rounded once.
// Bound: memory, each row read once and written once as 16 bits; 8 components, 16 bytes, a lane.
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
// than that.
template <typename T, Pages KV, int D>
__global__ __launch_bounds__(ET) void read_kernel(ReadArgs a) {
  constexpr int PPR = D / 8;  // pieces of a row
  constexpr int PB = page_bytes(KV, 8);
  const uint32_t per_token = uint32_t(a.n_kv) * PPR, side = per_token < ET ? ET / per_token : 1;
  const int lane = threadIdx.x & 63;
  const uint32_t which = per_token < ET ? threadIdx.x / per_token : 0;
  const uint32_t in = per_token < ET ? threadIdx.x % per_token : blockIdx.y * ET + threadIdx.x;
  const int64_t base = int64_t(blockIdx.x) * side * EU, t0 = base + which * EU;
  const int64_t first = base + (per_token < ET ? (threadIdx.x & ~63u) / per_token : 0) * EU;
  if (first >= a.n_tokens) return;  // the whole wavefront
  const bool live = t0 < a.n_tokens && which < side && in < per_token;
  const int32_t head = in / PPR, piece = in % PPR;
  const Requests requests(a.q_off, a.kv_len, a.n_req, first, lane);
  int at_request = 0;
  Request of[EU];
#pragma unroll
  for (int u = 0; u < EU; ++u) of[u] = requests.of(live ? (t0 + u < a.n_tokens ? t0 + u : a.n_tokens - 1) : first, at_request);
  if (!live) return;
  u32x4 x[EU][2];
  uint32_t e[EU][2];
  bool bad = false;
#pragma unroll
  for (int u = 0; u < EU; ++u) {
    const int64_t t = t0 + u;
    x[u][0] = x[u][1] = u32x4{0, 0, 0, 0};
    e[u][0] = e[u][1] = 127;
    if (t >= a.n_tokens) continue;
    const Request &q = of[u];
    const int64_t p = int64_t(q.len) - (q.to - t);
    const bool ok = t >= q.from && t < q.to && q.len >= 0 && q.len <= MAX_PLACES &&
                    int64_t(q.len) <= int64_t(a.cache.max_pages) * a.cache.ps.size;
    bad |= !ok;
    if (!ok || p < 0) continue;
    const int32_t place = int32_t(p), page = page_of(a.cache.ps, place);
    const int32_t id = a.cache.table[q.r * a.cache.table_stride + page], slot = place - page * a.cache.ps.size;
    if (uint32_t(id) >= uint32_t(a.cache.n_pages)) {
      bad = true;
      continue;
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      if (!a.out[s].data) continue;
      const PageSide &side = s ? a.cache.v : a.cache.k, &es = s ? a.cache.v_exp : a.cache.k_exp;
      const char *at = side.base + id * side.page + head * side.head + slot * side.token + piece * PB;
      if (KV == PAGES16) x[u][s] = *reinterpret_cast<const u32x4 *>(at);
      if (KV == PAGES8) {
        const u32x2 y = *reinterpret_cast<const u32x2 *>(at);
        x[u][s].x = y.x;
        x[u][s].y = y.y;
      }
      if (KV == PAGES4) {
        x[u][s].x = *reinterpret_cast<const uint32_t *>(at);
        e[u][s] = uint8_t(es.base[id * es.page + head * es.head + slot * es.token + piece / 4]);
      }
    }
  }
  if (bad) set_status(a.status, SMETRIC_EINVAL);
  float scale[2] = {1.0f, 1.0f};
  if (KV == PAGES8 && a.cache.k_scale) {
    scale[0] = a.cache.k_scale[head];
    scale[1] = a.cache.v_scale[head];
  }
#pragma unroll
  for (int u = 0; u < EU; ++u) {
    const int64_t t = t0 + u;
    if (t >= a.n_tokens) break;
#pragma unroll
    for (int s = 0; s < 2; ++s)
      if (a.out[s].data) {
        u32x4 *to = reinterpret_cast<u32x4 *>(a.out[s].data + t * a.out[s].token + head * a.out[s].head + 8 * piece);
        // past the caches: what is read back is more than they hold
        __builtin_nontemporal_store(widened<T, KV>(x[u][s], e[u][s], scale[s]), to);
      }
  }
}

template <typename T, Pages KV, int D>
int launch_d(const ReadArgs &a, hipStream_t stream) {
  const int64_t per_token = int64_t(a.n_kv) * (D / 8), side = per_token < ET ? ET / per_token : 1;
  const int64_t grid = (a.n_tokens + side * EU - 1) / (side * EU), wide = per_token < ET ? 1 : (per_token + ET - 1) / ET;
  if (grid > 0x7FFFFFFF || wide > 65535) return SMETRIC_EINVAL;
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
                   {heads_view(k_out), heads_view(v_out)}, status};
  return dtype == SMETRIC_BF16 ? launch_t<Bf16>(a, pages_of(cache), cache->head_dim, stream)
                               : launch_t<F16>(a, pages_of(cache), cache->head_dim, stream);
}
