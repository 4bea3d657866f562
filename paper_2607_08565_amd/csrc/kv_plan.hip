// The plan of an attention step: which rows and keys each workgroup takes, and the joining
// of the tiles whose keys were cut.
//
// The plan depends on the lengths alone, so one serves all layers of a step.  One workgroup
// makes it: the total of the tiles' key steps gives the length of a piece, then every tile
// writes its pieces at a place from a scan over the tiles.
#include <math.h>

#include "kv_attend.h"

namespace smk {
namespace {

constexpr int PT = 1024;

struct PlanArgs {
  const int64_t *q_off;
  const int32_t *kv_len;
  int32_t n_req, n_q, n_kv, group, rows, window, target, min_steps;
  int64_t n_tokens, max_tiles, max_items, max_splits, max_parts;
  PlanHdr *hdr;
  PlanItem *items;
  PlanSplit *splits;
  int32_t *status;
};

struct Tile {
  int32_t req, tile, n_new, kv_len, tok0, k0, k1, steps;  // req < 0: the number belongs to no tile
};
__device__ Tile tile_at(const PlanArgs &a, int64_t g) {
  Tile t{-1, 0, 0, 0, 0, 0, 0, 0};
  int32_t lo = 0, hi = a.n_req - 1;  // the last request whose numbers begin at or before g
  while (lo < hi) {
    const int32_t mid = (lo + hi + 1) / 2;
    if (a.q_off[mid] * a.group / a.rows + mid <= g)
      lo = mid;
    else
      hi = mid - 1;
  }
  const int64_t q0 = a.q_off[lo];
  const int64_t n = a.q_off[lo + 1] - q0, in = g - (q0 * a.group / a.rows + lo);
  const int64_t tiles = (n * a.group + a.rows - 1) / a.rows;
  if (in < 0 || in >= tiles) return t;
  t.req = lo;
  t.tile = int32_t(tiles - 1 - in);  // long ones first
  t.n_new = int32_t(n);
  t.tok0 = int32_t(q0);
  t.kv_len = a.kv_len[lo];
  const int32_t row0 = t.tile * a.rows;
  int32_t last = row0 + a.rows;
  if (last > t.n_new * a.group) last = t.n_new * a.group;
  const int32_t first = t.kv_len - t.n_new + row0 / a.group;  // places of the tile's first and last token
  t.k1 = t.kv_len - t.n_new + (last - 1) / a.group + 1;
  t.k0 = a.window > 0 && first - a.window + 1 > 0 ? first - a.window + 1 : 0;
  if (t.k1 <= t.k0) t.k0 = t.k1 = 0;
  t.steps = (t.k1 + KEY_STEP - 1) / KEY_STEP - t.k0 / KEY_STEP;
  return t;
}

// Sums of v over the workgroup's earlier threads, and of all, for two counts at once.
__device__ void scan2(int32_t &x, int32_t &y, int32_t &tx, int32_t &ty, int32_t (*sh)[PT / 64]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int32_t a = x, b = y;
#pragma unroll
  for (int m = 1; m < 64; m *= 2) {
    const int32_t ua = __shfl_up(a, m, 64), ub = __shfl_up(b, m, 64);
    if (lane >= m) {
      a += ua;
      b += ub;
    }
  }
  if (lane == 63) {
    sh[0][wave] = a;
    sh[1][wave] = b;
  }
  __syncthreads();
  int32_t pa = 0, pb = 0;
  tx = ty = 0;
  for (int w = 0; w < PT / 64; ++w) {
    if (w == wave) {
      pa = tx;
      pb = ty;
    }
    tx += sh[0][w];
    ty += sh[1][w];
  }
  x = pa + a - x;
  y = pb + b - y;
  __syncthreads();
}

__global__ __launch_bounds__(PT) void plan_kernel(PlanArgs a) {
  __shared__ int32_t sh[2][PT / 64];
  __shared__ unsigned long long total;
  __shared__ int bad;
  if (threadIdx.x == 0) {
    total = 0;
    bad = 0;
  }
  __syncthreads();
  bool wrong = false;
  for (int32_t r = threadIdx.x; r < a.n_req; r += PT) {
    const int64_t q0 = a.q_off[r], q1 = a.q_off[r + 1];
    const int32_t len = a.kv_len[r];
    wrong |= q0 < 0 || q1 < q0 || q1 > a.n_tokens || (r == 0 && q0 != 0) || (r == a.n_req - 1 && q1 != a.n_tokens) ||
             len < 0 || len > MAX_PLACES;
  }
  if (wrong) bad = 1;
  __syncthreads();
  int32_t n_items = 0, n_splits = 0, n_parts = 0;
  if (!bad) {
    unsigned long long mine = 0;
    for (int64_t g = threadIdx.x; g < a.max_tiles; g += PT) mine += tile_at(a, g).steps;
#pragma unroll
    for (int m = 1; m < 64; m *= 2) mine += __shfl_xor(mine, m, 64);
    if ((threadIdx.x & 63) == 0) atomicAdd(&total, mine);
    __syncthreads();
    const int64_t share = int64_t((total + a.target - 1) / a.target);
    const int32_t piece = share < a.min_steps ? a.min_steps : int32_t(share);
    for (int64_t g0 = 0; g0 < a.max_tiles; g0 += PT) {
      const int64_t g = g0 + threadIdx.x;
      Tile t{-1, 0, 0, 0, 0, 0, 0, 0};
      if (g < a.max_tiles) t = tile_at(a, g);
      const int32_t pieces = t.req < 0 ? 0 : t.steps <= piece ? 1 : (t.steps + piece - 1) / piece;
      int32_t at = pieces, cut = pieces > 1 ? pieces : 0, cut_at = cut, all, all_cut;
      scan2(at, cut_at, all, all_cut, sh);
      int32_t split = pieces > 1, none = 0, split_at, t0, t1;
      split_at = split;
      scan2(split_at, none, t0, t1, sh);
      const int32_t base = n_items + at, part0 = n_parts + cut_at;
      // even pieces: the last is not the shortest by much
      for (int32_t i = 0; i < pieces && base + i < a.max_items; ++i) {
        const int64_t s0 = int64_t(t.steps) * i / pieces, s1 = int64_t(t.steps) * (i + 1) / pieces;
        const int32_t k = t.k0 / KEY_STEP * KEY_STEP;
        a.items[base + i] =
            PlanItem{t.req,  t.tok0, t.n_new, t.kv_len, t.tile, i == 0 ? t.k0 : int32_t(k + s0 * KEY_STEP),
                     i == pieces - 1 ? t.k1 : int32_t(k + s1 * KEY_STEP), cut ? part0 + i : -1};
      }
      if (split && n_splits + split_at < a.max_splits)
        a.splits[n_splits + split_at] = PlanSplit{t.tok0, t.n_new, t.tile, part0, pieces, {0, 0, 0}};
      n_items += all;
      n_parts += all_cut;
      n_splits += t0;
    }
  }
  if (threadIdx.x == 0) {
    PlanHdr h{};
    h.err = bad ? SMETRIC_EINVAL : SMETRIC_OK;
    if (n_items > a.max_items || n_splits > a.max_splits || n_parts > a.max_parts) h.err = SMETRIC_EINTERNAL;
    h.n_items = n_items;
    h.n_splits = n_splits;
    h.n_req = a.n_req;
    h.n_q = a.n_q;
    h.n_kv = a.n_kv;
    h.rows = a.rows;
    h.window = a.window;
    h.n_tokens = a.n_tokens;
    *a.hdr = h;
    if (h.err) set_status(a.status, h.err);
  }
}

// Joins the parts of a cut tile: out = sum_p 2^(m_p - m) acc_p / sum_p 2^(m_p - m) l_p, in the
// order of the parts.  A workgroup takes one row of one key-value head at a time: D / 4
// threads a part, several parts side by side.
constexpr int32_t JOIN_GRID = 1024;
template <typename T, int D>
__global__ __launch_bounds__(256) void join_kernel(AttendArgs a) {
  constexpr int TPP = D / 4, SIDE = 256 / TPP;
  __shared__ f32x4 sh[256];
  __shared__ float shl[SIDE];
  if (!plan_fits(a)) return;
  const int64_t units = int64_t(a.hdr->n_splits) * a.n_kv * a.rows;
  const int32_t sub = threadIdx.x % TPP, side = threadIdx.x / TPP;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int32_t kvh = int32_t(u % a.n_kv), row = int32_t(u / a.n_kv % a.rows);
    const PlanSplit s = a.splits[u / a.n_kv / a.rows];
    const int32_t in_req = s.tile * a.rows + row;
    if (in_req >= s.n_new * a.group) continue;
    const int64_t step = int64_t(a.n_kv) * a.rows, at0 = (int64_t(s.part0) * a.n_kv + kvh) * a.rows + row;
    float m = -INFINITY;
    for (int32_t p = threadIdx.x & 63; p < s.n_parts; p += 64) m = fmaxf(m, a.parts.ml[at0 + p * step].x);
#pragma unroll
    for (int i = 1; i < 64; i *= 2) m = fmaxf(m, __shfl_xor(m, i, 64));
    const float ms = m == -INFINITY ? 0.0f : m;
    f32x4 acc{0, 0, 0, 0};
    float l = 0.0f;
#pragma unroll 4
    for (int32_t p = side; p < s.n_parts; p += SIDE) {
      const f32x2 ml = a.parts.ml[at0 + p * step];
      const f32x4 v = *reinterpret_cast<const f32x4 *>(a.parts.acc + (at0 + p * step) * D + sub * 4);
      const float w = exp2f(ml.x - ms);
      l = fmaf(w, ml.y, l);
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[i] = fmaf(w, v[i], acc[i]);
    }
    sh[threadIdx.x] = acc;
    if (sub == 0) shl[side] = l;
    __syncthreads();
    if (side == 0) {
#pragma unroll
      for (int i = 1; i < SIDE; ++i) {
        acc += sh[i * TPP + sub];
        l += shl[i];
      }
      const float inv = l == 0.0f ? 0.0f : 1.0f / l;
      const int64_t t = int64_t(s.tok0) + in_req / a.group;
      const int32_t head = kvh * a.group + in_req % a.group;
      *reinterpret_cast<u32x2 *>(a.out.data + t * a.out.token + head * a.out.head + sub * 4) =
          u32x2{T::pack(acc[0] * inv, acc[1] * inv), T::pack(acc[2] * inv, acc[3] * inv)};
      if (a.lse && sub == 0) a.lse[t * a.n_q + head] = lse_of<T>(m, l);
    }
    __syncthreads();
  }
}

template <typename T>
int launch_join(const AttendArgs &a, int32_t head_dim, int64_t max_splits, hipStream_t stream) {
  const int64_t units = max_splits * a.n_kv * a.rows;
  const dim3 grid(uint32_t(units < JOIN_GRID ? units : JOIN_GRID));
  if (head_dim == 64)
    join_kernel<T, 64><<<grid, 256, 0, stream>>>(a);
  else if (head_dim == 128)
    join_kernel<T, 128><<<grid, 256, 0, stream>>>(a);
  else
    join_kernel<T, 256><<<grid, 256, 0, stream>>>(a);
  return hip_status(hipGetLastError());
}

bool shape_ok(int32_t n_req, int64_t n_tokens, int32_t n_q, int32_t n_kv, int32_t head_dim, int32_t max_new) {
  return n_req >= 0 && n_tokens >= 0 && (n_req > 0 || n_tokens == 0) && n_kv >= 1 && n_q >= n_kv && n_q <= 65536 &&
         n_q % n_kv == 0 && n_tokens * (n_q / n_kv) < 0x7FFFFFFF && n_tokens <= 0x7FFFFFFF && max_new >= 1 &&
         (head_dim == 64 || head_dim == 128 || head_dim == 256);
}

}  // namespace
}  // namespace smk

using namespace smk;

extern "C" int smetric_attend_plan_bytes(int32_t n_req, int64_t n_tokens, int32_t n_q_heads, int32_t n_kv_heads,
                                         int32_t head_dim, int32_t max_new, uint64_t *plan_bytes, uint64_t *ws_bytes) {
  if (!plan_bytes || !ws_bytes || !shape_ok(n_req, n_tokens, n_q_heads, n_kv_heads, head_dim, max_new)) return SMETRIC_EINVAL;
  const PlanShape s = plan_shape(n_req, n_tokens, n_q_heads, n_kv_heads, head_dim, max_new);
  *plan_bytes = s.plan_bytes;
  *ws_bytes = s.ws_bytes;
  return SMETRIC_OK;
}

extern "C" int smetric_attend_plan(const int64_t *q_off, const int32_t *kv_len, int32_t n_req, int64_t n_tokens,
                                   int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t max_new,
                                   int32_t window, void *plan, uint64_t plan_bytes, int32_t *status, hipStream_t stream) {
  if (!shape_ok(n_req, n_tokens, n_q_heads, n_kv_heads, head_dim, max_new) || window < 0 || !plan ||
      (reinterpret_cast<uintptr_t>(plan) & 255) || (n_req > 0 && (!q_off || !kv_len)))
    return SMETRIC_EINVAL;
  const PlanShape s = plan_shape(n_req, n_tokens, n_q_heads, n_kv_heads, head_dim, max_new);
  if (plan_bytes < s.plan_bytes) return SMETRIC_EWORKSPACE;
  char *p = static_cast<char *>(plan);
  PlanArgs a{q_off, kv_len, n_req, n_q_heads, n_kv_heads, n_q_heads / n_kv_heads, s.rows, window, s.target,
             (s.rows == FEW_ROWS ? FEW_MIN_KEYS : MANY_MIN_KEYS) / KEY_STEP, n_tokens, n_req ? s.max_tiles : 0,
             s.max_items, s.max_splits, s.max_parts, reinterpret_cast<PlanHdr *>(p),
             reinterpret_cast<PlanItem *>(p + s.off_items), reinterpret_cast<PlanSplit *>(p + s.off_splits), status};
  plan_kernel<<<1, PT, 0, stream>>>(a);
  return hip_status(hipGetLastError());
}

extern "C" int smetric_attend(int32_t dtype, const smetric_kv_cache *cache, const smetric_batch *batch, int32_t n_q_heads,
                              const smetric_heads *q, const smetric_heads *out, float *lse, float scale, int32_t max_new,
                              int32_t window, const void *plan, uint64_t plan_bytes, void *workspace, uint64_t ws_bytes,
                              int32_t *status, hipStream_t stream) {
  if (!cache_ok(cache, dtype) || !batch_ok(batch) || window < 0 || !(scale > 0.0f) || !isfinite(scale) ||
      !shape_ok(batch->n_req, batch->n_tokens, n_q_heads, cache->n_kv_heads, cache->head_dim, max_new))
    return SMETRIC_EINVAL;
  if (batch->n_tokens == 0) return SMETRIC_OK;
  if (!heads_ok(q) || !heads_ok(out) || !plan || (reinterpret_cast<uintptr_t>(plan) & 255) ||
      (reinterpret_cast<uintptr_t>(workspace) & 255))
    return SMETRIC_EINVAL;
  const PlanShape s =
      plan_shape(batch->n_req, batch->n_tokens, n_q_heads, cache->n_kv_heads, cache->head_dim, max_new);
  if (plan_bytes < s.plan_bytes || ws_bytes < s.ws_bytes || !workspace) return SMETRIC_EWORKSPACE;
  if (s.max_items * cache->n_kv_heads > 0x7FFFFFFF) return SMETRIC_EINVAL;
  const char *p = static_cast<const char *>(plan);
  AttendArgs a{};
  a.hdr = reinterpret_cast<const PlanHdr *>(p);
  a.items = reinterpret_cast<const PlanItem *>(p + s.off_items);
  a.splits = reinterpret_cast<const PlanSplit *>(p + s.off_splits);
  a.cache = cache_view(cache, batch);
  a.q = heads_view(q);
  a.out = heads_view(out);
  a.lse = lse;
  const int64_t part_rows = s.max_parts * cache->n_kv_heads * s.rows;
  a.parts.acc = static_cast<float *>(workspace);
  a.parts.ml = reinterpret_cast<f32x2 *>(a.parts.acc + part_rows * cache->head_dim);
  a.n_tokens = batch->n_tokens;
  a.n_req = batch->n_req;
  a.n_q = n_q_heads;
  a.n_kv = cache->n_kv_heads;
  a.group = n_q_heads / cache->n_kv_heads;
  a.rows = s.rows;
  a.window = window;
  a.scale_log2 = scale * 1.4426950408889634f;
  a.status = status;
  const bool kv8 = cache->dtype == SMETRIC_E4M3;
  int rc = s.rows == FEW_ROWS ? launch_few(a, dtype, kv8, cache->head_dim, s.max_items, stream)
                              : launch_many(a, dtype, kv8, cache->head_dim, s.max_items, stream);
  if (rc != SMETRIC_OK) return rc;
  return dtype == SMETRIC_BF16 ? launch_join<Bf16>(a, cache->head_dim, s.max_splits, stream)
                               : launch_join<F16>(a, cache->head_dim, s.max_splits, stream);
}
