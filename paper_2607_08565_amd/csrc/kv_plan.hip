// The plan of an attention step: which rows and keys each workgroup takes, and the joining
// of the tiles whose keys were cut.
//
// The plan depends on the lengths alone, so one serves all layers of a step.  One workgroup
// makes it: it totals the tiles' costs (key steps, and what a tile costs besides), decides on
// shares or whole tiles, and every tile's thread writes its pieces at places from scans over the tiles,
// all threads together those of tiles that are cut often: 8 to 11 us also where one request of
// 131,072 tokens is all that is cut (34 us by the tile's thread alone).
#include <math.h>

#include "kv_attend.h"

namespace smk {
namespace {

constexpr int PT = 512;
constexpr int32_t STAGED = 2048;   // requests whose offsets and lengths are kept in LDS
constexpr int32_t LONG_CUTS = 8;   // cuts of a tile, of which there are fewer than `target` in all, at most 512
constexpr int32_t MAX_LONG = 512 / LONG_CUTS;
constexpr int32_t CUT_COST = 8;    // steps: what a share's partial results cost, see whole_tiles (12: up to 7 % slower)

struct PlanArgs {
  const int64_t *q_off;
  const int32_t *kv_len;
  int32_t n_req, n_q, n_kv, group, dim, rows, rows_log2, window, target, min_steps, edge_steps, tile_cost;
  int64_t n_tokens, max_tiles, max_items, max_groups, max_splits, max_parts;
  PlanHdr *hdr;
  PlanItem *items;
  PlanSplit *splits;
  int32_t *first;
  int32_t *status;
};

struct Tile {
  int32_t req, tile, n_new, kv_len, tok0, k0, k1, steps;  // req < 0: the number belongs to no tile
};
__device__ Tile tile_at(const PlanArgs &a, const int64_t *q_off, const int32_t *kv_len, int64_t g) {
  Tile t{-1, 0, 0, 0, 0, 0, 0, 0};
  int32_t lo = 0, hi = a.n_req - 1;  // the last request whose numbers begin at or before g
  while (lo < hi) {
    const int32_t mid = (lo + hi + 1) / 2;
    if ((q_off[mid] * a.group >> a.rows_log2) + mid <= g)
      lo = mid;
    else
      hi = mid - 1;
  }
  const int64_t q0 = q_off[lo];
  const int64_t n = q_off[lo + 1] - q0, in = g - ((q0 * a.group >> a.rows_log2) + lo);
  const int64_t tiles = (n * a.group + a.rows - 1) >> a.rows_log2;
  if (in < 0 || in >= tiles) return t;
  t.req = lo;
  t.tile = int32_t(tiles - 1 - in);  // long ones first
  t.n_new = int32_t(n);
  t.tok0 = int32_t(q0);
  t.kv_len = kv_len[lo];
  const uint32_t row0 = uint32_t(t.tile) << a.rows_log2;
  uint32_t last = row0 + a.rows;
  if (last > uint32_t(t.n_new) * a.group) last = uint32_t(t.n_new) * a.group;
  const int32_t first = t.kv_len - t.n_new + int32_t(row0 / uint32_t(a.group));  // places of the tile's first and last token
  t.k1 = t.kv_len - t.n_new + int32_t((last - 1) / uint32_t(a.group)) + 1;
  t.k0 = a.window > 0 && first - a.window + 1 > 0 ? first - a.window + 1 : 0;
  if (t.k1 <= t.k0) t.k0 = t.k1 = 0;
  t.steps = (t.k1 + KEY_STEP - 1) / KEY_STEP - t.k0 / KEY_STEP;
  return t;
}

// A tile's steps, and what it costs besides (its queries, first pages and output), in steps.
__device__ __forceinline__ int32_t cost_of(const PlanArgs &a, const Tile &t) {
  return (t.steps > 0 ? t.steps : 1) + a.tile_cost;
}

// floor(x / d) for 0 <= x < 2^52: a quotient in 64-bit floats is at most one off.
__device__ __forceinline__ int64_t quotient(int64_t x, int64_t d) {
  int64_t q = int64_t(double(x) / double(d));
  q -= q * d > x;
  q += (q + 1) * d <= x;
  return q;
}

// Sum of x over the workgroup's earlier threads; total: over all.
__device__ int64_t scan(int64_t x, int64_t &total, int64_t *sh) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t a = x;
#pragma unroll
  for (int m = 1; m < 64; m *= 2) {
    const int64_t u = __shfl_up(a, m, 64);
    if (lane >= m) a += u;
  }
  if (lane == 63) sh[wave] = a;
  __syncthreads();
  int64_t before = 0;
  total = 0;
  for (int w = 0; w < PT / 64; ++w) {
    const int64_t v = sh[w];
    before += w < wave ? v : 0;
    total += v;
  }
  __syncthreads();
  return before + a - x;
}

// Whether each tile gets a workgroup of its own.  Estimates, in steps: with n workgroups at
// once, whole tiles take ceil(tiles / n) rounds of the mean, at least the longest; or, as
// early ends are filled, the even share and half the longest.  Shares take the even share
// and what their cuts cost: partial sums written, read and joined, and a tile's start.
__device__ bool whole_tiles(int64_t cost, int64_t tiles, int32_t longest, int32_t n) {
  const int64_t share = quotient(cost + n - 1, n), rounds = quotient(tiles + n - 1, n);
  int64_t whole = tiles > 0 ? rounds * quotient(cost + tiles - 1, tiles) : 0;
  if (rounds > 1 && whole > share + longest / 2) whole = share + longest / 2;
  if (whole < longest) whole = longest;
  return whole <= share + CUT_COST;
}

// A tile's pieces and the workgroups whose shares begin in it, written by threads i, i + step, ...:
// shares' ends at multiples of `share`, of which w_lo .. w_hi cut the tile, whose costs begin at `at`.
struct Cut {
  Tile t;
  int32_t cuts, cost;
  int64_t at, w_lo, base, part0;
};
__device__ void write_pieces(const PlanArgs &a, const Cut &c, int64_t share, int64_t n_groups, int32_t i0, int32_t step) {
  const Tile &t = c.t;
  const int32_t k = t.k0 / KEY_STEP;
  for (int32_t i = i0; i <= c.cuts && c.base + i < a.max_items; i += step) {
    const int32_t c0 = i ? int32_t((c.w_lo + i - 1) * share - c.at) - a.tile_cost : 0;
    const int32_t c1 = i < c.cuts ? int32_t((c.w_lo + i) * share - c.at) - a.tile_cost : 0;
    a.items[c.base + i] = PlanItem{t.req, t.tok0, t.n_new, t.kv_len, t.tile, i == 0 ? t.k0 : (k + c0) * KEY_STEP,
                                   i == c.cuts ? t.k1 : (k + c1) * KEY_STEP, c.cuts ? int32_t(c.part0 + i) : -1};
  }
  for (int64_t w = quotient(c.at + share - 1, share) + i0; w * share < c.at + c.cost && w < n_groups && w < a.max_groups; w += step)
    a.first[w] = int32_t(c.base + (w < c.w_lo ? 0 : w > c.w_lo + c.cuts - 1 ? c.cuts + 1 : w - c.w_lo + 1));
}

__global__ __launch_bounds__(PT) void plan_kernel(PlanArgs a) {
  static_assert(FEW_ROWS == 1 << 4 && MANY_ROWS == 1 << 7, "rows_log2");
  __shared__ int64_t sh64[PT / 64];
  __shared__ int64_t off_l[STAGED + 1];
  __shared__ int32_t len_l[STAGED];
  // tiles of many pieces, which all threads write together (one thread's 130 of a long request take it 25 us)
  __shared__ Cut cuts_l[MAX_LONG];
  __shared__ int bad, longest, n_long;
  if (threadIdx.x == 0) bad = longest = n_long = 0;
  __syncthreads();
  bool wrong = false;
  const bool staged = a.n_req <= STAGED;
  for (int32_t r = threadIdx.x; r < a.n_req; r += PT) {
    const int64_t q0 = a.q_off[r], q1 = a.q_off[r + 1];
    const int32_t len = a.kv_len[r];
    wrong |= q0 < 0 || q1 < q0 || q1 > a.n_tokens || (r == 0 && q0 != 0) || (r == a.n_req - 1 && q1 != a.n_tokens) ||
             len < 0 || len > MAX_PLACES;
    if (staged) {
      off_l[r + 1] = q1;
      len_l[r] = len;
      if (r == 0) off_l[0] = q0;
    }
  }
  if (wrong) bad = 1;
  __syncthreads();
  const int64_t *q_off = staged ? off_l : a.q_off;
  const int32_t *kv_len = staged ? len_l : a.kv_len;
  int64_t n_items = 0, n_splits = 0, n_parts = 0, n_groups = 0;
  if (!bad) {
    int64_t mine = 0;
    int32_t top = 0, count = 0;
    Tile t{};
    for (int64_t g = threadIdx.x; g < a.max_tiles; g += PT) {
      t = tile_at(a, q_off, kv_len, g);
      if (t.req < 0) continue;
      const int32_t c = cost_of(a, t);
      mine += c;
      top = c > top ? c : top;
      ++count;
    }
    atomicMax(&longest, top);
    int64_t cost, tiles;
    const int64_t before = scan(mine, cost, sh64);
    if (a.max_tiles <= PT)
      tiles = __syncthreads_count(count);
    else
      scan(count, tiles, sh64);
    const int32_t least = a.min_steps + a.tile_cost;
    int64_t groups = quotient(cost + least - 1, least);
    if (groups > a.target) groups = a.target;
    if (groups < 1) groups = 1;
    const int64_t share = cost > 0 ? quotient(cost + groups - 1, groups) : 1;
    const bool whole = whole_tiles(cost, tiles, longest, a.target);
    n_groups = whole ? tiles : quotient(cost + share - 1, share);
    const int32_t edge = a.edge_steps + a.tile_cost;
    int64_t at0 = 0;
    for (int64_t g0 = 0; g0 < a.max_tiles; g0 += PT) {
      const int64_t g = g0 + threadIdx.x;
      if (a.max_tiles > PT || g >= a.max_tiles) t.req = -1;
      if (a.max_tiles > PT && g < a.max_tiles) t = tile_at(a, q_off, kv_len, g);
      const int64_t c = t.req < 0 ? 0 : cost_of(a, t);
      int64_t at = before;
      if (a.max_tiles > PT) {
        int64_t all;
        at = at0 + scan(c, all, sh64);
        at0 += all;
      }
      // shares' ends at multiples of `share`: w_lo .. w_hi cut this tile
      int64_t w_lo = 0, w_hi = -1;
      if (t.req >= 0 && !whole) {
        w_lo = quotient(at + edge + share - 1, share);
        w_hi = at + c < edge ? -1 : quotient(at + c - edge, share);
        if (w_hi >= n_groups) w_hi = n_groups - 1;
      }
      const int32_t cuts = w_hi >= w_lo ? int32_t(w_hi - w_lo + 1) : 0, pieces = t.req < 0 ? 0 : cuts + 1;
      // in one scan: pieces, those of cut tiles (at most 2 target, 16 bits), cut tiles (16 bits)
      int64_t all_n;
      const int64_t n = scan(int64_t(pieces) << 32 | int64_t(cuts ? pieces : 0) << 16 | (cuts > 0), all_n, sh64);
      const int64_t base = n_items + (n >> 32), part0 = n_parts + (n >> 16 & 0xFFFF), split_at = n_splits + (n & 0xFFFF);
      if (cuts && split_at < a.max_splits)
        a.splits[split_at] = PlanSplit{t.tok0, t.n_new, t.tile, int32_t(part0), pieces, {0, 0, 0}};
      if (t.req >= 0 && whole) {
        if (base < a.max_items) a.items[base] = PlanItem{t.req, t.tok0, t.n_new, t.kv_len, t.tile, t.k0, t.k1, -1};
        if (base < a.max_groups) a.first[base] = int32_t(base);
      } else if (t.req >= 0) {
        // (w_lo as the divisions above give it also where nothing is cut: `first` goes by it)
        const Cut cut{t, cuts, int32_t(c), at, w_lo, base, part0};
        if (cuts < LONG_CUTS)
          write_pieces(a, cut, share, n_groups, 0, 1);
        else
          cuts_l[atomicAdd(&n_long, 1)] = cut;
      }
      __syncthreads();
      const int32_t longs = n_long;
      for (int32_t i = 0; i < longs; ++i) write_pieces(a, cuts_l[i], share, n_groups, threadIdx.x, PT);
      __syncthreads();
      if (threadIdx.x == 0) n_long = 0;  // (the next scan's barriers come before it is counted on)
      n_items += all_n >> 32;
      n_parts += all_n >> 16 & 0xFFFF;
      n_splits += all_n & 0xFFFF;
    }
  }
  if (threadIdx.x == 0) {
    PlanHdr h{};
    h.err = bad ? SMETRIC_EINVAL : SMETRIC_OK;
    if (n_items > a.max_items || n_splits > a.max_splits || n_parts > a.max_parts || n_groups > a.max_groups)
      h.err = SMETRIC_EINTERNAL;
    else
      a.first[n_groups] = int32_t(n_items);
    h.n_items = int32_t(n_items);
    h.n_splits = int32_t(n_splits);
    h.n_groups = int32_t(n_groups);
    h.n_req = a.n_req;
    h.n_q = a.n_q;
    h.n_kv = a.n_kv;
    h.rows = a.rows;
    h.dim = a.dim;
    h.window = a.window;
    h.n_tokens = a.n_tokens;
    *a.hdr = h;
    if (h.err) set_status(a.status, h.err);
  }
}

// Joins the parts of a cut tile: out = sum_p 2^(m_p - m) acc_p / sum_p 2^(m_p - m) l_p, in the
// order of the parts, l_p the sums of rounded weights (PartView); lse takes those of unrounded ones.
// D / 4 threads hold a row.  Tiles of many rows: the workgroup takes as many rows at once (each of a few parts).  Tiles of few rows, which may have hundreds of
// parts, and of many where a few long requests share all of the parts: it takes one row's parts
// side by side (2 requests of 7 new tokens over 47,760, 14 heads on 2: 44 us, so 7).
constexpr int32_t JOIN_GRID = 2048;
template <typename T, int D, bool FEW>
__device__ __forceinline__ void write_row(const AttendArgs &a, const PlanSplit &s, int32_t in_req, int32_t kvh, int sub,
                                          f32x4 acc, float m, float l, float exact, float more) {
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  const int64_t t = int64_t(s.tok0) + in_req / a.group;
  const int32_t head = kvh * a.group + in_req % a.group;
  *reinterpret_cast<u32x2 *>(a.out.data + t * a.out.token + head * a.out.head + sub * 4) =
      u32x2{T::pack(acc[0] * inv, acc[1] * inv), T::pack(acc[2] * inv, acc[3] * inv)};
  if (a.lse && sub == 0) a.lse[t * a.n_q + head] = lse_of(m, exact, FEW ? T::FEW_SHIFT : T::MANY_SHIFT, more);
}
template <typename T, int D, bool FEW>
__global__ __launch_bounds__(256) void join_kernel(AttendArgs a) {
  constexpr int TPP = D / 4, SIDE = 256 / TPP, BLOCKS = FEW ? FEW_ROWS : MANY_ROWS / SIDE;
  __shared__ f32x4 sh[256];
  __shared__ f32x2 shl[SIDE];
  // a short request's joining is a chain of round trips: the first unit's split is asked for with the header
  PlanSplit s = a.splits[blockIdx.x / a.n_kv / BLOCKS];
  const PlanHdr h = *a.hdr;
  if (!plan_fits(a, h)) return;
  const int64_t tiles = int64_t(h.n_splits) * a.n_kv;
  const bool alone = FEW || tiles * MANY_ROWS <= gridDim.x;  // a row a workgroup, all at once
  const int32_t blocks_log2 = __builtin_ctz(!FEW && alone ? MANY_ROWS : BLOCKS);
  const int64_t units = tiles << blocks_log2;
  const int32_t sub = threadIdx.x % TPP, side = threadIdx.x / TPP;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int64_t in_tile = u / a.n_kv;
    const int32_t kvh = int32_t(u - in_tile * a.n_kv), block = int32_t(in_tile & ((1 << blocks_log2) - 1));
    if (u != blockIdx.x || (!FEW && alone)) s = a.splits[in_tile >> blocks_log2];
    const int32_t row = alone ? block : block * SIDE + side;
    const int32_t in_req = s.tile * a.rows + row;
    const int64_t step = int64_t(a.n_kv) * a.rows, at = (int64_t(s.part0) * a.n_kv + kvh) * a.rows + row;
    if (in_req >= s.n_new * a.group) continue;  // (alone: the whole workgroup)
    const f32x4 *ml = a.parts.ml + at;
    const float *parts = a.parts.acc + at * D + sub * 4;
    float m = -INFINITY;
    // (alone: a side's first part is asked for with the maxima)
    const bool has = alone && side < s.n_parts;
    const f32x4 ml0 = has ? ml[side * step] : f32x4{-INFINITY, 0.0f, 0.0f, 0.0f};
    const f32x4 v0 = has ? *reinterpret_cast<const f32x4 *>(parts + side * step * D) : f32x4{0, 0, 0, 0};
    if (alone) {
      for (int32_t p = threadIdx.x & 63; p < s.n_parts; p += 64) m = fmaxf(m, ml[p * step].x);
#pragma unroll
      for (int i = 1; i < 64; i *= 2) m = fmaxf(m, __shfl_xor(m, i, 64));
    } else {
      for (int32_t p = 0; p < s.n_parts; ++p) m = fmaxf(m, ml[p * step].x);
    }
    const float ms = m == -INFINITY ? 0.0f : m;
    f32x4 acc{0, 0, 0, 0};
    float l = 0.0f, exact = 0.0f;
    float more = ml0.w;  // (the same in all parts)
    if (has) {
      const float w = exp2f(ml0.x - ms);
      l = w * ml0.y;
      exact = w * ml0.z;
      acc = f32x4{w * v0[0], w * v0[1], w * v0[2], w * v0[3]};
    }
#pragma unroll 4
    for (int32_t p = alone ? side + SIDE : 0; p < s.n_parts; p += alone ? SIDE : 1) {
      const f32x4 x = ml[p * step];
      const f32x4 v = *reinterpret_cast<const f32x4 *>(parts + p * step * D);
      const float w = exp2f(x.x - ms);
      l = fmaf(w, x.y, l);
      exact = fmaf(w, x.z, exact);
      more = x.w;
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[i] = fmaf(w, v[i], acc[i]);
    }
    if (alone) {
      sh[threadIdx.x] = acc;
      if (sub == 0) shl[side] = f32x2{l, exact};
      __syncthreads();
      if (side == 0) {
#pragma unroll
        for (int i = 1; i < SIDE; ++i) {
          acc += sh[i * TPP + sub];
          l += shl[i].x;
          exact += shl[i].y;
        }
      }
    }
    if (!alone || side == 0) write_row<T, D, FEW>(a, s, in_req, kvh, sub, acc, m, l, exact, more);
    if (alone) __syncthreads();
  }
}

template <typename T, int D>
int launch_join_d(const AttendArgs &a, int64_t max_splits, hipStream_t stream) {
  constexpr int SIDE = 256 / (D / 4);
  const bool few = a.rows == FEW_ROWS;
  const int64_t units = max_splits * a.n_kv * (few ? FEW_ROWS : MANY_ROWS / SIDE);
  const dim3 grid(uint32_t(units < JOIN_GRID ? units : JOIN_GRID));
  if (few)
    join_kernel<T, D, true><<<grid, 256, 0, stream>>>(a);
  else
    join_kernel<T, D, false><<<grid, 256, 0, stream>>>(a);
  return hip_status(hipGetLastError());
}
template <typename T>
int launch_join(const AttendArgs &a, int32_t head_dim, int64_t max_splits, hipStream_t stream) {
  return head_dim == 64 ? launch_join_d<T, 64>(a, max_splits, stream)
                        : head_dim == 128 ? launch_join_d<T, 128>(a, max_splits, stream) : launch_join_d<T, 256>(a, max_splits, stream);
}

// A window of all places is none: what the kernels subtract from a place stays in 32 bits.
int32_t window_of(int32_t window) { return window >= MAX_PLACES ? 0 : window; }

// Caps that stay far from float32's ends, as their squares do.
constexpr float CAP_MIN = 0x1p-20f, CAP_MAX = 0x1p20f;

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
  PlanArgs a{q_off, kv_len, n_req, n_q_heads, n_kv_heads, n_q_heads / n_kv_heads, head_dim, s.rows, s.rows == FEW_ROWS ? 4 : 7, window_of(window), s.target,
             s.rows == FEW_ROWS ? FEW_MIN_STEPS : MANY_MIN_STEPS, s.rows == FEW_ROWS ? FEW_EDGE_STEPS : MANY_EDGE_STEPS,
             s.rows == FEW_ROWS ? FEW_TILE_COST : MANY_TILE_COST,
             n_tokens, n_req ? s.max_tiles : 0, s.max_items, s.max_groups, s.max_splits, s.max_parts,
             reinterpret_cast<PlanHdr *>(p), reinterpret_cast<PlanItem *>(p + s.off_items),
             reinterpret_cast<PlanSplit *>(p + s.off_splits), reinterpret_cast<int32_t *>(p + s.off_first), status};
  plan_kernel<<<1, PT, 0, stream>>>(a);
  return hip_status(hipGetLastError());
}

extern "C" int smetric_attend_scores(int32_t dtype, const smetric_kv_cache *cache, const smetric_batch *batch,
                                     int32_t n_q_heads, const smetric_heads *q, const smetric_heads *out, float *lse,
                                     float scale, const smetric_scores *scores, int32_t max_new, int32_t window,
                                     const void *plan, uint64_t plan_bytes, void *workspace, uint64_t ws_bytes,
                                     int32_t *status, hipStream_t stream) {
  if (!scores || !(scores->cap == 0.0f || (scores->cap >= CAP_MIN && scores->cap <= CAP_MAX)) ||
      reinterpret_cast<uintptr_t>(scores->slopes) % 4)
    return SMETRIC_EINVAL;
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
  if (s.max_groups * cache->n_kv_heads > 0x7FFFFFFF) return SMETRIC_EINVAL;
  const char *p = static_cast<const char *>(plan);
  AttendArgs a{};
  a.hdr = reinterpret_cast<const PlanHdr *>(p);
  a.items = reinterpret_cast<const PlanItem *>(p + s.off_items);
  a.splits = reinterpret_cast<const PlanSplit *>(p + s.off_splits);
  a.first = reinterpret_cast<const int32_t *>(p + s.off_first);
  a.cache = cache_view(cache, batch);
  a.q = heads_view(q);
  a.out = heads_view(out);
  a.lse = lse;
  const int64_t part_rows = s.max_parts * cache->n_kv_heads * s.rows;
  a.parts.acc = static_cast<float *>(workspace);
  a.parts.ml = reinterpret_cast<f32x4 *>(a.parts.acc + part_rows * cache->head_dim);
  a.n_tokens = batch->n_tokens;
  a.n_req = batch->n_req;
  a.n_q = n_q_heads;
  a.n_kv = cache->n_kv_heads;
  a.group = n_q_heads / cache->n_kv_heads;
  a.rows = s.rows;
  a.dim = cache->head_dim;
  a.window = window_of(window);
  a.scale_log2 = finite_factor(scale * LOG2E);
  a.cap_log2 = scores->cap * LOG2E;
  a.slopes = scores->slopes;
  a.status = status;
  const bool few = s.rows == FEW_ROWS;
  const auto launch = scores->cap > 0.0f || scores->slopes ? few ? launch_few_scores : launch_many_scores
                                                           : few ? launch_few : launch_many;
  const int rc = launch(a, dtype, pages_of(cache), cache->head_dim, s.max_groups, stream);
  if (rc != SMETRIC_OK) return rc;
  return dtype == SMETRIC_BF16 ? launch_join<Bf16>(a, cache->head_dim, s.max_splits, stream)
                               : launch_join<F16>(a, cache->head_dim, s.max_splits, stream);
}

extern "C" int smetric_attend(int32_t dtype, const smetric_kv_cache *cache, const smetric_batch *batch, int32_t n_q_heads,
                              const smetric_heads *q, const smetric_heads *out, float *lse, float scale, int32_t max_new,
                              int32_t window, const void *plan, uint64_t plan_bytes, void *workspace, uint64_t ws_bytes,
                              int32_t *status, hipStream_t stream) {
  const smetric_scores plain{0.0f, nullptr};
  return smetric_attend_scores(dtype, cache, batch, n_q_heads, q, out, lse, scale, &plain, max_new, window, plan, plan_bytes,
                               workspace, ws_bytes, status, stream);
}
