// The plan of an attention step and what its kernels share.  Not part of the ABI.
#pragma once

#include "kv_common.h"

namespace smk {

// Rows.  The n new tokens of a request and the G query heads that read one key-value head
// make n G rows of one matrix product, row = token * G + head: the heads share every key
// that is loaded.  Rows are cut into tiles, a tile's visible keys into parts:
//   few rows   16 rows a tile, one workgroup's wavefronts each taking keys of their own
//              (decoding, drafts): kv_few.hip
//   many rows  128 rows a tile, the wavefronts each taking rows of their own and sharing
//              the keys through LDS (prompts' chunks): kv_many.hip
constexpr int FEW_ROWS = 16, MANY_ROWS = 128;
constexpr int KEY_STEP = 64;  // parts begin at multiples of this many keys
inline int32_t rows_per_tile(int32_t n_q, int32_t n_kv, int32_t max_new) {
  return int64_t(max_new) * (n_q / n_kv) <= FEW_ROWS ? FEW_ROWS : MANY_ROWS;
}

// One piece of work: the keys [k0, k1) of one tile, for every key-value head.
struct PlanItem {
  int32_t req, tok0, n_new, kv_len;  // the request, its first new token, its lengths
  int32_t tile;
  int32_t k0, k1;
  int32_t part;  // slot for a partial result, -1: the tile's only piece, writes the output
};
struct PlanSplit {  // a tile of more than one piece
  int32_t tok0, n_new, tile, part0, n_parts, pad[3];
};
struct PlanHdr {
  int32_t err, n_items, n_splits, n_groups;
  int32_t n_req, n_q, n_kv, rows, window, dim;
  int64_t n_tokens;
  int32_t pad[20];
};
static_assert(sizeof(PlanHdr) == 128 && sizeof(PlanItem) == 32 && sizeof(PlanSplit) == 32, "plan layout");

// Workgroups of a step, over all key-value heads: as many as run at once (on each of 256
// compute units two, one with heads of 256: their registers), each with an equal share of the
// key steps in order, so that all end together; a share begins and ends within a tile, which is
// then in pieces, and may hold several tiles.  Heads of 64 would leave room for three, which is
// no faster (4 chunks of 2,048 over 8-bit pages: 732 us, with two 694); heads of 256 with twice
// as many shares as run at once: 2 chunks of 2,048 910 us for 858, 65,536 keys 59 for 53.
// Two exceptions: no share is smaller than MIN_STEPS, and a cut this near a tile's end goes to
// the end (EDGE_STEPS).  Few rows: a step is half a block of each wavefront, so two make the
// shortest share that occupies all four (one token over 1,025 keys: 5.8 us, with shares of four
// steps 8.3, of eight 11.6).  Many rows: a short chunk is a chain of steps of one workgroup, so
// two again (32 tokens over 1,032 keys: 17 us, with shares of eight steps 22; 64 over 4,064 at heads
// of 128 23 and 30; 30 over 2,030 at heads of 256 28 and 41; long chunks the same).
constexpr int32_t at_once(int32_t head_dim) { return head_dim == 256 ? 1 : 2; }
constexpr int32_t FEW_MIN_STEPS = 2, FEW_EDGE_STEPS = 1, FEW_TILE_COST = 0;
constexpr int32_t MANY_MIN_STEPS = 2, MANY_EDGE_STEPS = 1, MANY_TILE_COST = 2;

struct PlanShape {
  int32_t rows, target;  // rows per tile; workgroups aimed at per key-value head
  int64_t max_tiles, max_items, max_groups, max_splits, max_parts;
  uint64_t plan_bytes, ws_bytes;
  int64_t off_items, off_splits, off_first;
};
// Tiles: request r's are numbered from floor(q_off[r] G / rows) + r on, which leaves each
// request room for ceil(n G / rows) and needs no scan.  Shares have fewer than `target`
// inner ends, each of which cuts at most one tile: at most max_tiles + target pieces, target
// tiles of more than one, 2 target pieces of such tiles.
inline PlanShape plan_shape(int32_t n_req, int64_t n_tokens, int32_t n_q, int32_t n_kv, int32_t head_dim, int32_t max_new) {
  PlanShape s;
  s.rows = rows_per_tile(n_q, n_kv, max_new);
  s.target = 256 * at_once(head_dim) / n_kv;
  if (s.target < 1) s.target = 1;
  s.max_tiles = n_tokens * (n_q / n_kv) / s.rows + n_req;
  s.max_items = s.max_tiles + s.target;
  s.max_groups = s.max_tiles > s.target ? s.max_tiles : s.target;
  s.max_splits = s.target;
  s.max_parts = 2 * int64_t(s.target);
  s.off_items = sizeof(PlanHdr);
  s.off_splits = s.off_items + s.max_items * int64_t(sizeof(PlanItem));
  s.off_first = s.off_splits + s.max_splits * int64_t(sizeof(PlanSplit));
  s.plan_bytes = uint64_t(s.off_first + (s.max_groups + 1) * 4 + 255) / 256 * 256;
  // per part, key-value head and row: the sums over its keys, then their maximum and weights
  s.ws_bytes = uint64_t(s.max_parts) * n_kv * s.rows * (head_dim + 4) * 4;
  return s;
}

struct PartView {
  float *acc;  // [part][kv head][row][head_dim]
  f32x4 *ml;   // [part][kv head][row]: maximum (in powers of two), sum of rounded weights, of unrounded ones (for lse); what lse is more (Bias)
};
struct AttendArgs {
  const PlanHdr *hdr;
  const PlanItem *items;
  const PlanSplit *splits;
  const int32_t *first;  // workgroup -> its first piece
  CacheView cache;
  HeadsView q, out;
  float *lse;
  PartView parts;
  int64_t n_tokens;
  int32_t n_req, n_q, n_kv, group;  // group = n_q / n_kv
  int32_t rows, dim, window;
  float scale_log2;  // scale * log2(e)
  float cap_log2;    // cap * log2(e), 0: scores are not capped
  const float *slopes;  // of the query heads, or NULL
  int32_t *status;
};
__device__ __forceinline__ bool plan_fits(const AttendArgs &a, const PlanHdr &h) {
  return h.err == 0 && h.n_req == a.n_req && h.n_q == a.n_q && h.n_kv == a.n_kv && h.rows == a.rows &&
         h.dim == a.dim && h.window == a.window && h.n_tokens == a.n_tokens;
}

// lse from a row's maximum (in powers of two) and sum of weights times 2^shift; more: Bias.
__device__ __forceinline__ float lse_of(float m, float l, float shift, float more) {
  return l == 0.0f ? -INFINITY : (m + log2f(l * exp2f(-shift)) + more) * 0.693147180559945309f;
}

// Launches (one per file; those of other scores apart).  Grids cover plan_shape's bounds;
// workgroups past the plan's counts end at once.
int launch_few(const AttendArgs &a, int32_t dtype, Pages pages, int32_t head_dim, int64_t max_groups, hipStream_t stream);
int launch_many(const AttendArgs &a, int32_t dtype, Pages pages, int32_t head_dim, int64_t max_groups, hipStream_t stream);
int launch_few_scores(const AttendArgs &a, int32_t dtype, Pages pages, int32_t head_dim, int64_t max_groups, hipStream_t stream);
template <typename T>  // (a file each)
int launch_many_scored(const AttendArgs &a, Pages pages, int32_t head_dim, int64_t max_groups, hipStream_t stream);
template <>
int launch_many_scored<Bf16>(const AttendArgs &a, Pages pages, int32_t head_dim, int64_t max_groups, hipStream_t stream);
template <>
int launch_many_scored<F16>(const AttendArgs &a, Pages pages, int32_t head_dim, int64_t max_groups, hipStream_t stream);
inline int launch_many_scores(const AttendArgs &a, int32_t dtype, Pages pages, int32_t head_dim, int64_t max_groups, hipStream_t stream) {
  return dtype == SMETRIC_BF16 ? launch_many_scored<Bf16>(a, pages, head_dim, max_groups, stream)
                               : launch_many_scored<F16>(a, pages, head_dim, max_groups, stream);
}

// Where a place's keys and values are in memory, and the exponents of E2M1 pages.
struct Place {
  uint64_t k, v, k_exp, v_exp;
};
// A page outside the cache is page 0; returns whether it is one.
template <Pages KV>
__device__ __forceinline__ bool find_place(const AttendArgs &a, const int32_t *table, int32_t kvh, int32_t key, Place &p) {
  const int32_t page = page_of(a.cache.ps, key);
  int32_t id = table[page];
  const bool outside = uint32_t(id) >= uint32_t(a.cache.n_pages);
  if (outside) id = 0;
  const int32_t slot = key - page * a.cache.ps.size;
  const auto at = [&](const PageSide &s) {
    return reinterpret_cast<uint64_t>(s.base + kvh * s.head) + id * s.page + slot * s.token;
  };
  p.k = at(a.cache.k);
  p.v = at(a.cache.v);
  if (KV == PAGES4) {
    p.k_exp = at(a.cache.k_exp);
    p.v_exp = at(a.cache.v_exp);
  }
  return outside;
}

// What a lane takes of a row of E2M1 at once: 16 bytes, a group with one exponent; of the 32 bytes of
// a head of 64 half a group, so that 16 rows are a wavefront's load as with the others.
constexpr int piece4(int head_dim) { return head_dim == 64 ? 8 : 16; }
template <int BYTES>
__device__ __forceinline__ u32x4 load_piece(uint64_t p, uint32_t offset = 0) {
  if (BYTES == 16) return from_memory<u32x4>(p, offset);
  const u32x2 x = from_memory<u32x2>(p, offset);
  return u32x4{x.x, x.y, 0, 0};
}
__device__ __forceinline__ uint32_t load_exp(uint64_t p, uint32_t offset = 0) { return from_memory<uint8_t>(p, offset); }

// The four words of a lane's load of 4-bit components in the order in which they, widened, go to LDS as its
// 16-byte pieces: word n ^ flip as the n-th.  A write of 16 bytes a lane takes 8 lanes at a time (as the
// counters of conflicts say), which meet no bank twice if their pieces differ modulo 128 bytes:
// neighbouring lanes' pieces are 4 apart, and rows' exchanges alone leave some of them on one another.
__device__ __forceinline__ u32x4 flipped(u32x4 x, int flip) {
  x = flip & 2 ? u32x4{x.z, x.w, x.x, x.y} : x;
  return flip & 1 ? u32x4{x.y, x.x, x.w, x.z} : x;
}

// x, computed again in every step: what follows from it is not kept in registers across them.
__device__ __forceinline__ int again(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// A factor of scores as float32 holds it: 0 times it is 0, NaN stays.
__host__ __device__ __forceinline__ float finite_factor(float x) {
  return x > 0x1.fffffep127f ? 0x1.fffffep127f : x < -0x1.fffffep127f ? -0x1.fffffep127f : x;
}

// Other scores (smetric_attend_scores), in powers of two: of x = q . k, sc = scale log2(e) (and the keys'
// scale), the capped score, cap tanh(scale x / cap) = cap - 2 cap / (1 + exp(2 scale x / cap)): both ends
// come out of the exponential's own overflow to infinity and underflow to zero.  It loses some 2^-23 of
// the cap, which a score of the cap's size does as well, and smaller ones of caps up to CAP_NEAR can
// spare (2^-17).  Of larger caps scores below a quarter of it come from the series of tanh(u) = u (1 - u^2 / 3
// + 2 u^4 / 15 - 17 u^6 / 315 + 62 u^8 / 2835), whose next term is below 2^-26: far().
constexpr float LOG2E = 1.4426950408889634f;
constexpr float CAP_NEAR = 64.0f * LOG2E;
struct Capped {
  float rate, cap, top;  // of the exponent, 2 sc / cap; cap log2(e); that less m, which scores are taken from
  float sc, inverse;     // far(): 1 / (cap log2(e))
  __device__ __forceinline__ Capped(const AttendArgs &a, float sc_, float m = 0.0f)
      : rate(a.cap_log2 > 0.0f ? finite_factor(2.8853900817779268f * sc_ / a.cap_log2) : 0.0f), cap(a.cap_log2),
        top(a.cap_log2 - m), sc(sc_), inverse(1.0f / a.cap_log2) {}
  __device__ __forceinline__ float operator()(float x) const {
    return fmaf(-2.0f * cap, __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * rate)), top);
  }
  __device__ __forceinline__ float far(float x) const {  // (m: 0)
    const float y = x * sc, u = y * inverse, z = u * u;
    const float series = fmaf(z, fmaf(z, fmaf(z, 62.0f / 2835.0f, -17.0f / 315.0f), 2.0f / 15.0f), -1.0f / 3.0f);
    return fabsf(u) < 0.25f ? fmaf(y, z * series, y) : (*this)(x);
  }
};

// A row's bias by distance, in powers of two: slope (key - place), taken less the largest that the row sees, at its
// own place or, of slopes below zero, at its first key.  That leaves the output as it is, and the keys that count
// most have a small one, of which float32 holds much: of 65,536 keys with a slope of -1/2 they would have 32,768.
// What was taken off is added to lse.
struct Bias {
  float slope;
  int32_t from;  // the key with a bias of 0
  __device__ __forceinline__ Bias(float s, int32_t place, int32_t lo) : slope(s), from(s < 0.0f && lo > 0 ? lo : s < 0.0f ? 0 : place) {}
  __device__ __forceinline__ float more(int32_t place) const { return slope * float(from - place); }
};

// Whether one of eight 16-bit floats is infinite or NaN: its exponent is all ones, and adding
// the exponent's lowest bit to the exponent alone carries into the (cleared) sign bit.
template <typename T>
__device__ __forceinline__ bool any_not_finite(u32x4 x) {
  uint32_t c = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) c |= (x[i] & T::EXP) + T::ONE_EXP;
  return (c & 0x80008000u) != 0;
}

// Eight 16-bit floats, zeros for those that are not finite.
template <typename T>
__device__ __forceinline__ u32x4 finite_only(u32x4 x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] &= ~((((x[i] & T::EXP) + T::ONE_EXP) >> 15 & 0x00010001u) * 0xFFFFu);
  return x;
}
__device__ __forceinline__ bool is_finite(float x) { return fabsf(x) < INFINITY; }
// Components c .. c + 3 of a row of values in memory.
template <typename T, Pages KV>
__device__ __forceinline__ f32x4 four_values(const Place &p, int c) {
  u32x2 x;
  if (KV == PAGES4) {
    const uint32_t y = from_memory<uint16_t>(p.v + c / 2);
    const float e = power_of(load_exp(p.v_exp + c / GROUP4));
    x = u32x2{T::template from_e2m1<0>(y, e), T::template from_e2m1<1>(y, e)};
  } else if (KV == PAGES8) {
    const uint32_t y = from_memory<uint32_t>(p.v + c);
    x = u32x2{T::template from_e4m3<false>(y), T::template from_e4m3<true>(y)};
  } else {
    x = from_memory<u32x2>(p.v + 2 * c);
  }
  return f32x4{T::lo(x.x), T::hi(x.x), T::lo(x.y), T::hi(x.y)};
}

// 16 lanes read four rows' 16 columns of 16-bit values from LDS, each lane's address a row's
// (lane / 4) four columns (lane % 4): lane i gets column i of the four rows.
__device__ __forceinline__ u32x2 read_transposed(const char *lds) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                       (__attribute__((address_space(3))) s16x4 *)lds));
}
__device__ __forceinline__ uint64_t read_lane(uint64_t x, int lane) {
  return uint64_t(uint32_t(__builtin_amdgcn_readlane(uint32_t(x), lane))) |
         uint64_t(uint32_t(__builtin_amdgcn_readlane(uint32_t(x >> 32), lane))) << 32;
}

// A piece, in scalar registers: the compiler cannot know that a load through a pointer that
// it also sees stores beside is the same for all lanes.
__device__ __forceinline__ int32_t uniform(int32_t x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ PlanItem uniform(const PlanItem &p) {
  return PlanItem{uniform(p.req),  uniform(p.tok0), uniform(p.n_new), uniform(p.kv_len),
                  uniform(p.tile), uniform(p.k0),   uniform(p.k1),    uniform(p.part)};
}

// An invalid plan's outputs: zeros and -inf, dealt to all workgroups.
template <int D>
__device__ __forceinline__ void write_nothing(const AttendArgs &a) {
  const int64_t rows = a.n_tokens * a.n_q, step = int64_t(gridDim.x) * blockDim.x;
  for (int64_t i = int64_t(blockIdx.x) * blockDim.x + threadIdx.x; i < rows * (D / 8); i += step) {
    const int64_t row = i / (D / 8), t = row / a.n_q, h = row - t * a.n_q;
    *reinterpret_cast<u32x4 *>(a.out.data + t * a.out.token + h * a.out.head + (i % (D / 8)) * 8) = u32x4{0, 0, 0, 0};
    if (a.lse && i % (D / 8) == 0) a.lse[row] = -INFINITY;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) set_status(a.status, SMETRIC_EINVAL);
}

}  // namespace smk
