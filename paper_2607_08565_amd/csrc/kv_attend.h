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
  // per part, key-value head and row: the sums over its keys, then their maximum and weight
  s.ws_bytes = uint64_t(s.max_parts) * n_kv * s.rows * (head_dim + 2) * 4;
  return s;
}

struct PartView {
  float *acc;  // [part][kv head][row][head_dim]
  f32x2 *ml;   // [part][kv head][row]: maximum (in powers of two), sum of weights
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
  int32_t *status;
};
__device__ __forceinline__ bool plan_fits(const AttendArgs &a, const PlanHdr &h) {
  return h.err == 0 && h.n_req == a.n_req && h.n_q == a.n_q && h.n_kv == a.n_kv && h.rows == a.rows &&
         h.dim == a.dim && h.window == a.window && h.n_tokens == a.n_tokens;
}

// lse from a row's maximum (in powers of two) and sum of weights times 2^shift.
__device__ __forceinline__ float lse_of(float m, float l, float shift) {
  return l == 0.0f ? -INFINITY : (m + log2f(l * exp2f(-shift))) * 0.693147180559945309f;
}

// Launches (one per file).  Grids cover plan_shape's bounds; workgroups past the plan's
// counts end at once.
int launch_few(const AttendArgs &a, int32_t dtype, bool kv8, int32_t head_dim, int64_t max_groups, hipStream_t stream);
int launch_many(const AttendArgs &a, int32_t dtype, bool kv8, int32_t head_dim, int64_t max_groups, hipStream_t stream);

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
template <typename T, bool KV8>
__device__ __forceinline__ f32x4 four_values(uint64_t row, int c) {
  u32x2 x;
  if (KV8) {
    const uint32_t y = *reinterpret_cast<const uint32_t *>(row + c);
    x = u32x2{T::template from_e4m3<false>(y), T::template from_e4m3<true>(y)};
  } else {
    x = *reinterpret_cast<const u32x2 *>(row + 2 * c);
  }
  return f32x4{T::lo(x.x), T::hi(x.x), T::lo(x.y), T::hi(x.y)};
}

// 16 lanes read four rows' 16 columns of 16-bit values from LDS, each lane's address a row's
// (lane / 4) four columns (lane % 4): lane i gets column i of the four rows.
typedef __attribute__((ext_vector_type(4))) short s16x4;
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
