// Attention of many rows over a paged cache: the chunk of a prompt that is left after its hit.
//
// Mathematics (smetric_kv.h): out = sum_j p_j v_j / sum_j p_j with p_j = 2^(c s_j - m), c =
// scale log2(e), in one pass over the keys: m is the running maximum of c s_j, and what was
// summed before a larger one appears is scaled down by 2^(old - new).
//
// Bound: 4 head_dim operations per row and key that sees it, on the matrix cores; the keys of
// a tile are read once per 128 rows.  A wavefront holds 32 rows: their queries, their sums
// (O^T) and one step's scores stay in registers; 64 keys and values at a time go through LDS,
// where the workgroup's wavefronts share them, double-buffered, the next 64 on their way from
// memory (16-bit ones straight to LDS, past the registers) during the current ones' products.
// The products are S^T = K Q^T and O^T = V^T P^T: a lane holds scores of one row only, so its
// maximum takes one lane exchange, and its weights are where the second product wants them --
// the order in which S^T leaves the keys is the order in which V^T is read, transposed, from LDS.
// Weights are rounded to the activations' type for it, as the matrix cores take 16-bit operands;
// their sum is not.
//
// Measured: 4,096 tokens over 16,384 (32 heads of 128) 923 to 986 us, 1,041 to 976 TFLOP/s, from card to card; on the
// faster one the library's product of matrices of 16,384 reaches 1,402, of 8,192 1,173.  The matrix cores work half of the cycles
// and the vector instructions about as long (33 exponentials, 32 sums, 31 products and 16
// maxima a step of 32 matrix instructions), on two wavefronts that overlap them in part, at a
// clock that falls under the load (1.9 GHz).  With the keys always in the nearest cache it takes
// 5 % less, without the exponentials 8 %, without the maximum 5 %.  Heads of 64 do half the
// products for the same weights: 24 requests with up to 1,000 new tokens 108 to 112 us, 370 to 383 TFLOP/s.
#include <math.h>

#include <type_traits>

#include "kv_attend.h"

namespace smk {
namespace {

constexpr int MW = 4;         // wavefronts
constexpr int MT = 64 * MW;   // threads
constexpr int KT = KEY_STEP;  // keys of a step

__device__ __forceinline__ u32x2 swap32(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(a, b, false, false));
}

// Two times 64 lanes' 16 bytes, of keys and of values, from memory to 1 KB of LDS each, past the
// registers.  The instructions have no output the compiler could take for written; what waits for
// them is arrived().  (With the compiler's builtin, every later read of LDS waits for it, since
// both buffers are one array to the alias analysis.)  M0, which says where in LDS, is the
// compiler's: it is put back.  The waits are those that the hardware leaves to the program, where
// the compiler does not see into these lines: one instruction between a write of M0 and its load,
// and five between a vector instruction that writes a scalar register, as read_lane does, and a
// load that reads it.
__device__ __forceinline__ uint32_t lds_address(char *p) {
  return __builtin_amdgcn_readfirstlane(uint32_t(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char *)p)));
}
__device__ __forceinline__ void to_lds(uint64_t k, uint32_t k_offset, char *k_to, uint64_t v, uint32_t v_offset, char *v_to) {
  uint32_t kept;
  asm volatile(
      "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 2\n\tglobal_load_lds_dwordx4 %2, %3\n\t"
      "s_mov_b32 m0, %4\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %5, %6\n\ts_mov_b32 m0, %0"
      : "=&s"(kept)
      : "s"(lds_address(k_to)), "v"(k_offset), "s"(k), "s"(lds_address(v_to)), "v"(v_offset), "s"(v)
      : "memory");
}
__device__ __forceinline__ void to_lds(uint64_t k, char *k_to, uint64_t v, char *v_to) {
  uint32_t kept;
  asm volatile(
      "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, off\n\t"
      "s_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %4, off\n\ts_mov_b32 m0, %0"
      : "=&s"(kept)
      : "s"(lds_address(k_to)), "v"(k), "s"(lds_address(v_to)), "v"(v)
      : "memory");
}
__device__ __forceinline__ float max3(float a, float b, float c) {  // one instruction; NaN stays
  return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c);
}

// A row is scaled down only when its own maximum has grown by more than 2^SLACK: until then its
// weights are at most 2^SLACK instead of 1, which costs BF16 no precision and F16 that many of the
// powers of two below 1 (MANY_SHIFT), and most steps of a long request leave the sums alone.
constexpr float SLACK = 8.0f;

// Where a row's 16-byte pieces are in LDS: piece c at c ^ key_swap(row), c ^ value_swap(row).  A
// read of 16 bytes a lane takes 16 lanes at a time, 16 keys' piece c here: they have to lie in
// 16 places of 256 bytes, the banks' width.  A transposed read takes 32 lanes, 64 bytes of four
// rows that begin at a multiple of four: in four places of 64.
template <int D>
__device__ __forceinline__ int key_swap(int row) {
  return D == 64 ? row >> 1 & 7 : row & 15;
}
template <int D>
__device__ __forceinline__ int value_swap(int row) {
  return D == 64 ? 4 * (row >> 1 & 1) : 4 * (row & 3);
}

// The order in which a wavefront's instructions are issued is the order of the source between
// these: reads of LDS some products ahead, and weights between products, which the matrix
// cores take 32 cycles each for.
__device__ __forceinline__ void in_order() { __builtin_amdgcn_sched_barrier(0); }

// x, computed again in every step: what follows from it is not kept in registers across them.
__device__ __forceinline__ int again(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// What a wavefront keeps of its 32 rows; lane (half, col) holds row col's.
template <int D>
struct Rows {
  u32x4 q[D / 16];
  f32x16 o[D / 32];  // O^T: components 32 i + 8 (r / 4) + 4 half + r % 4
  float m, l;        // of the half's keys (l), of all (m)
  int32_t hi, lo;    // the keys [lo, hi) that the row sees
};

// The values of 16 keys of a step, V^T as the matrix instruction takes it: read in the order in
// which S^T leaves the keys.
template <int D>
struct Values {
  u32x2 lo[D / 32], hi[D / 32];
  __device__ __forceinline__ static int offset(int lane) {  // of column tile 0
    const int half = lane >> 5, j = lane & 15;
    const int r = 4 * half + j / 4, c = 2 * ((lane >> 4) & 1) + (j % 4) / 2;
    return r * 2 * D + ((c ^ value_swap<D>(r)) * 16) + (j & 1) * 8;
  }
  __device__ __forceinline__ void read(const char *vl, int off, int t, int i) {
    constexpr int ROWB = 2 * D;
    const char *x = vl + (off ^ (64 * i));  // (r + 8, r + 16: the same exchange)
    lo[i] = read_transposed(x + 16 * t * ROWB);
    hi[i] = read_transposed(x + (16 * t + 8) * ROWB);
  }
  __device__ __forceinline__ void read(const char *vl, int off, int t) {
#pragma unroll
    for (int i = 0; i < D / 32; ++i) read(vl, off, t, i);
  }
};

// One step's 64 keys: the scores.  S^T: lane (half, col) gets row col's scores of keys kb +
// 32 j + 8 (r / 4) + 4 half + r % 4, -inf for those that the row does not see (MASKED: there
// may be some).  Returns the row's largest, and the first 16 keys' values on their way.
template <typename T, int D, bool MASKED>
__device__ __forceinline__ float scores(const Rows<D> &w, const char *kl, const char *vl, int32_t kb, float sc, int lane,
                                        f32x16 (&s)[2], Values<D> &first) {
  constexpr int N = D / 8, AHEAD = 4, ROWB = 2 * D;
  const int l = again(lane), col = l & 31, swap = 16 * ((l >> 5) ^ key_swap<D>(col));
  const char *row = kl + col * ROWB;
  const auto piece = [&](int n) {  // (32 rows on: the same exchange)
    return *reinterpret_cast<const u32x4 *>(row + ((n / 2 * 32) ^ swap) + n % 2 * (32 * ROWB));
  };
  u32x4 k[AHEAD];
#pragma unroll
  for (int n = 0; n < AHEAD; ++n) k[n] = piece(n);
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int r = 0; r < 16; ++r) s[j][r] = 0.0f;
#pragma unroll
  for (int n = 0; n < N; ++n) {
    in_order();
    if (n == 0) __builtin_amdgcn_s_setprio(1);
    s[n % 2] = T::mfma32(k[n % AHEAD], w.q[n / 2], s[n % 2]);
    if (n + AHEAD < N) k[n % AHEAD] = piece(n + AHEAD);
  }
  in_order();
  __builtin_amdgcn_s_setprio(0);
  first.read(vl, Values<D>::offset(again(lane)), 0);
  if (MASKED) {
    const int half = lane >> 5;
    const int32_t hi = w.hi - kb - 4 * half, lo = w.lo - kb - 4 * half;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int32_t key = 32 * j + 8 * (r / 4) + r % 4;
        if (key >= hi || key < lo) s[j][r] = -INFINITY;
      }
  }
  float mx = max3(s[0][0], s[0][1], s[1][0]);
#pragma unroll
  for (int r = 2; r < 16; r += 2) mx = max3(mx, s[0][r], s[0][r + 1]);
#pragma unroll
  for (int r = 1; r < 15; r += 2) mx = max3(mx, s[1][r], s[1][r + 1]);
  mx = __builtin_elementwise_maximum(mx, s[1][15]);
  const u32x2 both = swap32(__float_as_uint(mx), __float_as_uint(mx));
  return __builtin_elementwise_maximum(__uint_as_float(both.x), __uint_as_float(both.y)) * sc;
}
template <typename T, int D>
__device__ __forceinline__ float exponent(const Rows<D> &w) {  // of weight 2^MANY_SHIFT
  return T::MANY_SHIFT - (w.m == -INFINITY ? 0.0f : w.m);
}

// The products of 16 keys' weights with their values, among them the next 16's weights and reads.
template <typename T, int D>
__device__ __forceinline__ void products(Rows<D> &w, const char *vl, float sc, int lane, const f32x16 (&s)[2],
                                         const Values<D> &first) {
  constexpr int DT = D / 32;
  const float base = exponent<T>(w);
  const int off = Values<D>::offset(again(lane));
  Values<D> v[2];
  u32x4 p[2];
  v[0] = first;
  const auto weights = [&](int t, int e) {
    const float x = __builtin_amdgcn_exp2f(fmaf(s[t / 2][8 * (t % 2) + 2 * e], sc, base));
    const float y = __builtin_amdgcn_exp2f(fmaf(s[t / 2][8 * (t % 2) + 2 * e + 1], sc, base));
    w.l += x + y;
    p[t % 2][e] = T::pack(x, y);
  };
#pragma unroll
  for (int e = 0; e < 4; ++e) weights(0, e);
#pragma unroll
  for (int t = 0; t < KT / 16; ++t)
#pragma unroll
    for (int i = 0; i < DT; ++i) {
      in_order();
      if (t == 0 && i == 0) __builtin_amdgcn_s_setprio(1);
      const Values<D> &x = v[t % 2];
      w.o[i] = T::mfma32(u32x4{x.lo[i].x, x.lo[i].y, x.hi[i].x, x.hi[i].y}, p[t % 2], w.o[i]);
      if (t + 1 < KT / 16) {
        v[(t + 1) % 2].read(vl, off, t + 1, i);
#pragma unroll
        for (int e = 4 * i / DT; e < 4 * (i + 1) / DT; ++e) weights(t + 1, e);
      }
    }
  in_order();
  __builtin_amdgcn_s_setprio(0);
}

// Where some row's maximum has grown by more than 2^SLACK: sums scaled down.  The branch
// around the products is part of the instruction sequence, so that for the compiler the sums
// are changed in one place and keep their registers; around a branch of its own it keeps
// them twice, which leaves no room for keys and values read ahead.  The products of the
// step before are long done: this step's scores, which came after them, have been read.  The
// next product may read what was scaled two instructions later, hence the wait at the end.
// (Heads of 256: the sums live in accumulation registers, and the operands here are vector ones, so
// that each step moves 128 sums here and back, besides 32 scores, for its 64 products.)
__device__ __forceinline__ void scale_down(f32x16 &o, float down, uint64_t grown) {
  float x[16];
#pragma unroll
  for (int r = 0; r < 16; ++r) x[r] = o[r];
  asm volatile(
      "s_cmp_eq_u64 %17, 0\n\ts_cbranch_scc1 .Lkept%=\n\t"
      "v_mul_f32 %0, %16, %0\n\tv_mul_f32 %1, %16, %1\n\tv_mul_f32 %2, %16, %2\n\tv_mul_f32 %3, %16, %3\n\t"
      "v_mul_f32 %4, %16, %4\n\tv_mul_f32 %5, %16, %5\n\tv_mul_f32 %6, %16, %6\n\tv_mul_f32 %7, %16, %7\n\t"
      "v_mul_f32 %8, %16, %8\n\tv_mul_f32 %9, %16, %9\n\tv_mul_f32 %10, %16, %10\n\tv_mul_f32 %11, %16, %11\n\t"
      "v_mul_f32 %12, %16, %12\n\tv_mul_f32 %13, %16, %13\n\tv_mul_f32 %14, %16, %14\n\tv_mul_f32 %15, %16, %15\n\t"
      "s_nop 1\n"
      ".Lkept%=:"
      : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3]), "+v"(x[4]), "+v"(x[5]), "+v"(x[6]), "+v"(x[7]), "+v"(x[8]),
        "+v"(x[9]), "+v"(x[10]), "+v"(x[11]), "+v"(x[12]), "+v"(x[13]), "+v"(x[14]), "+v"(x[15])
      : "v"(down), "s"(grown)
      : "scc");
#pragma unroll
  for (int r = 0; r < 16; ++r) o[r] = x[r];
}

// A step.  ENDS: not every row sees all of its keys.
template <typename T, int D, bool ENDS>
__device__ __forceinline__ void step(Rows<D> &w, const char *kl, const char *vl, int32_t kb, float sc, int lane) {
  f32x16 s[2];
  Values<D> first;
  const float mx = scores<T, D, ENDS>(w, kl, vl, kb, sc, lane, s, first);
  const uint64_t grown = __ballot(mx > w.m + SLACK);  // also the first time: m is -inf
  float down = 1.0f;
  if (grown) {  // only the rows that have grown: another one's scores change nothing in a row
    const bool mine = mx > w.m + SLACK;
    down = mine ? __builtin_amdgcn_exp2f(w.m - mx) : 1.0f;
    w.m = mine ? mx : w.m;
    w.l *= down;
  }
#pragma unroll
  for (int i = 0; i < D / 32; ++i) scale_down(w.o[i], down, grown);
  products<T>(w, vl, sc, lane, s, first);
}

// A wavefront's rows: the output, or the sums for the joining.
template <typename T, int D>
__device__ __forceinline__ void write_rows(const AttendArgs &a, const PlanItem &it, const Rows<D> &w, int32_t kvh, int wave,
                                           int lane, float vs) {
  constexpr int DT = D / 32;
  const int col = lane & 31, half = lane >> 5;
  const int32_t row = it.tile * MANY_ROWS + 32 * wave + col, tok = row / a.group, head = kvh * a.group + row % a.group;
  const bool has_row = row < it.n_new * a.group;
  if (it.part < 0) {
    const float inv = w.l == 0.0f ? 0.0f : vs / w.l;
    uint16_t *p = a.out.data + (int64_t(it.tok0) + tok) * a.out.token + head * a.out.head;
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
      for (int g = 0; g < 4; g += 2) {
        u32x4 x;
#pragma unroll
        for (int e = 0; e < 2; ++e) {  // halves trade 4 components: each then has 8 in a row
          const u32x2 z = swap32(T::pack(w.o[i][4 * g + 2 * e] * inv, w.o[i][4 * g + 2 * e + 1] * inv),
                                 T::pack(w.o[i][4 * g + 4 + 2 * e] * inv, w.o[i][4 * g + 4 + 2 * e + 1] * inv));
          x[e] = z.x;
          x[2 + e] = z.y;
        }
        if (has_row) *reinterpret_cast<u32x4 *>(p + 32 * i + 8 * g + 8 * half) = x;
      }
    if (a.lse && has_row && half == 0) a.lse[(int64_t(it.tok0) + tok) * a.n_q + head] = lse_of(w.m, w.l, T::MANY_SHIFT);
  } else if (has_row) {
    const int64_t slot = (int64_t(it.part) * a.n_kv + kvh) * MANY_ROWS + 32 * wave + col;
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<f32x4 *>(a.parts.acc + slot * D + 32 * i + 8 * g + 4 * half) =
            f32x4{w.o[i][4 * g] * vs, w.o[i][4 * g + 1] * vs, w.o[i][4 * g + 2] * vs, w.o[i][4 * g + 3] * vs};
    if (half == 0) a.parts.ml[slot] = f32x2{w.m, w.l};
  }
}

// What a row sees of a value that is not finite, added to what write_rows has written.  Weights
// are positive: infinities and NaN come through as they are.  A lane takes the components that it
// has written.  Rare, and here, where the sums' registers are free, at no cost to the steps.
template <typename T, bool KV8, int D>
__device__ __forceinline__ void add_not_finite(const AttendArgs &a, const PlanItem &it, uint64_t value, int32_t kvh, int wave,
                                               int lane, float vs) {
  const int col = lane & 31, half = lane >> 5;
  const int32_t row = it.tile * MANY_ROWS + 32 * wave + col, tok = row / a.group, head = kvh * a.group + row % a.group;
  const int64_t slot = (int64_t(it.part) * a.n_kv + kvh) * MANY_ROWS + 32 * wave + col;
#pragma unroll 1
  for (int n = 0; n < D / 8; ++n) {
    const int c = it.part < 0 ? 16 * (n / 2) + 8 * half + 4 * (n % 2) : 8 * n + 4 * half;
    const f32x4 v = four_values<T, KV8>(value, c);
    if (is_finite(v[0]) && is_finite(v[1]) && is_finite(v[2]) && is_finite(v[3])) continue;
    u32x2 *out = reinterpret_cast<u32x2 *>(a.out.data + (int64_t(it.tok0) + tok) * a.out.token + head * a.out.head + c);
    f32x4 *sum = reinterpret_cast<f32x4 *>(a.parts.acc + slot * D + c);
    f32x4 x = it.part < 0 ? f32x4{T::lo(out->x), T::hi(out->x), T::lo(out->y), T::hi(out->y)} : *sum;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (!is_finite(v[k])) x[k] += v[k] * vs;
    if (it.part < 0)
      *out = u32x2{T::pack(x[0], x[1]), T::pack(x[2], x[3])};
    else
      *sum = x;
  }
}

// WIDE: page_size is a multiple of 16, so 16 aligned keys are neighbours in one page.
template <typename T, bool KV8, int D, bool WIDE>
__global__ __launch_bounds__(MT, at_once(D)) void many_kernel(AttendArgs a) {
  constexpr int ESZ = KV8 ? 1 : 2;
  constexpr int LPR = D * ESZ / 16;   // lanes per row of keys or values
  constexpr int RPW = 64 / LPR;       // rows of a wavefront's load
  constexpr int RPL = RPW * MW;       // rows of a workgroup's load
  constexpr int NL = KT / RPL;        // loads of a lane per step and side
  constexpr int STEPS = D / 16, DT = D / 32;
  constexpr int ROWB = 2 * D;         // bytes of a row in LDS
  constexpr int SIDE = KT * ROWB;     // bytes of a step's keys, and of its values
  __shared__ __attribute__((aligned(1024))) char lds[4 * SIDE];  // a step's keys, values; the next one's
  __shared__ int32_t odd_piece;  // the last piece in which look_over has met a value that is not finite

  const int32_t kvh = blockIdx.x % a.n_kv, share = blockIdx.x / a.n_kv;
  // asked for together: a workgroup's start is a chain of round trips
  const PlanHdr hdr = *a.hdr;
  const int32_t first_piece = uniform(a.first[share]), last_piece = uniform(a.first[share + 1]);
  if (!plan_fits(a, hdr)) {
    write_nothing<D>(a);
    return;
  }
  if (share >= hdr.n_groups) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int col = lane & 31, half = lane >> 5;
  if (threadIdx.x == 0) odd_piece = -1;  // (a barrier follows before look_over)
  for (int32_t piece = first_piece; piece < last_piece; ++piece) {
    const PlanItem it = uniform(a.items[piece]);
    const int32_t row0 = it.tile * MANY_ROWS + 32 * wave;
    int32_t n_rows = it.n_new * a.group - row0;  // of this wavefront
    if (n_rows > 32) n_rows = 32;
    const bool too_long = int64_t(it.kv_len) > int64_t(a.cache.max_pages) * a.cache.ps.size;
    const int32_t k0 = uniform(too_long ? 0 : it.k0), k1 = uniform(too_long ? 0 : it.k1);
    if (too_long && threadIdx.x == 0) set_status(a.status, SMETRIC_EINVAL);

    Rows<D> w;
    const bool has_row = col < n_rows;
    const int32_t row = row0 + col, tok = row / a.group, head = kvh * a.group + row % a.group;
    const int32_t first = it.kv_len - it.n_new;  // the first new token's place
    w.hi = has_row ? first + tok + 1 : 0;
    w.lo = a.window > 0 ? first + tok + 1 - a.window : 0;
    // the wavefront's first and last row, and the tile's
    const int32_t min_hi = first + row0 / a.group + 1;
    const int32_t max_hi = n_rows > 0 ? first + (row0 + n_rows - 1) / a.group + 1 : 0;
    const int32_t min_lo = a.window > 0 ? min_hi - a.window : 0;
    const int32_t tile_min_hi = first + it.tile * MANY_ROWS / a.group + 1;
    int32_t tile_end = (it.tile + 1) * MANY_ROWS;
    if (tile_end > it.n_new * a.group) tile_end = it.n_new * a.group;
    const int32_t tile_max_lo = a.window > 0 ? first + (tile_end - 1) / a.group + 1 - a.window : 0;

    // Scores are masked, and their largest found, before they are multiplied, so the factor has to
    // be positive: another one's sign goes into the queries, and a NaN; zero becomes the smallest
    // normal number, which leaves all weights 1 for scores below 2^100.
    float sc = a.scale_log2;
    uint32_t flip = 0, nan = 0;
    if (KV8 && a.cache.k_scale) {
      sc *= a.cache.k_scale[kvh];
      if (!(sc > 0.0f)) {
        flip = sc < 0.0f ? 0x80008000u : 0;
        nan = sc != sc ? 0x7FFF7FFFu : 0;
        sc = sc < 0.0f ? -sc : sc == 0.0f ? 0x1p-126f : 1.0f;
      }
    }
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      w.q[s] = u32x4{0, 0, 0, 0};
      if (has_row)
        w.q[s] = *reinterpret_cast<const u32x4 *>(a.q.data + (int64_t(it.tok0) + tok) * a.q.token + head * a.q.head + s * 16 +
                                                  half * 8);
      if (KV8) w.q[s] = (w.q[s] ^ flip) | nan;
    }
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) w.o[i][r] = 0.0f;
    w.m = -INFINITY;
    w.l = 0.0f;
    const char *kbase = a.cache.k.base + kvh * a.cache.k.head;
    const char *vbase = a.cache.v.base + kvh * a.cache.v.head;
    const int32_t *table = a.cache.table + it.req * a.cache.table_stride;

    const int32_t kb0 = k0 / KT * KT, last_key = k1 - 1;
    u32x4 kr[KV8 ? NL : 1], vr[KV8 ? NL : 1];  // 8-bit keys and values on their way to LDS
    const int lrow = lane / LPR, lcol = lane % LPR;
    bool bad_page = false;
    // Where a place's keys and values are; a page outside the cache reads page 0.
    const auto find = [&](int32_t key, uint64_t &kp, uint64_t &vp) {
      const int32_t page = page_of(a.cache.ps, key);
      int32_t id = table[page];
      if (uint32_t(id) >= uint32_t(a.cache.n_pages)) {
        id = 0;
        bad_page = true;
      }
      const int32_t slot = key - page * a.cache.ps.size;
      kp = reinterpret_cast<uint64_t>(kbase) + id * a.cache.k.page + slot * a.cache.k.token;
      vp = reinterpret_cast<uint64_t>(vbase) + id * a.cache.v.page + slot * a.cache.v.token;
    };
    // WIDE: lane l knows where the 16 keys from known_from + 16 l on are, for 16 steps at a time
    uint64_t kp_l = 0, vp_l = 0;
    int32_t known_from = 0;
    const auto find_steps = [&](int32_t kb) {
      int32_t key = kb + 16 * lane;  // 16 keys outside [k0, k1) read a neighbour's places: in bounds, not seen
      key = key < last_key ? key : last_key;
      key = key > k0 ? key : k0;
      find(key & ~15, kp_l, vp_l);
      known_from = kb;
    };
    const uint32_t k_lane = uint32_t(lrow) * uint32_t(a.cache.k.token), v_lane = uint32_t(lrow) * uint32_t(a.cache.v.token);
    // From memory: 16-bit rows straight to LDS, each lane fetching the piece that belongs where
    // its 16 bytes land; 8-bit ones to registers, from which to_16 widens them.
    const auto load_step = [&](int32_t kb, char *kl) {
      char *vl = kl + SIDE;
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const int r = i * RPL + wave * RPW;  // the wavefront's first row
        const int kc = KV8 ? lcol : lcol ^ key_swap<D>(r + lrow), vc = KV8 ? lcol : lcol ^ value_swap<D>(r + lrow);
        uint64_t kp, vp;
        uint32_t ko = kc * 16, vo = vc * 16;
        if (WIDE) {
          const int from = (kb - known_from + r) / 16;
          kp = read_lane(kp_l, from);
          vp = read_lane(vp_l, from);
          ko += k_lane + uint32_t(r % 16) * uint32_t(a.cache.k.token);
          vo += v_lane + uint32_t(r % 16) * uint32_t(a.cache.v.token);
        } else {
          int32_t key = kb + r + lrow;
          key = key < last_key ? key : last_key;
          key = key > k0 ? key : k0;
          find(key, kp, vp);
        }
        if (KV8) {
          kr[i] = *reinterpret_cast<const u32x4 *>(kp + ko);
          vr[i] = *reinterpret_cast<const u32x4 *>(vp + vo);
        } else if (WIDE) {
          to_lds(kp, ko, kl + r * ROWB, vp, vo, vl + r * ROWB);
        } else {
          to_lds(kp + ko, kl + r * ROWB, vp + vo, vl + r * ROWB);
        }
      }
    };
    const auto to_16 = [&](char *kl) {
      char *vl = kl + SIDE;
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const int r = i * RPL + wave * RPW + lrow;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const u32x4 k = kr[i], v = vr[i];
          const uint32_t x = h ? k.z : k.x, y = h ? k.w : k.y, z = h ? v.z : v.x, u = h ? v.w : v.y;
          *reinterpret_cast<u32x4 *>(kl + r * ROWB + ((2 * lcol + h) ^ key_swap<D>(r)) * 16) =
              u32x4{T::template from_e4m3<false>(x), T::template from_e4m3<true>(x), T::template from_e4m3<false>(y),
                    T::template from_e4m3<true>(y)};
          *reinterpret_cast<u32x4 *>(vl + r * ROWB + ((2 * lcol + h) ^ value_swap<D>(r)) * 16) =
              u32x4{T::template from_e4m3<false>(z), T::template from_e4m3<true>(z), T::template from_e4m3<false>(u),
                    T::template from_e4m3<true>(u)};
        }
      }
    };
    // A step at the ends of what the rows see: values outside [k0, k1), which may be anything,
    // become zeros, as do those that are not finite -- 0 times them must not reach a row that does
    // not see them -- which add_not_finite adds to the rows that do.
    const auto look_over = [&](int32_t kb, char *vl) {
      constexpr int TPR = MT / KT, BYTES = ROWB / TPR;
      const int r = threadIdx.x / TPR;
      char *p = vl + r * ROWB + threadIdx.x % TPR * BYTES;
      const bool in = kb + r >= k0 && kb + r < k1;
      bool odd = false;
#pragma unroll
      for (int i = 0; i < BYTES; i += 16) {
        u32x4 &x = *reinterpret_cast<u32x4 *>(p + i);
        if (!in) {
          x = u32x4{0, 0, 0, 0};
        } else if (any_not_finite<T>(x)) {
          x = finite_only<T>(x);
          odd = true;
        }
      }
      if (odd) odd_piece = piece;
      __syncthreads();
    };
    const auto arrived = [] {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
    };
    int buf = 0;  // where the current step's keys and values are
    const auto here = [&] { return lds + buf * (2 * SIDE); };
    const auto there = [&] { return lds + (buf ^ 1) * (2 * SIDE); };
    const auto load_next = [&](int32_t kb) {
      const int32_t next = kb + KT;
      if (next >= k1) return;
      if (WIDE && next - known_from >= 64 * 16) find_steps(next);
      load_step(next, there());
    };
    // Steps from kb to `to`.  ENDS: not every row of the tile sees all of their keys.  Every
    // wavefront passes the same barriers: one a step, and those of look_over.
    const auto run = [&](auto ends, int32_t &kb, int32_t to) {
      constexpr bool ENDS = decltype(ends)::value;
      for (; kb < to; kb += KT, buf ^= 1) {
        load_next(kb);
        if (ENDS) look_over(kb, here() + SIDE);
        if (!ENDS || (n_rows > 0 && kb < max_hi && kb + KT > min_lo))
          step<T, D, ENDS>(w, here(), here() + SIDE, kb, sc, lane);
        if (KV8 && kb + KT < k1) to_16(there());
        arrived();
      }
    };

    // steps that every row of the tile sees whole lie between full0 and full1
    const int32_t full0 = (max(k0, tile_max_lo) + KT - 1) / KT * KT, full1 = min(k1, tile_min_hi) / KT * KT;
    if (kb0 < k1) {
      if (WIDE) find_steps(kb0);
      load_step(kb0, here());
      if (KV8) to_16(here());
      arrived();
      int32_t kb = kb0;
#pragma unroll 1
      for (int part = 0; part < 2; ++part) {
        run(std::true_type{}, kb, part ? k1 : min(full0, k1));
        if (!part) run(std::false_type{}, kb, full1);
      }
    }
    if (bad_page) set_status(a.status, SMETRIC_EINVAL);
    {
      const u32x2 both = swap32(__float_as_uint(w.l), __float_as_uint(w.l));
      w.l = __uint_as_float(both.x) + __uint_as_float(both.y);
    }
    const float vs = KV8 && a.cache.v_scale ? a.cache.v_scale[kvh] : 1.0f;
    write_rows<T>(a, it, w, kvh, wave, again(lane), vs);
    if (kb0 < k1 && odd_piece == piece) {  // (the next piece's first barrier comes after all have read it)
#pragma unroll 1
      for (int32_t key = k0; key < k1; ++key) {
        if (key >= full0 && key < full1) key = full1;
        if (key >= k1) break;
        uint64_t kp, vp;
        find(key, kp, vp);
        if (key < w.hi && key >= w.lo) add_not_finite<T, KV8, D>(a, it, vp, kvh, wave, lane, vs);
      }
    }
  }
}

template <typename T, bool KV8, int D>
int launch_d(const AttendArgs &a, int64_t max_groups, hipStream_t stream) {
  const dim3 grid(uint32_t(max_groups * a.n_kv)), block(MT);
  if (a.cache.ps.size % 16 == 0)
    many_kernel<T, KV8, D, true><<<grid, block, 0, stream>>>(a);
  else
    many_kernel<T, KV8, D, false><<<grid, block, 0, stream>>>(a);
  return hip_status(hipGetLastError());
}
template <typename T, bool KV8>
int launch_k(const AttendArgs &a, int32_t d, int64_t max_groups, hipStream_t stream) {
  return d == 64 ? launch_d<T, KV8, 64>(a, max_groups, stream)
                 : d == 128 ? launch_d<T, KV8, 128>(a, max_groups, stream) : launch_d<T, KV8, 256>(a, max_groups, stream);
}

}  // namespace

int launch_many(const AttendArgs &a, int32_t dtype, bool kv8, int32_t head_dim, int64_t max_groups, hipStream_t stream) {
  if (dtype == SMETRIC_BF16)
    return kv8 ? launch_k<Bf16, true>(a, head_dim, max_groups, stream) : launch_k<Bf16, false>(a, head_dim, max_groups, stream);
  return kv8 ? launch_k<F16, true>(a, head_dim, max_groups, stream) : launch_k<F16, false>(a, head_dim, max_groups, stream);
}

}  // namespace smk
