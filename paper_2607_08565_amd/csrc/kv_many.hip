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
// Weights are rounded to the activations' type for it, as the matrix cores take 16-bit operands, and
// so are those that they are divided by the sum of (WeightSum); lse has the sum of unrounded ones.
//
// Measured: 4,096 tokens over 16,384 (32 heads of 128) 919 to 953 us, 1,046 to 1,008 TFLOP/s, from card to card, with
// lse 942 to 990; the library's product of matrices of 16,384 reaches 1,330 to 1,400, of 8,192 1,170 to 1,270.  The matrix
// cores work half of the cycles and the vector instructions about as long (33 exponentials, 31 products,
// 16 maxima and, with lse, 32 sums a step of 40 matrix instructions), on two wavefronts that overlap them in part, at a
// clock that falls under the load (1.9 GHz).  With the keys always in the nearest cache it takes
// 5 % less, without the exponentials 8 %, without the maximum 5 %.  Heads of 64 do half the
// products for the same weights: 24 requests with up to 1,000 new tokens, with lse, 116 us, 357 TFLOP/s.
//
// 8- and 4-bit keys and values are widened on the way to LDS, 4-bit ones two at an instruction with their
// group's exponent, once for the 128 rows: over 4-bit pages the same 4,096 tokens take 915 to 941 us, with lse 943
// to 1,005, and 2 chunks of 2,048 at heads of 256 304, 315.  Scores that are capped or biased: enum Scores.  Capped,
// BF16, 4,096 over 16,384: 1,081 to 1,104 us, with lse 1,123 to 1,193; F16 1,183 to 1,204, 1,232 to 1,291; biased 995 to
// 1,031, 1,031 to 1,087; 2,048 over 8,048 with a window of 4,096 capped 168 to 177, 173 to 187.
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
// weights are at most 2^SLACK instead of 1, and most steps of a long request leave the sums alone.  The
// largest weight is then not 1, which rounding leaves as it is, but rounded as the others are (hence
// WeightSum), and F16 has that many powers of two fewer below 1 (MANY_SHIFT).
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

// Which of a lane's pieces of 4 bits goes there first (flipped): so that 8 lanes' pieces, of one or two rows, lie
// in 8 places of 128 bytes.  Without, 118 of 295 M cycles of LDS are conflicts (4,096 tokens over 16,384: 938 us, so
// 919; 2 chunks of 2,048 at heads of 256 348 us, so 309; at heads of 64, 2 to a place at most, 264 and 266).
// 8-bit pieces, where it takes away conflicts as well, it makes slower (2 chunks of 2,048: 221 us, so 230; at heads of 256 317 both).
template <int D, bool VALUES>
__device__ __forceinline__ int flip_of(int row, int lane_col) {
  if (D == 64) return row & 1;
  if (D == 256) return lane_col >> 1;
  return (VALUES ? row & 1 : 0) ^ 2 * (lane_col >> 1);  // (keys: their rows' exchange is by one already)
}

// The order in which a wavefront's instructions are issued is the order of the source between
// these: reads of LDS some products ahead, and weights between products, which the matrix
// cores take 32 cycles each for.
__device__ __forceinline__ void in_order() { __builtin_amdgcn_sched_barrier(0); }

// What is done to a product before it is a score (smetric_attend_scores):
//   BIASED  the bias, divided by the factor to come, is where the products' sums begin, instead of 0 (each of
//           head_dim / 16 products rounds it, but of the keys that count it is small: Bias)
//   CAPPED  capped by so little that the weights need no running maximum, with BF16, whose weights have
//           float32's range: scores are within cap of 0 in powers of two, and with m = 11 weights are
//           between 2^(-11 - cap) and 2^(cap - 11): times values between 2^(cap - 115) and 2^(115 - cap),
//           summed over 2^24 keys, they stay between float32's ends, 2^-126 and 2^128.  Caps up to 73
//           (50.5 natural) leave values 2^-42 to 2^42.  That saves the maxima, a subtraction and the sums'
//           scaling (2,048 tokens over 8,048: 195 us, without 175)
//   OTHER   capped and, maybe, biased then; FAR: caps above CAP_NEAR
// Capping takes five instructions a score, two of them at half rate, as long as the matrix cores take
// for it at heads of 128: so the first 32 keys' scores are capped during the other 32's products, and
// the others' (CAPPED) during those with the values (175 us, so 168).
enum Scores { PLAIN, BIASED, CAPPED, OTHER, FAR };
constexpr bool caps(Scores s) { return s >= CAPPED; }
constexpr bool caps_first(Scores s) { return s >= OTHER; }  // before a maximum is taken
constexpr float CAPPED_MOST = 73.0f, CAPPED_MAXIMUM = 11.0f;

// The sum of the weights that the products with the values take, rounded as they are: a sum of unrounded
// ones leaves equal values other than they are, by up to the weights' half step.  (lse has the unrounded
// ones' sum, 32 additions a step more.)  16 dot products with ones a step, each at half rate, or eight
// matrix products of 8 cycles with a matrix of ones (4 x 4 x 4: a lane's own four), MATRIX: 4,096 tokens
// over 16,384 of 4 bits with lse 1,005 us, with dot products 1,029, with a sum of unrounded ones 980; capped
// over BF16 pages 1,186 and 1,178; 2 chunks at heads of 256, where registers are short, 309 and 298.
template <int D, Scores S>
struct WeightSum {
  static constexpr bool MATRIX = D < 256 && !caps(S);
  std::conditional_t<MATRIX, f32x4, float> s;
  __device__ __forceinline__ WeightSum() : s{} {}
  // part i of n of 16 keys' 8 weights
  template <typename T>
  __device__ __forceinline__ void add(u32x4 p, int i, int n) {
    if constexpr (MATRIX) {
#pragma unroll
      for (int e = 2 * i / n; e < 2 * (i + 1) / n; ++e) s = T::add_four(u32x2{p[2 * e], p[2 * e + 1]}, s);
    } else {
#pragma unroll
      for (int e = 4 * i / n; e < 4 * (i + 1) / n; ++e) s = T::add_two(p[e], s);
    }
  }
  __device__ __forceinline__ float get() const {
    if constexpr (MATRIX)
      return s.x;
    else
      return s;
  }
};

// What a wavefront keeps of its 32 rows; lane (half, col) holds row col's.
template <int D, Scores S>
struct Rows {
  u32x4 q[D / 16];
  f32x16 o[D / 32];  // O^T: components 32 i + 8 (r / 4) + 4 half + r % 4
  float m;           // maximum
  WeightSum<D, S> l;  // of the half's keys: weights as the products take them, rounded
  float exact;       // the same unrounded (LSE)
  int32_t hi, lo;    // the keys [lo, hi) that the row sees
  float slope;       // other scores: a key's bias by distance, of the products' sums or in powers of two
  int32_t from;      // the key with a bias of 0
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
template <typename T, int D, bool MASKED, Scores S>
__device__ __forceinline__ float scores(const AttendArgs &a, const Rows<D, S> &w, const char *kl, const char *vl, int32_t kb,
                                        float sc, int lane, f32x16 (&s)[2], Values<D> &first) {
  constexpr int N = D / 8, AHEAD = 4, ROWB = 2 * D;
  constexpr bool CAP = caps(S);
  const int l = again(lane), col = l & 31, swap = 16 * ((l >> 5) ^ key_swap<D>(col));
  const char *row = kl + col * ROWB;
  const auto piece = [&](int n) {  // (32 rows on: the same exchange)
    const int j = CAP ? n / (N / 2) : n % 2, d = CAP ? n % (N / 2) : n / 2;
    return *reinterpret_cast<const u32x4 *>(row + ((d * 32) ^ swap) + j * (32 * ROWB));
  };
  u32x4 k[AHEAD];
#pragma unroll
  for (int n = 0; n < AHEAD; ++n) k[n] = piece(n);
  const float from = S == BIASED || caps_first(S) ? w.slope * float(kb + 4 * (lane >> 5) - w.from) : 0.0f;
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int r = 0; r < 16; ++r) s[j][r] = S == BIASED ? fmaf(w.slope, float(32 * j + 8 * (r / 4) + r % 4), from) : 0.0f;
  const Capped cap(a, sc, S == CAPPED ? CAPPED_MAXIMUM : 0.0f);
  const auto capped = [&](float x) { return S == FAR ? cap.far(x) : cap(x); };
#pragma unroll
  for (int n = 0; n < N; ++n) {
    in_order();
    if (n == 0) __builtin_amdgcn_s_setprio(1);
    if (CAP)
      s[n / (N / 2)] = T::mfma32(k[n % AHEAD], w.q[n % (N / 2)], s[n / (N / 2)]);
    else
      s[n % 2] = T::mfma32(k[n % AHEAD], w.q[n / 2], s[n % 2]);
    if (n + AHEAD < N) k[n % AHEAD] = piece(n + AHEAD);
    // the first 32 keys' scores during the others' products
    constexpr int PER = 32 / N;
    if (CAP && n > N / 2)
#pragma unroll
      for (int r = PER * (n - N / 2 - 1); r < PER * (n - N / 2); ++r) s[0][r] = capped(s[0][r]);
  }
  in_order();
  __builtin_amdgcn_s_setprio(0);
  first.read(vl, Values<D>::offset(again(lane)), 0);
  if (CAP) {
#pragma unroll
    for (int r = 16 - 32 / N; r < 16; ++r) s[0][r] = capped(s[0][r]);
    if (caps_first(S) || MASKED)  // (the others' among the products with the values: products)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[1][r] = capped(s[1][r]);
  }
  if (caps_first(S) && a.slopes) {
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[j][r] += fmaf(w.slope, float(32 * j + 8 * (r / 4) + r % 4), from);
  }
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
  if (S == CAPPED) return 0.0f;
  float mx = max3(s[0][0], s[0][1], s[1][0]);
#pragma unroll
  for (int r = 2; r < 16; r += 2) mx = max3(mx, s[0][r], s[0][r + 1]);
#pragma unroll
  for (int r = 1; r < 15; r += 2) mx = max3(mx, s[1][r], s[1][r + 1]);
  mx = __builtin_elementwise_maximum(mx, s[1][15]);
  const u32x2 both = swap32(__float_as_uint(mx), __float_as_uint(mx));
  return __builtin_elementwise_maximum(__uint_as_float(both.x), __uint_as_float(both.y)) * (caps_first(S) ? 1.0f : sc);
}
template <typename T, int D, Scores S>
__device__ __forceinline__ float exponent(const Rows<D, S> &w) {  // of weight 2^MANY_SHIFT
  return T::MANY_SHIFT - (w.m == -INFINITY ? 0.0f : w.m);
}

// The products of 16 keys' weights with their values, among them the next 16's weights and reads.
// Capped scores are the weights' exponents, the last 32 keys' (LATER) after capping, which is done here.
template <typename T, bool LATER, bool LSE, int D, Scores S>
__device__ __forceinline__ void products(const AttendArgs &a, Rows<D, S> &w, const char *vl, float sc, int lane,
                                         const f32x16 (&s)[2], const Values<D> &first) {
  constexpr int DT = D / 32;
  constexpr bool CAP = S == CAPPED;
  const float base = exponent<T>(w);
  const Capped capped(a, sc, CAP ? CAPPED_MAXIMUM : 0.0f);
  const int off = Values<D>::offset(again(lane));
  Values<D> v[2];
  u32x4 p[2];
  v[0] = first;
  const auto weights = [&](int t, int e) {
    const auto weight = [&](float z) {
      return __builtin_amdgcn_exp2f(!CAP ? fmaf(z, sc, base) : LATER && t >= 2 ? capped(z) : z);
    };
    const float x = weight(s[t / 2][8 * (t % 2) + 2 * e]), y = weight(s[t / 2][8 * (t % 2) + 2 * e + 1]);
    if (LSE) w.exact += x + y;
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
      w.l.template add<T>(p[t % 2], i, DT);
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
template <typename T, int D, bool ENDS, Scores S, bool LSE>
__device__ __forceinline__ void step(const AttendArgs &a, Rows<D, S> &w, const char *kl, const char *vl, int32_t kb, float sc,
                                     int lane) {
  f32x16 s[2];
  Values<D> first;
  const float mx = scores<T, D, ENDS, S>(a, w, kl, vl, kb, sc, lane, s, first);
  if (S != CAPPED) {
    const uint64_t grown = __ballot(mx > w.m + SLACK);  // also the first time: m is -inf
    float down = 1.0f;
    if (grown) {  // only the rows that have grown: another one's scores change nothing in a row
      const bool mine = mx > w.m + SLACK;
      down = mine ? __builtin_amdgcn_exp2f(w.m - mx) : 1.0f;
      w.m = mine ? mx : w.m;
      w.l.s *= down;
      w.exact *= down;
    }
#pragma unroll
    for (int i = 0; i < D / 32; ++i) scale_down(w.o[i], down, grown);
  }
  products<T, !ENDS, LSE>(a, w, vl, caps_first(S) ? 1.0f : sc, lane, s, first);
}

// A wavefront's rows: the output, or the sums for the joining.  l, exact: of both halves' keys.
template <typename T, bool LSE, int D, Scores S>
__device__ __forceinline__ void write_rows(const AttendArgs &a, const PlanItem &it, const Rows<D, S> &w, float l, float exact,
                                           float more, int32_t kvh, int wave, int lane, float vs) {
  constexpr int DT = D / 32;
  const int col = lane & 31, half = lane >> 5;
  const int32_t row = it.tile * MANY_ROWS + 32 * wave + col, tok = row / a.group, head = kvh * a.group + row % a.group;
  const bool has_row = row < it.n_new * a.group;
  if (it.part < 0) {
    const float inv = l == 0.0f ? 0.0f : vs / l;
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
    if (LSE && a.lse && has_row && half == 0) a.lse[(int64_t(it.tok0) + tok) * a.n_q + head] = lse_of(w.m, exact, T::MANY_SHIFT, more);
  } else if (has_row) {
    const int64_t slot = (int64_t(it.part) * a.n_kv + kvh) * MANY_ROWS + 32 * wave + col;
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<f32x4 *>(a.parts.acc + slot * D + 32 * i + 8 * g + 4 * half) =
            f32x4{w.o[i][4 * g] * vs, w.o[i][4 * g + 1] * vs, w.o[i][4 * g + 2] * vs, w.o[i][4 * g + 3] * vs};
    if (half == 0) a.parts.ml[slot] = f32x4{w.m, l, exact, more};
  }
}

// What a row sees of a value that is not finite, added to what write_rows has written.  Weights
// are positive: infinities and NaN come through as they are.  A lane takes the components that it
// has written.  Rare, and here, where the sums' registers are free, at no cost to the steps.
template <typename T, Pages KV, int D>
__device__ __forceinline__ void add_not_finite(const AttendArgs &a, const PlanItem &it, const Place &place, int32_t kvh, int wave,
                                               int lane, float vs) {
  const int col = lane & 31, half = lane >> 5;
  const int32_t row = it.tile * MANY_ROWS + 32 * wave + col, tok = row / a.group, head = kvh * a.group + row % a.group;
  const int64_t slot = (int64_t(it.part) * a.n_kv + kvh) * MANY_ROWS + 32 * wave + col;
#pragma unroll 1
  for (int n = 0; n < D / 8; ++n) {
    const int c = it.part < 0 ? 16 * (n / 2) + 8 * half + 4 * (n % 2) : 8 * n + 4 * half;
    const f32x4 v = four_values<T, KV>(place, c);
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

// Wavefronts a SIMD at least: heads of 64 leave registers for three, though a few values less than the compiler
// takes by itself with the two sums of weights (24 mixed requests over 4-bit pages with lse 114 us, so 109; 4
// chunks of 2,048 over 8-bit pages 275 without it, so 265).
constexpr int wavefronts(int head_dim) { return head_dim == 64 ? 3 : at_once(head_dim); }

// WIDE: page_size is a multiple of 16, so 16 aligned keys are neighbours in one page.  LSE: it is asked for.
template <typename T, Pages KV, int D, bool WIDE, Scores S, bool LSE>
__global__ __launch_bounds__(MT, wavefronts(D)) void many_kernel(AttendArgs a) {
  constexpr bool KV8 = KV == PAGES8, KV4 = KV == PAGES4;
  constexpr int PB = KV4 ? piece4(D) : 16;  // bytes of a lane's load
  constexpr int LPR = page_bytes(KV, D) / PB;  // lanes per row of keys or values
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

    Rows<D, S> w;
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
      sc = finite_factor(sc * a.cache.k_scale[kvh]);
      if (!(sc > 0.0f)) {
        flip = sc < 0.0f ? 0x80008000u : 0;
        nan = sc != sc ? 0x7FFF7FFFu : 0;
        sc = sc < 0.0f ? -sc : sc == 0.0f ? 0x1p-126f : 1.0f;
      }
    }
    // A bias divided by the factor stays in float32's range: where that is next to nothing, it takes
    // 2^66 of the queries (F16's become zeros: their scores are below 2^-20).
    const float smaller = S == BIASED && sc < 0x1p-60f ? 0x1p-66f : 1.0f;
    sc /= smaller;
    const Bias bias((S == BIASED || caps_first(S)) && a.slopes && has_row ? a.slopes[head] * LOG2E : 0.0f, first + tok, w.lo);
    w.from = bias.from;
    w.slope = S == BIASED ? bias.slope / sc : bias.slope;
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      w.q[s] = u32x4{0, 0, 0, 0};
      if (has_row)
        w.q[s] = *reinterpret_cast<const u32x4 *>(a.q.data + (int64_t(it.tok0) + tok) * a.q.token + head * a.q.head + s * 16 +
                                                  half * 8);
      if (KV8) w.q[s] = (w.q[s] ^ flip) | nan;
      if (S == BIASED && smaller != 1.0f)
#pragma unroll
        for (int e = 0; e < 4; ++e) w.q[s][e] = T::pack(T::lo(w.q[s][e]) * smaller, T::hi(w.q[s][e]) * smaller);
    }
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) w.o[i][r] = 0.0f;
    w.m = S == CAPPED ? CAPPED_MAXIMUM : -INFINITY;
    w.exact = 0.0f;
    const int32_t *table = a.cache.table + it.req * a.cache.table_stride;

    const int32_t kb0 = k0 / KT * KT, last_key = k1 - 1;
    u32x4 kr[KV == PAGES16 ? 1 : NL], vr[KV == PAGES16 ? 1 : NL];  // 8- and 4-bit keys and values on their way to LDS
    uint32_t kx[KV4 ? NL : 1], vx[KV4 ? NL : 1];                   // the exponents of 4-bit ones
    const int lrow = lane / LPR, lcol = lane % LPR;
    bool bad_page = false;
    const auto find = [&](int32_t key, Place &p) { bad_page |= find_place<KV>(a, table, kvh, key, p); };
    // WIDE: lane l knows where the 16 keys from known_from + 16 l on are, for 16 steps at a time
    Place at_l{};
    int32_t known_from = 0;
    const auto find_steps = [&](int32_t kb) {
      int32_t key = kb + 16 * lane;  // 16 keys outside [k0, k1) read a neighbour's places: in bounds, not seen
      key = key < last_key ? key : last_key;
      key = key > k0 ? key : k0;
      find(key & ~15, at_l);
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
        const int kc = KV != PAGES16 ? lcol : lcol ^ key_swap<D>(r + lrow);
        const int vc = KV != PAGES16 ? lcol : lcol ^ value_swap<D>(r + lrow);
        uint64_t kp, vp;
        uint32_t ko = kc * PB, vo = vc * PB;
        if (WIDE) {
          const int from = (kb - known_from + r) / 16;
          kp = read_lane(at_l.k, from);
          vp = read_lane(at_l.v, from);
          if (KV4) {
            const uint32_t row = r % 16 + lrow, g = D == 64 ? lcol / 2 : lcol;
            kx[i] = load_exp(read_lane(at_l.k_exp, from), (row * uint32_t(a.cache.k_exp.token) + g));
            vx[i] = load_exp(read_lane(at_l.v_exp, from), (row * uint32_t(a.cache.v_exp.token) + g));
          }
          ko += k_lane + uint32_t(r % 16) * uint32_t(a.cache.k.token);
          vo += v_lane + uint32_t(r % 16) * uint32_t(a.cache.v.token);
        } else {
          int32_t key = kb + r + lrow;
          key = key < last_key ? key : last_key;
          key = key > k0 ? key : k0;
          Place at;
          find(key, at);
          kp = at.k;
          vp = at.v;
          if (KV4) {
            kx[i] = load_exp(at.k_exp + (D == 64 ? lcol / 2 : lcol));
            vx[i] = load_exp(at.v_exp + (D == 64 ? lcol / 2 : lcol));
          }
        }
        if (KV != PAGES16) {
          kr[i] = load_piece<PB>(kp, ko);
          vr[i] = load_piece<PB>(vp, vo);
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
        const int fk = flip_of<D, false>(r, lcol), fv = flip_of<D, true>(r, lcol);
        const u32x4 k = KV4 ? flipped(kr[i], fk) : kr[i], v = KV4 ? flipped(vr[i], fv) : vr[i];
        if (KV4) {
          constexpr int N = PB / 4;
          const float ke = power_of(kx[i]), ve = power_of(vx[i]);
#pragma unroll
          for (int n = 0; n < N; ++n) {
            *reinterpret_cast<u32x4 *>(kl + r * ROWB + ((N * lcol + (n ^ fk)) ^ key_swap<D>(r)) * 16) = T::eight_e2m1(k[n], ke);
            *reinterpret_cast<u32x4 *>(vl + r * ROWB + ((N * lcol + (n ^ fv)) ^ value_swap<D>(r)) * 16) = T::eight_e2m1(v[n], ve);
          }
          continue;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
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
          step<T, D, ENDS, S, LSE>(a, w, here(), here() + SIDE, kb, sc, lane);
        if (KV != PAGES16 && kb + KT < k1) to_16(there());
        arrived();
      }
    };

    // steps that every row of the tile sees whole lie between full0 and full1
    const int32_t full0 = (max(k0, tile_max_lo) + KT - 1) / KT * KT, full1 = min(k1, tile_min_hi) / KT * KT;
    if (kb0 < k1) {
      if (WIDE) find_steps(kb0);
      load_step(kb0, here());
      if (KV != PAGES16) to_16(here());
      arrived();
      int32_t kb = kb0;
#pragma unroll 1
      for (int part = 0; part < 2; ++part) {
        run(std::true_type{}, kb, part ? k1 : min(full0, k1));
        if (!part) run(std::false_type{}, kb, full1);
      }
    }
    if (bad_page) set_status(a.status, SMETRIC_EINVAL);
    const auto halves = [](float x) {
      const u32x2 both = swap32(__float_as_uint(x), __float_as_uint(x));
      return __uint_as_float(both.x) + __uint_as_float(both.y);
    };
    const float l = halves(w.l.get()), exact = LSE ? halves(w.exact) : 0.0f;
    const float vs = KV8 && a.cache.v_scale ? a.cache.v_scale[kvh] : 1.0f;
    write_rows<T, LSE>(a, it, w, l, exact, bias.more(first + tok), kvh, wave, again(lane), vs);
    if (kb0 < k1 && odd_piece == piece) {  // (the next piece's first barrier comes after all have read it)
#pragma unroll 1
      for (int32_t key = k0; key < k1; ++key) {
        if (key >= full0 && key < full1) key = full1;
        if (key >= k1) break;
        Place at;
        find(key, at);
        if (key < w.hi && key >= w.lo) add_not_finite<T, KV, D>(a, it, at, kvh, wave, lane, vs);
      }
    }
  }
}

template <typename T, Pages KV, int D, Scores S>
int launch_s(const AttendArgs &a, int64_t max_groups, hipStream_t stream) {
  const dim3 grid(uint32_t(max_groups * a.n_kv)), block(MT);
  constexpr bool ALONE = S == FAR;  // (rare: one form for both)
  const bool lse = ALONE || a.lse;
  const auto kernel = a.cache.ps.size % 16 == 0 ? lse ? many_kernel<T, KV, D, true, S, true> : many_kernel<T, KV, D, true, S, ALONE>
                                                : lse ? many_kernel<T, KV, D, false, S, true> : many_kernel<T, KV, D, false, S, ALONE>;
  kernel<<<grid, block, 0, stream>>>(a);
  return hip_status(hipGetLastError());
}
template <typename T, Pages KV, int D>
int launch_d(const AttendArgs &a, int64_t max_groups, hipStream_t stream) {
#ifdef SCORED
  if constexpr (std::is_same_v<T, Bf16>)
    if (!a.slopes && a.cap_log2 <= CAPPED_MOST) return launch_s<T, KV, D, CAPPED>(a, max_groups, stream);
  if (!(a.cap_log2 > 0.0f)) return launch_s<T, KV, D, BIASED>(a, max_groups, stream);
  if (a.cap_log2 > CAP_NEAR) return launch_s<T, KV, D, FAR>(a, max_groups, stream);
  return launch_s<T, KV, D, OTHER>(a, max_groups, stream);
#else
  return launch_s<T, KV, D, PLAIN>(a, max_groups, stream);
#endif
}
template <typename T, Pages KV>
int launch_k(const AttendArgs &a, int32_t d, int64_t max_groups, hipStream_t stream) {
  return d == 64 ? launch_d<T, KV, 64>(a, max_groups, stream)
                 : d == 128 ? launch_d<T, KV, 128>(a, max_groups, stream) : launch_d<T, KV, 256>(a, max_groups, stream);
}
template <typename T>
int launch_t(const AttendArgs &a, Pages p, int32_t d, int64_t max_groups, hipStream_t stream) {
  return p == PAGES4   ? launch_k<T, PAGES4>(a, d, max_groups, stream)
         : p == PAGES8 ? launch_k<T, PAGES8>(a, d, max_groups, stream)
                       : launch_k<T, PAGES16>(a, d, max_groups, stream);
}

}  // namespace

#ifdef SCORED
template <>
int launch_many_scored<SCORED>(const AttendArgs &a, Pages pages, int32_t head_dim, int64_t max_groups, hipStream_t stream) {
  return launch_t<SCORED>(a, pages, head_dim, max_groups, stream);
}
#else
int launch_many(const AttendArgs &a, int32_t dtype, Pages pages, int32_t head_dim, int64_t max_groups, hipStream_t stream) {
  return dtype == SMETRIC_BF16 ? launch_t<Bf16>(a, pages, head_dim, max_groups, stream)
                               : launch_t<F16>(a, pages, head_dim, max_groups, stream);
}
#endif

}  // namespace smk
