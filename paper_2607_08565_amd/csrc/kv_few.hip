// Attention of few rows over a long paged cache: decoding steps and small drafts.
//
// Mathematics (smetric_kv.h): out = sum_j p_j v_j / sum_j p_j with p_j = 2^(c s_j - m), c =
// scale log2(e), in one pass over the keys: m is the running maximum of c s_j, and what was
// summed before a larger one appears is scaled down by 2^(old - new).
//
// Bound: every key and value is read once and used for at most 16 rows, 16 operations a
// byte, far below the card's 250: memory.  So a wavefront takes keys of its own, 32 at a
// time, and nothing but the end is shared: keys come from memory in the layout in which the
// matrix instruction takes them (a lane holds 8 components of one key), values through a
// piece of LDS of the wavefront's own, from which they are read transposed.  The product is
// formed as S^T = K Q^T: a lane then holds scores of one row only, its maximum takes two
// lane exchanges, and the weights are where the second product, O^T = V^T P^T, wants them:
// its order of keys is free as long as both operands use one, so the order in which S^T
// leaves them is used.  The next 32 keys' loads are in flight during all of it.  Weights are rounded
// to the activations' type for it, as the matrix cores take 16-bit operands, and the output is divided by the sum
// of rounded ones, so that equal values come out as they are; lse has the sum of unrounded ones.
//
// Measured: 32 requests decoding over 1.73 GB of cache 302 us, 5.7 TB/s (a copy of 4 GiB moves
// 4.8); 64 drafted tokens over 0.58 GB 115 us; 131,072 keys of 8 bits (134 MB) 37 us, 24
// of them here and the rest the joining; a lone token over 1,025 keys 9.6 us, two launches.
// 4 bits, where a lane's 16 bytes are a group of 32 components, widened two at an instruction with its
// exponent: the 32 requests (0.41 GB) 86 us, 4.8 TB/s, of which the kernel has 79, 5.2 TB/s; a lone
// token 9.0; 131,072 keys 24.7; 32 requests over 16,384 at heads of 64 71, over 8,192 at heads of 256, one
// wavefront a SIMD, 80.  Scores that are capped take 4 instructions more, two of them at half
// rate: at heads of 256 16 requests decoding over 1.33 GB 233 us, 5.7 TB/s; over the 4-bit pages of 32 101.
#include <math.h>

#include "kv_attend.h"

namespace smk {
namespace {

constexpr int FK = 32;    // keys of a wavefront's block
constexpr int NJ = FK / 16;
// Wavefronts of a workgroup.  The next block is on its way during a block's products: of 4-bit heads of 64
// that is 2 KB, and eight wavefronts on a compute unit keep 17 KB under way where 5.6 TB/s need some
// 45; with twice as many 32 requests decoding over 16,384 take 70 us for 85.  (Heads of 128 and 256 need the
// registers: with eight they spill.  Blocks of 64 keys: heads of 64 73 us, of 128 no faster, 87 for 85.)
constexpr int few_waves(Pages p, int head_dim) { return p == PAGES4 && head_dim == 64 ? 8 : 4; }

// Over the four lanes l, l ^ 16, l ^ 32, l ^ 48.
__device__ __forceinline__ float max4(float x) {
  const u32x2 a = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
  x = fmaxf(__uint_as_float(a.x), __uint_as_float(a.y));
  const u32x2 b = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false));
  return fmaxf(__uint_as_float(b.x), __uint_as_float(b.y));
}
__device__ __forceinline__ float sum4(float x) {
  const u32x2 a = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
  x = __uint_as_float(a.x) + __uint_as_float(a.y);
  const u32x2 b = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false));
  return __uint_as_float(b.x) + __uint_as_float(b.y);
}

// WIDE: page_size is a multiple of 16, so 16 aligned keys are neighbours in one page.
// SCORES: they are capped or have a bias by distance.
template <typename T, Pages KV, int D, bool WIDE, bool SCORES>
__global__ __launch_bounds__(64 * few_waves(KV, D), at_once(D) * few_waves(KV, D) / 4) void few_kernel(AttendArgs a) {
  constexpr int FW = few_waves(KV, D);        // wavefronts
  constexpr bool KV8 = KV == PAGES8, KV4 = KV == PAGES4;
  constexpr bool LATE = KV4 && !SCORES;       // scores are multiplied by their factor, positive here, on the way to weights
  constexpr int PB = KV4 ? piece4(D) : 16;    // bytes of a lane's load
  constexpr int ROW = page_bytes(KV, D);      // bytes of a row in memory
  constexpr int STEPS = D / 32;               // matrix steps over the components
  constexpr int KL = ROW / (4 * PB);          // loads of a lane for 16 keys
  constexpr int VL = FK * ROW / (64 * PB);    // loads of a lane for a block's values
  constexpr int VROW = ROW / PB;              // lanes per row of values
  constexpr int VRPI = 64 / VROW;             // rows per load
  constexpr int DT = D / 16;
  constexpr int PADDED = D + 4;               // floats of a row in the joining of the wavefronts
  // bytes of a wavefront's LDS: rows of values, later its sums; whole rows, as addresses are exchanged within one
  constexpr int SUMS = (16 * PADDED * 4 + 2 * D - 1) / (2 * D) * (2 * D), REGION = FK * 2 * D > SUMS ? FK * 2 * D : SUMS;
  constexpr int SWZ = D == 64 ? 3 : 7;
  __shared__ __attribute__((aligned(2 * D))) char lds[FW * REGION];
  __shared__ float ml[FW][16][3];  // maximum, sum of rounded weights, of unrounded ones
  __shared__ float more[SCORES ? 16 : 1];  // what lse is more

  const int32_t kvh = blockIdx.x % a.n_kv, share = blockIdx.x / a.n_kv;
  // asked for together: a workgroup's start is a chain of round trips
  const PlanHdr hdr = *a.hdr;
  const int32_t first_piece = uniform(a.first[share]), last_piece = uniform(a.first[share + 1]);
  const PlanItem guess = uniform(a.items[share]);  // the first piece of a share, where tiles do not end inside one before
  if (!plan_fits(a, hdr)) {
    write_nothing<D>(a);
    return;
  }
  if (share >= hdr.n_groups) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int col = lane & 15, grp = lane >> 4;
  for (int32_t piece = first_piece; piece < last_piece; ++piece) {
    const PlanItem it = piece == share ? guess : uniform(a.items[piece]);
    const int32_t row0 = it.tile * FEW_ROWS;
    int32_t n_rows = it.n_new * a.group - row0;
    if (n_rows > FEW_ROWS) n_rows = FEW_ROWS;
    const bool too_long = int64_t(it.kv_len) > int64_t(a.cache.max_pages) * a.cache.ps.size;
    const int32_t k0 = uniform(too_long ? 0 : it.k0), k1 = uniform(too_long ? 0 : it.k1);
    if (too_long && threadIdx.x == 0) set_status(a.status, SMETRIC_EINVAL);

    // this lane's row: its token's place gives the keys [lo, hi) that it sees
    const int32_t first_place = it.kv_len - it.n_new + row0 / a.group;
    const int32_t last_place = it.kv_len - it.n_new + (row0 + n_rows - 1) / a.group;
    const int32_t row = row0 + col;
    const int32_t tok = row / a.group, head = kvh * a.group + row % a.group;
    const bool has_row = col < n_rows;
    const int32_t place = it.kv_len - it.n_new + tok;
    const int32_t hi = has_row ? place + 1 : 0;
    const int32_t lo = a.window > 0 ? place - a.window + 1 : 0;
    const int32_t min_hi = first_place + 1, max_lo = a.window > 0 ? last_place - a.window + 1 : 0;
    const bool one_token = first_place == last_place;

    u32x4 q[STEPS];
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      // the components that the lane's pieces of keys hold, in their order
      constexpr int PER = PB * 8 / (KV4 ? 4 : KV8 ? 8 : 16) / 8;  // steps of a piece
      const int d = (s / PER) * (32 * PER) + grp * (8 * PER) + (s % PER) * 8;
      q[s] = u32x4{0, 0, 0, 0};
      if (has_row)
        q[s] = *reinterpret_cast<const u32x4 *>(a.q.data + (int64_t(it.tok0) + tok) * a.q.token + head * a.q.head + d);
    }
    const int32_t *table = a.cache.table + it.req * a.cache.table_stride;
    const float sc = KV8 && a.cache.k_scale ? finite_factor(a.scale_log2 * a.cache.k_scale[kvh]) : a.scale_log2;
    const Capped capped(a, sc);
    const Bias bias(SCORES && a.slopes && has_row ? a.slopes[head] * LOG2E : 0.0f, place, lo);
    char *my = lds + wave * REGION;
    // Where in LDS a lane's values go: 16-byte piece c of row r at c ^ 2 (r & SWZ), so that the transposed
    // reads, of eight rows' two pieces at a time, meet no bank twice.  What depends on the lane is
    // computed here; a load's and a piece's share is exchanged in (its bits lie within a row).
    constexpr int PIECES = 2 * D / 16 / VROW;  // 16-byte pieces in LDS of a lane's load
    const int r0 = lane / VROW, tr = 4 * grp + col / 4;
    const int flip = !KV4 ? 0 : D == 64 ? r0 & 1 : lane % VROW >> 1;  // (flipped)
    const int to = wave * REGION + r0 * (2 * D) + ((PIECES * (lane % VROW) + flip) ^ (2 * (r0 & SWZ))) * 16;
    const int from_t = wave * REGION + tr * (2 * D) + (((col % 4) / 2) ^ (2 * (tr & SWZ))) * 16 + (col & 1) * 8;

    const int32_t kb0 = k0 / KEY_STEP * KEY_STEP + FK * wave;
    const int32_t last_key = k1 - 1;
    u32x4 kr[NJ][KL], vr[VL];
    uint32_t kx[NJ][KL], vx[VL];  // E2M1: their exponents
    bool bad_page = false;
    const auto find = [&](int32_t key, Place &p) { bad_page |= find_place<KV>(a, table, kvh, key, p); };
    // WIDE: lane l knows where the 16 keys l % NJ of the wavefront's block l / NJ from known_from
    // on are
    Place at_l{};
    int32_t known_from = 0;
    const auto find_blocks = [&](int32_t kb) {
      int32_t key = kb + (lane / NJ) * (FK * FW) + (lane % NJ) * 16;
      key = key < last_key ? key : last_key;  // 16 keys outside [k0, k1) read a neighbour's places: in bounds, not seen
      key = key > k0 ? key : k0;
      find(key & ~15, at_l);
      known_from = kb;
    };
    // in E2M1 a group's exponent is that of the piece it lies in, or of the two pieces
    const auto group = [](int piece) { return D == 64 ? piece / 2 : piece; };
    const uint32_t k_lane = uint32_t(col) * uint32_t(a.cache.k.token) + grp * PB;
    const uint32_t v_lane = uint32_t(r0) * uint32_t(a.cache.v.token) + (lane % VROW) * PB;
    const uint32_t ke_lane = KV4 ? uint32_t(col) * uint32_t(a.cache.k_exp.token) + group(grp) : 0;
    const uint32_t ve_lane = KV4 ? uint32_t(r0) * uint32_t(a.cache.v_exp.token) + group(lane % VROW) : 0;
    const auto load_block = [&](int32_t kb) {
      if (WIDE) {
        const int from = (kb - known_from) / (FK * FW) * NJ;
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          const uint64_t kp = read_lane(at_l.k, from + j), vp = read_lane(at_l.v, from + j);
#pragma unroll
          for (int s = 0; s < KL; ++s) kr[j][s] = load_piece<PB>(kp, k_lane + s * (4 * PB));
#pragma unroll
          for (int i = 0; i < VL / NJ; ++i)
            vr[j * (VL / NJ) + i] = load_piece<PB>(vp, v_lane + uint32_t(i * VRPI) * uint32_t(a.cache.v.token));
          if (KV4) {
            const uint64_t ke = read_lane(at_l.k_exp, from + j), ve = read_lane(at_l.v_exp, from + j);
#pragma unroll
            for (int s = 0; s < KL; ++s) kx[j][s] = load_exp(ke, ke_lane + 4 * s);
#pragma unroll
            for (int i = 0; i < VL / NJ; ++i)
              vx[j * (VL / NJ) + i] = load_exp(ve, ve_lane + uint32_t(i * VRPI) * uint32_t(a.cache.v_exp.token));
          }
        }
      } else {
        int32_t key = kb + (lane & (FK - 1));
        key = key < last_key ? key : last_key;
        key = key > k0 ? key : k0;
        Place at;
        find(key, at);
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          const uint64_t p = __shfl(at.k, 16 * j + col) + grp * PB;
#pragma unroll
          for (int s = 0; s < KL; ++s) kr[j][s] = load_piece<PB>(p + s * (4 * PB));
          if (KV4) {
            const uint64_t e = __shfl(at.k_exp, 16 * j + col);
#pragma unroll
            for (int s = 0; s < KL; ++s) kx[j][s] = load_exp(e + group(grp + 4 * s));
          }
        }
#pragma unroll
        for (int i = 0; i < VL; ++i) {
          vr[i] = load_piece<PB>(__shfl(at.v, i * VRPI + r0) + (lane % VROW) * PB);
          if (KV4) vx[i] = load_exp(__shfl(at.v_exp, i * VRPI + r0) + group(lane % VROW));
        }
      }
    };

    f32x4 o[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i) o[i] = f32x4{0, 0, 0, 0};
    float m = -INFINITY, l = 0.0f, exact = 0.0f;
    bool odd = false;  // a value that rows see differently is not finite
    if (kb0 < k1) {
      if (WIDE) find_blocks(kb0);
      load_block(kb0);
    }
    for (int32_t kb = kb0; kb < k1; kb += FK * FW) {
      // S^T: lane (grp, col) gets row col's scores of keys kb + 16 j + 4 grp + r
      f32x4 s[NJ];
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        s[j] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int t = 0; t < STEPS; ++t) {
          u32x4 k;
          if (KV8) {
            const u32x4 w = kr[j][t / 2];
            const uint32_t x = t % 2 ? w.z : w.x, y = t % 2 ? w.w : w.y;
            k = u32x4{T::template from_e4m3<false>(x), T::template from_e4m3<true>(x), T::template from_e4m3<false>(y),
                      T::template from_e4m3<true>(y)};
          } else if (KV4) {
            constexpr int PER = PB / 4;  // steps of a piece
            k = T::eight_e2m1(kr[j][t / PER][t % PER], power_of(kx[j][t / PER]));
          } else {
            k = kr[j][t];
          }
          s[j] = T::mfma16(k, q[t], s[j]);
        }
      }
      const bool partial = kb < k0 || kb + FK > k1, masked = kb < max_lo || kb + FK > min_hi;
      // Values to LDS, as 16-bit rows; zeros in place of those that are not finite where rows differ
      // in what they see, as 0 times them must not reach a row that does not see them (added in the
      // end, from memory again, to the rows that do: weights are positive, infinities and NaN come
      // through as they are).
      const bool apart = masked && !one_token;
      wave_fence();
      const int to_now = KV4 ? again(to) : to, from_now = KV4 ? again(from_t) : from_t;
#pragma unroll
      for (int i = 0; i < VL; ++i) {
        u32x4 v = KV4 ? flipped(vr[i], flip) : vr[i], w[PIECES];
        uint32_t e = KV4 ? vx[i] : 0;
        if (partial && (kb + i * VRPI + r0 < k0 || kb + i * VRPI + r0 >= k1)) {
          v = u32x4{0, 0, 0, 0};
          e = 127;  // (it may be a NaN's, and 0 times that)
        }
        if (KV8) {
          w[0] = u32x4{T::template from_e4m3<false>(v.x), T::template from_e4m3<true>(v.x), T::template from_e4m3<false>(v.y),
                       T::template from_e4m3<true>(v.y)};
          w[PIECES - 1] = u32x4{T::template from_e4m3<false>(v.z), T::template from_e4m3<true>(v.z), T::template from_e4m3<false>(v.w),
                           T::template from_e4m3<true>(v.w)};
        } else if (KV4) {
#pragma unroll
          for (int n = 0; n < PIECES; ++n) w[n] = T::eight_e2m1(v[n], power_of(e));
        } else {
          w[0] = v;
        }
        if (apart) {
#pragma unroll
          for (int n = 0; n < PIECES; ++n)
            if (any_not_finite<T>(w[n])) {
              odd = true;
              w[n] = finite_only<T>(w[n]);
            }
        }
#pragma unroll
        for (int n = 0; n < PIECES; ++n)
          *reinterpret_cast<u32x4 *>(lds + (to_now ^ 16 * (n ^ (2 * ((i * VRPI) & SWZ)))) + i * VRPI * (2 * D)) = w[n];
      }
      wave_fence();
      const int32_t next = kb + FK * FW;
      if (next < k1) {
        if (WIDE && next - known_from >= 64 / NJ * FK * FW) find_blocks(next);
        load_block(next);
      }
      // weights
      float p[4 * NJ];
#pragma unroll
      for (int e = 0; e < 4 * NJ; ++e) p[e] = s[e / 4][e % 4];
      if (SCORES && capped.cap > CAP_NEAR) {
#pragma unroll
        for (int e = 0; e < 4 * NJ; ++e) p[e] = capped.far(p[e]);
      } else if (SCORES && capped.cap > 0.0f) {
#pragma unroll
        for (int e = 0; e < 4 * NJ; ++e) p[e] = capped(p[e]);
      } else if (!LATE) {
#pragma unroll
        for (int e = 0; e < 4 * NJ; ++e) p[e] *= sc;
      }
      if (SCORES && a.slopes) {
        const float from = bias.slope * float(kb + 4 * grp - bias.from);
#pragma unroll
        for (int e = 0; e < 4 * NJ; ++e) p[e] += fmaf(bias.slope, float(16 * (e / 4) + e % 4), from);
      }
      if (masked) {
#pragma unroll
        for (int e = 0; e < 4 * NJ; ++e) {
          const int32_t key = kb + 16 * (e / 4) + 4 * grp + e % 4;
          if (key >= hi || key < lo) p[e] = -INFINITY;
        }
      }
      float mx = p[0];
#pragma unroll
      for (int e = 1; e < 4 * NJ; ++e) mx = fmaxf(mx, p[e]);
      mx = max4(LATE ? mx * sc : mx);
      if (__any(mx > m)) {
        const float mn = fmaxf(m, mx);
        const float down = mn == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - mn);
        m = mn;
        l *= down;
        exact *= down;
#pragma unroll
        for (int i = 0; i < DT; ++i) o[i] *= down;
      }
      const float base = (m == -INFINITY ? 0.0f : m) - T::FEW_SHIFT;
#pragma unroll
      for (int e = 0; e < 4 * NJ; ++e) {
        p[e] = __builtin_amdgcn_exp2f(LATE ? fmaf(p[e], sc, -base) : p[e] - base);
        exact += p[e];
      }
#pragma unroll
      for (int t = 0; t < NJ / 2; ++t) {
        const u32x4 pw{T::pack(p[8 * t], p[8 * t + 1]), T::pack(p[8 * t + 2], p[8 * t + 3]), T::pack(p[8 * t + 4], p[8 * t + 5]),
                       T::pack(p[8 * t + 6], p[8 * t + 7])};
#pragma unroll
        for (int e = 0; e < 4; ++e) l = T::add_two(pw[e], l);
#pragma unroll
        for (int i = 0; i < DT; ++i) {
          const char *x = lds + (from_now ^ 32 * i) + t * 32 * (2 * D);
          const u32x2 v0 = read_transposed(x), v1 = read_transposed(x + 16 * (2 * D));  // r + 16: the same exchange
          o[i] = T::mfma16(u32x4{v0.x, v0.y, v1.x, v1.y}, pw, o[i]);
        }
      }
    }
    if (!one_token && __any(odd)) {
#pragma unroll 1
      for (int32_t kb = kb0; kb < k1; kb += FK * FW) {
        if (kb >= max_lo && kb + FK <= min_hi) continue;
#pragma unroll 1
        for (int32_t key = max(kb, k0); key < min(kb + FK, k1); ++key) {
          Place at;
          find(key, at);
          const bool seen = key < hi && key >= lo;
#pragma unroll
          for (int i = 0; i < DT; ++i) {
            const f32x4 v = four_values<T, KV>(at, 16 * i + 4 * grp);
#pragma unroll
            for (int k = 0; k < 4; ++k) o[i][k] = seen && !is_finite(v[k]) ? o[i][k] + v[k] : o[i][k];
            __builtin_amdgcn_sched_barrier(0);  // (rare: in few registers)
          }
        }
      }
    }
    if (bad_page) set_status(a.status, SMETRIC_EINVAL);

    // join the wavefronts
    l = sum4(l);
    exact = sum4(exact);
    wave_fence();
#pragma unroll
    for (int i = 0; i < DT; ++i)
      *reinterpret_cast<f32x4 *>(my + (col * PADDED + 16 * i + 4 * grp) * 4) = o[i];
    if (grp == 0) {
      ml[wave][col][0] = m;
      ml[wave][col][1] = l;
      ml[wave][col][2] = exact;
      if (SCORES && wave == 0) more[col] = bias.more(place);
    }
    __syncthreads();
    constexpr int N = D / 16;  // components of a thread
    const int jr = threadIdx.x / 16, jc = threadIdx.x % 16 * N;
    if (jr < n_rows) {
      float mm = ml[0][jr][0];
#pragma unroll
      for (int w = 1; w < FW; ++w) mm = fmaxf(mm, ml[w][jr][0]);
      const float ms = mm == -INFINITY ? 0.0f : mm;
      float acc[N], ll = 0.0f, le = 0.0f;
#pragma unroll
      for (int i = 0; i < N; ++i) acc[i] = 0.0f;
#pragma unroll
      for (int w = 0; w < FW; ++w) {
        const float f = __builtin_amdgcn_exp2f(ml[w][jr][0] - ms);
        ll = fmaf(f, ml[w][jr][1], ll);
        le = fmaf(f, ml[w][jr][2], le);
        const float *x = reinterpret_cast<const float *>(lds + w * REGION) + jr * PADDED + jc;
#pragma unroll
        for (int i = 0; i < N; ++i) acc[i] = fmaf(f, x[i], acc[i]);
      }
      const float vs = KV8 && a.cache.v_scale ? a.cache.v_scale[kvh] : 1.0f;
      if (it.part < 0) {
        const float inv = ll == 0.0f ? 0.0f : vs / ll;
        const int32_t jrow = row0 + jr, jt = jrow / a.group, jh = kvh * a.group + jrow % a.group;
        uint16_t *p = a.out.data + (int64_t(it.tok0) + jt) * a.out.token + jh * a.out.head + jc;
#pragma unroll
        for (int i = 0; i < N; i += 4)
          *reinterpret_cast<u32x2 *>(p + i) =
              u32x2{T::pack(acc[i] * inv, acc[i + 1] * inv), T::pack(acc[i + 2] * inv, acc[i + 3] * inv)};
        if (a.lse && jc == 0) a.lse[(int64_t(it.tok0) + jt) * a.n_q + jh] = lse_of(mm, le, T::FEW_SHIFT, SCORES ? more[jr] : 0.0f);
      } else {
        const int64_t slot = (int64_t(it.part) * a.n_kv + kvh) * FEW_ROWS + jr;
#pragma unroll
        for (int i = 0; i < N; i += 4)
          *reinterpret_cast<f32x4 *>(a.parts.acc + slot * D + jc + i) =
              f32x4{acc[i] * vs, acc[i + 1] * vs, acc[i + 2] * vs, acc[i + 3] * vs};
        if (jc == 0) a.parts.ml[slot] = f32x4{mm, ll, le, SCORES ? more[jr] : 0.0f};
      }
    }
    __syncthreads();  // the next piece's values go where these sums were
  }
}

#ifdef SCORED
constexpr bool OTHER_SCORES = true;
#else
constexpr bool OTHER_SCORES = false;
#endif
template <typename T, Pages KV, int D>
int launch_d(const AttendArgs &a, int64_t max_groups, hipStream_t stream) {
  const dim3 grid(uint32_t(max_groups * a.n_kv)), block(64 * few_waves(KV, D));
  if (a.cache.ps.size % 16 == 0)
    few_kernel<T, KV, D, true, OTHER_SCORES><<<grid, block, 0, stream>>>(a);
  else
    few_kernel<T, KV, D, false, OTHER_SCORES><<<grid, block, 0, stream>>>(a);
  return hip_status(hipGetLastError());
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
int launch_few_scores(
#else
int launch_few(
#endif
    const AttendArgs &a, int32_t dtype, Pages pages, int32_t head_dim, int64_t max_groups, hipStream_t stream) {
  return dtype == SMETRIC_BF16 ? launch_t<Bf16>(a, pages, head_dim, max_groups, stream)
                               : launch_t<F16>(a, pages, head_dim, max_groups, stream);
}

}  // namespace smk
