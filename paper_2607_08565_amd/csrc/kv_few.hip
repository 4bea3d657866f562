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
// to the activations' type for it, as the matrix cores take 16-bit operands; their sum is not.
//
// Measured: 32 requests decoding over 1.73 GB of cache 305 us, 5.7 TB/s (a copy of 4 GiB moves
// 4.8); 64 drafted tokens over 0.58 GB 117 us; 131,072 keys of 8 bits (134 MB) 31 to 35 us, 24
// of them here and the rest the joining; a lone token over 1,025 keys 9.5 us, two launches.
#include <math.h>

#include "kv_attend.h"

namespace smk {
namespace {

constexpr int FW = 4;     // wavefronts
constexpr int FK = 32;    // keys of a wavefront's block

__device__ __forceinline__ void wave_fence() {  // orders the wavefront's LDS accesses; no instruction
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}
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
template <typename T, bool KV8, int D, bool WIDE>
__global__ __launch_bounds__(64 * FW, at_once(D)) void few_kernel(AttendArgs a) {
  constexpr int ESZ = KV8 ? 1 : 2;
  constexpr int STEPS = D / 32;               // matrix steps over the components
  constexpr int KL = D * ESZ / 64;            // 16-byte loads of a lane for 16 keys
  constexpr int VL = FK * D * ESZ / 1024;     // 16-byte loads of a lane for a block's values
  constexpr int VROW = D * ESZ / 16;          // lanes per row of values
  constexpr int VRPI = 64 / VROW;             // rows per load
  constexpr int DT = D / 16;
  constexpr int PADDED = D + 4;               // floats of a row in the joining of the wavefronts
  constexpr int REGION = 16 * PADDED * 4;     // bytes of a wavefront's LDS: 32 rows of values, later its sums
  constexpr int SWZ = D == 64 ? 3 : 7;
  static_assert(REGION >= FK * D * 2, "values fit");
  __shared__ __attribute__((aligned(16))) char lds[FW * REGION];
  __shared__ float ml[FW][16][2];

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
  const int col = lane & 15, grp = lane >> 4;
  for (int32_t piece = first_piece; piece < last_piece; ++piece) {
    const PlanItem it = uniform(a.items[piece]);
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
      const int d = KV8 ? (s / 2) * 64 + grp * 16 + (s % 2) * 8 : s * 32 + grp * 8;
      q[s] = u32x4{0, 0, 0, 0};
      if (has_row)
        q[s] = *reinterpret_cast<const u32x4 *>(a.q.data + (int64_t(it.tok0) + tok) * a.q.token + head * a.q.head + d);
    }
    const char *kbase = a.cache.k.base + kvh * a.cache.k.head;
    const char *vbase = a.cache.v.base + kvh * a.cache.v.head;
    const int32_t *table = a.cache.table + it.req * a.cache.table_stride;
    const float sc = a.scale_log2 * (KV8 && a.cache.k_scale ? a.cache.k_scale[kvh] : 1.0f);
    char *my = lds + wave * REGION;

    const int32_t kb0 = k0 / KEY_STEP * KEY_STEP + FK * wave;
    const int32_t last_key = k1 - 1;
    u32x4 kr[2][KL], vr[VL];
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
    // WIDE: lane l knows where the 16 keys l % 2 of the wavefront's block l / 2 from known_from
    // on are
    uint64_t kp_l = 0, vp_l = 0;
    int32_t known_from = 0;
    const auto find_blocks = [&](int32_t kb) {
      int32_t key = kb + (lane >> 1) * (FK * FW) + (lane & 1) * 16;
      key = key < last_key ? key : last_key;  // 16 keys outside [k0, k1) read a neighbour's places: in bounds, not seen
      key = key > k0 ? key : k0;
      find(key & ~15, kp_l, vp_l);
      known_from = kb;
    };
    const auto load_block = [&](int32_t kb) {
      if (WIDE) {
        const int from = (kb - known_from) / (FK * FW) * 2;
        const uint32_t ko = uint32_t(col) * uint32_t(a.cache.k.token) + grp * 16;
        const uint32_t vo = uint32_t(lane / VROW) * uint32_t(a.cache.v.token) + (lane % VROW) * 16;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const char *kp = reinterpret_cast<const char *>(read_lane(kp_l, from + j));
          const char *vp = reinterpret_cast<const char *>(read_lane(vp_l, from + j));
#pragma unroll
          for (int s = 0; s < KL; ++s) kr[j][s] = *reinterpret_cast<const u32x4 *>(kp + ko + s * 64);
#pragma unroll
          for (int i = 0; i < VL / 2; ++i)
            vr[j * (VL / 2) + i] =
                *reinterpret_cast<const u32x4 *>(vp + vo + uint32_t(i * VRPI) * uint32_t(a.cache.v.token));
        }
      } else {
        int32_t key = kb + (lane & 31);
        key = key < last_key ? key : last_key;
        key = key > k0 ? key : k0;
        uint64_t kp, vp;
        find(key, kp, vp);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const char *p = reinterpret_cast<const char *>(__shfl(kp, 16 * j + col)) + grp * 16;
#pragma unroll
          for (int s = 0; s < KL; ++s) kr[j][s] = *reinterpret_cast<const u32x4 *>(p + s * 64);
        }
#pragma unroll
        for (int i = 0; i < VL; ++i)
          vr[i] = *reinterpret_cast<const u32x4 *>(reinterpret_cast<const char *>(__shfl(vp, i * VRPI + lane / VROW)) +
                                                   (lane % VROW) * 16);
      }
    };

    f32x4 o[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i) o[i] = f32x4{0, 0, 0, 0};
    float m = -INFINITY, l = 0.0f;
    bool odd = false;  // a value that rows see differently is not finite
    if (kb0 < k1) {
      if (WIDE) find_blocks(kb0);
      load_block(kb0);
    }
    for (int32_t kb = kb0; kb < k1; kb += FK * FW) {
      // S^T: lane (grp, col) gets row col's scores of keys kb + 16 j + 4 grp + r
      f32x4 s[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        s[j] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int t = 0; t < STEPS; ++t) {
          u32x4 k;
          if (KV8) {
            const u32x4 w = kr[j][t / 2];
            const uint32_t x = t % 2 ? w.z : w.x, y = t % 2 ? w.w : w.y;
            k = u32x4{T::template from_e4m3<false>(x), T::template from_e4m3<true>(x), T::template from_e4m3<false>(y),
                      T::template from_e4m3<true>(y)};
          } else {
            k = kr[j][t];
          }
          s[j] = T::mfma16(k, q[t], s[j]);
        }
      }
      const bool partial = kb < k0 || kb + FK > k1, masked = kb < max_lo || kb + FK > min_hi;
      // values to LDS, as 16-bit rows whose 16-byte pieces are exchanged within the row; zeros in
      // place of those that are not finite where rows differ in what they see, as 0 times them must
      // not reach a row that does not see them (added in the end, from memory again, to the rows that
      // do: weights are positive, infinities and NaN come through as they are)
      const bool apart = masked && !one_token;
      const auto finite = [&](u32x4 x) {
        if (!apart || !any_not_finite<T>(x)) return x;
        odd = true;
        return finite_only<T>(x);
      };
      wave_fence();
#pragma unroll
      for (int i = 0; i < VL; ++i) {
        const int r = i * VRPI + lane / VROW, c = lane % VROW;
        u32x4 v = vr[i];
        if (partial && (kb + r < k0 || kb + r >= k1)) v = u32x4{0, 0, 0, 0};
        if (KV8) {
          const u32x4 x{T::template from_e4m3<false>(v.x), T::template from_e4m3<true>(v.x),
                        T::template from_e4m3<false>(v.y), T::template from_e4m3<true>(v.y)};
          const u32x4 y{T::template from_e4m3<false>(v.z), T::template from_e4m3<true>(v.z),
                        T::template from_e4m3<false>(v.w), T::template from_e4m3<true>(v.w)};
          *reinterpret_cast<u32x4 *>(my + r * (2 * D) + (((2 * c) ^ (2 * (r & SWZ))) * 16)) = finite(x);
          *reinterpret_cast<u32x4 *>(my + r * (2 * D) + (((2 * c + 1) ^ (2 * (r & SWZ))) * 16)) = finite(y);
        } else {
          *reinterpret_cast<u32x4 *>(my + r * (2 * D) + ((c ^ (2 * (r & SWZ))) * 16)) = finite(v);
        }
      }
      wave_fence();
      const int32_t next = kb + FK * FW;
      if (next < k1) {
        if (WIDE && next - known_from >= 32 * FK * FW) find_blocks(next);
        load_block(next);
      }
      // weights
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = s[e / 4][e % 4] * sc;
      if (masked) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int32_t key = kb + 16 * (e / 4) + 4 * grp + e % 4;
          if (key >= hi || key < lo) p[e] = -INFINITY;
        }
      }
      float mx = p[0];
#pragma unroll
      for (int e = 1; e < 8; ++e) mx = fmaxf(mx, p[e]);
      mx = max4(mx);
      if (__any(mx > m)) {
        const float mn = fmaxf(m, mx);
        const float down = mn == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - mn);
        m = mn;
        l *= down;
#pragma unroll
        for (int i = 0; i < DT; ++i) o[i] *= down;
      }
      const float base = (m == -INFINITY ? 0.0f : m) - T::FEW_SHIFT;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[e] = __builtin_amdgcn_exp2f(p[e] - base);
        l += p[e];
      }
      const u32x4 pw{T::pack(p[0], p[1]), T::pack(p[2], p[3]), T::pack(p[4], p[5]), T::pack(p[6], p[7])};
#pragma unroll
      for (int i = 0; i < DT; ++i) {
        const int r = 4 * grp + col / 4, c = 2 * i + (col % 4) / 2;
        const char *x = my + r * (2 * D) + ((c ^ (2 * (r & SWZ))) * 16) + (col & 1) * 8;
        const u32x2 v0 = read_transposed(x), v1 = read_transposed(x + 16 * (2 * D));  // r + 16: the same exchange
        o[i] = T::mfma16(u32x4{v0.x, v0.y, v1.x, v1.y}, pw, o[i]);
      }
    }
    if (!one_token && __any(odd)) {
#pragma unroll 1
      for (int32_t kb = kb0; kb < k1; kb += FK * FW) {
        if (kb >= max_lo && kb + FK <= min_hi) continue;
#pragma unroll 1
        for (int32_t key = max(kb, k0); key < min(kb + FK, k1); ++key) {
          uint64_t kp, vp;
          find(key, kp, vp);
          const bool seen = key < hi && key >= lo;
#pragma unroll
          for (int i = 0; i < DT; ++i) {
            const f32x4 v = four_values<T, KV8>(vp, 16 * i + 4 * grp);
#pragma unroll
            for (int k = 0; k < 4; ++k) o[i][k] = seen && !is_finite(v[k]) ? o[i][k] + v[k] : o[i][k];
          }
        }
      }
    }
    if (bad_page) set_status(a.status, SMETRIC_EINVAL);

    // join the wavefronts
    l = sum4(l);
    wave_fence();
#pragma unroll
    for (int i = 0; i < DT; ++i)
      *reinterpret_cast<f32x4 *>(my + (col * PADDED + 16 * i + 4 * grp) * 4) = o[i];
    if (grp == 0) {
      ml[wave][col][0] = m;
      ml[wave][col][1] = l;
    }
    __syncthreads();
    constexpr int N = D / 16;  // components of a thread
    const int jr = threadIdx.x / 16, jc = threadIdx.x % 16 * N;
    if (jr < n_rows) {
      float mm = ml[0][jr][0];
#pragma unroll
      for (int w = 1; w < FW; ++w) mm = fmaxf(mm, ml[w][jr][0]);
      const float ms = mm == -INFINITY ? 0.0f : mm;
      float acc[N], ll = 0.0f;
#pragma unroll
      for (int i = 0; i < N; ++i) acc[i] = 0.0f;
#pragma unroll
      for (int w = 0; w < FW; ++w) {
        const float f = __builtin_amdgcn_exp2f(ml[w][jr][0] - ms);
        ll = fmaf(f, ml[w][jr][1], ll);
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
        if (a.lse && jc == 0) a.lse[(int64_t(it.tok0) + jt) * a.n_q + jh] = lse_of(mm, ll, T::FEW_SHIFT);
      } else {
        const int64_t slot = (int64_t(it.part) * a.n_kv + kvh) * FEW_ROWS + jr;
#pragma unroll
        for (int i = 0; i < N; i += 4)
          *reinterpret_cast<f32x4 *>(a.parts.acc + slot * D + jc + i) =
              f32x4{acc[i] * vs, acc[i + 1] * vs, acc[i + 2] * vs, acc[i + 3] * vs};
        if (jc == 0) a.parts.ml[slot] = f32x2{mm, ll};
      }
    }
    __syncthreads();  // the next piece's values go where these sums were
  }
}

template <typename T, bool KV8, int D>
int launch_d(const AttendArgs &a, int64_t max_groups, hipStream_t stream) {
  const dim3 grid(uint32_t(max_groups * a.n_kv)), block(64 * FW);
  if (a.cache.ps.size % 16 == 0)
    few_kernel<T, KV8, D, true><<<grid, block, 0, stream>>>(a);
  else
    few_kernel<T, KV8, D, false><<<grid, block, 0, stream>>>(a);
  return hip_status(hipGetLastError());
}
template <typename T, bool KV8>
int launch_k(const AttendArgs &a, int32_t d, int64_t max_groups, hipStream_t stream) {
  return d == 64 ? launch_d<T, KV8, 64>(a, max_groups, stream)
                 : d == 128 ? launch_d<T, KV8, 128>(a, max_groups, stream) : launch_d<T, KV8, 256>(a, max_groups, stream);
}

}  // namespace

int launch_few(const AttendArgs &a, int32_t dtype, bool kv8, int32_t head_dim, int64_t max_groups, hipStream_t stream) {
  if (dtype == SMETRIC_BF16)
    return kv8 ? launch_k<Bf16, true>(a, head_dim, max_groups, stream) : launch_k<Bf16, false>(a, head_dim, max_groups, stream);
  return kv8 ? launch_k<F16, true>(a, head_dim, max_groups, stream) : launch_k<F16, false>(a, head_dim, max_groups, stream);
}

}  // namespace smk
