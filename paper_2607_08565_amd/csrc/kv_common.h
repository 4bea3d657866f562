// Internal definitions shared by the paged-cache kernels: 16-, 8- and 4-bit floats, page
// addressing, and the plan of an attention step.  Not part of the ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "smetric_kv.h"

namespace smk {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
typedef __attribute__((ext_vector_type(4))) _Float16 f16x4;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;

constexpr int32_t MAX_PLACES = 1 << 24;  // cached tokens of a request
constexpr float E4M3_MAX = 448.0f;
constexpr int GROUP4 = 32;  // components of E2M1 pages with one exponent

// What pages hold: the activations' 16 bits, E4M3 or E2M1.
enum Pages { PAGES16 = 0, PAGES8 = 1, PAGES4 = 2 };
constexpr int page_bytes(Pages p, int components) {
  return p == PAGES16 ? 2 * components : p == PAGES8 ? components : components / 2;
}

// Activation types: one struct per type with what the kernels ask of it.
struct Bf16 {
  typedef bf16x8 V8;
  static constexpr uint32_t EXP = 0x7F807F80u, ONE_EXP = 0x00800080u;  // exponent bits, their lowest (both halves)
  static constexpr uint32_t EXP4_MIN = 127 - 125, EXP4_MAX = 127 + 125;  // exponents whose E2M1 values it holds exactly
  // weights are held times a power of two, for few rows and for many (whose maximum may lag by 2^8)
  static constexpr float FEW_SHIFT = 0.0f, MANY_SHIFT = 0.0f;
  __device__ static __forceinline__ float lo(uint32_t x) { return __uint_as_float(x << 16); }
  __device__ static __forceinline__ float hi(uint32_t x) { return __uint_as_float(x & 0xFFFF0000u); }
  __device__ static __forceinline__ uint32_t pack(float a, float b) {  // to nearest even, v_cvt_pk_bf16_f32
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){a, b}, bf16x2));
  }
  // Sums in float32 of packed weights as the products take them (checked: rounded as additions are):
  // s and two of them; c (each of its components) and four
  __device__ static __forceinline__ float add_two(uint32_t x, float s) {
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, x), __builtin_bit_cast(bf16x2, 0x3F803F80u), s, false);
  }
  __device__ static __forceinline__ f32x4 add_four(u32x2 x, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(__builtin_bit_cast(s16x4, u32x2{0x3F803F80u, 0x3F803F80u}),
                                                  __builtin_bit_cast(s16x4, x), c, 0, 0, 0);
  }
  // two of the four E4M3 values in x
  template <bool HIGH>
  __device__ static __forceinline__ uint32_t from_e4m3(uint32_t x) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.0f, HIGH));
  }
  // Two of the eight E2M1 values in x, times scale, a power of two given as a float (its exponent
  // is what is read; all ones: NaN), rounded to nearest: checked for every byte and exponent.
  template <int PAIR>
  __device__ static __forceinline__ uint32_t from_e2m1(uint32_t x, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, PAIR));
  }
  // eight of them
  __device__ static __forceinline__ u32x4 eight_e2m1(uint32_t x, float scale) {
    return u32x4{from_e2m1<0>(x, scale), from_e2m1<1>(x, scale), from_e2m1<2>(x, scale), from_e2m1<3>(x, scale)};
  }
  __device__ static __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(V8, a), __builtin_bit_cast(V8, b), c, 0, 0, 0);
  }
  __device__ static __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(V8, a), __builtin_bit_cast(V8, b), c, 0, 0, 0);
  }
};
struct F16 {
  typedef f16x8 V8;
  static constexpr uint32_t EXP = 0x7C007C00u, ONE_EXP = 0x04000400u;
  static constexpr uint32_t EXP4_MIN = 127 - 23, EXP4_MAX = 127 + 13;
  // as large as the type allows (2^15), for it holds weights below 2^-14 with fewer than 11 bits
  static constexpr float FEW_SHIFT = 15.0f, MANY_SHIFT = 7.0f;
  __device__ static __forceinline__ float lo(uint32_t x) { return float(__builtin_bit_cast(f16x2, x).x); }
  __device__ static __forceinline__ float hi(uint32_t x) { return float(__builtin_bit_cast(f16x2, x).y); }
  __device__ static __forceinline__ uint32_t pack(float a, float b) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){a, b}, f16x2));
  }
  __device__ static __forceinline__ float add_two(uint32_t x, float s) {  // (subnormal ones as they are, as the products take them)
    return __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, x), __builtin_bit_cast(f16x2, 0x3C003C00u), s, false);
  }
  __device__ static __forceinline__ f32x4 add_four(u32x2 x, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_4x4x4f16(__builtin_bit_cast(f16x4, u32x2{0x3C003C00u, 0x3C003C00u}),
                                              __builtin_bit_cast(f16x4, x), c, 0, 0, 0);
  }
  template <bool HIGH>
  __device__ static __forceinline__ uint32_t from_e4m3(uint32_t x) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, 1.0f, HIGH));
  }
  template <int PAIR>
  __device__ static __forceinline__ uint32_t from_e2m1(uint32_t x, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(x, scale, PAIR));
  }
  // eight of them
  __device__ static __forceinline__ u32x4 eight_e2m1(uint32_t x, float scale) {
    return u32x4{from_e2m1<0>(x, scale), from_e2m1<1>(x, scale), from_e2m1<2>(x, scale), from_e2m1<3>(x, scale)};
  }
  __device__ static __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(V8, a), __builtin_bit_cast(V8, b), c, 0, 0, 0);
  }
  __device__ static __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(V8, a), __builtin_bit_cast(V8, b), c, 0, 0, 0);
  }
};

// An exponent byte as the power of two that it stands for (255: all exponent bits, NaN to from_e2m1;
// 0: zero's bits, which from_e2m1 takes for 2^-127).
__device__ __forceinline__ float power_of(uint32_t e) { return __uint_as_float(e << 23); }

// Orders a wavefront's LDS accesses; no instruction.
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

__device__ __forceinline__ void set_status(int32_t *status, int err) {
  if (status) atomicCAS(status, 0, err);
}

// Place -> page: floor(p / size) for p < 2^24 and size <= 2^16 as one 64-bit product.  With
// inv = floor(2^40 / size) + 1, p inv / 2^40 exceeds p / size by at most p / 2^40 < 2^-16,
// less than the 1 / size that p / size stays below the next whole number.
struct PageSize {
  uint64_t inv;
  int32_t size;
};
inline PageSize page_size_of(int32_t size) { return {(uint64_t(1) << 40) / uint32_t(size) + 1, size}; }
__device__ __forceinline__ int32_t page_of(PageSize s, int32_t p) { return int32_t((uint64_t(uint32_t(p)) * s.inv) >> 40); }

// One of the cache's two sides, strides in bytes.
struct PageSide {
  char *base;
  int64_t page, head, token;
};
struct CacheView {
  PageSide k, v;
  PageSide k_exp, v_exp;  // E2M1 pages' exponents
  const float *k_scale, *v_scale;
  const int32_t *table;
  int64_t table_stride;
  int32_t n_pages, max_pages;
  PageSize ps;
};
struct HeadsView {  // strides in elements of 16 bits
  uint16_t *data;
  int64_t token, head;
};

// From an address that is known to be memory's: a load that might be LDS's counts as one of both, and
// then every read of LDS waits for the keys and values on their way.
template <typename V>
__device__ __forceinline__ V from_memory(uint64_t p, uint32_t offset = 0) {
  return *(const __attribute__((address_space(1))) V *)((const __attribute__((address_space(1))) char *)p + offset);
}

// The request of a token t, the last r with q_off[r] <= t, and its numbers.
struct Request {
  int32_t r, len;    // kv_len
  int64_t from, to;  // its tokens
};
// Where a wavefront finds its tokens' requests: 64 of them from that of its first token on, each lane
// holding one's numbers, so that they come from memory in one round instead of a chain of loads.
// All lanes make it and ask it together.
struct Requests {
  const int64_t *q_off;
  const int32_t *kv_len;
  int32_t n_req, lo, len;
  int64_t from, to;
  // first: the first token, the same for all lanes.  They bisect until 64 requests are left: no
  // round up to 64 requests, one up to 4,096.
  __device__ __forceinline__ Requests(const int64_t *__restrict__ off, const int32_t *__restrict__ lens, int32_t n,
                                      int64_t first, int lane)
      : q_off(off), kv_len(lens), n_req(n), lo(0) {
    int32_t hi = n_req;  // the answer is in [lo, hi), if anywhere
    while (hi - lo > 64) {
      const int32_t step = (hi - lo + 63) / 64;
      const int32_t at = lo + lane * step;
      const int k = __popcll(__ballot(at < hi && q_off[at] <= first));
      if (k == 0) break;
      lo += (k - 1) * step;
      hi = lo + step < hi ? lo + step : hi;
    }
    const int32_t at = lo + lane < n_req ? lo + lane : n_req - 1;
    from = q_off[at];
    to = q_off[at + 1];
    len = kv_len[at];
  }
  // In order: t is at least what the lane asked for before, `in` where that was found (0 at first).
  __device__ __forceinline__ Request of(int64_t t, int &in) const {
    int64_t z = __shfl(to, in);
    for (;;) {
      const bool on = z <= t && in < 63 && lo + in + 1 < n_req;
      if (!__any(on)) break;
      in += on;
      z = __shfl(to, in);
    }
    Request q{lo + in, __shfl(len, in), __shfl(from, in), z};
    if (z <= t && q.r + 1 < n_req) {  // past the 64
      while (q.r + 1 < n_req && q_off[q.r + 1] <= t) ++q.r;
      q = Request{q.r, kv_len[q.r], q_off[q.r], q_off[q.r + 1]};
    }
    return q;
  }
};

// Host checks shared by the entry points (defined with the append).
bool heads_ok(const smetric_heads *h);
bool cache_ok(const smetric_kv_cache *c, int32_t dtype);
bool batch_ok(const smetric_batch *b);
CacheView cache_view(const smetric_kv_cache *c, const smetric_batch *b);
inline HeadsView heads_view(const smetric_heads *h) {
  return h ? HeadsView{static_cast<uint16_t *>(h->data), h->token_stride, h->head_stride} : HeadsView{nullptr, 0, 0};
}
inline Pages pages_of(const smetric_kv_cache *c) {
  return c->dtype == SMETRIC_E4M3 ? PAGES8 : c->dtype == SMETRIC_E2M1 ? PAGES4 : PAGES16;
}
inline int hip_status(hipError_t e) { return e == hipSuccess ? SMETRIC_OK : SMETRIC_EHIP; }

}  // namespace smk
