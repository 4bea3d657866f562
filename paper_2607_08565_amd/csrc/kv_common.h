// Internal definitions shared by the paged-cache kernels: 16- and 8-bit floats, page
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
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;

constexpr int32_t MAX_PLACES = 1 << 24;  // cached tokens of a request
constexpr float E4M3_MAX = 448.0f;

// Activation types: one struct per type with what the kernels ask of it.
struct Bf16 {
  typedef bf16x8 V8;
  static constexpr uint32_t EXP = 0x7F807F80u, ONE_EXP = 0x00800080u;  // exponent bits, their lowest (both halves)
  // weights are held times a power of two, for few rows and for many (whose maximum may lag by 2^8)
  static constexpr float FEW_SHIFT = 0.0f, MANY_SHIFT = 0.0f;
  __device__ static __forceinline__ float lo(uint32_t x) { return __uint_as_float(x << 16); }
  __device__ static __forceinline__ float hi(uint32_t x) { return __uint_as_float(x & 0xFFFF0000u); }
  __device__ static __forceinline__ uint32_t pack(float a, float b) {  // to nearest even, v_cvt_pk_bf16_f32
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){a, b}, bf16x2));
  }
  // two of the four E4M3 values in x
  template <bool HIGH>
  __device__ static __forceinline__ uint32_t from_e4m3(uint32_t x) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.0f, HIGH));
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
  // as large as the type allows (2^15), for it holds weights below 2^-14 with fewer than 11 bits
  static constexpr float FEW_SHIFT = 15.0f, MANY_SHIFT = 7.0f;
  __device__ static __forceinline__ float lo(uint32_t x) { return float(__builtin_bit_cast(f16x2, x).x); }
  __device__ static __forceinline__ float hi(uint32_t x) { return float(__builtin_bit_cast(f16x2, x).y); }
  __device__ static __forceinline__ uint32_t pack(float a, float b) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){a, b}, f16x2));
  }
  template <bool HIGH>
  __device__ static __forceinline__ uint32_t from_e4m3(uint32_t x) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, 1.0f, HIGH));
  }
  __device__ static __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(V8, a), __builtin_bit_cast(V8, b), c, 0, 0, 0);
  }
  __device__ static __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(V8, a), __builtin_bit_cast(V8, b), c, 0, 0, 0);
  }
};

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

// Host checks shared by the entry points (defined with the append).
bool heads_ok(const smetric_heads *h);
bool cache_ok(const smetric_kv_cache *c, int32_t dtype);
bool batch_ok(const smetric_batch *b);
CacheView cache_view(const smetric_kv_cache *c, const smetric_batch *b);
inline HeadsView heads_view(const smetric_heads *h) {
  return h ? HeadsView{static_cast<uint16_t *>(h->data), h->token_stride, h->head_stride} : HeadsView{nullptr, 0, 0};
}
inline int hip_status(hipError_t e) { return e == hipSuccess ? SMETRIC_OK : SMETRIC_EHIP; }

}  // namespace smk
