// What the serving kernels share: 16-bit types, conversions, division.
#pragma once

#include <hip/hip_runtime.h>

#include "kvx_serve.h"

namespace kvx_dev {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f16v __attribute__((ext_vector_type(16)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));

constexpr int kBadBlock = 1, kBadArgument = 2;  // bits of a stream's error word (kvx_check)

__device__ __forceinline__ uint32_t divide(uint32_t n, kvx::Divisor f) {
  if (f.m == 0) return n;
  const uint32_t t = __umulhi(n, f.m);
  return (t + ((n - t) >> 1)) >> f.s;
}

struct Bf16 {
  using T = __bf16;
  static __device__ __forceinline__ f4 mfma16(u4 a, u4 b, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8, a),
                                                   __builtin_bit_cast(bf8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ f16v mfma32(u4 a, u4 b, f16v c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8, a),
                                                   __builtin_bit_cast(bf8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    const bf2 v = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, v);
  }
  static __device__ __forceinline__ float low(uint32_t v) { return __uint_as_float(v << 16); }
  static __device__ __forceinline__ float high(uint32_t v) {
    return __uint_as_float(v & 0xFFFF0000u);
  }
  // two 8-bit words (bytes 0, 1 or 2, 3 of v) as a pair
  template <bool HI>
  static __device__ __forceinline__ uint32_t from_e4m3(uint32_t v) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, 1.0f, HI));
  }
  static constexpr uint32_t kInf = 0x7F80u;  // infinity; above it NaN
  // log2 of how far softmax weights may be above 1 when they are first rounded to this type (kvx_attn_dev.h)
  static constexpr float kLift = 0.0f;
};

struct F16 {
  using T = _Float16;
  static __device__ __forceinline__ f4 mfma16(u4 a, u4 b, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, a),
                                                  __builtin_bit_cast(h8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ f16v mfma32(u4 a, u4 b, f16v c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8, a),
                                                  __builtin_bit_cast(h8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    const h2 v = {(_Float16)a, (_Float16)b};
    return __builtin_bit_cast(uint32_t, v);
  }
  static __device__ __forceinline__ float low(uint32_t v) {
    return (float)__builtin_bit_cast(h2, v)[0];
  }
  static __device__ __forceinline__ float high(uint32_t v) {
    return (float)__builtin_bit_cast(h2, v)[1];
  }
  template <bool HI>
  static __device__ __forceinline__ uint32_t from_e4m3(uint32_t v) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v, 1.0f, HI));
  }
  static constexpr uint32_t kInf = 0x7C00u;
  static constexpr float kLift = 7.0f;
};

// Eight 8-bit words as eight 16-bit ones.
template <class T>
__device__ __forceinline__ u4 widen(uint32_t a, uint32_t b) {
  u4 r;
  r.x = T::template from_e4m3<false>(a);
  r.y = T::template from_e4m3<true>(a);
  r.z = T::template from_e4m3<false>(b);
  r.w = T::template from_e4m3<true>(b);
  return r;
}

}  // namespace kvx_dev
