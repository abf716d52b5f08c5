// Codes of the paged 8-bit cache on the device (include/jpi_cache.h).
#pragma once

#include "jpi_cache_internal.h"
#include "jpi_device.h"

namespace jpi {
namespace {

typedef unsigned int u32;
typedef u32 u32x2 __attribute__((ext_vector_type(2)));
typedef u32 u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

template <bool E4M3>
struct Code;

template <>
struct Code<true> {
  static constexpr float TOP = 448.f;
  static constexpr u32 TOP_FRACTION = 0x600000;  // 448 = 1.75 * 2^8
  static constexpr int TOP_EXPONENT = 8;
  static __device__ __forceinline__ u32 encode4(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (u32)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
  }
  static __device__ __forceinline__ void decode4(u32 w, float (&f)[4]) {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    f[0] = lo[0], f[1] = lo[1], f[2] = hi[0], f[3] = hi[1];
  }
  // eight codes as bf16, which holds them exactly
  static __device__ __forceinline__ bf16x8 widen8(u32 a, u32 b) {
    const bf16x2 x = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, false), y = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, true);
    const bf16x2 z = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, false), w = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, true);
    return bf16x8{x[0], x[1], y[0], y[1], z[0], z[1], w[0], w[1]};
  }
};

template <>
struct Code<false> {
  static constexpr float TOP = 127.f;
  static constexpr u32 TOP_FRACTION = 0x7e0000;  // 127 = 1.984375 * 2^6
  static constexpr int TOP_EXPONENT = 6;
  static __device__ __forceinline__ u32 encode4(float a, float b, float c, float d) {
    const u32 x = (u32)(int)rintf(a) & 255, y = (u32)(int)rintf(b) & 255, z = (u32)(int)rintf(c) & 255, w = (u32)(int)rintf(d);
    return x | y << 8 | z << 16 | w << 24;
  }
  static __device__ __forceinline__ void decode4(u32 w, float (&f)[4]) {
    f[0] = (float)(int8_t)w, f[1] = (float)(int8_t)(w >> 8), f[2] = (float)(int8_t)(w >> 16), f[3] = (float)((int)w >> 24);
  }
  static __device__ __forceinline__ bf16x8 widen8(u32 a, u32 b) {
    float x[4], y[4];
    decode4(a, x), decode4(b, y);
    return bf16x8{(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3], (__bf16)y[0], (__bf16)y[1], (__bf16)y[2], (__bf16)y[3]};
  }
};

// The least 2^e, e >= -126, with TOP * 2^e >= x, for a finite x >= 0 given by its bits
template <bool E4M3>
__device__ __forceinline__ float scale_for(u32 bits) {
  typedef Code<E4M3> C;
  // a subnormal x needs an exponent far below -126
  const int e = (int)(bits >> 23) - 127 - C::TOP_EXPONENT + ((bits & 0x7fffff) > C::TOP_FRACTION ? 1 : 0);
  return __builtin_bit_cast(float, (u32)(max(e, -126) + 127) << 23);
}

__device__ __forceinline__ int clamp_len(int n, int most) { return min(max(n, 0), most); }

}  // namespace
}  // namespace jpi
