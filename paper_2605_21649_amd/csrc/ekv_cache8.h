// The cache held in 8 bits: OCP E4M3 codes with a power-of-two scale per page and KV head, on the device.
#pragma once
#include "ekv_device.h"

namespace ekv {

struct e4m3_t { uint8_t bits; };

// 8 channels of a row of codes
template <> struct Raw8<e4m3_t> { uint2 a; };
__device__ __forceinline__ void load_raw8(const e4m3_t* p, Raw8<e4m3_t>& r) { r.a = *reinterpret_cast<const uint2*>(p); }

typedef __attribute__((ext_vector_type(2))) float f32x2_t;
// values of the codes, without the scale (exact)
__device__ __forceinline__ void widen8(const Raw8<e4m3_t>& r, float (&x)[8]) {
  const f32x2_t a = __builtin_amdgcn_cvt_pk_f32_fp8((int)r.a.x, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)r.a.x, true);
  const f32x2_t c = __builtin_amdgcn_cvt_pk_f32_fp8((int)r.a.y, false), d = __builtin_amdgcn_cvt_pk_f32_fp8((int)r.a.y, true);
  x[0] = a[0]; x[1] = a[1]; x[2] = b[0]; x[3] = b[1];
  x[4] = c[0]; x[5] = c[1]; x[6] = d[0]; x[7] = d[1];
}

constexpr float kMaxCode = 448.0f;              // largest finite value of the format
constexpr int kScaleLow = -100, kScaleHigh = 119;   // exponents of scales: code * scale stays a normal, finite float32 and bf16

// Exponent of the least power of two s with amax <= 448 s = 1.75 * 2^8 s, kept in range; amax finite, >= 0.
__device__ __forceinline__ int scale_exponent(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  return min(max(e, kScaleLow), kScaleHigh);
}
__device__ __forceinline__ float two_to(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Codes of two numbers that were divided by the scale: to nearest, ties to even; the clamp keeps what lies beyond the largest
// code at it (the instruction would make it NaN), and infinities and NaN become the format's NaN.
__device__ __forceinline__ uint32_t code_of(float x) { return __builtin_fabsf(x) < INFINITY ? __float_as_uint(__builtin_amdgcn_fmed3f(x, -kMaxCode, kMaxCode)) : 0x7fc00000u; }
__device__ __forceinline__ uint2 codes8(const float (&x)[8]) {
  auto f = [&](int i) { return __uint_as_float(code_of(x[i])); };
  uint2 r;
  r.x = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f(2), f(3), __builtin_amdgcn_cvt_pk_fp8_f32(f(0), f(1), 0, false), true);
  r.y = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f(6), f(7), __builtin_amdgcn_cvt_pk_fp8_f32(f(4), f(5), 0, false), true);
  return r;
}

}  // namespace ekv
