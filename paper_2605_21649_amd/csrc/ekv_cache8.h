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

// Codes of 8 numbers divided by a power of two s: to nearest, ties to even, NaN for infinities and NaN (the conversion makes a
// code of its own of each pair; it gives NaN for what lies beyond the largest code too, so with CLAMP numbers are first kept within).
typedef __attribute__((ext_vector_type(2))) short s16x2_t;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float s) {
  s16x2_t r = {0, 0};
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, a, b, s, false);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, c, d, s, true);
  return __builtin_bit_cast(uint32_t, r);
}
__device__ __forceinline__ uint32_t codes4(uint32_t ab, uint32_t cd, float s) {      // of two pairs of bf16
  s16x2_t r = {0, 0};
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2_t, ab), s, false);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2_t, cd), s, true);
  return __builtin_bit_cast(uint32_t, r);
}
__device__ __forceinline__ uint2 codes8(const Raw8<float>& x, float s) {
  return make_uint2(codes4(x.a.x, x.a.y, x.a.z, x.a.w, s), codes4(x.b.x, x.b.y, x.b.z, x.b.w, s));
}
__device__ __forceinline__ uint2 codes8(const Raw8<bf16_t>& x, float s) {
  return make_uint2(codes4(x.a.x, x.a.y, s), codes4(x.a.z, x.a.w, s));
}
// Numbers beyond +-448 s (what rounding to the largest scale leaves) at it; s >= 2^-100, so that the limit is a normal number
__device__ __forceinline__ uint2 codes8_clamped(const float (&v)[8], float s) {
  const float most = kMaxCode * s;
  float x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = __builtin_fabsf(v[i]) < INFINITY ? __builtin_amdgcn_fmed3f(v[i], -most, most) : v[i];
  return make_uint2(codes4(x[0], x[1], x[2], x[3], s), codes4(x[4], x[5], x[6], x[7], s));
}
// The codes' values times s, a power of two (exact)
__device__ __forceinline__ void values8(const uint2& c, float s, float (&x)[8]) {
  const f32x2_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c.x, s, false), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c.x, s, true);
  const f32x2_t d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c.y, s, false), e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c.y, s, true);
  x[0] = a[0]; x[1] = a[1]; x[2] = b[0]; x[3] = b[1];
  x[4] = d[0]; x[5] = d[1]; x[6] = e[0]; x[7] = e[1];
}
// The largest magnitude of 8 numbers as bits, which order as magnitudes do; NaN above infinity.  bf16: a pair of 16-bit maxima.
__device__ __forceinline__ uint32_t max_bits(const Raw8<float>& x, uint32_t m) {
  auto b = [](float f) { return __float_as_uint(f) & 0x7fffffffu; };
  m = max(m, max(b(x.a.x), b(x.a.y)));
  m = max(m, max(b(x.a.z), b(x.a.w)));
  m = max(m, max(b(x.b.x), b(x.b.y)));
  return max(m, max(b(x.b.z), b(x.b.w)));
}
__device__ __forceinline__ uint32_t max_bits(const Raw8<bf16_t>& x, uint32_t m) {
  typedef __attribute__((ext_vector_type(2))) unsigned short u16x2_t;
  auto b = [](uint32_t w) { return __builtin_bit_cast(u16x2_t, w & 0x7fff7fffu); };
  u16x2_t p = __builtin_bit_cast(u16x2_t, m);
  p = __builtin_elementwise_max(p, b(x.a.x));
  p = __builtin_elementwise_max(p, b(x.a.y));
  p = __builtin_elementwise_max(p, b(x.a.z));
  p = __builtin_elementwise_max(p, b(x.a.w));
  return __builtin_bit_cast(uint32_t, p);
}
template <typename T> __device__ __forceinline__ uint32_t max_as_float_bits(uint32_t m) {
  return sizeof(T) == 4 ? m : max(m & 0xffffu, m >> 16) << 16;
}

}  // namespace ekv
