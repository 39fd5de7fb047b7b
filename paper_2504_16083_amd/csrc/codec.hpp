// The cache's codes (include/mmi_cache.h): groups of 32 channels with one
// power-of-two scale each, codes of 8 or 4 bits.
#pragma once

#include "../../include/mmi_cache.h"
#include "device.hpp"

namespace mmi {

typedef __attribute__((ext_vector_type(2))) __bf16 bf16v2;
typedef __attribute__((__vector_size__(16))) unsigned int u32x4;
typedef __attribute__((__vector_size__(8))) unsigned int u32x2;

template <int TYPE>
struct Codec {
  static constexpr int ROW = TYPE == MMI_CACHE_BF16 ? 256 : TYPE == MMI_CACHE_FP4 ? 64 : 128;   // bytes a row
  static constexpr int CH = 16 * 128 / ROW;      // channels of 16 bytes of codes
  static constexpr bool SCALED = TYPE != MMI_CACHE_BF16;
};

// Largest magnitude, as bfloat16 bits, whose nearest code stays below 2^128
// (rounding up to 2^128 would read back as an infinity): larger ones are cut.
template <int TYPE>
__device__ __forceinline__ int most_bits() {
  return TYPE == MMI_CACHE_FP8 ? 0x7f70 : TYPE == MMI_CACHE_INT8 ? 0x7f7e : 0x7f40;
}

// Scale byte of a group whose largest |x| has these bits as bfloat16 (signs
// cleared): the smallest e >= -126 with |x| <= M 2^e, M = mant 2^top; 255 if
// an infinity or a NaN is among them. M's seven mantissa bits decide whether
// |x|'s own exponent does.
template <int TYPE>
__device__ __forceinline__ int scale_byte(int amax) {
  constexpr int top = TYPE == MMI_CACHE_FP8 ? 8 : TYPE == MMI_CACHE_INT8 ? 6 : 2;
  constexpr int mant = TYPE == MMI_CACHE_FP8 ? 0x60 : TYPE == MMI_CACHE_INT8 ? 0x7e : 0x40;
  if (amax >= 0x7f80) return 255;
  amax = min(amax, most_bits<TYPE>());
  return max(1, (amax >> 7) - top + ((amax & 0x7f) > mant ? 1 : 0));
}

// 2^(127 - b): what a value is multiplied with to get its code's value (b >= 1).
__device__ __forceinline__ float scale_inverse(int b) { return __uint_as_float((uint32_t)(254 - b) << 23); }

// The scale of byte b (255: NaN; 0, which no write leaves: zero).
__device__ __forceinline__ float scale_value(uint32_t b) {
  return __uint_as_float(b == 255 ? 0x7fc00000u : b << 23);
}

// Two values that the codes can hold up to rounding, as codes (ties to even).
template <int TYPE>
__device__ __forceinline__ uint32_t encode8(float x0, float x1, float x2, float x3) {
  if (TYPE == MMI_CACHE_FP8) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(x0, x1, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x2, x3, w, true);
  }
  const int a = (int)rintf(x0), b = (int)rintf(x1), c = (int)rintf(x2), d = (int)rintf(x3);
  return (uint32_t)(a & 255) | (uint32_t)(b & 255) << 8 | (uint32_t)(c & 255) << 16 | (uint32_t)d << 24;
}

// The 8 values of bytes 0-3 of w0 and of w1 (8-bit codes) times the scale s.
template <int TYPE>
__device__ __forceinline__ bf16x8 decode8(uint32_t w0, uint32_t w1, float s) {
  bf16x8 r;
  if (TYPE == MMI_CACHE_FP8) {
    const bf16v2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, s, false);
    const bf16v2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, s, true);
    const bf16v2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, s, false);
    const bf16v2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, s, true);
    r[0] = a[0]; r[1] = a[1]; r[2] = b[0]; r[3] = b[1];
    r[4] = c[0]; r[5] = c[1]; r[6] = d[0]; r[7] = d[1];
  } else {
    // bytes + 128 convert to fp32 in one instruction each (b s + (128 s) would
    // save one more, but 128 s is no number for the largest scales)
    const uint32_t u0 = w0 ^ 0x80808080u, u1 = w1 ^ 0x80808080u;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      r[e] = (__bf16)(((float)((e < 4 ? u0 : u1) >> (8 * (e & 3)) & 255u) - 128.0f) * s);
  }
  return r;
}

// The 8 values of w's four bytes of E2M1 pairs times the scale s.
__device__ __forceinline__ bf16x8 decode4(uint32_t w, float s) {
  const bf16v2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0);
  const bf16v2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1);
  const bf16v2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2);
  const bf16v2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3);
  bf16x8 r;
  r[0] = a[0]; r[1] = a[1]; r[2] = b[0]; r[3] = b[1];
  r[4] = c[0]; r[5] = c[1]; r[6] = d[0]; r[7] = d[1];
  return r;
}

}  // namespace mmi
