// 4-bit values of the key / value cache: e2m1 codes (0, 1/2, 1, 3/2, 2, 3, 4, 6; bit 3 is the sign)
// with a power-of-two scale byte per 32 channels of a token and head.
//
// Why these: gfx950 converts two such codes and their scale to 16 bits in one instruction; every value
// is exact in bfloat16, and in float16 from 2^-23 to 2^13; and a block belongs to one token, so a token
// that is appended moves nothing of the tokens before it (a scale over tokens would have their four bits
// rounded again each time it grew).
#pragma once
#include "e4m3.h"

namespace nv {

constexpr int KV4_BLOCK = 32;  // channels of a scale

// Scale byte of a block whose largest magnitude is amax (infinite: the block holds something that is
// not finite, and is NaN): the smallest e >= 1 with amax <= 6 * 2^(e - 127).  6 = 1.5 * 2^2: a mantissa
// above .5 (0x400000) carries into the next exponent.  At most 253 for what is finite.
__device__ __forceinline__ int scale_byte4(float amax) {
  const int e = ((__float_as_int(amax) + 0x3FFFFF) >> 23) - 2;
  return amax == INFINITY ? 255 : e < 1 ? 1 : e;
}

// |x|, infinite where x is NaN.
__device__ __forceinline__ float abs_or_inf(float x) {
  const float a = fabsf(x);
  return a <= 3.402823466e38f ? a : INFINITY;
}

// Codes of eight values times inv = 2^(127 - e) (v_cvt_scalef32_pk_fp4_f32 rounds to nearest even and
// keeps the sign of what becomes zero); zeros in a NaN block.
__device__ __forceinline__ uint32_t codes4x8(const float (&x)[8], float inv) {
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0] * inv, x[1] * inv, 1.f, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2] * inv, x[3] * inv, 1.f, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4] * inv, x[5] * inv, 1.f, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6] * inv, x[7] * inv, 1.f, 3);
}

// Eight codes times a scale (a power of two) as 16-bit values; not for NaN scales.
template <typename T>
struct Half8;
template <>
struct Half8<_Float16> {
  typedef half8 Vec;
  static __device__ __forceinline__ Vec of(uint32_t w, float s) {
    const half2v a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 0),
                 b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 1),
                 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 2),
                 d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 3);
    return Vec{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
  }
  static __device__ __forceinline__ floatx4 mul(Vec a, Vec b, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
};
template <>
struct Half8<__bf16> {
  typedef bf16x8 Vec;
  static __device__ __forceinline__ Vec of(uint32_t w, float s) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0),
                 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1),
                 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2),
                 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3);
    return Vec{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
  }
  static __device__ __forceinline__ floatx4 mul(Vec a, Vec b, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
};

}  // namespace nv
