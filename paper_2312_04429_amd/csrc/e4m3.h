// 8-bit values shared by the 8-bit operators: e4m3 codes with a power-of-two scale per block.
//
// Why powers of two: the scaled matrix instruction applies them at no cost; e4m3 keeps its
// three mantissa bits at every magnitude, so a finer scale would only move the bottom of its
// range by a fraction of a binade; and a block's scale can grow later by moving codes exactly
// (all but those that become subnormal).
#pragma once
#include <type_traits>

#include "common.h"

namespace nv {

typedef int intx8 __attribute__((ext_vector_type(8)));

// Columns c .. c + 7 of a row of n (those past its end: zeros, not stored) as one vector.  VEC: n
// and the row's start keep the eight together and 16-byte aligned; without, the vector is aligned as
// its elements are (global memory takes that: 5003 rows of 1001 in nv_op_rmsnorm8 took 28.8 us
// element by element), and only a row's last columns move one by one.
template <typename T>
struct alignas(16) Vec8 {
  T v[8];
};
template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) Any8 {
  T v[8];
};
template <bool VEC, typename T>
__device__ __forceinline__ void load8(const T* row, int c, int n, float (&x)[8]) {
  if (VEC ? c < n : c + 8 <= n) {
    const auto t = *(const std::conditional_t<VEC, Vec8<T>, Any8<T>>*)(row + c);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)t.v[i];
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = !VEC && c + i < n ? (float)row[c + i] : 0.f;
  }
}
template <bool VEC, typename T>
__device__ __forceinline__ void store8(T* row, int c, int n, const float (&x)[8]) {
  if (VEC ? c < n : c + 8 <= n) {
    std::conditional_t<VEC, Vec8<T>, Any8<T>> t;
#pragma unroll
    for (int i = 0; i < 8; ++i) t.v[i] = (T)x[i];
    *(decltype(t)*)(row + c) = t;
  } else if (!VEC) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < n) row[c + i] = (T)x[i];
  }
}

// |x|, and 0 where x is not finite: what a block's scale looks at.
__device__ __forceinline__ float finite_abs(float x) {
  const float a = fabsf(x);
  return a <= 3.402823466e38f ? a : 0.f;
}

// Scale byte of a block whose largest finite magnitude is amax: the smallest e >= 1 with
// amax <= 448 * 2^(e - 127).  448 = 1.75 * 2^8: a mantissa above .75 (0x600000) carries into
// the next exponent.  At most 247, as amax is below 2^128.
__device__ __forceinline__ int scale_byte(float amax) {
  const int e = ((__float_as_int(amax) + 0x1FFFFF) >> 23) - 8;
  return e < 1 ? 1 : e;
}

// 2^(e - 127) of a scale byte (0: a subnormal float; 255: NaN).
__device__ __forceinline__ float scale_value(int e) {
  return e == 255 ? __int_as_float(0x7FC00000) : e == 0 ? __int_as_float(0x00400000)
                                                        : __int_as_float(e << 23);
}

// Codes of two values that are scaled already (|x| <= 448, or not finite: NaN).
// v_cvt_pk_fp8_f32 rounds to nearest even, subnormal codes included.
__device__ __forceinline__ float code_value(float x, float inv) {
  return finite_abs(x) == fabsf(x) ? x * inv : __int_as_float(0x7FC00000);
}
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float inv) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(code_value(a, inv), code_value(b, inv), 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(code_value(c, inv), code_value(d, inv), r, true);
}

// Eight scaled codes to columns c .. c + 7 of a row of n bytes.
template <bool VEC>
__device__ __forceinline__ void store_codes8(uint8_t* row, int c, int n, const float (&x)[8],
                                             float inv) {
  const uint32_t lo = codes4(x[0], x[1], x[2], x[3], inv), hi = codes4(x[4], x[5], x[6], x[7], inv);
  struct __attribute__((packed, aligned(1))) Any { uint32_t lo, hi; };
  if (VEC ? c < n : c + 8 <= n) {
    if constexpr (VEC) *(uint2*)(row + c) = make_uint2(lo, hi);
    else *(Any*)(row + c) = Any{lo, hi};
  } else if (!VEC) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < n) row[c + i] = (uint8_t)((i < 4 ? lo : hi) >> (8 * (i & 3)));
  }
}
// 2^(127 - e) for a scale byte e in [1, 253].
__device__ __forceinline__ float scale_inverse(int e) { return __int_as_float((254 - e) << 23); }

// Largest of x over the 16 lanes of a row of the wave.
__device__ __forceinline__ float row16_max(float v) {
  v = fmaxf(v, dpp_f<0xB1>(v));   // quad_perm [1, 0, 3, 2]
  v = fmaxf(v, dpp_f<0x4E>(v));   // quad_perm [2, 3, 0, 1]
  v = fmaxf(v, dpp_f<0x124>(v));  // row_ror:4
  return fmaxf(v, dpp_f<0x128>(v));  // row_ror:8
}

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

}  // namespace nv
