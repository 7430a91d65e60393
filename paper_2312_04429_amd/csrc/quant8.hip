// Into and out of the 8-bit form, and the root-mean-square norm that ends in it.
//
// All three are bound by HBM: each value is read once into registers, its block's largest
// magnitude is found there (a block of 128 columns is 16 lanes of 8 values: four DPP maxima,
// no LDS), and codes leave as 8-byte stores, one scale byte per block.  Measured: 8192 x 5120
// float16 into codes 26 us (4.8 TB/s read and written), back to bfloat16 22 (5.8); 10240 x 1280
// float32 in blocks of 128 rows 13 (5.0); the norm of 16384 x 1280 with residual 31 (4.7).
#include <algorithm>

#include "common.h"
#include "e4m3.h"

namespace nv {
namespace {

// Blocks of 1 x 128: 16 lanes a block, blocks in row order.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) quant8_rows_k(const T* __restrict__ x, int64_t ldx,
                                                     int64_t M, int K, uint8_t* __restrict__ q,
                                                     int64_t ldq, uint8_t* __restrict__ scales) {
  const int nb = (K + 127) / 128, lane16 = threadIdx.x & 15;
  const int64_t total = M * nb;
  for (int64_t u = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4); u < total;
       u += (int64_t)gridDim.x * 16) {
    const int64_t m = u / nb;
    const int c = (int)(u - m * nb) * 128 + lane16 * 8;
    float v[8];
    load8<VEC>(x + m * ldx, c, K, v);
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = fmaxf(top, finite_abs(v[i]));
    const int e = scale_byte(row16_max(top));
    store_codes8<VEC>(q + m * ldq, c, K, v, scale_inverse(e));
    if (lane16 == 0) scales[u] = (uint8_t)e;
  }
}

// Blocks of 128 x 128: a workgroup each, 16 rows a pass, the whole block in registers.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) quant8_tiles_k(const T* __restrict__ x, int64_t ldx,
                                                      int64_t M, int K, uint8_t* __restrict__ q,
                                                      int64_t ldq, uint8_t* __restrict__ scales) {
  __shared__ float part[4];
  const int nb = (K + 127) / 128;
  const int64_t total = (M + 127) / 128 * nb;
  for (int64_t u = blockIdx.x; u < total; u += gridDim.x) {
    const int64_t mb = u / nb, m0 = mb * 128 + (threadIdx.x >> 4);
    const int c = (int)(u - mb * nb) * 128 + (threadIdx.x & 15) * 8;
    float v[8][8];
    float top = 0.f;
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      const int64_t m = m0 + p * 16;
      load8<VEC>(x + m * ldx, c, m < M ? K : 0, v[p]);
#pragma unroll
      for (int i = 0; i < 8; ++i) top = fmaxf(top, finite_abs(v[p][i]));
    }
    top = rows_max(row16_max(top));
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = top;
    __syncthreads();
    const int e = scale_byte(fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3])));
    const float inv = scale_inverse(e);
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      const int64_t m = m0 + p * 16;
      store_codes8<VEC>(q + m * ldq, c, m < M ? K : 0, v[p], inv);
    }
    if (threadIdx.x == 0) scales[u] = (uint8_t)e;
    __syncthreads();
  }
}

// Eight values a thread; a block's scale byte is read by its 16 lanes at once.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) dequant8_k(const uint8_t* __restrict__ q, int64_t ldq,
                                                  const uint8_t* __restrict__ scales, int64_t M,
                                                  int K, int rows_shift, T* __restrict__ out,
                                                  int64_t ldo) {
  const int nb = (K + 127) / 128, lane16 = threadIdx.x & 15;
  const int64_t total = M * nb;
  for (int64_t u = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4); u < total;
       u += (int64_t)gridDim.x * 16) {
    const int64_t m = u / nb;
    const int b = (int)(u - m * nb), c = b * 128 + lane16 * 8;
    const float s = scale_value(scales[(m >> rows_shift) * nb + b]);
    const uint8_t* row = q + m * ldq;
    uint2 w = make_uint2(0, 0);
    struct __attribute__((packed, aligned(1))) Any { uint32_t lo, hi; };
    if (VEC ? c < K : c + 8 <= K) {
      if constexpr (VEC) w = *(const uint2*)(row + c);
      else w = make_uint2(((const Any*)(row + c))->lo, ((const Any*)(row + c))->hi);
    } else if (!VEC) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (c + i < K) (i < 4 ? w.x : w.y) |= (uint32_t)row[c + i] << (8 * (i & 3));
    }
    float v[8];
    const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w.x, false);
    const auto b2 = __builtin_amdgcn_cvt_pk_f32_fp8((int)w.x, true);
    const auto c2 = __builtin_amdgcn_cvt_pk_f32_fp8((int)w.y, false);
    const auto d = __builtin_amdgcn_cvt_pk_f32_fp8((int)w.y, true);
    v[0] = a[0] * s, v[1] = a[1] * s, v[2] = b2[0] * s, v[3] = b2[1] * s;
    v[4] = c2[0] * s, v[5] = c2[1] * s, v[6] = d[0] * s, v[7] = d[1] * s;
    store8<VEC>(out + m * ldo, c, K, v);
  }
}

struct NormArgs {
  const void *x, *r;
  const float* w;
  void* h;
  uint8_t *q, *scales;
  int64_t ldx, ldr, ldh, ldq, M;
  int D;
  float eps;
};

// y = s w / sqrt(mean(s^2) + eps), s = x + r, one pass: a row's values stay in registers
// (NCH chunks of 8 a thread) between the sum of squares and the codes.  The mean is of the
// float32 sum, not of its 16-bit copy h: one rounding less.  WPR waves share a row; with one,
// a workgroup takes four rows and needs no barrier.
template <typename T, int WPR, int NCH, bool VEC>
__global__ void __launch_bounds__(WPR == 1 ? 256 : WPR * 64) rmsnorm8_k(NormArgs a) {
  constexpr int NT = WPR * 64, RPB = WPR == 1 ? 4 : 1;
  __shared__ float part[2][WPR];
  const int t = threadIdx.x % NT, nb = (a.D + 127) / 128;
  int flip = 0;
  float w[NCH][8];
#pragma unroll
  for (int c = 0; c < NCH; ++c) load8<VEC>(a.w, (c * NT + t) * 8, a.D, w[c]);
  for (int64_t m = (int64_t)blockIdx.x * RPB + (RPB == 1 ? 0 : threadIdx.x / NT); m < a.M;
       m += (int64_t)gridDim.x * RPB) {
    float s[NCH][8];
    float ss = 0.f;
#pragma unroll
    for (int c = 0; c < NCH; ++c)
      load8<VEC>((const T*)a.x + m * a.ldx, (c * NT + t) * 8, a.D, s[c]);
    if (a.r) {
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        float r[8];
        load8<VEC>((const T*)a.r + m * a.ldr, (c * NT + t) * 8, a.D, r);
#pragma unroll
        for (int i = 0; i < 8; ++i) s[c][i] += r[i];
      }
    }
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) ss += s[c][i] * s[c][i];
    if (a.h) {
#pragma unroll
      for (int c = 0; c < NCH; ++c)
        store8<VEC>((T*)a.h + m * a.ldh, (c * NT + t) * 8, a.D, s[c]);
    }
    ss = wave_sum(ss);
    if constexpr (WPR > 1) {  // two slots in turn: one barrier a row
      if ((threadIdx.x & 63) == 0) part[flip][threadIdx.x >> 6] = ss;
      __syncthreads();
      ss = 0.f;
#pragma unroll
      for (int w = 0; w < WPR; ++w) ss += part[flip][w];
      flip ^= 1;
    }
    const float rstd = 1.0f / sqrtf(ss / (float)a.D + a.eps);
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int col = (c * NT + t) * 8;
      float top = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        s[c][i] = s[c][i] * rstd * w[c][i];
        top = fmaxf(top, finite_abs(s[c][i]));
      }
      const int e = scale_byte(row16_max(top));
      store_codes8<VEC>(a.q + m * a.ldq, col, a.D, s[c], scale_inverse(e));
      if ((t & 15) == 0 && col < a.D) a.scales[m * nb + (col >> 7)] = (uint8_t)e;
    }
  }
}

// Workgroups of the norm: a thread keeps its weights and takes every NORM_GRID-th row (or four), so
// they are read once (16384 x 1280: 36.2 us with a workgroup for each four rows and the weights read
// beside each, 30.2 to 30.9 us with 1024 or 2048 workgroups that keep them).
constexpr int64_t NORM_GRID = 2048;
unsigned grid_of(int64_t units) { return (unsigned)std::min<int64_t>(std::max<int64_t>(units, 1), 1 << 20); }

template <typename T>
void quant8_launch(const void* x, int64_t ldx, int64_t M, int K, int block_rows, void* q,
                   int64_t ldq, uint8_t* scales, bool vec, hipStream_t s) {
  const int64_t nb = ceil_div(K, 128);
  const dim3 grid(grid_of(block_rows == 1 ? ceil_div(M * nb, 16) : ceil_div(M, 128) * nb));
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, (const T*)x, ldx, M, K, (uint8_t*)q, ldq,
                       scales);
  };
  if (block_rows == 1)
    vec ? go(quant8_rows_k<T, true>) : go(quant8_rows_k<T, false>);
  else
    vec ? go(quant8_tiles_k<T, true>) : go(quant8_tiles_k<T, false>);
}

template <typename T>
void dequant8_launch(const void* q, int64_t ldq, const uint8_t* scales, int64_t M, int K,
                     int block_rows, void* out, int64_t ldo, bool vec, hipStream_t s) {
  const dim3 grid(grid_of(ceil_div(M * ceil_div(K, 128), 16)));
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, (const uint8_t*)q, ldq, scales, M, K,
                       block_rows == 1 ? 0 : 7, (T*)out, ldo);
  };
  vec ? go(dequant8_k<T, true>) : go(dequant8_k<T, false>);
}

template <typename T, int WPR, int NCH>
void norm_go(const NormArgs& a, bool vec, hipStream_t s) {
  const int64_t groups = WPR == 1 ? ceil_div(a.M, 4) : a.M;
  const dim3 grid((unsigned)std::min<int64_t>(groups, NORM_GRID)), block(WPR == 1 ? 256 : WPR * 64);
  if (vec)
    hipLaunchKernelGGL((rmsnorm8_k<T, WPR, NCH, true>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((rmsnorm8_k<T, WPR, NCH, false>), grid, block, 0, s, a);
}

template <typename T>
void norm_launch(const NormArgs& a, bool vec, hipStream_t s) {
  if (a.D <= 512) return norm_go<T, 1, 1>(a, vec, s);
  if (a.D <= 1024) return norm_go<T, 1, 2>(a, vec, s);
  if (a.D <= 1536) return norm_go<T, 1, 3>(a, vec, s);
  if (a.D <= 2048) return norm_go<T, 1, 4>(a, vec, s);
  if (a.D <= 4096) return norm_go<T, 4, 2>(a, vec, s);
  if (a.D <= 8192) return norm_go<T, 4, 4>(a, vec, s);
  return norm_go<T, 16, 4>(a, vec, s);
}

// Columns of a row: what the kernels' 32-bit column numbers reach, the last block's past its end
// included.
constexpr int32_t K_MAX = 0x7FFFFF00;
bool half_type(int32_t t) { return t == NV_F16 || t == NV_BF16; }

}  // namespace
}  // namespace nv

using namespace nv;

extern "C" int32_t nv_op_quant8(const void* x, int32_t x_dtype, int64_t ldx, int64_t M, int32_t K,
                                int32_t block_rows, void* q, int64_t ldq, uint8_t* scales,
                                void* stream) {
  clear_error();
  NV_CHECK_ARG(M >= 0 && K >= 1, "need M >= 0 and K >= 1");
  NV_CHECK_ARG(x_dtype == NV_F32 || half_type(x_dtype), "x_dtype must be NV_F32, NV_F16 or NV_BF16");
  NV_CHECK_ARG(block_rows == 1 || block_rows == 128, "block_rows must be 1 or 128");
  NV_CHECK_ARG(ldx >= K && ldq >= K, "row strides shorter than K");
  if (K > K_MAX) {
    set_error("rows of more than 2^31 - 256 columns");
    return NV_ERR_UNSUPPORTED;
  }
  if (M == 0) return NV_OK;
  NV_CHECK_ARG(x && q && scales, "null pointer argument");
  const bool vec = K % 8 == 0 && ldx % 8 == 0 && ldq % 8 == 0 && aligned16(x) &&
                   (uintptr_t)q % 8 == 0;
  hipStream_t s = (hipStream_t)stream;
  if (x_dtype == NV_F32) quant8_launch<float>(x, ldx, M, K, block_rows, q, ldq, scales, vec, s);
  else if (x_dtype == NV_F16)
    quant8_launch<_Float16>(x, ldx, M, K, block_rows, q, ldq, scales, vec, s);
  else quant8_launch<__bf16>(x, ldx, M, K, block_rows, q, ldq, scales, vec, s);
  NV_LAUNCH_CHECK("quant8");
  return NV_OK;
}

extern "C" int32_t nv_op_dequant8(const void* q, int64_t ldq, const uint8_t* scales, int64_t M,
                                  int32_t K, int32_t block_rows, void* out, int32_t out_dtype,
                                  int64_t ldo, void* stream) {
  clear_error();
  NV_CHECK_ARG(M >= 0 && K >= 1, "need M >= 0 and K >= 1");
  NV_CHECK_ARG(out_dtype == NV_F32 || half_type(out_dtype),
               "out_dtype must be NV_F32, NV_F16 or NV_BF16");
  NV_CHECK_ARG(block_rows == 1 || block_rows == 128, "block_rows must be 1 or 128");
  NV_CHECK_ARG(ldo >= K && ldq >= K, "row strides shorter than K");
  if (K > K_MAX) {
    set_error("rows of more than 2^31 - 256 columns");
    return NV_ERR_UNSUPPORTED;
  }
  if (M == 0) return NV_OK;
  NV_CHECK_ARG(q && scales && out, "null pointer argument");
  const bool vec = K % 8 == 0 && ldo % 8 == 0 && ldq % 8 == 0 && aligned16(out) &&
                   (uintptr_t)q % 8 == 0;
  hipStream_t s = (hipStream_t)stream;
  if (out_dtype == NV_F32)
    dequant8_launch<float>(q, ldq, scales, M, K, block_rows, out, ldo, vec, s);
  else if (out_dtype == NV_F16)
    dequant8_launch<_Float16>(q, ldq, scales, M, K, block_rows, out, ldo, vec, s);
  else dequant8_launch<__bf16>(q, ldq, scales, M, K, block_rows, out, ldo, vec, s);
  NV_LAUNCH_CHECK("dequant8");
  return NV_OK;
}

extern "C" int32_t nv_op_rmsnorm8(const void* x, int64_t ldx, const void* residual, int64_t ldr,
                                  int32_t dtype, const float* weight, float eps, int64_t M,
                                  int32_t D, void* h, int64_t ldh, void* q, int64_t ldq,
                                  uint8_t* scales, void* stream) {
  clear_error();
  NV_CHECK_ARG(M >= 0 && D >= 1, "need M >= 0 and D >= 1");
  NV_CHECK_ARG(half_type(dtype), "dtype must be NV_F16 or NV_BF16");
  NV_CHECK_ARG(eps >= 0.f && eps <= 3.402823466e38f, "eps must be finite and not negative");
  NV_CHECK_ARG(ldx >= D && ldq >= D && (!residual || ldr >= D) && (!h || ldh >= D),
               "row strides shorter than D");
  if (D > 32768) {
    set_error("rows of more than 32768 columns");
    return NV_ERR_UNSUPPORTED;
  }
  if (M == 0) return NV_OK;
  NV_CHECK_ARG(x && weight && q && scales, "null pointer argument");
  const NormArgs a{x,   residual, weight, h,   (uint8_t*)q, scales,
                   ldx, ldr,      ldh,    ldq, M,           D,      eps};
  const bool vec = D % 8 == 0 && ldx % 8 == 0 && ldq % 8 == 0 && aligned16(x) &&
                   aligned16(weight) && (uintptr_t)q % 8 == 0 &&
                   (!residual || (ldr % 8 == 0 && aligned16(residual))) &&
                   (!h || (ldh % 8 == 0 && aligned16(h)));
  if (dtype == NV_F16) norm_launch<_Float16>(a, vec, (hipStream_t)stream);
  else norm_launch<__bf16>(a, vec, (hipStream_t)stream);
  NV_LAUNCH_CHECK("rmsnorm8");
  return NV_OK;
}
