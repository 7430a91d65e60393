// Attention over a paged cache in shares of a row's pages: the partial results and what joins them.
#pragma once
#include <algorithm>

#include "e4m3.h"
#include "kv8.h"

namespace nv {
namespace {

// The shares of a query's pages, in order.  A workgroup per query: the shares' weights first, then
// GROUPS threads per four channels that take every GROUPS-th share's means and meet in LDS.  A share
// that held nothing has no means (its maximum is -inf, its sum 0).
template <typename T>
__global__ void __launch_bounds__(256) attn_join_k(Kv8AttnArgs a) {
  __shared__ float fac[KV8_MAX_SPLITS];
  __shared__ float red[4][2];
  __shared__ __align__(16) floatx4 part[256];
  const int tid = threadIdx.x, group = a.heads / a.kv_heads, nq = a.dh / 4, groups = 256 / nq;
  const int cols = a.S * group;
  const int64_t u = blockIdx.x, rh = u / cols;
  const int c = (int)(u - rh * cols);
  const float* ml = a.part_ml + u * a.splits * 2;
  float m = -INFINITY, l = 0.f;
  if (tid < a.splits) m = ml[tid * 2], l = ml[tid * 2 + 1];
  float top = rows_max(row16_max(m));
  if ((tid & 63) == 0) red[tid >> 6][0] = top;
  __syncthreads();
  top = fmaxf(fmaxf(red[0][0], red[1][0]), fmaxf(red[2][0], red[3][0]));
  const float base = top == -INFINITY ? 0.f : top;
  const float f = __builtin_amdgcn_exp2f(m - base) * l;
  if (tid < a.splits) fac[tid] = m == -INFINITY && l == 0.f ? -1.f : f;  // -1: no means
  const float ls = wave_sum(f);  // the same tree in every call
  if ((tid & 63) == 0) red[tid >> 6][1] = ls;
  __syncthreads();
  const float sum = (red[0][1] + red[1][1]) + (red[2][1] + red[3][1]);
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  const int g = tid / nq, d = (tid - g * nq) * 4;
  floatx4 o = {0.f, 0.f, 0.f, 0.f};
  if (g < groups)
#pragma unroll 4
    for (int s = g; s < a.splits; s += groups)
      if (fac[s] != -1.f) o += fac[s] * inv * *(const floatx4*)(a.part_o + (u * a.splits + s) * a.dh + d);
  part[tid] = o;
  __syncthreads();
  if (tid >= nq) return;
  for (int i = 1; i < groups && i < a.splits; ++i) o += part[i * nq + tid];
  const int64_t row = rh / a.kv_heads, h = rh % a.kv_heads * group + c % group;
  struct alignas(8) Quad { T v[4]; } out;
#pragma unroll
  for (int r = 0; r < 4; ++r) out.v[r] = (T)o[r];
  *(Quad*)((T*)a.out + row * a.o_row + c / group * a.ldo + h * a.dh + d) = out;
}

// The same with few shares: one thread per four channels.
template <typename T>
__global__ void __launch_bounds__(256) attn_join_few_k(Kv8AttnArgs a) {
  const int group = a.heads / a.kv_heads, nq = a.dh / 4;
  const int64_t cols = (int64_t)a.S * group, total = a.rows * a.kv_heads * cols * nq;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total;
       i += (int64_t)gridDim.x * 256) {
    const int64_t u = i / nq, rh = u / cols, c = u - rh * cols;
    const int d = (int)(i - u * nq) * 4;
    const float* ml = a.part_ml + u * a.splits * 2;
    float m[KV8_FEW], f[KV8_FEW];
    float top = -INFINITY, ls = 0.f;
#pragma unroll
    for (int s = 0; s < KV8_FEW; ++s) {
      m[s] = s < a.splits ? ml[s * 2] : -INFINITY;
      f[s] = s < a.splits ? ml[s * 2 + 1] : 0.f;
      top = fmaxf(top, m[s]);
    }
    const float base = top == -INFINITY ? 0.f : top;
    bool none[KV8_FEW];
#pragma unroll
    for (int s = 0; s < KV8_FEW; ++s) {
      none[s] = m[s] == -INFINITY && f[s] == 0.f;
      f[s] *= __builtin_amdgcn_exp2f(m[s] - base);
      ls += f[s];
    }
    const float inv = ls == 0.f ? 0.f : 1.f / ls;
    floatx4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < KV8_FEW; ++s)
      if (!none[s]) o += f[s] * inv * *(const floatx4*)(a.part_o + (u * a.splits + s) * a.dh + d);
    const int64_t row = rh / a.kv_heads, h = rh % a.kv_heads * group + c % group;
    struct alignas(8) Quad { T v[4]; } out;
#pragma unroll
    for (int r = 0; r < 4; ++r) out.v[r] = (T)o[r];
    *(Quad*)((T*)a.out + row * a.o_row + c / group * a.ldo + h * a.dh + d) = out;
  }
}

template <typename T>
void attn_join(const Kv8AttnArgs& a, hipStream_t s) {
  const int64_t queries = (int64_t)a.rows * a.heads * a.S;
  if (a.splits > KV8_FEW)
    hipLaunchKernelGGL(attn_join_k<T>, dim3((unsigned)queries), dim3(256), 0, s, a);
  else if (a.splits > 1)
    hipLaunchKernelGGL(attn_join_few_k<T>,
                       dim3((unsigned)std::min<int64_t>(ceil_div(queries * (a.dh / 4), 256), 1 << 20)),
                       dim3(256), 0, s, a);
}

// Partial results.
size_t part_bytes(const Kv8Plan& p, int64_t rows, int S, int heads, int dh, size_t* ml_at) {
  if (p.splits == 1) return 0;
  const int64_t queries = rows * S * heads;
  const size_t o = align_up((size_t)queries * p.splits * dh * 4, 256);
  if (ml_at) *ml_at = o;
  return o + align_up((size_t)queries * p.splits * 8, 256);
}

}  // namespace
}  // namespace nv
