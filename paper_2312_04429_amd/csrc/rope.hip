// Queries and keys between their product and the cache: a norm for each head and the rotation by
// position, in one pass over both.
//
//   y = x w / sqrt(mean(x^2) + eps) over the dh channels of a head (without a norm: y = x)
//   (u, v) -> (u cos t - v sin t, v cos t + u sin t) for each pair i of an axis, t = position freqs[i]
//
// An angle is a float64 product, brought to turns of [0, 1) there: float32 would leave a token 200000
// places in with 14 bits of its angle.
#include <algorithm>

#include "common.h"
#include "e4m3.h"

namespace nv {
namespace {

constexpr int ROPE_AXES = 4, ROPE_DH = 256;

struct RopeArgs {
  const void *q, *k;
  void *qo, *ko;
  int64_t ldq, q_row, ldqo, qo_row, ldk, k_row, ldko, ko_row;
  const float *qw, *kw;
  const int32_t* pos;
  int64_t ldpos, pos_row;
  const double* freqs;
  int q_heads, k_heads, dh, S, n_axes, rot, norm;
  int axis[ROPE_AXES];  // channels of an axis
  float eps;
  int64_t tokens;
};

// A workgroup per TT tokens: first the tokens' cosines and sines, each computed once for all heads,
// into LDS; then GROUP lanes a head, eight channels a lane.
template <typename T, int GROUP, bool HALVES, bool VEC>
__global__ void __launch_bounds__(256) qk_rope_k(RopeArgs a, int tt) {
  extern __shared__ __align__(16) char lds[];
  float2* cs = (float2*)lds;                             // [tt][rot / 2]
  float* rows = (float*)(cs + (int64_t)tt * (a.rot / 2));  // halves: [256][8] normed values
  const int tid = threadIdx.x, pairs = a.rot / 2, heads = a.q_heads + a.k_heads;
  const int64_t first = (int64_t)blockIdx.x * tt;
  const int n = (int)std::min<int64_t>(tt, a.tokens - first);
  for (int i = tid; i < n * pairs; i += 256) {
    const int64_t tok = first + i / pairs, row = tok / a.S, s = tok - row * a.S;
    const int p = i % pairs;
    int axis = 0, end = a.axis[0] / 2;
    while (p >= end) end += a.axis[++axis] / 2;
    const double turns = (double)a.pos[row * a.pos_row + s * a.ldpos + axis] * a.freqs[p] *
                         0.15915494309189533577;
    float sn, c;
    sincospif(2.f * (float)(turns - floor(turns)), &sn, &c);
    cs[i] = make_float2(c, sn);
  }
  __syncthreads();
  const int g = tid % GROUP, c0 = g * 8, dh = a.dh;
  const bool in = c0 < dh;
  // halves: where a channel's pair is, for the eight channels of this lane
  int pair[8], mate[8];
  if (HALVES) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      int at = 0, axis = 0;
      pair[j] = -1, mate[j] = 0;
      if (c0 + j < a.rot) {
        while (c0 + j >= at + a.axis[axis]) at += a.axis[axis++];
        const int l = c0 + j - at, h = a.axis[axis] / 2;
        pair[j] = at / 2 + (l < h ? l : l - h);
        mate[j] = l < h ? h : -h;
      }
    }
  }
  for (int u = tid / GROUP; u < n * heads; u += 256 / GROUP) {
    const int t = u / heads, hd = u - t * heads;
    const int64_t tok = first + t, row = tok / a.S, s = tok - row * a.S;
    const bool is_k = hd >= a.q_heads;
    const int h = is_k ? hd - a.q_heads : hd;
    const T* src = (const T*)(is_k ? a.k : a.q) + row * (is_k ? a.k_row : a.q_row) +
                   s * (is_k ? a.ldk : a.ldq) + (int64_t)h * dh;
    T* dst = (T*)(is_k ? a.ko : a.qo) + row * (is_k ? a.ko_row : a.qo_row) +
             s * (is_k ? a.ldko : a.ldqo) + (int64_t)h * dh;
    float x[8];
    load8<VEC>(src, c0, dh, x);
    if (a.norm) {
      float sq = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) sq += x[j] * x[j];
#pragma unroll
      for (int m = 1; m < GROUP; m *= 2) sq += __shfl_xor(sq, m);
      const float f = 1.f / sqrtf(sq / (float)dh + a.eps);
      const float* w = is_k ? a.kw : a.qw;
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = x[j] * f * (w && in ? w[c0 + j] : 1.f);
    }
    float y[8];
    const float2* c = cs + t * pairs;
    if (HALVES) {
      float* mine = rows + (tid - g) * 8;  // this head's channels
#pragma unroll
      for (int j = 0; j < 8; ++j) mine[c0 + j] = x[j];
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // read by lanes of the same wave
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        y[j] = x[j];
        if (pair[j] >= 0) {
          const float2 r = c[pair[j]];
          const float o = mine[c0 + j + mate[j]];
          y[j] = x[j] * r.x + (mate[j] > 0 ? -o : o) * r.y;
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    } else {
#pragma unroll
      for (int j = 0; j < 8; j += 2) {
        y[j] = x[j], y[j + 1] = x[j + 1];
        if (c0 + j < a.rot) {
          const float2 r = c[(c0 + j) / 2];
          y[j] = x[j] * r.x - x[j + 1] * r.y;
          y[j + 1] = x[j + 1] * r.x + x[j] * r.y;
        }
      }
    }
    if (in) store8<VEC>(dst, c0, dh, y);
  }
}

}  // namespace
}  // namespace nv

using namespace nv;

extern "C" int32_t nv_op_qk_rope(const void* q, int64_t ldq, int64_t q_row_stride, void* q_out,
                                 int64_t ldqo, int64_t qo_row_stride, int32_t q_heads,
                                 const float* q_weight, const void* k, int64_t ldk,
                                 int64_t k_row_stride, void* k_out, int64_t ldko,
                                 int64_t ko_row_stride, int32_t k_heads, const float* k_weight,
                                 int32_t dtype, int32_t rows, int32_t S, int32_t dh,
                                 const int32_t* pos, int64_t ldpos, int64_t pos_row_stride,
                                 int32_t n_axes, const int32_t* axes, const double* freqs,
                                 int32_t halves, int32_t norm, float eps, void* stream) {
  clear_error();
  NV_CHECK_ARG(rows >= 0 && S >= 0 && q_heads >= 0 && k_heads >= 0, "negative sizes");
  NV_CHECK_ARG(dtype == NV_F16 || dtype == NV_BF16, "dtype must be NV_F16 or NV_BF16");
  NV_CHECK_ARG(halves == 0 || halves == 1, "halves must be 0 or 1");
  NV_CHECK_ARG(norm == 0 || norm == 1, "norm must be 0 or 1");
  NV_CHECK_ARG(norm || (!q_weight && !k_weight), "weights without a norm");
  NV_CHECK_ARG(!norm || (eps >= 0.f && eps - eps == 0.f), "eps must be finite and not negative");
  if (dh < 8 || dh > ROPE_DH || dh % 8) {
    set_error("dh must be a multiple of 8 from 8 to 256");
    return NV_ERR_UNSUPPORTED;
  }
  NV_CHECK_ARG(n_axes >= 0 && (n_axes == 0 || axes), "need n_axes >= 0, and their channels");
  if (n_axes > ROPE_AXES) {
    set_error("more than 4 axes");
    return NV_ERR_UNSUPPORTED;
  }
  RopeArgs a{};
  for (int i = 0; i < n_axes; ++i) {
    NV_CHECK_ARG(axes[i] >= 0 && axes[i] % 2 == 0 && axes[i] <= dh, "an axis has an even number of channels");
    a.axis[i] = axes[i], a.rot += axes[i];
  }
  NV_CHECK_ARG(a.rot <= dh, "the axes have more channels than a head");
  NV_CHECK_ARG(ldq >= 0 && q_row_stride >= 0 && ldk >= 0 && k_row_stride >= 0 && ldpos >= 0 &&
                   pos_row_stride >= 0, "negative strides");
  NV_CHECK_ARG(ldqo >= (int64_t)q_heads * dh && ldko >= (int64_t)k_heads * dh && qo_row_stride >= 0 &&
                   ko_row_stride >= 0, "negative strides, or rows of an output shorter than heads * dh");
  if (rows == 0 || S == 0 || q_heads + (int64_t)k_heads == 0) return NV_OK;
  NV_CHECK_ARG((q_heads == 0 || (q && q_out)) && (k_heads == 0 || (k && k_out)) &&
                   (a.rot == 0 || (pos && freqs)), "null pointer argument");
  const int64_t heads = (int64_t)q_heads + k_heads;
  if (heads > (1 << 20)) {
    set_error("more than 2^20 heads");
    return NV_ERR_UNSUPPORTED;
  }
  a.q = q, a.ldq = ldq, a.q_row = q_row_stride, a.qo = q_out, a.ldqo = ldqo, a.qo_row = qo_row_stride;
  a.k = k, a.ldk = ldk, a.k_row = k_row_stride, a.ko = k_out, a.ldko = ldko, a.ko_row = ko_row_stride;
  a.qw = q_weight, a.kw = k_weight, a.pos = pos, a.ldpos = ldpos, a.pos_row = pos_row_stride;
  a.freqs = freqs, a.q_heads = q_heads, a.k_heads = k_heads, a.dh = dh, a.S = S, a.n_axes = n_axes;
  a.norm = norm, a.eps = eps, a.tokens = (int64_t)rows * S;
  int group = 1;
  while (group * 8 < dh) group *= 2;
  const int tt = (int)std::max<int64_t>(1, std::min<int64_t>(16, 1024 / (heads * group)));
  const int64_t wgs = ceil_div(a.tokens, tt);
  if (wgs > 8388607) {
    set_error("more tokens than a grid holds");
    return NV_ERR_UNSUPPORTED;
  }
  auto ok = [](const void* p, int64_t ld, int64_t row) {
    return !p || (aligned16(p) && (ld | row) % 8 == 0);
  };
  const bool vec = ok(q_heads ? q : nullptr, ldq, q_row_stride) &&
                   ok(q_heads ? q_out : nullptr, ldqo, qo_row_stride) &&
                   ok(k_heads ? k : nullptr, ldk, k_row_stride) &&
                   ok(k_heads ? k_out : nullptr, ldko, ko_row_stride);
  const size_t lds = (size_t)tt * (a.rot / 2) * 8 + (halves ? 8192 : 0);
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)wgs), dim3(256), lds, (hipStream_t)stream, a, tt);
  };
  auto pick = [&](auto t, auto g) {
    typedef decltype(t) T;
    constexpr int G = decltype(g)::value;
    if (halves) vec ? go(qk_rope_k<T, G, true, true>) : go(qk_rope_k<T, G, true, false>);
    else vec ? go(qk_rope_k<T, G, false, true>) : go(qk_rope_k<T, G, false, false>);
  };
  auto sized = [&](auto t) {
    switch (group) {
      case 1: return pick(t, std::integral_constant<int, 1>());
      case 2: return pick(t, std::integral_constant<int, 2>());
      case 4: return pick(t, std::integral_constant<int, 4>());
      case 8: return pick(t, std::integral_constant<int, 8>());
      case 16: return pick(t, std::integral_constant<int, 16>());
      default: return pick(t, std::integral_constant<int, 32>());
    }
  };
  if (dtype == NV_F16) sized(_Float16());
  else sized(__bf16());
  NV_LAUNCH_CHECK("qk_rope_k");
  return NV_OK;
}
