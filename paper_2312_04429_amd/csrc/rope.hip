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

// How a channel's pair lies to it: NEXT: beside it; HALF8: in the other half of its axis, all axes of 16
// channels or multiples of it, so that eight neighbours have eight neighbours; HALF: anywhere.
enum Pairs { NEXT, HALF8, HALF };

// Sum over the GROUP lanes of a head, on the vector unit.
template <int GROUP>
__device__ __forceinline__ float group_sum(float v) {
  if (GROUP > 1) v += dpp_f<0xB1>(v);   // quad_perm [1, 0, 3, 2]
  if (GROUP > 2) v += dpp_f<0x4E>(v);   // quad_perm [2, 3, 0, 1]
  if (GROUP > 4) v += dpp_f<0x141>(v);  // row_half_mirror
  if (GROUP > 8) v += dpp_f<0x140>(v);  // row_mirror
  if (GROUP > 16) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  }
  return v;
}

// A workgroup takes tt tokens and `steps` steps of 64 / GROUP heads from blockIdx.y * steps on: first the
// tokens' cosines and sines, each computed once for all heads, into LDS; then a wave a step, GROUP lanes
// a head, eight channels a lane.  A wave's token is uniform: its addresses are scalar arithmetic (with a
// 64-bit division by S a lane and step, 16384 tokens of 40 heads of 128 took 158 us).  Bound by HBM: those
// tokens, bfloat16, three axes: 335 MB in 78 us (4.3 TB/s); 8346 tokens of 40 heads of 64, float16: 22 us
// (3.8); 32 single tokens of 40 heads of 128: 4.9 us, launch and the way from a position to its angles.
// Halves cost their way through LDS: 16384 tokens of 40 heads of 128, bfloat16, NEXT 77 us, HALF8 92, HALF 87; 4096
// tokens 24, 31 and 27; 8346 of 64 channels 22, 28 and 27.
template <typename T, int GROUP, Pairs P, bool VEC>
__global__ void __launch_bounds__(256) qk_rope_k(RopeArgs a, int tt, int steps) {
  constexpr int HPW = 64 / GROUP;  // heads of a step
  extern __shared__ __align__(16) char lds[];
  const int tid = threadIdx.x, pairs = a.rot / 2, pitch = (pairs + 3) & ~3;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int heads = a.q_heads + a.k_heads, dh = a.dh;
  float2* cs = (float2*)lds;                             // [tt][pitch]
  float* mine = (float*)(cs + tt * pitch) + wave * 512;  // HALF8, HALF: 64 lanes' channels
  const int64_t first = (int64_t)blockIdx.x * tt;
  const int n = (int)std::min<int64_t>(tt, a.tokens - first);
  const int64_t row0 = first / a.S;
  const int s0 = (int)(first - row0 * a.S);
  for (int i = tid; i < n * pairs; i += 256) {
    const int t = i / pairs, p = i - t * pairs;
    int s = s0 + t;  // below 2^31 + 16
    int64_t row = row0;
    if ((unsigned)s >= (unsigned)a.S) row += (unsigned)s / (unsigned)a.S, s = (unsigned)s % (unsigned)a.S;
    int axis = 0, end = a.axis[0] / 2;
    while (p >= end) end += a.axis[++axis] / 2;
    const double turns = (double)a.pos[row * a.pos_row + s * a.ldpos + axis] * a.freqs[p] *
                         0.15915494309189533577;
    float sn, c;
    sincospif(2.f * (float)(turns - floor(turns)), &sn, &c);
    cs[t * pitch + p] = make_float2(c, sn);
  }
  const int g = lane % GROUP, c0 = g * 8;
  const bool in = c0 < dh;
  float wq[8], wk[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    wq[j] = a.qw && in ? a.qw[c0 + j] : 1.f;
    wk[j] = a.kw && in ? a.kw[c0 + j] : 1.f;
  }
  // where the pairs of this lane's channels are: their index, and how far the other channel is
  constexpr int NP = P == HALF ? 8 : 1;
  int pair[NP], mate[NP];
#pragma unroll
  for (int j = 0; j < NP; ++j) {
    int at = 0, axis = 0;
    pair[j] = -1, mate[j] = 0;
    if (c0 + j >= a.rot) continue;
    if (P == NEXT) {
      pair[j] = c0 / 2;
    } else {
      while (c0 + j >= at + a.axis[axis]) at += a.axis[axis++];
      const int l = c0 + j - at, h = a.axis[axis] / 2;
      pair[j] = at / 2 + (l < h ? l : l - h);
      mate[j] = l < h ? h : -h;
    }
  }
  __syncthreads();
  const int step0 = blockIdx.y * steps;
  const int ns = std::min(steps, (heads + HPW - 1) / HPW - step0);
  int t = 0, st = wave, s = s0;
  int64_t row = row0;
  while (true) {
    while (st >= ns) {  // uniform
      st -= ns, ++t;
      if (++s == a.S) s = 0, ++row;
    }
    if (t >= n) break;
    const int hd = (step0 + st) * HPW + lane / GROUP;
    const bool is_k = hd >= a.q_heads, on = in && hd < heads;
    const int64_t at = (int64_t)(is_k ? hd - a.q_heads : hd) * dh;
    const T* src = (is_k ? (const T*)a.k + (row * a.k_row + s * a.ldk)
                         : (const T*)a.q + (row * a.q_row + s * a.ldq)) + at;
    T* dst = (is_k ? (T*)a.ko + (row * a.ko_row + s * a.ldko)
                   : (T*)a.qo + (row * a.qo_row + s * a.ldqo)) + at;
    float x[8], y[8];
    load8<VEC>(src, c0, on ? dh : 0, x);
    if (a.norm) {
      float sq = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) sq += x[j] * x[j];
      const float f = rsqrtf(group_sum<GROUP>(sq) / (float)dh + a.eps);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = x[j] * f * (is_k ? wk[j] : wq[j]);
    }
    const float2* c = cs + t * pitch;
    if constexpr (P == NEXT) {
      float4 r[2];  // of four pairs: cosine, sine, cosine, sine
      r[0] = *(const float4*)(c + std::max(pair[0], 0)), r[1] = *(const float4*)(c + std::max(pair[0], 0) + 2);
      const float co[4] = {r[0].x, r[0].z, r[1].x, r[1].z}, si[4] = {r[0].y, r[0].w, r[1].y, r[1].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bool turns = c0 + 2 * j < a.rot;
        const float u = x[2 * j], v = x[2 * j + 1];
        y[2 * j] = turns ? u * co[j] - v * si[j] : u;
        y[2 * j + 1] = turns ? v * co[j] + u * si[j] : v;
      }
    } else {
      float* own = mine + lane * 8;
      *(float4*)own = make_float4(x[0], x[1], x[2], x[3]);
      *(float4*)(own + 4) = make_float4(x[4], x[5], x[6], x[7]);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // read by lanes of the same wave
      if constexpr (P == HALF8) {
        float o[8], co[8], si[8];
        const float2* cp = c + std::max(pair[0], 0);
        *(float4*)o = *(const float4*)(own + mate[0]), *(float4*)(o + 4) = *(const float4*)(own + mate[0] + 4);
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
          const float4 r = *(const float4*)(cp + j);
          co[j] = r.x, si[j] = r.y, co[j + 1] = r.z, si[j + 1] = r.w;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
          y[j] = pair[0] < 0 ? x[j] : x[j] * co[j] + (mate[0] > 0 ? -o[j] : o[j]) * si[j];
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float2 r = c[std::max(pair[j], 0)];
          const float o = own[j + mate[j]];
          y[j] = pair[j] < 0 ? x[j] : x[j] * r.x + (mate[j] > 0 ? -o : o) * r.y;
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    if (on) store8<VEC>(dst, c0, dh, y);
    st += 4;
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
  // About ten steps a wave pay for the tokens' angles and the workgroup's start, but a step is 1 us of
  // latency: tokens share a workgroup only where there are 1024 workgroups without, and where there are
  // not 512 the heads are dealt out too (40 heads of 64, ten steps always: 256 tokens 9.4 us, 1024 10.1, 8192
  // 20.0; a step always: 4.4, 10.2 and 62; so: 4.3, 7.3 and 20.3; tokens shared from 4096 on: 22.7).
  const int64_t all = ceil_div(heads, 64 / group), least = std::max<int64_t>(1, 4 / all);
  const int tt = (int)std::max(least, std::min<int64_t>({16, 40 / all, a.tokens / 1024}));
  const int64_t parts = std::min(ceil_div(all, 4), ceil_div(512, ceil_div(a.tokens, tt)));
  const int steps = (int)ceil_div(all, parts);
  const int64_t wgs = ceil_div(a.tokens, tt);
  if (wgs > 8388607) {
    set_error("more tokens than a grid holds");
    return NV_ERR_UNSUPPORTED;
  }
  const dim3 grid((unsigned)wgs, (unsigned)ceil_div(all, steps));
  auto ok = [](const void* p, int64_t ld, int64_t row) {
    return !p || (aligned16(p) && (ld | row) % 8 == 0);
  };
  const bool vec = ok(q_heads ? q : nullptr, ldq, q_row_stride) &&
                   ok(q_heads ? q_out : nullptr, ldqo, qo_row_stride) &&
                   ok(k_heads ? k : nullptr, ldk, k_row_stride) &&
                   ok(k_heads ? k_out : nullptr, ldko, ko_row_stride);
  // channels without a pair look at the first ones
  const size_t lds = (size_t)tt * ((a.rot / 2 + 3) & ~3) * 8 + 32 + (halves ? 8192 : 0);
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(256), lds, (hipStream_t)stream, a, tt, steps);
  };
  bool by16 = true;
  for (int i = 0; i < n_axes; ++i) by16 &= axes[i] % 16 == 0;
  auto pick = [&](auto t, auto g) {
    typedef decltype(t) T;
    constexpr int G = decltype(g)::value;
    if (!halves) vec ? go(qk_rope_k<T, G, NEXT, true>) : go(qk_rope_k<T, G, NEXT, false>);
    else if (by16) vec ? go(qk_rope_k<T, G, HALF8, true>) : go(qk_rope_k<T, G, HALF8, false>);
    else vec ? go(qk_rope_k<T, G, HALF, true>) : go(qk_rope_k<T, G, HALF, false>);
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
