// Keys and values kept in 8 bits: appending tokens to their pages, and attention over them.
//
// Page: 64 tokens of one sequence.  Keys [head][64][dh] and values [head][dh][64] as e4m3
// codes, one scale byte per page and head for each.
//
// Attention multiplies 16-bit matrices: codes convert exactly (three mantissa bits), queries are
// taken as they are, in their type, and scales stay out of the 16-bit operands: a page's key scale
// multiplies its scores in float32, its value scale the accumulators' common unit.  The second
// product is float16 for either type: a probability loses 2^-11 there, 2^-8 in bfloat16 (32 rows of up
// to 8192 tokens, bfloat16: error against float64 0.0022 -> 0.0017, of which 0.0017 is the result's own
// rounding).  Float16 has no small numbers, so the largest probability of a row stands at 2^15, or
// 2^9 to 2^15 under many queries, instead of 1: one is rounded to 2^-11 of itself, or to 2^-34 of the
// largest where it is subnormal (below 2^-23 of it).  The sum takes the same rounded ones: a tail that
// rounding moves, moves the sum with it.
// S^T = K Q^T is computed, so an accumulator entry's column is a query and the softmax state is a
// lane's own; key row r of 16-key tile t is token 16 (r / 4) + 4 t + r % 4 of the page, so that
// lane group kc ends up with tokens 16 kc .. 16 kc + 15: the probabilities are then the second
// product's operand as they stand, against 16 consecutive bytes of a value row.  Nothing passes
// through LDS until waves merge.
#include <algorithm>

#include "common.h"
#include "e4m3.h"
#include "kv8.h"
#include "kv_join.h"

namespace nv {
namespace {

constexpr int PAGE = NV_KV8_PAGE;
constexpr int KV8_FEW_TOKENS = 4;  // of a row, that a wave appends on its own
constexpr float LOG2E = 1.4426950408889634f;

// ------------------------------------------------------------------------------------ append

// Four codes at another scale (old value * 2^d, d < 0).
__device__ __forceinline__ uint32_t recode4(uint32_t w, float f) {
  const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
  const auto b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  return codes4(a[0], a[1], b[0], b[1], f);
}

// What a call appends to the slot-th page that a row's tokens touch: tokens t0 .. t1 - 1 of it, from
// src on, ld apart.  False: nothing.
template <typename T>
struct Appended {
  const T* src;
  int64_t ld;
  uint8_t *codes, *scale;
  int t0, t1;
  __device__ __forceinline__ bool find(const Kv8AppendArgs& a, int64_t row, int head, bool is_v,
                                       int slot) {
    const int64_t pos = a.pos[row];
    const int cnt = a.count ? std::min(std::max(a.count[row], 0), a.T) : a.T;
    if (pos < 0) return false;
    const int64_t p = pos / PAGE + slot, first = p * PAGE;
    const int64_t lo = std::max(pos, first), hi = std::min(pos + cnt, first + PAGE);
    if (lo >= hi || p >= a.table_w) return false;
    const int64_t page = a.table[row * a.table_w + p];
    if (page < 0 || page >= a.n_pages) return false;
    t0 = (int)(lo - first), t1 = (int)(hi - first);
    ld = is_v ? a.ldv : a.ldk;
    src = (const T*)(is_v ? a.v : a.k) + row * (is_v ? a.v_row : a.k_row) + (lo - pos) * ld +
          (int64_t)head * a.dh;
    const int64_t ph = page * a.heads + head;
    codes = (is_v ? a.vp : a.kp) + ph * PAGE * a.dh;
    scale = (is_v ? a.vs : a.ks) + ph;
    return true;
  }
};

// Up to KV8_FEW_TOKENS tokens a row: a wave for what a workgroup does below.  Its lanes take eight
// channels of a token each, and nothing waits for a barrier (200 rows of one token, 8 heads of 128:
// 16.7 us with the kernel below, 7.1 here).
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) kv8_append_few_k(Kv8AppendArgs a, int64_t units, int slots) {
  constexpr int MAXU = (KV8_FEW_TOKENS * 160 / 8 + 63) / 64;
  const int lane = threadIdx.x & 63;
  int64_t id = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (id >= units) return;
  const bool is_v = id & 1;
  id >>= 1;
  const int head = (int)(id % a.heads);
  id /= a.heads;
  Appended<T> t;
  if (!t.find(a, id / slots, head, is_v, (int)(id % slots))) return;
  const int dh = a.dh, nch = dh / 8, n = (t.t1 - t.t0) * nch, t0 = t.t0;
  const int old = t0 > 0 ? *t.scale : 0;
  float v[MAXU][8];
  float top = 0.f;
#pragma unroll
  for (int u = 0; u < MAXU; ++u) {
    const int i = u * 64 + lane, k = i / nch;
    load8<VEC>(t.src + k * t.ld, (i - k * nch) * 8, i < n ? dh : 0, v[u]);
#pragma unroll
    for (int j = 0; j < 8; ++j) top = fmaxf(top, finite_abs(v[u][j]));
  }
  const int e = std::max(old, scale_byte(rows_max(row16_max(top))));
  const float inv = ldexpf(1.f, 127 - e), move = ldexpf(1.f, old - e);
  if (t0 > 0 && e > old) {  // the old codes to the larger scale
    if (!is_v) {
      for (int i = lane; i < t0 * nch; i += 64) {
        uint2* w = (uint2*)(t.codes + i * 8);
        *w = make_uint2(recode4(w->x, move), recode4(w->y, move));
      }
    } else {
      const int nw = (t0 + 3) / 4;  // the last word of a channel may hold new tokens: single codes
      for (int i = lane; i < dh * nw; i += 64) {
        const int c = i / nw, b = (i - c * nw) * 4;
        uint8_t* to = t.codes + c * PAGE + b;
        const uint32_t w = recode4(*(const uint32_t*)to, move);
        if (b + 4 <= t0) *(uint32_t*)to = w;
        else
          for (int k = 0; b + k < t0; ++k) to[k] = (uint8_t)(w >> (8 * k));
      }
    }
  }
#pragma unroll
  for (int u = 0; u < MAXU; ++u) {
    const int i = u * 64 + lane, k = i / nch, c = (i - k * nch) * 8;
    if (i >= n) continue;
    if (!is_v) {
      store_codes8<true>(t.codes + t0 * dh, i * 8, n * 8, v[u], inv);
    } else {
      const uint32_t w0 = codes4(v[u][0], v[u][1], v[u][2], v[u][3], inv);
      const uint32_t w1 = codes4(v[u][4], v[u][5], v[u][6], v[u][7], inv);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        t.codes[(c + j) * PAGE + t0 + k] = (uint8_t)((j < 4 ? w0 : w1) >> (8 * (j & 3)));
    }
  }
  if (lane == 0 && (t0 == 0 || e > old)) *t.scale = (uint8_t)e;
}

__device__ __forceinline__ float block_max(float v, float* part) {
  v = rows_max(row16_max(v));
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  return fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
}

// A workgroup per (row, touched page, head) and tensor: the new tokens' values stay in registers
// between their largest magnitude and their codes.  A thread takes eight channels of single tokens
// for keys, and of four neighbouring tokens for values: their codes of one channel are a word of the
// transposed page, sixteen lanes write a whole row of it, and nothing passes through LDS (through it,
// byte by byte, 8 prompts of 2000 tokens, 8 heads of 128, took 28.8 us, so 23.6).  Bound by launch and
// latency for single tokens; for prompts (3.8 TB/s) by its loads' way: waves wait 58 % of their cycles.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) kv8_append_k(Kv8AppendArgs a) {
  __shared__ float part[4];
  const int tid = threadIdx.x;
  const bool is_v = blockIdx.y & 1;
  Appended<T> at;
  if (!at.find(a, blockIdx.z, blockIdx.y >> 1, is_v, blockIdx.x)) return;  // uniform
  const int dh = a.dh, nch = dh / 8, t0 = at.t0, t1 = at.t1;
  const T* src = at.src;
  const int64_t ld = at.ld;
  uint8_t *codes = at.codes, *scale = at.scale;
  const int old = t0 > 0 ? *scale : 0;  // before block_max's barrier: thread 0 writes it after
  float top = 0.f;
  int e;
  if (!is_v) {
    constexpr int MAXU = 64 * 160 / 8 / 256;
    const int units = (t1 - t0) * nch;
    float v[MAXU][8];
#pragma unroll
    for (int u = 0; u < MAXU; ++u) {
      const int i = u * 256 + tid;
      if (u * 256 >= units) break;  // uniform
      const int t = i / nch, c = (i - t * nch) * 8;
      load8<VEC>(src + t * ld, c, i < units ? dh : 0, v[u]);
#pragma unroll
      for (int j = 0; j < 8; ++j) top = fmaxf(top, finite_abs(v[u][j]));
    }
    e = std::max(old, scale_byte(block_max(top, part)));
    const float inv = ldexpf(1.f, 127 - e), move = ldexpf(1.f, old - e);
    if (t0 > 0 && e > old)
      for (int i = tid; i < t0 * nch; i += 256) {
        uint2* w = (uint2*)(codes + i * 8);
        *w = make_uint2(recode4(w->x, move), recode4(w->y, move));
      }
#pragma unroll
    for (int u = 0; u < MAXU; ++u) {
      const int i = u * 256 + tid;
      if (u * 256 >= units) break;
      if (i < units) store_codes8<true>(codes + t0 * dh, i * 8, units * 8, v[u], inv);
    }
  } else {
    constexpr int MAXU = (16 * 160 / 8 + 255) / 256;
    float v[MAXU][4][8];
#pragma unroll
    for (int u = 0; u < MAXU; ++u) {
      const int t = (tid & 15) * 4, c = (u * 16 + (tid >> 4)) * 8;  // c >= dh: no channels
      if (u * 128 >= dh) break;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const bool there = c < dh && t + k >= t0 && t + k < t1;
        load8<VEC>(src + (t + k - t0) * ld, c, there ? dh : 0, v[u][k]);
#pragma unroll
        for (int j = 0; j < 8; ++j) top = fmaxf(top, finite_abs(v[u][k][j]));
      }
    }
    e = std::max(old, scale_byte(block_max(top, part)));
    const float inv = ldexpf(1.f, 127 - e), move = ldexpf(1.f, old - e);
    const bool grow = t0 > 0 && e > old;
#pragma unroll
    for (int u = 0; u < MAXU; ++u) {
      const int t = (tid & 15) * 4, c = (u * 16 + (tid >> 4)) * 8;
      if (u * 128 >= dh) break;
      // words of new codes; single ones at [t0, t1)'s ends; words with old codes to move if the scale
      // grew: what else is in them stays
      if (c >= dh || t >= t1 || (t + 4 <= t0 && !grow)) continue;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        uint32_t* to = (uint32_t*)(codes + (c + j) * PAGE + t);
        uint32_t w = codes4(v[u][0][j], v[u][1][j], v[u][2][j], v[u][3][j], inv);
        if (!grow && (t < t0 || t + 4 > t1)) {
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (t + k >= t0 && t + k < t1) ((uint8_t*)to)[k] = (uint8_t)(w >> (8 * k));
          continue;
        }
        if (t < t0 || t + 4 > t1) {
          const uint32_t was = *to, kept = grow ? recode4(was, move) : was, fresh = w;
          w = 0;
#pragma unroll
          for (int k = 0; k < 4; ++k)
            w |= (t + k < t0 ? kept : t + k < t1 ? fresh : was) & (0xFFu << (8 * k));
        }
        *to = w;
      }
    }
  }
  if (tid == 0 && (t0 == 0 || e > old)) *scale = (uint8_t)e;
}

// --------------------------------------------------------------------------------- attention

// Four pairs of 16-bit values as one operand.
template <typename Vec, typename P>
__device__ __forceinline__ Vec pack8(P a, P b, P c, P d) {
  return __builtin_bit_cast(Vec, u32x4{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b),
                                       __builtin_bit_cast(uint32_t, c), __builtin_bit_cast(uint32_t, d)});
}

template <typename T>
struct Mma;
template <>
struct Mma<_Float16> {
  typedef half8 Vec;
  static __device__ __forceinline__ floatx4 mul(Vec a, Vec b, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
  // eight codes times the power of two s
  static __device__ __forceinline__ Vec codes(uint32_t lo, uint32_t hi, float s) {
    return pack8<Vec>(__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, s, false),
                      __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, s, true),
                      __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, s, false),
                      __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, s, true));
  }
};
template <>
struct Mma<__bf16> {
  typedef bf16x8 Vec;
  static __device__ __forceinline__ floatx4 mul(Vec a, Vec b, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ Vec codes(uint32_t lo, uint32_t hi, float s) {
    return pack8<Vec>(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, false),
                      __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, true),
                      __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, false),
                      __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, true));
  }
};

// Head dimension in 32-wide steps.  A whole 64 is two steps of which lane group kc takes dims
// 16 kc .. 16 kc + 15 (one 16-byte load); the rest go 8 a group, dims past dh zero.
template <int DH>
struct Dims {
  static constexpr int FULL = DH / 64, REST = DH % 64, STEPS = 2 * FULL + (REST + 31) / 32;
  static constexpr int DV = (DH + 15) / 16;  // 16-channel tiles of the output
  static __device__ __forceinline__ int dim(int step, int kc) {
    return step < 2 * FULL ? (step / 2) * 64 + kc * 16 + (step & 1) * 8
                           : FULL * 64 + (step - 2 * FULL) * 32 + kc * 8;
  }
};

// Bytes of w (tokens t .. t + 15) at or past n tokens become zero.
__device__ __forceinline__ u32x4 keep_tokens(u32x4 w, int n) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int k = n - j * 4;
    if (k < 4) w[j] = k <= 0 ? 0 : w[j] & ((1u << (8 * k)) - 1);
  }
  return w;
}

// Nonzero where a byte of w is a NaN code (0x7F, 0xFF): that byte's bit 7.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) {
  return ((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
}

// Pages p0 .. p1 - 1 of share `split` of a tile's pages: equal parts of at least KV8_SHARE pages, so a
// short row's last shares may be empty.
__device__ __forceinline__ void share_of(int pages, int split, int splits, int* p0, int* p1) {
  const int n = std::max(KV8_SHARE, (pages + splits - 1) / splits);
  *p0 = (int)std::min<int64_t>((int64_t)split * n, pages);
  *p1 = std::min(*p0 + n, pages);
}

// One wave's running softmax over 16 queries: reference (probabilities are 2^(score - m)), their sum,
// accumulators O^T in units of 2^(unit - 127).  The unit is a query's own: it follows the scales of the
// pages that the query sees, and no others.
template <int DH>
struct State {
  float m, l;
  int unit;
  floatx4 acc[Dims<DH>::DV];
};

// The value exponents that convert exactly beside the unit: codes are 2^-9 .. 448, times
// 2^-5 .. 2^7 still normal float16 numbers.
constexpr int UNIT_LO = -5, UNIT_HI = 7;

// The largest probability is at most 2^P_TOP, which float16 holds.
constexpr float P_TOP = 15.f;

// The reference under which a score of `top` has the probability 2^room (room <= P_TOP): top - room, or
// top itself where the scores are so large that this rounds to more than P_TOP below it.
__device__ __forceinline__ float reference(float top, float room) {
  const float low = top - room;
  return top - low > P_TOP ? top : low;
}

// Sums over the 64 keys of a page out of the matrix unit, of the probabilities as rounded: a row of ones.
__device__ __forceinline__ floatx4 add_probs(const half8* fp, floatx4 sum) {
  half8 ones;
#pragma unroll
  for (int i = 0; i < 8; ++i) ones[i] = (_Float16)1.f;
  return Mma<_Float16>::mul(ones, fp[1], Mma<_Float16>::mul(ones, fp[0], sum));
}

// A lane's part of a page of one head: codes of keys 16 (li / 4) + 4 t + li % 4 and of 16 tokens of
// channels 16 j + li, and the two scale bytes.
template <int DH>
struct PageCodes {
  u32x4 k[4][Dims<DH>::FULL + 1];                              // [FULL]: not used
  uint2 kr[4][Dims<DH>::STEPS - 2 * Dims<DH>::FULL + 1];       // [REST]: not used
  u32x4 v[Dims<DH>::DV];
  int ke, ve;
  __device__ __forceinline__ void load_keys(const Kv8AttnArgs& a, int64_t ph, int li, int kc) {
    using D = Dims<DH>;
    const uint8_t* kp = a.kp + ph * PAGE * DH + (16 * (li >> 2) + (li & 3)) * DH;
    ke = a.ks[ph];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
#pragma unroll
      for (int b = 0; b < D::FULL; ++b) k[t][b] = *(const u32x4*)(kp + 4 * t * DH + b * 64 + kc * 16);
#pragma unroll
      for (int b = 2 * D::FULL; b < D::STEPS; ++b) {
        const int d = D::dim(b, kc);
        kr[t][b - 2 * D::FULL] = d < DH ? *(const uint2*)(kp + 4 * t * DH + d) : make_uint2(0, 0);
      }
    }
  }
  __device__ __forceinline__ void load_values(const Kv8AttnArgs& a, int64_t ph, int li, int kc) {
    using D = Dims<DH>;
    const uint8_t* vp = a.vp + ph * PAGE * DH + li * PAGE + kc * 16;
    ve = a.vs[ph];
#pragma unroll
    for (int j = 0; j < D::DV; ++j)
      v[j] = DH % 16 == 0 || j * 16 + li < DH ? *(const u32x4*)(vp + j * 16 * PAGE)
                                              : u32x4{0, 0, 0, 0};
  }
};

// A page's 64 tokens, from token j0 of the sequence, into the state.  lim: tokens this lane's
// query sees (at least one query sees some of the page); len: tokens of the sequence; some: whether
// some query sees only part of them.  keys_done runs once the keys' registers are free again.
template <typename T, int DH, typename Done>
__device__ __forceinline__ void page_step(State<DH>& st, const typename Mma<T>::Vec* fq,
                                          PageCodes<DH>& pc, float scale2, int j0, int lim, int len,
                                          bool some, int kc, Done&& keys_done) {
  using D = Dims<DH>;
  using M = Mma<T>;
  using V = Mma<_Float16>;
  u32x4(&v)[D::DV] = pc.v;
  const int ke = __builtin_amdgcn_readfirstlane(pc.ke);
  const int ve = __builtin_amdgcn_readfirstlane(pc.ve);
  floatx4 s[4];
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    s[t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int b = 0; b < D::FULL; ++b) {
      s[t] = M::mul(M::codes(pc.k[t][b][0], pc.k[t][b][1], 1.f), fq[2 * b], s[t]);
      s[t] = M::mul(M::codes(pc.k[t][b][2], pc.k[t][b][3], 1.f), fq[2 * b + 1], s[t]);
    }
#pragma unroll
    for (int b = 2 * D::FULL; b < D::STEPS; ++b) {
      const uint2 w = pc.kr[t][b - 2 * D::FULL];
      s[t] = M::mul(M::codes(w.x, w.y, 1.f), fq[b], s[t]);
    }
  }
  keys_done();
  const float f = scale2 * scale_value(ke);
  float top = -INFINITY;
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      s[t][r] *= f;
      if (some && j0 + 16 * kc + 4 * t + r >= lim) s[t][r] = -INFINITY;
      top = fmaxf(top, s[t][r]);
    }
  const float mnew = fmaxf(st.m, reference(rows_max(top), P_TOP)), base = mnew == -INFINITY ? 0.f : mnew;
  const float alpha = __builtin_amdgcn_exp2f(st.m - base);
  if (__ballot(mnew != st.m)) {
#pragma unroll
    for (int j = 0; j < D::DV; ++j) st.acc[j] *= alpha;
    st.l *= alpha;
    st.m = mnew;
  }
  half8 fp[2];
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      fp[t >> 1][(t & 1) * 4 + r] = (_Float16)__builtin_amdgcn_exp2f(s[t][r] - base);
  st.l += add_probs(fp, floatx4{0.f, 0.f, 0.f, 0.f})[0];
  if (ve == 255) {  // a NaN scale: every code of the page is NaN, the unit stays
#pragma unroll
    for (int j = 0; j < D::DV; ++j) v[j] = u32x4{0x7F7F7F7F, 0x7F7F7F7F, 0x7F7F7F7F, 0x7F7F7F7F};
  }
  if (some) {
    // Tokens behind the sequence may hold anything: zeros.  A NaN among those before that some
    // query does not see must not reach it (0 * NaN): NaN codes become zeros, and a product of
    // indicators (is NaN) x (is seen) finds the outputs that they do reach.
    uint32_t any = 0;
#pragma unroll
    for (int j = 0; j < D::DV; ++j) {
      v[j] = keep_tokens(v[j], len - j0 - kc * 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) any |= nan_bytes(v[j][i]);
    }
    if (__ballot(any != 0)) {
      half8 seen[2];
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          seen[t >> 1][(t & 1) * 4 + r] = (_Float16)(j0 + 16 * kc + 4 * t + r < lim ? 1.f : 0.f);
#pragma unroll
      for (int j = 0; j < D::DV; ++j) {
        u32x4 ind;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t n = nan_bytes(v[j][i]) >> 7;  // 1 in each NaN byte
          ind[i] = n * 0x38;                           // code of 1.0
          v[j][i] &= ~(n * 0xFF);
        }
        floatx4 hit = {0.f, 0.f, 0.f, 0.f};
        hit = V::mul(V::codes(ind[0], ind[1], 1.f), seen[0], hit);
        hit = V::mul(V::codes(ind[2], ind[3], 1.f), seen[1], hit);
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (hit[r] > 0.f) st.acc[j][r] = __int_as_float(0x7FC00000);
      }
    }
  }
  // Queries that see the page have one unit (they saw the same pages before it), but for pages that
  // come late (attn_kv8_tall_k).
  const bool sees = lim > j0;
  const int unit = __builtin_amdgcn_readlane(st.unit, __builtin_ctzll(__ballot(sees)));
  const int d = ve == 255 ? 0 : ve - unit;
  if (d < UNIT_LO || d > UNIT_HI || __ballot(sees && st.unit != unit)) {
    // far from the unit: its own accumulators, added at their size; far above, it becomes the unit
    const int own = ve == 255 ? 0 : ve - st.unit;
    const bool up = sees && own > UNIT_HI;
    const float was = up ? ldexpf(1.f, -own) : 1.f, g = up ? 1.f : sees ? ldexpf(1.f, own) : 0.f;
    if (up) st.unit = ve;
#pragma unroll
    for (int j = 0; j < D::DV; ++j) {
      floatx4 o = {0.f, 0.f, 0.f, 0.f};
      o = V::mul(V::codes(v[j][0], v[j][1], 1.f), fp[0], o);
      o = V::mul(V::codes(v[j][2], v[j][3], 1.f), fp[1], o);
      st.acc[j] = st.acc[j] * was + o * g;
    }
    return;
  }
  const float g = __int_as_float((127 + d) << 23);
#pragma unroll
  for (int j = 0; j < D::DV; ++j) {
    st.acc[j] = V::mul(V::codes(v[j][0], v[j][1], g), fp[0], st.acc[j]);
    st.acc[j] = V::mul(V::codes(v[j][2], v[j][3], g), fp[1], st.acc[j]);
  }
}

// A workgroup takes 16 queries of one row and kv head (query heads of the group innermost) and
// share of the row's pages, dealt out to its four waves; their states meet in LDS.  With more
// than one share the means go to the workspace and attn_join_k adds them in order.  Bound by HBM:
// one query over 200000 tokens, 8 heads of 128, 75 us (5.4 TB/s); 32 rows of 2048 to 8192 tokens 76.
template <typename T, int DH>
__global__ void __launch_bounds__(256) attn_kv8_k(Kv8AttnArgs a) {
  using D = Dims<DH>;
  typedef typename Mma<T>::Vec Vec;
  constexpr int NW = 4, CH = D::DV * 16;
  __shared__ float sm[NW][16], sl[NW][16];
  __shared__ __align__(16) float so[NW][16][CH + 4];
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, kc = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int id = blockIdx.x;
  const int split = id % a.splits;
  id /= a.splits;
  const int ct = id % a.col_tiles;
  id /= a.col_tiles;
  const int head = id % a.kv_heads, row = id / a.kv_heads;
  const int group = a.heads / a.kv_heads, cols = a.S * group, c0 = ct * 16;
  const int col = std::min(c0 + li, cols - 1), qs = col / group, qh = head * group + col % group;
  const int len = (int)std::min<int64_t>(std::max(a.lens[row], 0), (int64_t)a.table_w * PAGE);
  const int64_t q0 = a.qpos ? (int64_t)a.qpos[row] + 1 : len;  // tokens that query 0 sees
  auto sees = [&](int s) {
    return (int)std::max<int64_t>(0, std::min<int64_t>(len, a.qpos ? q0 + s : len));
  };
  const int lim = sees(qs), least = sees(c0 / group);
  const int most = sees((std::min(c0 + 16, cols) - 1) / group);
  int p0, p1;
  share_of((most + PAGE - 1) / PAGE, split, a.splits, &p0, &p1);

  Vec fq[D::STEPS];
  const T* qrow = (const T*)a.q + (int64_t)row * a.q_row + (int64_t)qs * a.ldq + (int64_t)qh * DH;
#pragma unroll
  for (int b = 0; b < D::STEPS; ++b) {
    const int d = D::dim(b, kc);
    fq[b] = d < DH ? *(const Vec*)(qrow + d) : Vec{};
  }
  State<DH> st;
  st.m = -INFINITY, st.l = 0.f, st.unit = 1;
#pragma unroll
  for (int j = 0; j < D::DV; ++j) st.acc[j] = floatx4{0.f, 0.f, 0.f, 0.f};
  const float scale2 = a.scale * LOG2E;
  // The next page's keys are requested as soon as this one's are multiplied, its values after this
  // one's, into the same registers; its table entry was read a page earlier.
  const int32_t* table = a.table + (int64_t)row * a.table_w;
  int pn = p0 + wave, entry = pn < p1 ? table[pn] : 0;
  auto take = [&](int& p) {  // page and head of the next page that is there; -1: none left
    while (pn < p1) {
      p = pn;
      const int64_t page = __builtin_amdgcn_readfirstlane(entry);
      pn += NW;
      if (pn < p1) entry = table[pn];
      if (page >= 0 && page < a.n_pages) return page * a.kv_heads + head;
    }
    return (int64_t)-1;
  };
  PageCodes<DH> pc;
  int p = 0;
  int64_t ph = take(p);
  if (ph >= 0) pc.load_keys(a, ph, li, kc), pc.load_values(a, ph, li, kc);
  while (ph >= 0) {
    const int j0 = p * PAGE;
    const int64_t next = take(p);
    page_step<T, DH>(st, fq, pc, scale2, j0, lim, len, j0 + PAGE > least, kc, [&] {
      if (next >= 0) pc.load_keys(a, next, li, kc);
    });
    if (next >= 0) pc.load_values(a, next, li, kc);
    ph = next;
  }
  // The waves' states, in wave order: means, which are no larger than the values, and their weights (a
  // sum in its final size may pass float32 where the mean does not).
  const float l = st.l, us = scale_value(st.unit), mean = l == 0.f ? 0.f : 1.f / l;
  if (kc == 0) sm[wave][li] = st.m, sl[wave][li] = l;
#pragma unroll
  for (int j = 0; j < D::DV; ++j) *(floatx4*)&so[wave][li][j * 16 + kc * 4] = st.acc[j] * mean * us;
  __syncthreads();
  for (int i = tid; i < 16 * (CH / 4); i += 256) {
    const int c = i / (CH / 4), d = i % (CH / 4) * 4;
    if (c0 + c >= cols || d >= DH) continue;
    float m = sm[0][c];
#pragma unroll
    for (int w = 1; w < NW; ++w) m = fmaxf(m, sm[w][c]);
    const float base = m == -INFINITY ? 0.f : m;
    float f[NW], ls = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) ls += f[w] = __builtin_amdgcn_exp2f(sm[w][c] - base) * sl[w][c];
    const float inv = ls == 0.f ? 0.f : 1.f / ls;
    floatx4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < NW; ++w) o += f[w] * inv * *(const floatx4*)&so[w][c][d];
    if (a.splits == 1) {
      const int qi = (c0 + c) / group, h = head * group + (c0 + c) % group;
      struct alignas(8) Quad { T v[4]; } out;
#pragma unroll
      for (int r = 0; r < 4; ++r) out.v[r] = (T)o[r];
      *(Quad*)((T*)a.out + (int64_t)row * a.o_row + (int64_t)qi * a.ldo + (int64_t)h * DH + d) = out;
    } else {
      const int64_t slot = (((int64_t)row * a.kv_heads + head) * cols + c0 + c) * a.splits + split;
      if (m != -INFINITY || ls != 0.f) *(floatx4*)(a.part_o + slot * DH + d) = o;
      if (d == 0) a.part_ml[slot * 2] = m, a.part_ml[slot * 2 + 1] = ls;
    }
  }
}

// Many queries of a head: four waves of QB * 16 queries share every page.  A page's codes come two
// pages ahead into registers and are converted once, on their way into a double-buffered LDS
// (16-bit: the products then read operands as they stand); key rows lie in the order in which
// page_step takes them, so 16 rows are 16 consecutive ones.  A page that not every query sees whole
// has its scores masked and its values behind the sequence zeroed; one with a NaN value among the
// others waits until the loop is over and goes through page_step, which keeps it from the queries
// that do not see it, and so does one whose values are too small beside the others'.  Workgroups run in
// order of falling work under a causal limit: the last queries of every head first, which counts where
// not all of them are resident at once.
// 2 x 2048 queries, 16 heads of 128 on 4, over 4096 tokens: 154 us (890 TFLOP/s); per SIMD the matrix
// unit is busy 41 % of the time and the vector unit 44 %, mostly one after the other.  Under a causal
// limit behind 2048 tokens 133 to 138, from an empty cache 72: the 64 or 32 pages of the last tiles, at
// 2.1 to 2.4 us a page, while the shorter tiles beside them end early (all 512 are resident).
template <typename T, int DH, int QB>
__global__ void __launch_bounds__(256, 2) attn_kv8_tall_k(Kv8AttnArgs a) {
  using D = Dims<DH>;
  using M = Mma<T>;
  typedef typename M::Vec Vec;
  using V = Mma<_Float16>;
  constexpr int NW = 4, NT = NW * 64, COLS = NW * QB * 16;
  constexpr int CW = DH % 16 ? 8 : 16;                       // codes of a key chunk
  constexpr int KCH = DH / CW, KCN = PAGE * KCH, VCN = DH * 4;  // chunks of a page (values: 16 codes)
  constexpr int KPT = (KCN + NT - 1) / NT, VPT = (VCN + NT - 1) / NT;
  constexpr int KROW = (DH / 8) % 2 ? DH : DH + 8, VROW = PAGE + 8;  // odd counts of 16-byte chunks
  constexpr int VR = D::DV * 16;
  __shared__ __align__(16) T sk[2][PAGE * KROW];
  __shared__ __align__(16) _Float16 sv[2][VR * VROW];
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, kc = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  __shared__ uint32_t nan_pages;  // bit i: page least / 64 + i waits (at most COLS / 64 + 2 pages)
  const int rh = blockIdx.x % (a.rows * a.kv_heads);  // a multiple of 8: one XCD's L2 for a head
  const int rest = blockIdx.x / (a.rows * a.kv_heads), split = rest / a.col_tiles;
  const int ct = a.col_tiles - 1 - rest % a.col_tiles;
  const int head = rh % a.kv_heads, row = rh / a.kv_heads;
  const int group = a.heads / a.kv_heads, cols = a.S * group, c0 = ct * COLS;
  const int len = (int)std::min<int64_t>(std::max(a.lens[row], 0), (int64_t)a.table_w * PAGE);
  const int64_t q0 = a.qpos ? (int64_t)a.qpos[row] + 1 : len;  // tokens that query 0 sees
  auto sees = [&](int c) {                                     // tokens that column c sees
    c = std::min(c, cols - 1) / group;
    return (int)std::max<int64_t>(0, std::min<int64_t>(len, a.qpos ? q0 + c : len));
  };
  const int32_t* table = a.table + (int64_t)row * a.table_w;
  const float scale2 = a.scale * LOG2E;

  Vec fq[QB][D::STEPS];
  State<DH> st[QB];
  floatx4 sum[QB];  // of a lane's query, four times
  int lim[QB];
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    const int col = std::min(c0 + (wave * QB + qb) * 16 + li, cols - 1);
    lim[qb] = sees(col);
    const T* qrow = (const T*)a.q + (int64_t)row * a.q_row + (int64_t)(col / group) * a.ldq +
                    (int64_t)(head * group + col % group) * DH;
#pragma unroll
    for (int b = 0; b < D::STEPS; ++b) {
      const int d = D::dim(b, kc);
      fq[qb][b] = d < DH ? *(const Vec*)(qrow + d) : Vec{};
    }
    st[qb].m = -INFINITY, st[qb].unit = 1, sum[qb] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < D::DV; ++j) st[qb].acc[j] = floatx4{0.f, 0.f, 0.f, 0.f};
  }

  // the page at hand: its place, scales, and how its values enter the accumulators
  struct Page { int64_t ph; int p, ke, ve; };
  const int least = sees(c0);
  int pnext, pages;  // the next page of this share, and its end
  share_of((sees(c0 + COLS - 1) + PAGE - 1) / PAGE, split, a.splits, &pnext, &pages);
  const int first = pnext;
  const int wave_least = sees(c0 + wave * QB * 16), wave_most = sees(c0 + (wave + 1) * QB * 16 - 1);
  // The next page that is there (p.ph < 0: none left).  Its table entry was read at the last call:
  // the page's address does not wait for memory.
  int entry = pnext < pages ? table[pnext] : 0;
  auto take = [&](Page& p) {
    p.ph = -1;
    while (pnext < pages) {
      const int64_t page = __builtin_amdgcn_readfirstlane(entry);
      p.p = pnext++;
      if (pnext < pages) entry = table[pnext];
      if (page < 0 || page >= a.n_pages) continue;
      p.ph = page * a.kv_heads + head;
      p.ke = a.ks[p.ph], p.ve = a.vs[p.ph];
      break;
    }
  };
  struct Chunk { uint32_t w[CW / 4]; };
  Chunk rk[KPT];
  u32x4 rv[VPT];
  auto fetch = [&](const Page& p) {
    const uint8_t* kp = a.kp + p.ph * PAGE * DH;
    const uint8_t* vp = a.vp + p.ph * PAGE * DH;
#pragma unroll
    for (int i = 0; i < KPT; ++i)
      if (KCN % NT == 0 || tid + i * NT < KCN)
        __builtin_memcpy(&rk[i], __builtin_assume_aligned(kp + (tid + i * NT) * CW, CW), CW);
#pragma unroll
    for (int i = 0; i < VPT; ++i)
      if (VCN % NT == 0 || tid + i * NT < VCN) rv[i] = *(const u32x4*)(vp + (tid + i * NT) * 16);
  };
  auto stash = [&](const Page& p, int buf, float vscale) {
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
      const int c = tid + i * NT, key = c / KCH;
      if (KCN % NT != 0 && c >= KCN) break;
      // key 16 g + 4 t + r goes to row 16 t + 4 g + r
      T* to = sk[buf] + ((key >> 2 & 3) * 16 + (key >> 4) * 4 + (key & 3)) * KROW + c % KCH * CW;
      *(Vec*)to = M::codes(rk[i].w[0], rk[i].w[1], 1.f);
      if constexpr (CW == 16) *(Vec*)(to + 8) = M::codes(rk[i].w[2], rk[i].w[3], 1.f);
    }
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int c = tid + i * NT;
      if (VCN % NT != 0 && c >= VCN) break;
      if (p.ve == 255) rv[i] = u32x4{0x7F7F7F7F, 0x7F7F7F7F, 0x7F7F7F7F, 0x7F7F7F7F};
      if (p.p * PAGE + PAGE > least) {  // uniform
        rv[i] = keep_tokens(rv[i], len - p.p * PAGE - (c & 3) * 16);
        if (nan_bytes(rv[i][0]) | nan_bytes(rv[i][1]) | nan_bytes(rv[i][2]) | nan_bytes(rv[i][3]))
          atomicOr(&nan_pages, 1u << (p.p - least / PAGE));
      }
      _Float16* to = sv[buf] + (c >> 2) * VROW + (c & 3) * 16;
      *(half8*)to = V::codes(rv[i][0], rv[i][1], vscale);
      *(half8*)(to + 8) = V::codes(rv[i][2], rv[i][3], vscale);
    }
  };
  if (DH % 16)  // channels past dh: zeros
    for (int i = tid; i < 2 * (VR - DH) * VROW; i += NT)
      sv[i / ((VR - DH) * VROW)][DH * VROW + i % ((VR - DH) * VROW)] = (_Float16)0.f;

  // Unit of the accumulators, the same in every wave, of the queries that see the page at hand.  A
  // page's exponent beside it is folded into its converted values where that is exact; one far above
  // becomes the unit (of the queries that see it: the others keep theirs); for one far below the
  // accumulators are brought to its size and back (exact too: a term is below 2^31, so they stay
  // below 2^126), and one further below than that waits until the loop is over (sums of its own here
  // cost every page 4 %).
  constexpr int FAR = -64;
  int unit = 1;
  bool late = false;                               // some page waits for its distance
  struct How { float conv, pre, post; bool late; };  // factors: values; accumulators before, after
  auto how = [&](const Page& p) {
    const int d = p.ve == 255 ? 0 : p.ve - unit;
    How h{1.f, 1.f, 1.f, d < FAR};
    if (d > UNIT_HI) h.pre = ldexpf(1.f, -d), unit = p.ve;
    else if (h.late) late = true;
    else if (d < UNIT_LO) h.pre = ldexpf(1.f, -d), h.post = ldexpf(1.f, d);
    else h.conv = __int_as_float((127 + d) << 23);
    return h;
  };

  auto attend = [&](const Page& p, int buf, int j0, bool some) {
    const T* K_ = sk[buf];
    const _Float16* V_ = sv[buf];
    const float f = scale2 * scale_value(p.ke);
    // Key fragments are requested TG tiles at a time, VG tiles of values before the softmax, whose
    // arithmetic covers their way (left to itself the compiler reads each just before its
    // multiply, and a SIMD has two waves to fill the wait with): all of them where 256 registers
    // hold them.
    constexpr int TG = DH >= 128 ? 2 : 4, VG = DH >= 128 ? D::DV / 2 : D::DV;
    floatx4 s[QB][4];
#pragma unroll
    for (int t0 = 0; t0 < 4; t0 += TG) {
      Vec fk[TG][D::STEPS];
#pragma unroll
      for (int t = 0; t < TG; ++t)
#pragma unroll
        for (int b = 0; b < D::STEPS; ++b) {
          const int d = D::dim(b, kc);  // past dh: the row's first codes against zeros
          fk[t][b] = *(const Vec*)(K_ + ((t0 + t) * 16 + li) * KROW + (d < DH ? d : 0));
        }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int t = 0; t < TG; ++t)
#pragma unroll
        for (int b = 0; b < D::STEPS; ++b)
#pragma unroll
          for (int qb = 0; qb < QB; ++qb)
            s[qb][t0 + t] =
                M::mul(fk[t][b], fq[qb][b], b ? s[qb][t0 + t] : floatx4{0.f, 0.f, 0.f, 0.f});
    }
    const _Float16* vr = V_ + li * VROW + kc * 16;
    auto value = [&](int j, int h2) { return *(const half8*)(vr + j * 16 * VROW + h2 * 8); };
    half8 fv[VG][2];
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int j = 0; j < VG; ++j) fv[j][0] = value(j, 0), fv[j][1] = value(j, 1);
    __builtin_amdgcn_sched_barrier(0);
    // Scores relative to the query's reference.  It moves only when a probability would pass 2^P_TOP,
    // and then to where the largest is 2^LOW: low enough that few pages move it, high enough for what
    // is small beside it (2 x 2048 queries of 16 heads on 4096 tokens, scores of spread 4: 161.8 us
    // with 7, 165 with 9 and 10, 171 with 12; spread 1: 157 to 159 with any).
    constexpr float LOW = 9.f;
    bool grow = false;
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      const float base = st[qb].m == -INFINITY ? 0.f : st[qb].m;
      float top = -INFINITY;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          s[qb][t][r] = fmaf(s[qb][t][r], f, -base);
          top = fmaxf(top, s[qb][t][r]);
        }
      if (some) {  // uniform
        const int n = lim[qb] - j0 - 16 * kc;
        top = -INFINITY;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            if (4 * t + r >= n) s[qb][t][r] = -INFINITY;
            top = fmaxf(top, s[qb][t][r]);
          }
      }
      grow |= !(top <= P_TOP) || st[qb].m == -INFINITY;
    }
    if (__ballot(grow)) {
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        float top = -INFINITY;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r) top = fmaxf(top, s[qb][t][r]);
        top = rows_max(top);
        const bool fresh = st[qb].m == -INFINITY;
        const float low = reference(top, LOW);
        const float move = low == -INFINITY ? 0.f : fresh ? low : fmaxf(low, 0.f);
        const float mnew = fresh ? low : st[qb].m + move;
        const float alpha = fresh ? 0.f : __builtin_amdgcn_exp2f(-move);
        st[qb].m = mnew;
        sum[qb] *= alpha;
#pragma unroll
        for (int j = 0; j < D::DV; ++j) st[qb].acc[j] *= alpha;
#pragma unroll
        for (int t = 0; t < 4; ++t) s[qb][t] -= move;
      }
    }
    half8 fp[QB][2];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          fp[qb][t >> 1][(t & 1) * 4 + r] = (_Float16)__builtin_amdgcn_exp2f(s[qb][t][r]);
      sum[qb] = add_probs(fp[qb], sum[qb]);
    }
#pragma unroll
    for (int j = 0; j < D::DV; ++j) {
      const half8 v0 = j < VG ? fv[j < VG ? j : 0][0] : value(j, 0);
      const half8 v1 = j < VG ? fv[j < VG ? j : 0][1] : value(j, 1);
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) st[qb].acc[j] = V::mul(v0, fp[qb][0], st[qb].acc[j]);
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) st[qb].acc[j] = V::mul(v1, fp[qb][1], st[qb].acc[j]);
    }
  };

  auto multiply = [&](const Page& p, const How& h, int buf) {
    const int j0 = p.p * PAGE;
    const bool some = j0 + PAGE > wave_least;  // some query of the wave sees part of it
    if (h.pre != 1.f) {
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        const bool sees = lim[qb] > j0;
        const float f = sees || h.post != 1.f ? h.pre : 1.f;
        if (sees && h.post == 1.f) st[qb].unit = p.ve;
#pragma unroll
        for (int j = 0; j < D::DV; ++j) st[qb].acc[j] *= f;
      }
    }
    if (j0 < wave_most && !h.late &&
        !(j0 + PAGE > least && (nan_pages >> (p.p - least / PAGE) & 1)))
      attend(p, buf, j0, some);
    if (h.post != 1.f) {
#pragma unroll
      for (int qb = 0; qb < QB; ++qb)
#pragma unroll
        for (int j = 0; j < D::DV; ++j) st[qb].acc[j] *= h.post;
    }
  };

  Page cur, ahead;
  How hc{1.f, 1.f, 1.f, false};
  if (tid == 0) nan_pages = 0;
  __syncthreads();
  take(cur);
  if (cur.ph >= 0) {
    fetch(cur);
    hc = how(cur);
    stash(cur, 0, hc.conv);
    take(ahead);
    if (ahead.ph >= 0) fetch(ahead);
    int buf = 0;
    while (true) {
      __syncthreads();  // the page is in LDS; the other buffer is read no more
      multiply(cur, hc, buf);
      if (ahead.ph < 0) break;
      hc = how(ahead);
      stash(ahead, buf ^ 1, hc.conv);
      cur = ahead;
      take(ahead);
      if (ahead.ph >= 0) fetch(ahead);
      buf ^= 1;
    }
  }
  const uint32_t nans = __builtin_amdgcn_readfirstlane(nan_pages);
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    st[qb].l = sum[qb][0];
    // the pages that wait: the units again in order tell which are too far below theirs
    int seen_unit = 1;
    for (int p = late ? first : nans ? least / PAGE : pages; p < pages; ++p) {
      bool waits = p >= least / PAGE && (nans >> (p - least / PAGE) & 1);
      if (late) {
        const int64_t page = __builtin_amdgcn_readfirstlane(table[p]);
        if (page < 0 || page >= a.n_pages) continue;
        const int ve = __builtin_amdgcn_readfirstlane(a.vs[page * a.kv_heads + head]);
        if (ve != 255 && ve > seen_unit + UNIT_HI) seen_unit = ve;
        waits |= ve - seen_unit < FAR;
      }
      if (!waits || !__ballot(lim[qb] > p * PAGE)) continue;
      const int64_t ph = (int64_t)table[p] * a.kv_heads + head;  // there: its codes were read
      PageCodes<DH> pc;
      pc.load_keys(a, ph, li, kc);
      pc.load_values(a, ph, li, kc);
      page_step<T, DH>(st[qb], fq[qb], pc, scale2, p * PAGE, lim[qb], len, true, kc, [] {});
    }
    const float us = scale_value(st[qb].unit);
    const int col = c0 + (wave * QB + qb) * 16 + li;
    const float l = st[qb].l;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    if (col >= cols) continue;
    if (a.splits > 1) {
      const int64_t slot = ((int64_t)rh * cols + col) * a.splits + split;
#pragma unroll
      for (int j = 0; j < D::DV; ++j) {
        const int d = j * 16 + kc * 4;
        if ((DH % 16 == 0 || d < DH) && (st[qb].m != -INFINITY || l != 0.f))
          *(floatx4*)(a.part_o + slot * DH + d) = st[qb].acc[j] * inv * us;
      }
      if (kc == 0) a.part_ml[slot * 2] = st[qb].m, a.part_ml[slot * 2 + 1] = l;
      continue;
    }
    T* to = (T*)a.out + (int64_t)row * a.o_row + (int64_t)(col / group) * a.ldo +
            (int64_t)(head * group + col % group) * DH;
#pragma unroll
    for (int j = 0; j < D::DV; ++j) {
      const int d = j * 16 + kc * 4;
      if (DH % 16 && d >= DH) continue;
      struct alignas(8) Quad { T v[4]; } out;
#pragma unroll
      for (int r = 0; r < 4; ++r) out.v[r] = (T)(st[qb].acc[j][r] * inv * us);
      *(Quad*)(to + d) = out;
    }
  }
}

template <typename T, int DH>
hipError_t attn_go(const Kv8AttnArgs& a, hipStream_t s) {
  const int64_t wgs = (int64_t)a.rows * a.kv_heads * a.col_tiles * a.splits;
  const dim3 grid((unsigned)wgs);
  if (a.tall == 0) hipLaunchKernelGGL((attn_kv8_k<T, DH>), grid, dim3(256), 0, s, a);
  else if (a.tall == 1) hipLaunchKernelGGL((attn_kv8_tall_k<T, DH, 1>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((attn_kv8_tall_k<T, DH, 2>), grid, dim3(256), 0, s, a);
  attn_join<T>(a, s);
  return hipGetLastError();
}

template <typename T>
hipError_t attn_launch_t(const Kv8AttnArgs& a, hipStream_t s) {
  switch (a.dh) {
    case 16: return attn_go<T, 16>(a, s);
    case 32: return attn_go<T, 32>(a, s);
    case 40: return attn_go<T, 40>(a, s);
    case 64: return attn_go<T, 64>(a, s);
    case 80: return attn_go<T, 80>(a, s);
    case 128: return attn_go<T, 128>(a, s);
    case 160: return attn_go<T, 160>(a, s);
    default: return hipErrorInvalidValue;
  }
}

bool head_dim_ok(int dh) {
  return dh == 16 || dh == 32 || dh == 40 || dh == 64 || dh == 80 || dh == 128 || dh == 160;
}

}  // namespace
}  // namespace nv

using namespace nv;

extern "C" int32_t nv_op_kv8_append(const void* k, int64_t ldk, int64_t k_row_stride, const void* v,
                                    int64_t ldv, int64_t v_row_stride, int32_t dtype, int32_t rows,
                                    int32_t T, int32_t heads, int32_t dh, void* kp, void* vp,
                                    uint8_t* ks, uint8_t* vs, int64_t n_pages,
                                    const int32_t* table, int32_t table_w, const int32_t* pos,
                                    const int32_t* count, void* stream) {
  clear_error();
  NV_CHECK_ARG(rows >= 0 && rows <= 65535 && T >= 0 && heads >= 1 && heads <= 32767,
               "need 0 <= rows <= 65535, T >= 0 and 1 <= heads <= 32767");
  NV_CHECK_ARG(dtype == NV_F16 || dtype == NV_BF16, "dtype must be NV_F16 or NV_BF16");
  NV_CHECK_ARG(n_pages >= 0 && table_w >= 0, "negative sizes");
  NV_CHECK_ARG(ldk >= 0 && ldv >= 0 && k_row_stride >= 0 && v_row_stride >= 0, "negative strides");
  if (!head_dim_ok(dh)) {
    set_error("dh must be 16, 32, 40, 64, 80, 128 or 160");
    return NV_ERR_UNSUPPORTED;
  }
  if (rows == 0 || T == 0 || n_pages == 0 || table_w == 0) return NV_OK;
  NV_CHECK_ARG(k && v && kp && vp && ks && vs && table && pos, "null pointer argument");
  NV_CHECK_ARG(aligned16(kp) && aligned16(vp), "kp and vp must be 16-byte aligned");
  const Kv8AppendArgs a{k, v, (uint8_t*)kp, (uint8_t*)vp, ks, vs,
                        ldk, k_row_stride, ldv, v_row_stride, n_pages, table, pos, count,
                        T, heads, dh, table_w};
  const bool vec = (ldk | ldv | k_row_stride | v_row_stride) % 8 == 0 && aligned16(k) && aligned16(v);
  const int64_t touched = std::min<int64_t>(((int64_t)T + PAGE - 2) / PAGE + 1, table_w);
  if (touched > 0xFFFFFF) {  // 256 threads each: below 2^32 in all
    set_error("tokens for more than 2^24 - 1 pages of a row");
    return NV_ERR_UNSUPPORTED;
  }
  const dim3 grid((unsigned)touched, heads * 2, rows);
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, (hipStream_t)stream, a);
  };
  const int64_t units = touched * heads * 2 * rows;  // below 2^33
  auto few = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)ceil_div(units, 4)), dim3(256), 0, (hipStream_t)stream,
                       a, units, (int)touched);
  };
  if (T <= KV8_FEW_TOKENS && units <= (1 << 25)) {
    if (dtype == NV_F16) vec ? few(kv8_append_few_k<_Float16, true>) : few(kv8_append_few_k<_Float16, false>);
    else vec ? few(kv8_append_few_k<__bf16, true>) : few(kv8_append_few_k<__bf16, false>);
  } else {
    if (dtype == NV_F16) vec ? go(kv8_append_k<_Float16, true>) : go(kv8_append_k<_Float16, false>);
    else vec ? go(kv8_append_k<__bf16, true>) : go(kv8_append_k<__bf16, false>);
  }
  NV_LAUNCH_CHECK("kv8_append_k");
  return NV_OK;
}

extern "C" size_t nv_op_attention_kv8_workspace(int32_t rows, int32_t S, int32_t heads,
                                                int32_t kv_heads, int32_t dh, int32_t table_w) {
  if (rows < 1 || S < 1 || heads < 1 || kv_heads < 1 || heads % kv_heads || !head_dim_ok(dh) ||
      table_w < 0)
    return 0;
  return part_bytes(kv8_plan(rows, S, heads, kv_heads, dh, table_w), rows, S, heads, dh,
                    nullptr);
}

extern "C" int32_t nv_op_attention_kv8(const void* q, int64_t ldq, int64_t q_row_stride,
                                       int32_t dtype, const void* kp, const void* vp,
                                       const uint8_t* ks, const uint8_t* vs, int64_t n_pages,
                                       const int32_t* table, int32_t table_w, const int32_t* lens,
                                       const int32_t* qpos, int32_t rows, int32_t S, int32_t heads,
                                       int32_t kv_heads, int32_t dh, float scale, void* out,
                                       int64_t ldo, int64_t o_row_stride, void* workspace,
                                       size_t workspace_bytes, void* stream) {
  clear_error();
  NV_CHECK_ARG(rows >= 0 && S >= 0 && heads >= 1 && kv_heads >= 1 && heads % kv_heads == 0,
               "need rows, S >= 0 and heads a positive multiple of kv_heads");
  NV_CHECK_ARG(dtype == NV_F16 || dtype == NV_BF16, "dtype must be NV_F16 or NV_BF16");
  NV_CHECK_ARG(n_pages >= 0 && table_w >= 0 && table_w <= 0x7FFFFFFF / PAGE,
               "need n_pages >= 0 and 0 <= table_w < 2^25");
  NV_CHECK_ARG(scale - scale == 0.f, "scale must be finite");
  if (!head_dim_ok(dh)) {
    set_error("dh must be 16, 32, 40, 64, 80, 128 or 160");
    return NV_ERR_UNSUPPORTED;
  }
  NV_CHECK_ARG(ldq >= 0 && q_row_stride >= 0 && ldo >= (int64_t)heads * dh && o_row_stride >= 0,
               "negative strides, or rows of out shorter than heads * dh");
  if (rows == 0 || S == 0) return NV_OK;
  NV_CHECK_ARG(q && lens && out && (table_w == 0 || table) &&
                   (n_pages == 0 || (kp && vp && ks && vs)), "null pointer argument");
  if ((ldq | q_row_stride | ldo | o_row_stride) % 8 || !aligned16(q) || !aligned16(out)) {
    set_error("q and out need 16-byte aligned buffers and strides in multiples of 8");
    return NV_ERR_UNSUPPORTED;
  }
  NV_CHECK_ARG(aligned16(kp) && aligned16(vp), "kp and vp must be 16-byte aligned");
  const Kv8Plan p = kv8_plan(rows, S, heads, kv_heads, dh, table_w);
  if ((int64_t)S * (heads / kv_heads) > 0x7FFFFFF0 ||
      (double)rows * kv_heads * p.col_tiles * p.splits > 8388607.0) {
    set_error("more queries than a grid holds");
    return NV_ERR_UNSUPPORTED;
  }
  size_t ml_at = 0;
  const size_t need = part_bytes(p, rows, S, heads, dh, &ml_at);
  if (need && (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 255))) {
    set_error("workspace missing, misaligned or smaller than nv_op_attention_kv8_workspace()");
    return NV_ERR_WORKSPACE;
  }
  Kv8AttnArgs a{};
  a.q = q, a.ldq = ldq, a.q_row = q_row_stride;
  a.kp = (const uint8_t*)kp, a.vp = (const uint8_t*)vp, a.ks = ks, a.vs = vs;
  a.n_pages = n_pages, a.table = table, a.table_w = table_w, a.lens = lens, a.qpos = qpos;
  a.rows = rows, a.S = S, a.heads = heads, a.kv_heads = kv_heads, a.dh = dh, a.scale = scale;
  a.out = out, a.ldo = ldo, a.o_row = o_row_stride;
  a.col_tiles = p.col_tiles, a.splits = p.splits, a.tall = p.tall;
  if (need) {
    a.part_o = (float*)workspace;
    a.part_ml = (float*)((uint8_t*)workspace + ml_at);
  }
  const hipStream_t s = (hipStream_t)stream;
  NV_HIP_TRY(dtype == NV_F16 ? attn_launch_t<_Float16>(a, s) : attn_launch_t<__bf16>(a, s));
  return NV_OK;
}
