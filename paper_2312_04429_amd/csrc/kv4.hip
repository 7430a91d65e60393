// Keys and values kept in 4 bits: appending tokens to their pages, reading them back, and attention
// over them.
//
// Page: 64 tokens of one sequence, keys and values alike [head][64][dh / 2] bytes of two e2m1 codes and
// [head][64][ceil(dh / 32)] scale bytes.  A token's codes and scales are bytes of its own, so tokens are
// written in any order and over again without touching others.
#include <algorithm>

#include "common.h"
#include "e2m1.h"
#include "kv4.h"
#include "kv_join.h"

namespace nv {
namespace {

constexpr int PAGE = NV_KV4_PAGE;
constexpr float LOG2E = 1.4426950408889634f;

__host__ __device__ constexpr int blocks_of(int dh) { return (dh + KV4_BLOCK - 1) / KV4_BLOCK; }

// The place of token t of a call's row: unit page * heads + head, times 64, plus the token's slot in the
// page; -1: not held, or not asked for.
template <typename Args>
__device__ __forceinline__ int64_t place_of(const Args& a, int64_t row, int t, int head) {
  const int64_t pos = a.pos[row];
  const int cnt = a.count ? std::min(std::max(a.count[row], 0), a.T) : a.T;
  const int64_t p = (pos + t) / PAGE;
  if (pos < 0 || t >= cnt || p >= a.table_w) return -1;
  const int64_t page = a.table[row * a.table_w + p];
  if (page < 0 || page >= a.n_pages) return -1;
  return (page * a.heads + head) * PAGE + (pos + t) % PAGE;
}

// ------------------------------------------------------------------------------------ append

// Four lanes a block of 32 channels, eight channels of keys and values each; a head's tokens one after
// another, as a page has them, so that a workgroup writes whole lines.  Bound by launch and latency for single
// tokens (64 of 8 heads of 128: 3.4 us), by HBM for prompts (11680 tokens of 8 heads of 128, float16: 60 MB
// in 13.8 us, 4.4 TB/s; with keys and values in workgroups of their own 16.5, with two units a lane 15.1).
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) kv4_append_k(Kv4AppendArgs a) {
  const int64_t row = blockIdx.y;
  const uint32_t nb = blocks_of(a.dh), lanes = nb * 4;  // of a token's head
  const uint32_t id = blockIdx.x * 256u + threadIdx.x, u = id / lanes;  // below 2^32: checked
  const uint32_t head = u / (uint32_t)a.T, t = u - head * a.T, c = (id - u * lanes) * 8;
  const int64_t at = head < (uint32_t)a.heads ? place_of(a, row, (int)t, head) : -1;
  const bool on = at >= 0 && c < (uint32_t)a.dh;
  float x[2][8];
  load8<VEC>((const T*)a.k + row * a.k_row + t * a.ldk + (int64_t)head * a.dh, c, on ? a.dh : 0, x[0]);
  load8<VEC>((const T*)a.v + row * a.v_row + t * a.ldv + (int64_t)head * a.dh, c, on ? a.dh : 0, x[1]);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float top = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = fmaxf(top, abs_or_inf(x[i][j]));
    top = fmaxf(top, dpp_f<0xB1>(top));  // quad_perm [1, 0, 3, 2]
    top = fmaxf(top, dpp_f<0x4E>(top));  // quad_perm [2, 3, 0, 1]
    if (!on) continue;
    const int e = scale_byte4(top);
    *(uint32_t*)((i ? a.vp : a.kp) + at * (a.dh / 2) + c / 2) =
        e == 255 ? 0u : codes4x8(x[i], scale_inverse(e));
    if (c % KV4_BLOCK == 0) (i ? a.vs : a.ks)[at * nb + c / KV4_BLOCK] = (uint8_t)e;
  }
}

// -------------------------------------------------------------------------------------- read

// Units of eight channels from which on a lane takes two at once: their way from a position over the
// table to the tokens is waited for once (8 rows of 8 heads of 128, one unit and two: 512 tokens, 2^19 units,
// 5.4 and 5.6 us; 1024, 8.7 and 8.8; 2048, 14.9 and 14.8; 4096, 38 and 34 with outputs in turn).
constexpr int64_t READ_TWO = 1 << 21;

// Eight channels of a token's keys and values a lane, N times; a token's heads one after another, as the
// output has them.  Bound by HBM's writes: 8 x 4096 tokens of 8 heads of 128 (134 MB out) 34 us with operands
// and outputs in turn (one unit a lane: 37 to 39; a head's tokens one after another: 40).
template <typename T, bool VEC, int N>
__global__ void __launch_bounds__(256) kv4_read_k(Kv4ReadArgs a) {
  const int64_t row = blockIdx.y;
  const uint32_t nb = blocks_of(a.dh), nch = a.dh / 8;
  uint32_t t[N], col[N], w[N][2];
  int e[N][2];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const uint32_t id = (blockIdx.x * N + n) * 256u + threadIdx.x, u = id / nch;  // below 2^32: checked
    t[n] = u / (uint32_t)a.heads;
    const uint32_t head = u - t[n] * a.heads, c = (id - u * nch) * 8;
    col[n] = head * a.dh + c;
    const int64_t at = t[n] < (uint32_t)a.T ? place_of(a, row, (int)t[n], head) : -1;
    w[n][0] = w[n][1] = 0, e[n][0] = e[n][1] = 127;
    if (at >= 0) {
      w[n][0] = *(const uint32_t*)(a.kp + at * (a.dh / 2) + c / 2), e[n][0] = a.ks[at * nb + c / KV4_BLOCK];
      w[n][1] = *(const uint32_t*)(a.vp + at * (a.dh / 2) + c / 2), e[n][1] = a.vs[at * nb + c / KV4_BLOCK];
    }
  }
#pragma unroll
  for (int n = 0; n < N; ++n) {
    if (t[n] >= (uint32_t)a.T) return;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float x[8];
      const float s = scale_value(e[n][i]);
      const half8 v = Half8<_Float16>::of(w[n][i], 1.f);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = (float)v[j] * s;
      T* to = i ? (T*)a.v + row * a.v_row + t[n] * a.ldv : (T*)a.k + row * a.k_row + t[n] * a.ldk;
      store8<VEC>(to, col[n], a.heads * a.dh, x);
    }
  }
}

// --------------------------------------------------------------------------------- attention
//
// S^T = K Q^T is computed, so an accumulator entry's column is a query and the softmax state is a
// lane's own; accumulators of two 16-token tiles are then the second product's operand as they stand,
// against values of the same tokens.

// Head dimension in 32-wide steps, of which lane group kc takes eight channels.  NEAR: those of all steps
// are neighbours (its codes of a token are one load); otherwise a step's 32 are (16-byte units in LDS that
// groups of lanes read at once lie in different banks).
template <int DH>
struct Dims {
  static constexpr int STEPS = (DH + 31) / 32, NB = blocks_of(DH), DV = (DH + 15) / 16;
  template <bool NEAR = true>
  static __device__ __forceinline__ int dim(int step, int kc) {
    return NEAR ? kc * 8 * STEPS + step * 8 : step * 32 + kc * 8;
  }
};

// Pages p0 .. p1 - 1 of share `split` of a tile's pages: equal parts of at least KV8_SHARE pages, so a
// short row's last shares may be empty.
__device__ __forceinline__ void share_of(int pages, int split, int splits, int* p0, int* p1) {
  const int n = std::max(KV8_SHARE, (pages + splits - 1) / splits);
  *p0 = (int)std::min<int64_t>((int64_t)split * n, pages);
  *p1 = std::min(*p0 + n, pages);
}

// One wave's running softmax over 16 queries: reference (probabilities are 2^(score - m)), their sum,
// accumulators O^T.
template <int DH>
struct State {
  float m, l;
  floatx4 acc[Dims<DH>::DV];
};

// Probabilities enter the second product in float16: 2^-11 of themselves is lost, of those that the sum is made
// of too, so that a mean stays one.  One query over 200000 tokens, float16: 2.8e-4 from float64 where a result
// rounded once is 2.1e-4; as sums of two float16 numbers 2.1e-4, for 2 to 10 % of the time.  With
// bfloat16 results it does not show.  The largest probability is at most 2^P_TOP, which float16 holds.
constexpr float P_TOP = 15.f;

// The reference under which a score of `top` has the probability 2^room (room <= P_TOP): top - room, or
// top itself where the scores are so large that this rounds to more than P_TOP below it.
__device__ __forceinline__ float reference(float top, float room) {
#pragma clang fp contract(off)  // top is a rounded product, and has to be the same one in both lines
  const float low = top - room;
  return top - low > P_TOP ? top : low;
}

// x as the sum of two bfloat16 numbers: 16 bits of it, and float16 exactly.
__device__ __forceinline__ void split_bf16(float x, __bf16* hi, __bf16* lo) {
  *hi = (__bf16)x;
  const float d = x - (float)*hi;
  *lo = (__bf16)(d - d == 0.f ? d : 0.f);  // not finite: all of it is in hi
}

// A page's 64 tokens into the state, whatever is in it: bfloat16 operands, which hold every code times
// every scale; float16 queries, and probabilities, as sums of two.  Everything comes from global memory
// as it is needed.  j0: the page's first token; lim: tokens this lane's query sees; len: tokens of
// the sequence.  A NaN block of values reaches the queries that see its token, in its 32 channels.
// Written for few registers, not speed: where every page goes this way one query over 200000 tokens takes
// 498 us for 43, 2 x 2048 queries over 4096 3900 for 140; with one such page a row 77 and 303.
template <typename T, int DH, bool NEAR>
__device__ __forceinline__ void page_any(State<DH>& st, const typename Half8<T>::Vec* fq,
                                         const Kv4AttnArgs& a, int64_t ph, float scale2, int j0,
                                         int lim, int len, int li, int kc) {
  using D = Dims<DH>;
  using B = Half8<__bf16>;
  // Nothing of this is to be computed ahead of a loop over pages and kept in registers there.
  asm volatile("" : "+v"(li), "+v"(kc));
  const uint8_t *kp = a.kp + ph * PAGE * (DH / 2), *ks = a.ks + ph * PAGE * D::NB;
  const uint8_t *vp = a.vp + ph * PAGE * (DH / 2), *vs = a.vs + ph * PAGE * D::NB;
  floatx4 s[4];
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    s[t] = floatx4{0.f, 0.f, 0.f, 0.f};
    const int tok = 16 * t + li;
#pragma unroll
    for (int b = 0; b < D::STEPS; ++b) {
      const int d = D::template dim<NEAR>(b, kc);
      bf16x8 k = {}, qh, ql;
      auto fb = fq[b];
      asm volatile("" : "+v"(fb));
      if (d < DH) {
        const int e = ks[tok * D::NB + d / KV4_BLOCK];
        k = B::of(*(const uint32_t*)(kp + (tok * DH + d) / 2), scale_value(e == 255 ? 127 : e));
        if (e == 255) k = __builtin_bit_cast(bf16x8, u32x4{0x7FC07FC0, 0x7FC07FC0, 0x7FC07FC0, 0x7FC07FC0});
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        __bf16 hi, lo;
        split_bf16((float)fb[i], &hi, &lo);
        qh[i] = hi, ql[i] = lo;
      }
      s[t] = B::mul(k, qh, s[t]);
      if (std::is_same<T, _Float16>::value) s[t] = B::mul(k, ql, s[t]);
      __builtin_amdgcn_sched_barrier(0);  // few registers, not speed: this is the rare way
    }
  }
  float top = -INFINITY;
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      s[t][r] *= scale2;
      if (j0 + 16 * t + 4 * kc + r >= lim) s[t][r] = -INFINITY;
      top = fmaxf(top, s[t][r]);
    }
  const float mnew = fmaxf(st.m, reference(rows_max(top), P_TOP)), base = mnew == -INFINITY ? 0.f : mnew;
  const float alpha = __builtin_amdgcn_exp2f(st.m - base);
  st.m = mnew;
  // The larger codes of scales 253 and 254 are 2^128 and more, infinite in bfloat16, and would reach queries
  // that do not see their token (0 * infinity): with such a scale the page's values count as eighths,
  // its probabilities eightfold.
  bool wide = false;
#pragma unroll
  for (int b = 0; b < D::NB; ++b) {
    const int tok = 16 * kc + li;
    wide |= j0 + tok < len && (unsigned)(vs[tok * D::NB + b] - 253) <= 1u;
  }
  const bool eighths = __ballot(wide);
  const int less = eighths ? 3 : 0;
  const float times = eighths ? 8.f : 1.f;
  float sum = 0.f;
  bf16x8 ph8[2], pl8[2];
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float p = __builtin_amdgcn_exp2f(s[t][r] - base) * times;
      __bf16 hi, lo;
      split_bf16(p, &hi, &lo);
      ph8[t >> 1][(t & 1) * 4 + r] = hi, pl8[t >> 1][(t & 1) * 4 + r] = lo;
      sum += (float)hi + (float)lo;
    }
  st.l = st.l * alpha + rows_sum(sum) / times;
  float nan[D::NB];
#pragma unroll
  for (int b = 0; b < D::NB; ++b) {
    nan[b] = 0.f;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int tok = 16 * t + 4 * kc + r;
        if (j0 + tok < lim && vs[tok * D::NB + b] == 255) nan[b] = 1.f;
      }
    nan[b] = rows_max(nan[b]);
    __builtin_amdgcn_sched_barrier(0);
  }
#pragma unroll
  for (int j = 0; j < D::DV; ++j) {
    const int c = 16 * j + li;
    st.acc[j] *= alpha;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      bf16x8 v;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int tok = 32 * h + 4 * kc + (i < 4 ? i : i + 12);
        v[i] = (__bf16)0.f;
        if (j0 + tok < len && c < DH) {
          const int e = vs[tok * D::NB + c / KV4_BLOCK] - less;
          const uint32_t w = vp[(tok * DH + c) / 2];
          const bf16x2 two = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale_value(e), 0);
          if ((unsigned)e < 255u - less) v[i] = two[c & 1];
        }
      }
      st.acc[j] = B::mul(v, ph8[h], st.acc[j]);
      st.acc[j] = B::mul(v, pl8[h], st.acc[j]);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (nan[j / 2] != 0.f)
#pragma unroll
      for (int r = 0; r < 4; ++r) st.acc[j][r] = __int_as_float(0x7FC00000);
  }
}

// What the kernels below read a page in: units of CW channels of a token, UPT of them a token, for keys
// and values alike.
template <int DH>
struct Units {
  static constexpr int CW = DH % 32 == 0 ? 32 : DH % 16 == 0 ? 16 : 8, UPT = DH / CW, N = PAGE * UPT;
  struct Codes { uint32_t w[CW / 8]; };
  static __device__ __forceinline__ Codes load(const uint8_t* codes, int i) {
    Codes c;
    __builtin_memcpy(&c, __builtin_assume_aligned(codes + i * (CW / 2), CW / 2), CW / 2);
    return c;
  }
  static __device__ __forceinline__ int scale(const uint8_t* scales, int i) {
    return scales[i / UPT * blocks_of(DH) + i % UPT * CW / KV4_BLOCK];
  }
};

// Scale bytes whose codes a 16-bit type holds exactly (a block of zeros does with any but 255, but is
// not asked for here: its codes are).
template <typename T>
__device__ __forceinline__ bool exact(int e) {
  return std::is_same<T, _Float16>::value ? (unsigned)(e - 104) <= 36u : (unsigned)(e - 1) <= 253u;
}
template <typename T, int DH>
__device__ __forceinline__ bool exact(int e, const typename Units<DH>::Codes& c) {
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < Units<DH>::CW / 8; ++i) any |= c.w[i];
  return exact<T>(e) | ((e != 255) & ((any & 0x77777777u) == 0));
}
__device__ __forceinline__ float scale_bits(int e) { return __int_as_float(e << 23); }

// A page's values in LDS, token after token in float16; a row is an odd number of 32-byte steps, so that
// the 16 rows of a transposed read lie in different banks.
template <int DH>
struct Values {
  static constexpr int ROW = (Dims<DH>::DV | 1) == Dims<DH>::DV ? (Dims<DH>::DV + 2) * 16
                                                                 : (Dims<DH>::DV + 1) * 16;
  static __device__ __forceinline__ void store(_Float16* to, int i, const typename Units<DH>::Codes& c,
                                               float scale) {
    using U = Units<DH>;
    to += i / U::UPT * ROW + i % U::UPT * U::CW;
#pragma unroll
    for (int k = 0; k < U::CW / 8; ++k) *(half8*)(to + k * 8) = Half8<_Float16>::of(c.w[k], scale);
  }
  // Channels 16 j + li of tokens 32 h + 4 kc .. + 3 and 16 further: four rows of 16 channels a lane
  // group, turned on their way (ds_read_b64_tr_b16).
  static __device__ __forceinline__ half8 load(const _Float16* v, int j, int h, int li, int kc) {
    typedef __attribute__((ext_vector_type(4))) short Short4;
    typedef __attribute__((address_space(3))) Short4* Lds;
    const _Float16* p = v + (32 * h + 4 * kc + (li >> 2)) * ROW + 16 * j + (li & 3) * 4;
    const Short4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)p),
                 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(p + 16 * ROW));
    return __builtin_bit_cast(half8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
  }
};

// Sums over the 64 keys of a page out of the matrix unit, of the probabilities as rounded: a row of ones.
__device__ __forceinline__ floatx4 add_probs(const half8* fp, floatx4 sum) {
  half8 ones;
#pragma unroll
  for (int i = 0; i < 8; ++i) ones[i] = (_Float16)1.f;
  return Half8<_Float16>::mul(ones, fp[1], Half8<_Float16>::mul(ones, fp[0], sum));
}

// A lane's part of a page of one head: codes of keys 16 t + li, channels 8 STEPS kc .., and units of
// values, with their scales.
template <int DH>
struct PageCodes {
  using D = Dims<DH>;
  using U = Units<DH>;
  static constexpr bool ONE = 32 % (8 * D::STEPS) == 0;  // a lane's keys have one scale
  static constexpr int KE = ONE ? 1 : D::STEPS, VU = (U::N + 63) / 64;
  struct Key { uint32_t w[D::STEPS]; };
  Key k[4];
  typename U::Codes v[VU];
  int ke[4][KE], ve[VU];
  __device__ __forceinline__ void load_keys(const Kv4AttnArgs& a, int64_t ph, int li, int kc) {
    const uint8_t *kp = a.kp + ph * PAGE * (DH / 2) + li * (DH / 2) + kc * 4 * D::STEPS,
                  *ks = a.ks + ph * PAGE * D::NB + li * D::NB;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      if (DH % 32 == 0) {
        __builtin_memcpy(&k[t], __builtin_assume_aligned(kp + t * 16 * (DH / 2), 4), sizeof(Key));
      } else {
#pragma unroll
        for (int b = 0; b < D::STEPS; ++b)
          k[t].w[b] = D::dim(b, kc) < DH ? *(const uint32_t*)(kp + t * 16 * (DH / 2) + b * 4) : 0u;
      }
#pragma unroll
      for (int b = 0; b < KE; ++b)
        ke[t][b] = D::dim(b, kc) < DH ? ks[t * 16 * D::NB + D::dim(b, kc) / KV4_BLOCK] : 127;
    }
  }
  __device__ __forceinline__ void load_values(const Kv4AttnArgs& a, int64_t ph, int lane) {
    const uint8_t *vp = a.vp + ph * PAGE * (DH / 2), *vs = a.vs + ph * PAGE * D::NB;
#pragma unroll
    for (int i = 0; i < VU; ++i) {
      v[i] = U::load(vp, i * 64 + lane);
      ve[i] = U::scale(vs, i * 64 + lane);
    }
  }
  // Scales of tokens from n on become 1: what is there may be anything.
  __device__ __forceinline__ void cut(int n, int lane, int li) {
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int b = 0; b < KE; ++b)
        if (16 * t + li >= n) ke[t][b] = 127;
#pragma unroll
    for (int i = 0; i < VU; ++i)
      if ((i * 64 + lane) / U::UPT >= n) ve[i] = 127;
  }
  // Whether 16-bit operands hold all of it.
  template <typename T>
  __device__ __forceinline__ bool exact16() const {
    bool ok = true;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int b = 0; b < KE; ++b) ok &= exact<T>(ke[t][b]);
#pragma unroll
    for (int i = 0; i < VU; ++i) ok &= exact<_Float16>(ve[i]);
    if (!__ballot(!ok)) return true;
    ok = true;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int b = 0; b < D::STEPS; ++b) {
        const int e = ke[t][ONE ? 0 : b];
        ok &= exact<T>(e) || (e != 255 && (k[t].w[b] & 0x77777777u) == 0);
      }
#pragma unroll
    for (int i = 0; i < VU; ++i) ok &= exact<_Float16, DH>(ve[i], v[i]);
    return !__ballot(!ok);
  }
};

// A page's 64 tokens into the state, in 16-bit operands that hold them.  lim: tokens this lane's query
// sees; some: whether some query sees only part of the page.  keys_done and values_done run once the
// keys' and the values' registers are free again.
template <typename T, int DH, typename KeysDone, typename ValuesDone>
__device__ __forceinline__ void page_step(State<DH>& st, const typename Half8<T>::Vec* fq,
                                          PageCodes<DH>& pc, _Float16* lds, float scale2, int j0,
                                          int lim, bool some, int lane, int li, int kc,
                                          KeysDone&& keys_done, ValuesDone&& values_done) {
  using D = Dims<DH>;
  using M = Half8<T>;
  using PC = PageCodes<DH>;
  floatx4 s[4];
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    s[t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int b = 0; b < D::STEPS; ++b)
      s[t] = M::mul(M::of(pc.k[t].w[b], scale_bits(pc.ke[t][PC::ONE ? 0 : b])), fq[b], s[t]);
  }
  keys_done();
#pragma unroll
  for (int i = 0; i < PC::VU; ++i) Values<DH>::store(lds, i * 64 + lane, pc.v[i], scale_bits(pc.ve[i]));
  values_done();
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // a wave's LDS is its own
  float top = -INFINITY;
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      top = fmaxf(top, s[t][r]);
    }
  if (some) {  // uniform
    top = -INFINITY;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        if (j0 + 16 * t + 4 * kc + r >= lim) s[t][r] = -INFINITY;
        top = fmaxf(top, s[t][r]);
      }
  }
  // Scores are multiplied by the scale inside the exponent, where the product is not rounded, and measured
  // against the reference in the same way.  It moves only when a probability would pass 2^P_TOP.  A new one
  // comes from rounded products: from 2^23 on those differ by 1/2 and more from the others (2^29: by 32, past
  // float16 either way), so this page's scores are rounded, too (below, the largest probability is 2^(P_TOP +
  // 1/4)); a later page's that pass P_TOP without being rounded come back here.
  float rest = scale2;
  if (__ballot(fmaf(rows_max(top), scale2, -st.m) > P_TOP)) {  // at the start: infinite
    const float largest = rows_max(top * scale2), size = fabsf(largest);
    const float mnew = fmaxf(st.m, reference(largest, P_TOP));
    const float alpha = __builtin_amdgcn_exp2f(st.m - (mnew == -INFINITY ? 0.f : mnew));
#pragma unroll
    for (int j = 0; j < D::DV; ++j) st.acc[j] *= alpha;
    st.l *= alpha;
    st.m = mnew;
    if (__ballot(size >= 0x1p23f && size < INFINITY)) {
#pragma unroll
      for (int t = 0; t < 4; ++t) s[t] *= scale2;
      rest = 1.f;
    }
  }
  const float base = st.m == -INFINITY ? 0.f : st.m;
  half8 fp[2];
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      fp[t >> 1][(t & 1) * 4 + r] = (_Float16)__builtin_amdgcn_exp2f(fmaf(s[t][r], rest, -base));
  st.l += add_probs(fp, floatx4{0.f, 0.f, 0.f, 0.f})[0];
#pragma unroll
  for (int j = 0; j < D::DV; ++j)
#pragma unroll
    for (int h = 0; h < 2; ++h)
      st.acc[j] = Half8<_Float16>::mul(Values<DH>::load(lds, j, h, li, kc), fp[h], st.acc[j]);
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// A workgroup takes 16 queries of one row and kv head (query heads of the group innermost) and
// share of the row's pages, dealt out to its four waves; their states meet in LDS.  With more
// than one share the means go to the workspace and attn_join_k adds them in order.  Keys are converted
// from registers into the first product's operand; values pass through a wave's own LDS, where they are
// turned.  Bound by HBM and its latency: one query over 200000 tokens, 8 heads of 128, 44 us (217 MB, 4.9
// TB/s) with two waves a SIMD, 60 with one; a page costs a wave 330 vector instructions, 128 of them
// conversions.  32 rows of 2048 to 8192 tokens: 44 us, the longest rows' tail.
template <typename T, int DH>
__global__ void __launch_bounds__(256) attn_kv4_k(Kv4AttnArgs a) {
  using D = Dims<DH>;
  typedef typename Half8<T>::Vec Vec;
  constexpr int NW = 4, CH = D::DV * 16;
  constexpr int VALS = PAGE * Values<DH>::ROW * 2, OUT = 16 * (CH + 4) * 4;  // bytes of a wave
  __shared__ float sm[NW][16], sl[NW][16];
  __shared__ __align__(16) char lds[NW * (VALS > OUT ? VALS : OUT)];
  float(*so)[16][CH + 4] = (float(*)[16][CH + 4])lds;  // once no wave reads values any more
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
    // the scale's sign to the queries, so that the largest product is the largest score
#pragma unroll
    for (int i = 0; i < 8; ++i)
      fq[b][i] = a.scale > 0.f ? fq[b][i] : a.scale < 0.f ? -fq[b][i] : fq[b][i] * (T)0.f;
  }
  State<DH> st;
  st.m = -INFINITY, st.l = 0.f;
#pragma unroll
  for (int j = 0; j < D::DV; ++j) st.acc[j] = floatx4{0.f, 0.f, 0.f, 0.f};
  const float scale2 = a.scale == 0.f ? 1.f : fabsf(a.scale) * LOG2E;
  // The next page's keys are requested as soon as this one's are multiplied, its values once this one's
  // are in LDS, into the same registers; its table entry was read a page earlier.
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
  _Float16* vals = (_Float16*)(lds + wave * VALS);
  PageCodes<DH> pc;
  int p = 0;
  int64_t ph = take(p);
  if (ph >= 0) pc.load_keys(a, ph, li, kc), pc.load_values(a, ph, lane);
  bool late = false;  // some page waits
  while (ph >= 0) {
    const int j0 = p * PAGE;
    const int64_t next = take(p);
    auto keys = [&] { if (next >= 0) pc.load_keys(a, next, li, kc); };
    auto values = [&] { if (next >= 0) pc.load_values(a, next, lane); };
    if (j0 + PAGE > len) pc.cut(len - j0, lane, li);
    if (pc.template exact16<T>()) {
      page_step<T, DH>(st, fq, pc, vals, scale2, j0, lim, j0 + PAGE > least, lane, li, kc, keys, values);
    } else {
      late = true;
      keys(), values();
    }
    ph = next;
  }
  // Pages that 16 bits do not hold, or with a NaN: the same rule tells which they are.  (In the loop above
  // their code would cost the others a tenth in copies of registers.)
  for (pn = p0 + wave; late && pn < p1; pn += NW) {
    const int64_t page = __builtin_amdgcn_readfirstlane(table[pn]);
    if (page < 0 || page >= a.n_pages) continue;
    const int j0 = pn * PAGE;
    pc.load_keys(a, page * a.kv_heads + head, li, kc);
    pc.load_values(a, page * a.kv_heads + head, lane);
    pc.cut(len - j0, lane, li);
    if (!pc.template exact16<T>())
      page_any<T, DH, true>(st, fq, a, page * a.kv_heads + head, scale2, j0, lim, len, li, kc);
  }
  __syncthreads();
  // The waves' states, in wave order: means, which are no larger than the values, and their weights (a
  // sum in its final size may pass float32 where the mean does not).
  const float l = st.l, mean = l == 0.f ? 0.f : 1.f / l;
  if (kc == 0) sm[wave][li] = st.m, sl[wave][li] = l;
#pragma unroll
  for (int j = 0; j < D::DV; ++j) *(floatx4*)&so[wave][li][j * 16 + kc * 4] = st.acc[j] * mean;
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

// Many queries of a head: NW waves of QB * 16 queries share every page.  A page's codes come two
// pages ahead into registers and are converted once, on their way into a double-buffered LDS
// (16-bit: the products then read operands as they stand, values turned).  A page that not every query
// sees whole has its scores masked; one that 16 bits do not hold (or with a NaN) waits until the loop is
// over and goes through page_any.
// 2 x 2048 queries, 16 heads of 128 on 4, over 4096 tokens: 138 us (1000 TFLOP/s, where a large library
// product reaches 1290); behind 2048 of them under a causal limit 115, from an empty cache 54.  Per SIMD the
// matrix unit is busy 42 % of the time and the vector unit 42 %; what is not exponentials runs beside products
// only in part.  Left out one at a time: conversion and LDS writes -29 us, the products -27 and -22, key reads
// -17, scores' arithmetic -9, exponentials and value reads -7 each.
template <typename T, int DH, int NW, int QB>
__global__ void __launch_bounds__(NW * 64, 2) attn_kv4_tall_k(Kv4AttnArgs a) {
  using D = Dims<DH>;
  using M = Half8<T>;
  typedef typename M::Vec Vec;
  using V = Half8<_Float16>;
  using U = Units<DH>;
  constexpr int NT = NW * 64, COLS = NW * QB * 16;
  constexpr int UPL = (2 * U::N + NT - 1) / NT;  // units of keys, then of values, a lane
  constexpr int KROW = D::STEPS * 32 + 16, VSIZE = PAGE * Values<DH>::ROW;
  __shared__ __align__(16) T sk[2][PAGE * KROW];
  __shared__ __align__(16) _Float16 sv[2][VSIZE];
  __shared__ int waits[4];  // [n & 3]: n + 1 if the n-th page waits
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, kc = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rh = blockIdx.x % (a.rows * a.kv_heads);  // a multiple of 8: one XCD's L2 for a head
  const int rest = blockIdx.x / (a.rows * a.kv_heads), split = rest / a.col_tiles;
  // Longest first, where not all are resident at once (two a compute unit; one past 128 channels, where the
  // pairing below is without effect); where they are, a compute unit's second workgroup is as short as its
  // first is long (a causal limit from 2048 of 4096 tokens: 126 -> 117 us).
  const int nth = rest % a.col_tiles, half = (a.col_tiles + 1) / 2;
  const int ct = nth < half || gridDim.x > 512 ? a.col_tiles - 1 - nth : nth - half;
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
  float sum[QB];
  int lim[QB];
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    const int col = std::min(c0 + (wave * QB + qb) * 16 + li, cols - 1);
    lim[qb] = sees(col);
    const T* qrow = (const T*)a.q + (int64_t)row * a.q_row + (int64_t)(col / group) * a.ldq +
                    (int64_t)(head * group + col % group) * DH;
#pragma unroll
    for (int b = 0; b < D::STEPS; ++b) {
      const int d = D::template dim<false>(b, kc);
      fq[qb][b] = d < DH ? *(const Vec*)(qrow + d) : Vec{};
    }
    st[qb].m = -INFINITY, sum[qb] = 0.f;
#pragma unroll
    for (int j = 0; j < D::DV; ++j) st[qb].acc[j] = floatx4{0.f, 0.f, 0.f, 0.f};
  }

  // The pages in turn, ph < 0: none left.  A page's table entry was read when the one before it was
  // taken: its address does not wait for memory.
  struct Page { int64_t ph; int p; };
  int pnext, pages;  // the next page of this share, and its end
  share_of((sees(c0 + COLS - 1) + PAGE - 1) / PAGE, split, a.splits, &pnext, &pages);
  const int first = pnext;
  const int wave_least = sees(c0 + wave * QB * 16);
  int entry = pnext < pages ? table[pnext] : 0;
  auto take = [&] {
    Page p{-1, 0};
    while (pnext < pages) {
      const int64_t page = __builtin_amdgcn_readfirstlane(entry);
      p.p = pnext++;
      if (pnext < pages) entry = table[pnext];
      if (page < 0 || page >= a.n_pages) continue;
      p.ph = page * a.kv_heads + head;
      break;
    }
    return p;
  };
  struct Coded {
    typename U::Codes w;
    int e;
  };
  Coded code[UPL] = {};
  auto is_value = [&](int i) {  // the same in all lanes of a wave
    return U::N % NT == 0 ? i * NT >= U::N : __builtin_amdgcn_readfirstlane(i * NT + tid) >= U::N;
  };
  auto in_page = [&](int i) { return 2 * U::N % NT == 0 || i * NT + tid < 2 * U::N; };
  auto fetch = [&](Coded (&code)[UPL], const Page& pk, const Page& pv) {  // a page's keys, another's values
#pragma unroll
    for (int i = 0; i < UPL; ++i) {
      const bool is_v = is_value(i);
      const int64_t ph = is_v ? pv.ph : pk.ph;
      if (ph < 0 || !in_page(i)) continue;
      const int n = i * NT + tid - (is_v ? U::N : 0);
      code[i].w = U::load((is_v ? a.vp : a.kp) + ph * PAGE * (DH / 2), n);
      code[i].e = U::scale((is_v ? a.vs : a.ks) + ph * PAGE * D::NB, n);
    }
  };
  // The i-th unit into LDS, as 16-bit values.  What they do not hold is zeros there, and its page, the
  // n-th, waits.
  bool bad_k = false, bad_v = false;
  auto stash = [&](const Coded& c, int i, const Page& pk, const Page& pv, int bk, int bv) {
    const bool is_v = is_value(i);
    if (!in_page(i)) return;
    const int u = i * NT + tid - (is_v ? U::N : 0), tok = u / U::UPT;
    // what is behind the sequence may be anything
    const int e = (is_v ? pv.p : pk.p) * PAGE + tok < len ? c.e : 127;
    const bool ok = is_v ? exact<_Float16, DH>(e, c.w) : exact<T, DH>(e, c.w);
    const float f = ok ? scale_bits(e) : 0.f;
    if (is_v) {
      bad_v |= !ok;
      Values<DH>::store(sv[bv], u, c.w, f);
    } else {
      bad_k |= !ok;
      T* to = sk[bk] + tok * KROW + u % U::UPT * U::CW;
#pragma unroll
      for (int k = 0; k < U::CW / 8; ++k) *(Vec*)(to + k * 8) = M::of(c.w.w[k], f);
    }
  };
  auto stashed = [&](int nk, int nv) {
    if (bad_k) waits[nk & 3] = nk + 1;
    if (bad_v) waits[nv & 3] = nv + 1;
    bad_k = bad_v = false;
  };
  auto stash_all = [&](const Coded (&code)[UPL], const Page& p, int n) {
#pragma unroll
    for (int i = 0; i < UPL; ++i) stash(code[i], i, p, p, n, n);
    stashed(n, n);
  };

  // S = Q K^T, 16 keys at a time
  Vec fk[2][D::STEPS];
  auto load_keys = [&](int buf, int t) {
#pragma unroll
    for (int b = 0; b < D::STEPS; ++b) {
      const int d = D::template dim<false>(b, kc);  // past dh: the row's first channels against zeros
      fk[t & 1][b] = *(const Vec*)(sk[buf] + (t * 16 + li) * KROW + (d < DH ? d : 0));
    }
  };
  auto score = [&](floatx4 (&s)[QB][4], int t) {
#pragma unroll
    for (int b = 0; b < D::STEPS; ++b)
#pragma unroll
      for (int qb = 0; qb < QB; ++qb)
        s[qb][t] = M::mul(fk[t & 1][b], fq[qb][b], b ? s[qb][t] : floatx4{0.f, 0.f, 0.f, 0.f});
  };
  // Scores relative to the query's reference, and the largest of a lane's.
  float top[QB];
  auto relate = [&](floatx4 (&s)[QB][4], int tile) {
    const int qb = tile / 4, t = tile % 4;
    const float base = st[qb].m == -INFINITY ? 0.f : st[qb].m;
    if (t == 0) top[qb] = -INFINITY;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      s[qb][t][r] = fmaf(s[qb][t][r], scale2, -base);
      top[qb] = fmaxf(top[qb], s[qb][t][r]);
    }
  };
  bool late = false;  // some page waits
  // Masks, and the reference.  It moves only when a probability would pass 2^P_TOP, and then to where the
  // largest is 2^LOW: low enough that few pages move it, high enough for what is small beside it.
  auto settle = [&](floatx4 (&s)[QB][4], const Page& cur, int n) {
    constexpr float LOW = 9.f;
    const int j0 = cur.p * PAGE;
    const bool wait = __builtin_amdgcn_readfirstlane(waits[n & 3]) == n + 1;
    late |= wait;
    if (wait || j0 + PAGE > wave_least) {  // uniform
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        const int sees_of = wait ? 0 : lim[qb] - j0 - 4 * kc;
        top[qb] = -INFINITY;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            if (16 * t + r >= sees_of) s[qb][t][r] = -INFINITY;
            top[qb] = fmaxf(top[qb], s[qb][t][r]);
          }
      }
    }
    bool grow = false;
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) grow |= !(top[qb] <= P_TOP) || st[qb].m == -INFINITY;
    if (__ballot(grow)) {
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        const float most = rows_max(top[qb]);
        const bool fresh = st[qb].m == -INFINITY;
        const float low = reference(most, LOW);
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
  };
  half8 fp[QB][2];
  auto probs = [&](const floatx4 (&s)[QB][4], int t) {
#pragma unroll
    for (int qb = 0; qb < QB; ++qb)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        fp[qb][t >> 1][(t & 1) * 4 + r] = (_Float16)__builtin_amdgcn_exp2f(s[qb][t][r]);
  };
  half8 fv[2][2];
  auto load_values = [&](int buf, int j) {
#pragma unroll
    for (int h = 0; h < 2; ++h) fv[j & 1][h] = Values<DH>::load(sv[buf], j, h, li, kc);
  };
  auto add_values = [&](int j) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) st[qb].acc[j] = V::mul(fv[j & 1][h], fp[qb][h], st[qb].acc[j]);
  };

  // Page n in step n.  Its keys were multiplied in the step before; in this one its exponentials run
  // beside the product of page n + 1's keys, whose scores take their place, and the values' product beside
  // those scores' arithmetic and the conversion of page n + 2's keys and n + 1's values, whose codes came
  // a step ahead.  Page n's values are in sv[n & 1], page n + 1's keys in sk[n + 1 & 1]; what is written
  // was read in the step before.  Within a step the order is kept (left to itself the compiler requests
  // every operand at the start, and spills): the operands of the next 16 keys or channels are on their way
  // during these products.
  Page p0 = take();
  if (tid < 4) waits[tid] = 0;
  if (p0.ph >= 0) {
    Page p1 = take(), p2 = take();
    floatx4 s[QB][4];
    Coded second[UPL] = {};
    fetch(code, p0, p0), fetch(second, p1, p1);
    __syncthreads();  // waits
    stash_all(code, p0, 0);
    stash_all(second, p1, 1);  // page 1's values once more in step 0
    fetch(code, p2, p1);
    __syncthreads();
#pragma unroll
    for (int t = 0; t < 4; ++t) load_keys(0, t), score(s, t);
#pragma unroll
    for (int i = 0; i < QB * 4; ++i) relate(s, i);
    __syncthreads();
    int n = 0;
    while (p1.ph >= 0) {
      const int now = n & 1;
      load_keys(now ^ 1, 0);
      settle(s, p0, n);
      probs(s, 0);
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        if (t < 3) load_keys(now ^ 1, t + 1);
        else load_values(now, 0);
        score(s, t);
        if (t < 3) probs(s, t + 1);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) sum[qb] += add_probs(fp[qb], floatx4{0.f, 0.f, 0.f, 0.f})[0];
#pragma unroll
      for (int j = 0; j < D::DV; ++j) {
        if (j + 1 < D::DV) load_values(now, j + 1);
        add_values(j);
#pragma unroll
        for (int i = j * QB * 4 / D::DV; i < (j + 1) * QB * 4 / D::DV; ++i) relate(s, i);
        if (j < UPL) stash(code[j], j, p2, p1, now, now ^ 1);
        __builtin_amdgcn_sched_barrier(0);
      }
      stashed(n + 2, n + 1);
      p0 = p1, p1 = p2, p2 = take(), ++n;
      fetch(code, p2, p1);
      __syncthreads();
    }
    settle(s, p0, n);
#pragma unroll
    for (int t = 0; t < 4; ++t) probs(s, t);
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) sum[qb] += add_probs(fp[qb], floatx4{0.f, 0.f, 0.f, 0.f})[0];
#pragma unroll
    for (int j = 0; j < D::DV; ++j) load_values(n & 1, j), add_values(j);
  }
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) st[qb].l = sum[qb];
  // The pages that wait: the same rule tells which they are.
  for (int p = first; late && p < pages; ++p) {
    const int64_t page = __builtin_amdgcn_readfirstlane(table[p]);
    if (page < 0 || page >= a.n_pages) continue;
    const int64_t ph = page * a.kv_heads + head;
    bool wait = false;
    for (int i = lane; i < 2 * U::N; i += 64) {
      const bool is_v = i >= U::N;
      const int n = is_v ? i - U::N : i;
      if (p * PAGE + n / U::UPT >= len) continue;
      const auto c = U::load((is_v ? a.vp : a.kp) + ph * PAGE * (DH / 2), n);
      const int e = U::scale((is_v ? a.vs : a.ks) + ph * PAGE * D::NB, n);
      wait |= is_v ? !exact<_Float16, DH>(e, c) : !exact<T, DH>(e, c);
    }
    if (!__ballot(wait)) continue;
    auto take_in = [&](auto n) {  // (a loop of two would be kept, its state in memory)
      constexpr int qb = decltype(n)::value;
      if (__ballot(lim[qb] > p * PAGE))
        page_any<T, DH, false>(st[qb], fq[qb], a, ph, scale2, p * PAGE, lim[qb], len, li, kc);
    };
    take_in(std::integral_constant<int, 0>());
    if constexpr (QB > 1) take_in(std::integral_constant<int, 1>());
  }
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
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
          *(floatx4*)(a.part_o + slot * DH + d) = st[qb].acc[j] * inv;
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
      for (int r = 0; r < 4; ++r) out.v[r] = (T)(st[qb].acc[j][r] * inv);
      *(Quad*)(to + d) = out;
    }
  }
}

template <typename T, int DH>
hipError_t attn_go(const Kv4AttnArgs& a, hipStream_t s) {
  const int64_t wgs = (int64_t)a.rows * a.kv_heads * a.col_tiles * a.splits;
  const dim3 grid((unsigned)wgs);
  if (a.tall == 0) hipLaunchKernelGGL((attn_kv4_k<T, DH>), grid, dim3(256), 0, s, a);
  else if (a.tall == 1) hipLaunchKernelGGL((attn_kv4_tall_k<T, DH, 4, 1>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((attn_kv4_tall_k<T, DH, 4, 2>), grid, dim3(256), 0, s, a);
  attn_join<T>(a, s);
  return hipGetLastError();
}

template <typename T>
hipError_t attn_launch_t(const Kv4AttnArgs& a, hipStream_t s) {
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

// What append and read check alike.  NV_OK, or the error that is set.
int32_t check_tokens(int32_t dtype, bool f32, int32_t rows, int32_t T, int32_t heads, int32_t dh,
                     int64_t n_pages, int32_t table_w, int64_t ldk, int64_t k_row, int64_t ldv,
                     int64_t v_row, int64_t lanes) {
  NV_CHECK_ARG(rows >= 0 && rows <= 65535 && T >= 0 && heads >= 1 && heads <= 32767,
               "need 0 <= rows <= 65535, T >= 0 and 1 <= heads <= 32767");
  NV_CHECK_ARG(dtype == NV_F16 || dtype == NV_BF16 || (f32 && dtype == NV_F32),
               f32 ? "dtype must be NV_F32, NV_F16 or NV_BF16" : "dtype must be NV_F16 or NV_BF16");
  NV_CHECK_ARG(n_pages >= 0 && table_w >= 0, "negative sizes");
  NV_CHECK_ARG(ldk >= 0 && ldv >= 0 && k_row >= 0 && v_row >= 0, "negative strides");
  if (!head_dim_ok(dh)) {
    set_error("dh must be 16, 32, 40, 64, 80, 128 or 160");
    return NV_ERR_UNSUPPORTED;
  }
  if ((int64_t)T * heads * lanes > 0xFFFFFE00ll) {  // threads of a grid's first dimension
    set_error("more tokens of a row than a grid holds");
    return NV_ERR_UNSUPPORTED;
  }
  return NV_OK;
}

}  // namespace
}  // namespace nv

using namespace nv;

extern "C" int32_t nv_op_kv4_append(const void* k, int64_t ldk, int64_t k_row_stride, const void* v,
                                    int64_t ldv, int64_t v_row_stride, int32_t dtype, int32_t rows,
                                    int32_t T, int32_t heads, int32_t dh, void* kp, void* vp,
                                    uint8_t* ks, uint8_t* vs, int64_t n_pages,
                                    const int32_t* table, int32_t table_w, const int32_t* pos,
                                    const int32_t* count, void* stream) {
  clear_error();
  const int64_t lanes = 4 * blocks_of(std::max(dh, 1));
  const int32_t st = check_tokens(dtype, false, rows, T, heads, dh, n_pages, table_w, ldk,
                                  k_row_stride, ldv, v_row_stride, lanes);
  if (st != NV_OK) return st;
  if (rows == 0 || T == 0 || n_pages == 0 || table_w == 0) return NV_OK;
  NV_CHECK_ARG(k && v && kp && vp && ks && vs && table && pos, "null pointer argument");
  NV_CHECK_ARG(aligned16(kp) && aligned16(vp), "kp and vp must be 16-byte aligned");
  const Kv4AppendArgs a{k, v, (uint8_t*)kp, (uint8_t*)vp, ks, vs,
                        ldk, k_row_stride, ldv, v_row_stride, n_pages, table, pos, count,
                        T, heads, dh, table_w};
  const bool vec = (ldk | ldv | k_row_stride | v_row_stride) % 8 == 0 && aligned16(k) && aligned16(v);
  const dim3 grid((unsigned)ceil_div((int64_t)T * heads * lanes, 256), rows);
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, (hipStream_t)stream, a);
  };
  if (dtype == NV_F16) vec ? go(kv4_append_k<_Float16, true>) : go(kv4_append_k<_Float16, false>);
  else vec ? go(kv4_append_k<__bf16, true>) : go(kv4_append_k<__bf16, false>);
  NV_LAUNCH_CHECK("kv4_append_k");
  return NV_OK;
}

extern "C" int32_t nv_op_kv4_read(const void* kp, const void* vp, const uint8_t* ks,
                                  const uint8_t* vs, int64_t n_pages, const int32_t* table,
                                  int32_t table_w, const int32_t* pos, const int32_t* count,
                                  int32_t rows, int32_t T, int32_t heads, int32_t dh, void* k,
                                  int64_t ldk, int64_t k_row_stride, void* v, int64_t ldv,
                                  int64_t v_row_stride, int32_t dtype, void* stream) {
  clear_error();
  const int64_t lanes = std::max(dh, 0) / 8;
  const int32_t st = check_tokens(dtype, true, rows, T, heads, dh, n_pages, table_w, ldk,
                                  k_row_stride, ldv, v_row_stride, lanes);
  if (st != NV_OK) return st;
  NV_CHECK_ARG(ldk >= (int64_t)heads * dh && ldv >= (int64_t)heads * dh,
               "rows of an output shorter than heads * dh");
  if (rows == 0 || T == 0) return NV_OK;
  NV_CHECK_ARG(k && v && pos && (table_w == 0 || table) && (n_pages == 0 || (kp && vp && ks && vs)),
               "null pointer argument");
  NV_CHECK_ARG(aligned16(kp) && aligned16(vp), "kp and vp must be 16-byte aligned");
  const Kv4ReadArgs a{(const uint8_t*)kp, (const uint8_t*)vp, ks, vs, n_pages, table, pos, count,
                      k, v, ldk, k_row_stride, ldv, v_row_stride, T, heads, dh, table_w};
  const bool vec = (ldk | ldv | k_row_stride | v_row_stride) % 8 == 0 && aligned16(k) && aligned16(v);
  const int64_t units = (int64_t)T * heads * lanes;
  auto go = [&](auto kernel, int n) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)ceil_div(units, 256 * n), rows), dim3(256), 0,
                       (hipStream_t)stream, a);
  };
  auto pick = [&](auto t) {
    typedef decltype(t) Ty;
    if (units * rows < READ_TWO) vec ? go(kv4_read_k<Ty, true, 1>, 1) : go(kv4_read_k<Ty, false, 1>, 1);
    else vec ? go(kv4_read_k<Ty, true, 2>, 2) : go(kv4_read_k<Ty, false, 2>, 2);
  };
  if (dtype == NV_F32) pick(float());
  else if (dtype == NV_F16) pick(_Float16());
  else pick(__bf16());
  NV_LAUNCH_CHECK("kv4_read_k");
  return NV_OK;
}

extern "C" size_t nv_op_attention_kv4_workspace(int32_t rows, int32_t S, int32_t heads,
                                                int32_t kv_heads, int32_t dh, int32_t table_w) {
  if (rows < 1 || S < 1 || heads < 1 || kv_heads < 1 || heads % kv_heads || !head_dim_ok(dh) ||
      table_w < 0)
    return 0;
  return part_bytes(kv4_plan(rows, S, heads, kv_heads, dh, table_w), rows, S, heads, dh,
                    nullptr);
}

extern "C" int32_t nv_op_attention_kv4(const void* q, int64_t ldq, int64_t q_row_stride,
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
  const Kv8Plan p = kv4_plan(rows, S, heads, kv_heads, dh, table_w);
  if ((int64_t)S * (heads / kv_heads) > 0x7FFFFFF0 ||
      (double)rows * kv_heads * p.col_tiles * p.splits > 8388607.0) {
    set_error("more queries than a grid holds");
    return NV_ERR_UNSUPPORTED;
  }
  size_t ml_at = 0;
  const size_t need = part_bytes(p, rows, S, heads, dh, &ml_at);
  if (need && (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 255))) {
    set_error("workspace missing, misaligned or smaller than nv_op_attention_kv4_workspace()");
    return NV_ERR_WORKSPACE;
  }
  Kv4AttnArgs a{};
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
