// Matrix product of 8-bit matrices: out[m][n] = sum_k x[m][k] w[n][k] over e4m3 codes with a
// power-of-two scale per 128 columns of a row of x and per 128 x 128 block of w.
//
// v_mfma_scale_f32_16x16x128_f8f6f4 multiplies 16 x 16 x 128 codes and takes the scale byte of
// every row's 32 codes: a 128-deep tile is one block of both operands, so its scales enter the
// instruction itself and the float32 sums run over all of K without a multiply of their own.
// The order of the 128 codes within a lane's registers is the same for both operands and
// otherwise free: a lane takes 16-byte chunks kc and kc + 4 of its row.
//
// Tiles of 128 codes (128-byte rows) move global -> LDS with 16-byte buffer loads, chunk c of
// row r at slot c ^ (r & 7), in a ring of STAGES buffers.
#include <algorithm>

#include "common.h"
#include "e4m3.h"
#include "linear8.h"

namespace nv {
namespace {

constexpr uint32_t OOB = 0x80000000u;  // past every descriptor's range: loads return zeros

__device__ inline __amdgpu_buffer_rsrc_t make_rsrc(const void* p, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), (short)0, (int)bytes, 0x00020000);
}
__device__ inline void lds_dma16(__amdgpu_buffer_rsrc_t r, uint32_t off, void* lds_wave_base,
                                 uint32_t soff) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)lds_wave_base,
                                           16, off, soff, 0, 0);
}
// All but the newest N of the wave's loads have landed, and its LDS reads are done.
template <int N>
__device__ inline void wait_loads() {
  static_assert(N >= 0 && N < 64, "vmcnt range");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4));
}
// Each wave has waited for its own loads of the tile about to be read: the barrier publishes it.
__device__ inline void ring_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Codes at or past K of a lane's two chunks (k0 and k0 + 64 of the row) become zeros: what lies
// behind a row's K codes may be anything, NaN among it.
__device__ __forceinline__ void mask_tail(intx8& f, int left) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int n = left - (j & 3) * 4 - (j >> 2) * 64;  // codes of this dword that count
    if (n < 4) f[j] = n <= 0 ? 0 : f[j] & ((1 << (8 * n)) - 1);
  }
}

// bias, residual, rounding and store of columns n .. n + 3 of row m
template <typename T>
__device__ __forceinline__ void store_quad(const Linear8Args& g, int64_t m, int n, floatx4 v) {
  struct alignas(8) Quad { T v[4]; };
  T* o = (T*)g.out + m * g.ldo + n;
  const T* r = (const T*)g.residual + m * g.ldr + n;
  if (g.vec && n + 4 <= g.N) {
    if (g.bias) v += *(const floatx4*)(g.bias + n);
    if (g.residual) {
      const Quad q = *(const Quad*)r;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] += (float)q.v[i];
    }
    Quad q;
#pragma unroll
    for (int i = 0; i < 4; ++i) q.v[i] = (T)v[i];
    *(Quad*)o = q;
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (n + i < g.N) {
      float s = v[i];
      if (g.bias) s += g.bias[n + i];
      if (g.residual) s += (float)r[i];
      o[i] = (T)s;
    }
}

template <typename T, int BM, int BN, int WGM, int WGN, int STAGES>
__global__ void __launch_bounds__(WGM * WGN * 64) linear8_k(Linear8Args g) {
  constexpr int NW = WGM * WGN, NT = NW * 64;
  constexpr int WM = BM / WGM, WN = BN / WGN, FM = WM / 16, FN = WN / 16;
  constexpr int GA = BM / 8, PER = (BM + BN) / 8 / NW;  // 8-row groups; groups a wave loads
  constexpr int TILE = (BM + BN) * 128;
  static_assert((BM + BN) / 8 % NW == 0 && GA % NW == 0 && 128 % WN == 0 && FM % 4 == 0, "tile");
  extern __shared__ __align__(16) unsigned char smem[];
  uint8_t* ring = smem;
  uint8_t* sxs = smem + STAGES * TILE;         // [S8_TILES][BM]: tile, wave row, lane, row block
  uint8_t* sws = sxs + S8_TILES * BM;          // [S8_TILES][BN / WN]
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, kc = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / WGN, wn = wave % WGN;
  const int ntn = (g.N + BN - 1) / BN, mtn = (int)((g.M + BM - 1) / BM);
  const int tile = xcd_remap(blockIdx.x, gridDim.x);
  const int64_t m0 = (int64_t)(g.n_major ? tile % mtn : tile / ntn) * BM;
  const int n0 = (g.n_major ? tile / mtn : tile % ntn) * BN;
  const int KB = (g.K + 127) / 128;
  const int kt0 = (int)((int64_t)KB * blockIdx.y / gridDim.y);
  const int kt1 = (int)((int64_t)KB * (blockIdx.y + 1) / gridDim.y);
  const int k16 = (g.K + 15) & ~15;

  // descriptors start at the tile's first row, so any matrix fits their 2 GiB
  const int mrows = (int)std::min<int64_t>(BM, g.M - m0), nrows = std::min(BN, g.N - n0);
  const __amdgpu_buffer_rsrc_t rx =
      make_rsrc(g.x + m0 * g.ldx, (uint32_t)((mrows - 1) * g.ldx + k16));
  const __amdgpu_buffer_rsrc_t rw =
      make_rsrc(g.w + (int64_t)n0 * g.ldw, (uint32_t)((nrows - 1) * g.ldw + k16));
  const int lrow = lane >> 3, cch = ((lane & 7) ^ lrow) * 16;  // this lane's byte of the 128
  uint32_t voff[PER];
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int gi = j * NW + wave, r = (gi < GA ? gi : gi - GA) * 8 + lrow;
    voff[j] = gi < GA ? (r < mrows ? (uint32_t)(r * g.ldx + cch) : OOB)
                      : (r < nrows ? (uint32_t)(r * g.ldw + cch) : OOB);
  }
  // tile kt into ring buffer `slot` (past the last tile: that one again, never multiplied, so
  // that every wave keeps the same number of loads in flight)
  auto issue = [&](int kt, int slot) {
    kt = std::min(kt, kt1 - 1);
    uint8_t* dst = ring + slot * TILE;
    const uint32_t k0 = (uint32_t)kt * 128;
    const bool in = k0 + cch < (uint32_t)g.K;  // chunks wholly past K are not read
#pragma unroll
    for (int j = 0; j < PER; ++j)
      lds_dma16(j * NW < GA ? rx : rw, in ? voff[j] : OOB, dst + (j * NW + wave) * 1024, k0);
  };
  // scale bytes of tiles kb .. kb + S8_TILES - 1, those of a lane's FM rows side by side
  auto stage_scales = [&](int kb) {
    const int n = std::min(S8_TILES, kt1 - kb);
    for (int i = tid; i < n * BM; i += NT) {
      const int r = i / n, t = i - r * n;
      const int64_t m = std::min<int64_t>(m0 + r, g.M - 1);
      sxs[t * BM + (r / WM) * WM + (r & 15) * FM + (r % WM) / 16] = g.xs[m * KB + kb + t];
    }
    for (int i = tid; i < n * WGN; i += NT) {
      const int c = i / n, t = i - c * n;
      const int nb = std::min(n0 + c * WN, g.N - 1) >> 7;
      sws[t * WGN + c] = g.ws[(int64_t)nb * KB + kb + t];
    }
  };

  floatx4 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
  const int arow = (wm * WM + li) * 128, brow = (BM + wn * WN + li) * 128;
  const int s0 = (kc ^ (li & 7)) * 16, s1 = ((4 + kc) ^ (li & 7)) * 16;
  auto frag = [&](const uint8_t* __restrict__ row) {
    const u32x4 lo = *(const u32x4*)(row + s0), hi = *(const u32x4*)(row + s1);
    return intx8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3],
                 (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
  };

#pragma unroll
  for (int s = 0; s < STAGES - 1; ++s) issue(kt0 + s, s);
  int slot = 0;
  for (int kt = kt0; kt < kt1; ++kt) {
    const int sk = (kt - kt0) % S8_TILES;
    if (sk == 0) {
      __syncthreads();  // the last tiles' scales have been read
      stage_scales(kt);
      __syncthreads();
    }
    wait_loads<(STAGES - 2) * PER>();
    ring_barrier();
    issue(kt + STAGES - 1, slot == 0 ? STAGES - 1 : slot - 1);
    const uint8_t* t = ring + slot * TILE;
    intx8 fa[FM], fb[FN];
    int sx[FM / 4];
#pragma unroll
    for (int i = 0; i < FM / 4; ++i)
      sx[i] = *(const int*)(sxs + sk * BM + wm * WM + li * FM + i * 4);
    const int sw = sws[sk * WGN + wn];
#pragma unroll
    for (int j = 0; j < FN; ++j) fb[j] = frag(t + brow + j * 2048);
#pragma unroll
    for (int i = 0; i < FM; ++i) fa[i] = frag(t + arow + i * 2048);
    if ((kt + 1) * 128 > g.K) {
#pragma unroll
      for (int j = 0; j < FN; ++j) mask_tail(fb[j], g.K - kt * 128 - kc * 16);
#pragma unroll
      for (int i = 0; i < FM; ++i) mask_tail(fa[i], g.K - kt * 128 - kc * 16);
    }
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) {
#define NV_MFMA8(SEL)                                                                             \
  acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb[j], fa[i], acc[i][j], 0, 0, 0, \
                                                               sw, SEL, sx[i / 4])
        if ((i & 3) == 0) NV_MFMA8(0);
        if ((i & 3) == 1) NV_MFMA8(1);
        if ((i & 3) == 2) NV_MFMA8(2);
        if ((i & 3) == 3) NV_MFMA8(3);
#undef NV_MFMA8
      }
    slot = slot + 1 == STAGES ? 0 : slot + 1;
  }
  wait_loads<0>();  // loads past the last tile land before the workgroup's LDS is given back

#pragma unroll
  for (int i = 0; i < FM; ++i) {
    const int64_t m = m0 + wm * WM + i * 16 + li;
    if (m >= g.M) continue;
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      const int n = n0 + wn * WN + j * 16 + kc * 4;
      if (n >= g.N) continue;
      if (gridDim.y == 1) {
        store_quad<T>(g, m, n, acc[i][j]);
      } else {  // partial sums, rows of Np = N rounded up to 4
        const int64_t Np = (g.N + 3) & ~3;
        *(floatx4*)(g.partial + ((int64_t)blockIdx.y * g.M + m) * Np + n) = acc[i][j];
      }
    }
  }
}

// The shares of K in order, then the epilogue.
template <typename T>
__global__ void __launch_bounds__(256) linear8_sum_k(Linear8Args g, int splits) {
  const int nq = (g.N + 3) / 4;
  const int64_t total = g.M * nq;
  for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < total;
       u += (int64_t)gridDim.x * 256) {
    const int64_t m = u / nq;
    const float* p = g.partial + u * 4;
    floatx4 v = *(const floatx4*)p;
    for (int s = 1; s < splits; ++s) v += *(const floatx4*)(p + (int64_t)s * total * 4);
    store_quad<T>(g, m, (int)(u - m * nq) * 4, v);
  }
}

template <typename T, int BM, int BN, int WGM, int WGN, int STAGES>
hipError_t go(Linear8Args g, int splits, hipStream_t s) {
  constexpr size_t lds = (size_t)STAGES * (BM + BN) * 128 + S8_TILES * (BM + WGN);
  static_assert(lds <= 160 * 1024, "LDS per workgroup");
  const hipError_t e = hipFuncSetAttribute((const void*)linear8_k<T, BM, BN, WGM, WGN, STAGES>,
                                           hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  if (e != hipSuccess) return e;
  const int64_t tiles = ceil_div(g.M, BM) * ceil_div(g.N, BN);
  if (tiles > 0x7FFFFFFF / (WGM * WGN * 64)) return hipErrorInvalidValue;
  g.n_major = (int64_t)g.N > g.M;
  hipLaunchKernelGGL((linear8_k<T, BM, BN, WGM, WGN, STAGES>), dim3((unsigned)tiles, splits),
                     dim3(WGM * WGN * 64), lds, s, g);
  if (splits > 1) {
    const int64_t quads = g.M * ((g.N + 3) / 4);
    hipLaunchKernelGGL(linear8_sum_k<T>, dim3((unsigned)std::min<int64_t>(ceil_div(quads, 256), 1 << 20)),
                       dim3(256), 0, s, g, splits);
  }
  return hipGetLastError();
}

template <typename T>
hipError_t launch(const Linear8Args& g, const Linear8Plan& p, hipStream_t s) {
  return go<T, 128, 128, 2, 2, 2>(g, p.splits, s);
}

}  // namespace
}  // namespace nv

using namespace nv;

extern "C" size_t nv_op_linear8_workspace(int64_t M, int32_t N, int32_t K) {
  if (M < 1 || N < 1 || K < 1 || M > 0x7FFFFFFF) return 0;
  const Linear8Plan p = linear8_plan(M, N, K);
  return p.splits > 1 ? (size_t)p.splits * (size_t)M * (size_t)((N + 3) / 4) * 16 : 0;
}

extern "C" int32_t nv_op_linear8(const void* x, int64_t ldx, const uint8_t* xs, const void* w,
                                 int64_t ldw, const uint8_t* ws, const float* bias,
                                 const void* residual, int64_t ldr, void* out, int64_t ldo,
                                 int32_t dtype, int64_t M, int32_t N, int32_t K, void* workspace,
                                 size_t workspace_bytes, void* stream) {
  clear_error();
  NV_CHECK_ARG(M >= 0 && M <= 0x7FFFFFFF && N >= 1 && K >= 1,
               "need 0 <= M <= 2^31 - 1, N >= 1 and K >= 1");
  NV_CHECK_ARG(dtype == NV_F16 || dtype == NV_BF16, "dtype must be NV_F16 or NV_BF16");
  NV_CHECK_ARG(ldx >= K && ldw >= K && ldo >= N && (!residual || ldr >= N),
               "row strides shorter than the rows");
  if (ldx % 16 || ldw % 16 || ((uintptr_t)x | (uintptr_t)w) % 16) {
    set_error("x and w need 16-byte aligned rows (strides in multiples of 16 bytes)");
    return NV_ERR_UNSUPPORTED;
  }
  if (ldx > (1 << 22) || ldw > (1 << 22)) {
    set_error("rows of x and w more than 4 MiB apart");
    return NV_ERR_UNSUPPORTED;
  }
  if (M == 0) return NV_OK;
  NV_CHECK_ARG(x && xs && w && ws && out, "null pointer argument");
  const size_t need = nv_op_linear8_workspace(M, N, K);
  if (need && (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 255))) {
    set_error("workspace missing, misaligned or smaller than nv_op_linear8_workspace()");
    return NV_ERR_WORKSPACE;
  }
  Linear8Args g{};
  g.x = (const uint8_t*)x, g.w = (const uint8_t*)w, g.xs = xs, g.ws = ws;
  g.ldx = ldx, g.ldw = ldw, g.ldr = ldr, g.ldo = ldo;
  g.bias = bias, g.residual = residual, g.out = out, g.partial = (float*)workspace;
  g.M = M, g.N = N, g.K = K;
  g.vec = ldo % 4 == 0 && (uintptr_t)out % 8 == 0 && (!bias || aligned16(bias)) &&
          (!residual || (ldr % 4 == 0 && (uintptr_t)residual % 8 == 0));
  const Linear8Plan p = linear8_plan(M, N, K);
  const hipStream_t s = (hipStream_t)stream;
  const hipError_t e = dtype == NV_F16 ? launch<_Float16>(g, p, s) : launch<__bf16>(g, p, s);
  if (e == hipErrorInvalidValue) {
    set_error("more output tiles than a grid holds");
    return NV_ERR_UNSUPPORTED;
  }
  NV_HIP_TRY(e);
  return NV_OK;
}
