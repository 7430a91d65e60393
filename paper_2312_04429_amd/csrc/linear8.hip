// Matrix product of 8-bit matrices: out[m][n] = sum_k x[m][k] w[n][k] over e4m3 codes with a
// power-of-two scale per 128 columns of a row of x and per 128 x 128 block of w.
//
// v_mfma_scale_f32_16x16x128_f8f6f4 multiplies 16 x 16 x 128 codes and takes the scale byte of
// every row's 32 codes: a 128-deep tile is one block of both operands, so its scales enter the
// instruction itself and the float32 sums run over all of K without a multiply of their own.
// The order of the 128 codes within a lane's registers is the same for both operands and
// otherwise free: a lane takes 16-byte chunks kc and kc + 4 of its row.
//
// Precision: the unit cuts each product to 2^-13 of the largest exponent among its group of eight
// consecutive k before it adds them (towards zero; measured), and adds the groups in float32: of a
// product next to the group's largest nothing is lost, of one 2^-10 of it less than an eighth, where
// its code had lost a sixteenth.
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
__device__ inline void lds_dma16(__amdgpu_buffer_rsrc_t r, uint32_t off, void* lds_wave_base) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)lds_wave_base,
                                           16, off, 0, 0, 0);
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

// bias, residual, rounding and store of columns n .. n + 3 of row m (those below N)
template <typename T>
__device__ __forceinline__ void store_quad(const Linear8Args& g, int64_t m, int n, floatx4 v) {
  struct __attribute__((packed, aligned(sizeof(T)))) Quad { T v[4]; };
  struct __attribute__((packed, aligned(4))) Quad32 { float v[4]; };
  T* o = (T*)g.out + m * g.ldo + n;
  const T* r = (const T*)g.residual + m * g.ldr + n;
  if (n + 4 <= g.N) {
    if (g.bias) {
      const Quad32 b = *(const Quad32*)(g.bias + n);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] += b.v[i];
    }
    Quad q;
    if (g.residual) {
      q = *(const Quad*)r;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] += (float)q.v[i];
    }
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

// One output tile.  The loop is rotated by half a tile: while
// the first half of a wave's row blocks is multiplied, the fragments of the second half are
// read; then all of the tile's reads are out, one barrier hands its buffer back and publishes the
// next tile, and the second half's multiplies run between the reads of the next tile's first
// fragments and the requests for the tile STAGES on.  Everything within a tile is in program
// order (with one wave a SIMD nothing else fills a gap).
//
// KT teams of waves share out the tile's K in contiguous parts, each with a ring of its own; a team
// that runs out multiplies zeros (loads out of range), so all keep step with the barriers, and
// the epilogue adds the teams' sums in order.
//
// Measured: 8192 x 10240 x 5120 with bias 333 us in calls back to back (2580 TFLOP/s; graph replays of
// a few calls, at a lower clock: 365, and 403 for 8192^3): the multiplies take 59 % of its cycles, and
// each round of 256 tiles adds about 14 us outside its steps, 6 of them the results' stores.
// 2000 x 1280 x 5120 22 us: 160 tiles of 128 x 128 on 256 compute units, each bound by the 96 KB of LDS
// that its waves read a step (two teams of 64 x 64 waves read 64 but hold two buffers each, and took 28).
template <typename T, int BM, int BN, int WGM, int WGN, int KT, int STAGES>
__global__ void __launch_bounds__(KT * WGM * WGN * 64) linear8_k(Linear8Args g) {
  constexpr int NW = WGM * WGN, NT = NW * 64;  // waves and threads of a team
  constexpr int WM = BM / WGM, WN = BN / WGN, FM = WM / 16, FN = WN / 16;
  constexpr int GA = BM / 8, PER = (BM + BN) / 8 / NW;  // 8-row groups; groups a wave loads
  constexpr int TILE = (BM + BN) * 128;
  constexpr int HALF = FM / 2;                // row blocks before the barrier, and after
  constexpr int FB = (FN + HALF - 1) / HALF;  // column fragments of the next tile read per row block
  static_assert((BM + BN) / 8 % NW == 0 && GA % NW == 0 && 128 % WN == 0, "tile");
  static_assert(FM == 2 || FM % 4 == 0, "row blocks");
  // Two buffers of large tiles: see the step below.
  constexpr bool EARLY = STAGES == 2 && BM == 256;
  static_assert(!EARLY || WM / 16 % NW == 0, "sets of loads");
  extern __shared__ __align__(16) unsigned char smem[];
  const int tid = threadIdx.x % NT, lane = tid & 63, li = lane & 15, kc = lane >> 4;
  const int team = KT == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / NT);
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / WGN, wn = wave % WGN;
  uint8_t* ring = smem + team * STAGES * TILE;
  uint8_t* sxs = smem + KT * STAGES * TILE + team * S8_TILES * (BM + WGN);
                                               // [S8_TILES][BM]: tile, wave row, lane, row block
  uint8_t* sws = sxs + S8_TILES * BM;          // [S8_TILES][WGN]
  const int ntn = (g.N + BN - 1) / BN, mtn = (int)((g.M + BM - 1) / BM);
  // An XCD's tiles run in bands of GROUP tile columns, row after row: those that run at once then
  // form a near-square block, and their rows of x and w meet in its L2.
  constexpr int GROUP = BN >= 256 ? 4 : 8;
  const int tile = xcd_remap(blockIdx.x, gridDim.x);
  const int band = tile / (GROUP * mtn), in_band = tile - band * GROUP * mtn;
  const int width = std::min(GROUP, ntn - band * GROUP);
  const int64_t m0 = (int64_t)(in_band / width) * BM;
  const int n0 = (band * GROUP + in_band % width) * BN;
  const int KB = (g.K + 127) / 128;
  const int steps = (KB + KT - 1) / KT;  // of every team
  const int kt0 = std::min(team * steps, KB), kt1 = std::min(kt0 + steps, KB);
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
    // a tile's rows past the matrix: its last row again (their sums are not stored)
    voff[j] = gi < GA ? (uint32_t)(std::min(r, mrows - 1) * g.ldx + cch)
                      : (uint32_t)(std::min(r, nrows - 1) * g.ldw + cch);
  }
  // Groups j0 .. j1 - 1 of tile kt into ring buffer `slot`.  Chunks wholly past K, and tiles past
  // the last one (issued all the same: every wave keeps its number of loads in flight), are out
  // of range: zeros.
  auto load_group = [&](int kt, int slot, int j) {
    const uint32_t k0 = kt < kt1 && kt * 128 + cch < g.K ? (uint32_t)kt * 128 : OOB;
    lds_dma16(j * NW < GA ? rx : rw, voff[j] + k0, ring + slot * TILE + (j * NW + wave) * 1024);
  };
  auto issue = [&](int kt, int slot, int j0, int j1) {
#pragma unroll
    for (int j = j0; j < j1; ++j) load_group(kt, slot, j);
  };
  // EARLY: a tile's groups in two sets: its columns and the first half of every wave's rows (read
  // in the second half of the step before), and the rest.
  auto late = [](int j) { return j * NW < GA && (j * NW % (WM / 8)) * 2 >= WM / 8; };
  auto issue_set = [&](int kt, int slot, bool rest, int part, int parts) {
    constexpr int NR = GA / NW / 2, NF = PER - NR;  // groups of the sets
    const int n = rest ? NR : NF, a = part * n / parts, b = (part + 1) * n / parts;
    int i = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j)
      if (late(j) == rest) {
        if (i >= a && i < b) load_group(kt, slot, j);
        ++i;
      }
  };
  // scale bytes of tiles kb .. kb + S8_TILES - 1, those of a lane's FM rows side by side
  // (a team without tiles left: those of the last tile, for its zeros)
  auto stage_scales = [&](int kb) {
    const int n = std::max(1, std::min(S8_TILES, kt1 - kb));
    kb = std::min(kb, KB - 1);
    constexpr int RT = NT / BM > 0 ? NT / BM : 1;  // threads that share a row
    for (int r = tid / RT; r < BM; r += NT / RT) {
      const uint8_t* src = g.xs + std::min<int64_t>(m0 + r, g.M - 1) * KB + kb;
      uint8_t* dst = sxs + (r / WM) * WM + (r & 15) * FM + (r % WM) / 16;
      if (n >= 16) {  // 16 at a time, the last ones ending with the row
#pragma unroll
        for (int t = tid % RT * 16; t < S8_TILES; t += RT * 16)
          if (t < n) {
            const int t0 = std::min(t, n - 16);
            uint8_t v[16];
            __builtin_memcpy(v, src + t0, 16);
#pragma unroll
            for (int i = 0; i < 16; ++i) dst[(t0 + i) * BM] = v[i];
          }
      } else {
        for (int t = tid % RT; t < n; t += RT) dst[t * BM] = src[t];
      }
    }
    for (int i = tid; i < n * WGN; i += NT) {
      const int t = i / WGN, c = i % WGN;
      sws[i] = g.ws[(int64_t)(std::min(n0 + c * WN, g.N - 1) >> 7) * KB + kb + t];
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
  struct Scales { int x[(FM + 3) / 4], w; };
  auto scales = [&](int kt) {
    Scales s;
    const int t = std::max(std::min(kt, kt1 - 1) - kt0, 0) % S8_TILES;  // past the end: staged ones
    const uint8_t* p = sxs + t * BM + wm * WM + li * FM;
#pragma unroll
    for (int i = 0; i < (FM + 3) / 4; ++i)
      s.x[i] = FM >= 4 ? *(const int*)(p + i * 4) : (int)*(const uint16_t*)p;
    s.w = sws[t * WGN + wn];
    return s;
  };
  intx8 fa[FM], fb0[FN], fb1[FN];
  auto mul = [&](int i, int j, const Scales& s, const intx8(&fb)[FN]) {
#define NV_MFMA8(SEL)                                                                             \
  acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb[j], fa[i], acc[i][j], 0, 0, 0, \
                                                               s.w, SEL, s.x[i / 4])
    if ((i & 3) == 0) NV_MFMA8(0);
    if ((i & 3) == 1) NV_MFMA8(1);
    if ((i & 3) == 2) NV_MFMA8(2);
    if ((i & 3) == 3) NV_MFMA8(3);
#undef NV_MFMA8
  };

#pragma unroll
  for (int s = 0; s < STAGES; ++s) {
    if constexpr (EARLY) issue_set(kt0 + s, s, false, 0, 1), issue_set(kt0 + s, s, true, 0, 1);
    else issue(kt0 + s, s, 0, PER);
  }
  stage_scales(kt0);
  wait_loads<0>();  // the scales' bytes are the newest loads
  ring_barrier();
  const uint8_t* cur = ring;
  Scales sc = scales(kt0);
#pragma unroll
  for (int j = 0; j < FN; ++j) fb0[j] = frag(cur + brow + j * 2048);
#pragma unroll
  for (int i = 0; i < HALF; ++i) fa[i] = frag(cur + arow + i * 2048);
  // A last chunk that ends within its 16 bytes: its tile is not multiplied in the loop (one team
  // only: the launcher gives such a K no others).
  const bool cut = KT == 1 && g.K % 16 && kt1 == KB;
  const int full = kt0 + steps - (cut ? 1 : 0);
  int slot = 0, kt = kt0;
  // With EARLY a second barrier ends the step: the next tile's columns and first rows have then
  // been read by every wave, and their place takes tile kt + 3's half a tile before the rest: every
  // load has one and a half tiles of time instead of one (graph replays: 8192^3 418 -> 403 us,
  // 8192 x 8192 x 2048 146 -> 143, 8192 x 10240 x 5120 367 -> 365).
  if constexpr (EARLY) {
    wait_loads<0>();
    ring_barrier();
  }
  auto step = [&](const intx8(&fb)[FN], intx8(&fn)[FN]) {
    const uint8_t* t = ring + slot * TILE;
    const int next = slot + 1 == STAGES ? 0 : slot + 1;
    const uint8_t* tn = ring + next * TILE;
#pragma unroll
    for (int i = 0; i < HALF; ++i) {
      fa[HALF + i] = frag(t + arow + (HALF + i) * 2048);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        mul(i, j, sc, fb);
        if constexpr (EARLY) {
          issue_set(kt + 2, slot, false, i * FN + j, HALF * FN);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    // this wave's loads of tile kt + 1 (what is read below, with EARLY), its reads of kt
    wait_loads<EARLY ? PER : (STAGES - 2) * PER>();
    ring_barrier();
    const Scales sn = scales(kt + 1);
#pragma unroll
    for (int i = 0; i < HALF; ++i) {
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        mul(HALF + i, j, sc, fb);
        if (j < FB && i * FB + j < FN) fn[i * FB + j] = frag(tn + brow + (i * FB + j) * 2048);
        if (j == (FB < FN ? FB : FN - 1)) fa[i] = frag(tn + arow + i * 2048);
        if constexpr (EARLY) issue_set(kt + 2, slot, true, i * FN + j, HALF * FN);
        else issue(kt + STAGES, slot, (i * FN + j) * PER / (HALF * FN),
                   (i * FN + j + 1) * PER / (HALF * FN));
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    if constexpr (EARLY) {
      wait_loads<PER>();  // the rest of tile kt + 1; this wave's reads of it
      ring_barrier();
    }
    sc = sn;
    slot = next;
    ++kt;
  };
  while (kt < full) {
    const int end = std::min(full, kt + S8_TILES);
    for (; kt + 1 < end;) {
      step(fb0, fb1);
      step(fb1, fb0);
    }
    if (kt < end) {
      step(fb0, fb1);
#pragma unroll
      for (int j = 0; j < FN; ++j) fb0[j] = fb1[j];
    }
    if (kt < kt0 + steps && (kt - kt0) % S8_TILES == 0) {  // the next tiles' scales
      __syncthreads();
      stage_scales(kt);
      __syncthreads();
      sc = scales(kt);
    }
  }
  if (cut) {  // the short tile: fragments re-read, codes past K cut
    const uint8_t* t = ring + slot * TILE;
    const int left = g.K - full * 128 - kc * 16;
#pragma unroll
    for (int j = 0; j < FN; ++j) mask_tail(fb0[j] = frag(t + brow + j * 2048), left);
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      mask_tail(fa[i] = frag(t + arow + i * 2048), left);
#pragma unroll
      for (int j = 0; j < FN; ++j) mul(i, j, sc, fb0);
    }
  }
  wait_loads<0>();  // loads past the last tile land before the LDS is used again
  ring_barrier();

  // Epilogue through LDS, a wave (and team) in its own part: rows of float32 sums (16-byte chunk c of row r
  // at slot c ^ (r & 7)), then 8 columns of a row a lane, so that outputs and residuals move in
  // whole lines (straight from the accumulators a store touches 16 rows, 32 bytes each).
  constexpr int CH = WN / 4;                                   // 16-byte chunks of a row
  constexpr int FIT = STAGES * TILE / NW / (WN * 4) / 16;      // row blocks that fit at a time
  constexpr int IB = FIT >= FM ? FM : FIT >= 4 ? 4 : FIT >= 2 ? 2 : 1;
  constexpr int ROWS = IB * 16, LPR = WN / 8;                  // rows a pass, lanes a row
  static_assert(FIT >= 1 && FM % IB == 0 && WN >= 32, "epilogue passes");
  // a wave finishes its rows for all teams, or the teams take every KT-th group of rows
  constexpr int STEP = 64 / LPR, ALL = ROWS / STEP, SETS = ALL >= KT ? ALL / KT : 1;
  constexpr int U = SETS >= 4 ? 4 : SETS;
  static_assert(ALL >= 1 && (ALL < KT || ALL % KT == 0) && SETS % U == 0, "rows of a team");
  float* mine = (float*)(ring + wave * (STAGES * TILE / NW));
  const float* first = (const float*)(smem + wave * (STAGES * TILE / NW));  // team 0's part
  const int c = lane % LPR * 2, n = n0 + wn * WN + c * 4;
  const bool whole = n + 8 <= g.N;
  floatx4 blo = {0.f, 0.f, 0.f, 0.f}, bhi = blo;
  if (whole && g.bias) {
    const Any8<float> b = *(const Any8<float>*)(g.bias + n);
#pragma unroll
    for (int e = 0; e < 4; ++e) blo[e] = b.v[e], bhi[e] = b.v[4 + e];
  }
#pragma unroll
  for (int i0 = 0; i0 < FM; i0 += IB) {
#pragma unroll
    for (int i = i0; i < i0 + IB; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j)
        *(floatx4*)(mine + ((i - i0) * 16 + li) * WN + ((j * 4 + kc) ^ (li & 7)) * 4) = acc[i][j];
    if (KT > 1) __syncthreads();
    else __builtin_amdgcn_wave_barrier();
    const int64_t mw = m0 + wm * WM + i0 * 16;
    for (int r0 = team * SETS * STEP + lane / LPR; r0 < std::min((team + 1) * SETS * STEP, ROWS);
         r0 += STEP * U) {
      floatx4 lo[U], hi[U];
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const int r = r0 + k * STEP;
        lo[k] = *(const floatx4*)(first + r * WN + (c ^ (r & 7)) * 4);
        hi[k] = *(const floatx4*)(first + r * WN + ((c + 1) ^ (r & 7)) * 4);
#pragma unroll
        for (int t = 1; t < KT; ++t) {
          const float* p = first + t * (STAGES * TILE / 4) + r * WN;
          lo[k] += *(const floatx4*)(p + (c ^ (r & 7)) * 4);
          hi[k] += *(const floatx4*)(p + ((c + 1) ^ (r & 7)) * 4);
        }
      }
      if (whole) {
        Any8<T> q[U];  // rows start anywhere: vectors aligned as their elements
        if (g.residual) {
#pragma unroll
          for (int k = 0; k < U; ++k) {
            const int64_t m = std::min<int64_t>(mw + r0 + k * STEP, g.M - 1);
            q[k] = *(const Any8<T>*)((const T*)g.residual + m * g.ldr + n);
          }
        } else {
#pragma unroll
          for (int k = 0; k < U; ++k) q[k] = Any8<T>{};
        }
#pragma unroll
        for (int k = 0; k < U; ++k) {
          const int64_t m = mw + r0 + k * STEP;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            q[k].v[e] = (T)(lo[k][e] + blo[e] + (float)q[k].v[e]);
            q[k].v[4 + e] = (T)(hi[k][e] + bhi[e] + (float)q[k].v[4 + e]);
          }
          if (m < g.M) *(Any8<T>*)((T*)g.out + m * g.ldo + n) = q[k];
        }
      } else {
#pragma unroll
        for (int k = 0; k < U; ++k) {
          const int64_t m = mw + r0 + k * STEP;
          if (m < g.M && n < g.N) store_quad<T>(g, m, n, lo[k]);
          if (m < g.M && n + 4 < g.N) store_quad<T>(g, m, n + 4, hi[k]);
        }
      }
    }
    if (KT > 1) __syncthreads();
    else __builtin_amdgcn_wave_barrier();
  }
}

// At most 16 rows of x: bound by the bytes of w, which go straight from memory to registers.  A
// workgroup takes 16 columns and all of K; its eight waves take 128-deep tiles in turn (two at a time,
// all their loads out before the first multiply) and their sums meet in LDS, in wave order.
template <typename T>
__global__ void __launch_bounds__(512) linear8_few_k(Linear8Args g) {
  constexpr int NW = 8, U = 2, ROW = 16 + 4;
  __shared__ __align__(16) float part[NW][16 * ROW];
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, kc = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n0 = blockIdx.x * 16;
  const int KB = (g.K + 127) / 128, k16 = (g.K + 15) & ~15;
  const int64_t row = std::min<int64_t>(li, g.M - 1), col = std::min(n0 + li, g.N - 1);
  const uint8_t *xr = g.x + row * g.ldx, *xsr = g.xs + row * KB;
  const uint8_t *wr = g.w + col * g.ldw, *wsr = g.ws + (int64_t)(n0 >> 7) * KB;
  floatx4 acc = {0.f, 0.f, 0.f, 0.f};
  auto load = [&](const uint8_t* codes, int kt) {  // chunks past the row's codes: its last one again
    const u32x4 lo = *(const u32x4*)(codes + std::min(kt * 128 + kc * 16, k16 - 16));
    const u32x4 hi = *(const u32x4*)(codes + std::min(kt * 128 + 64 + kc * 16, k16 - 16));
    return intx8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3],
                 (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
  };
  for (int k0 = wave; k0 < KB; k0 += NW * U) {
    intx8 fx[U], fw[U];
    int sx[U], sw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int kt = std::min(k0 + u * NW, KB - 1);
      fw[u] = load(wr, kt), sw[u] = wsr[kt];
      fx[u] = load(xr, kt), sx[u] = xsr[kt];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int kt = k0 + u * NW;
      if (kt >= KB) break;  // uniform
      if ((kt + 1) * 128 > g.K) {
        mask_tail(fw[u], g.K - kt * 128 - kc * 16);
        mask_tail(fx[u], g.K - kt * 128 - kc * 16);
      }
      acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fw[u], fx[u], acc, 0, 0, 0, sw[u], 0,
                                                             sx[u]);
    }
  }
  *(floatx4*)&part[wave][li * ROW + kc * 4] = acc;
  __syncthreads();
  const int m = tid / 4, c = tid % 4 * 4;
  if (tid >= 64 || m >= g.M || n0 + c >= g.N) return;
  floatx4 v = *(const floatx4*)&part[0][m * ROW + c];
#pragma unroll
  for (int w = 1; w < NW; ++w) v += *(const floatx4*)&part[w][m * ROW + c];
  store_quad<T>(g, m, n0 + c, v);
}

template <typename T, int BM, int BN, int WGM, int WGN, int KT, int STAGES>
hipError_t go(const Linear8Args& g, hipStream_t s) {
  constexpr size_t lds = (size_t)KT * (STAGES * (BM + BN) * 128 + S8_TILES * (BM + WGN));
  static_assert(lds <= 160 * 1024, "LDS per workgroup");
  const hipError_t e = hipFuncSetAttribute((const void*)linear8_k<T, BM, BN, WGM, WGN, KT, STAGES>,
                                           hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((linear8_k<T, BM, BN, WGM, WGN, KT, STAGES>),
                     dim3((unsigned)(ceil_div(g.M, BM) * ceil_div(g.N, BN))),
                     dim3(KT * WGM * WGN * 64), lds, s, g);
  return hipGetLastError();
}

template <typename T>
hipError_t launch(const Linear8Args& g, int form, hipStream_t s) {
  switch (form) {
    case L8_FEW:
      hipLaunchKernelGGL(linear8_few_k<T>, dim3((unsigned)ceil_div(g.N, 16)), dim3(512), 0, s, g);
      return hipGetLastError();
    case 1: return go<T, 32, 32, 1, 1, 4, 4>(g, s);
    case 2: return go<T, 32, 64, 1, 2, 1, 4>(g, s);
    case 3: return go<T, 64, 64, 2, 2, 1, 4>(g, s);
    case 4: return go<T, 64, 128, 1, 4, 1, 3>(g, s);
    case 5: return go<T, 128, 128, 2, 2, 1, 2>(g, s);
    case 6: return go<T, 128, 128, 2, 4, 1, 4>(g, s);
    default: return go<T, 256, 256, 2, 2, 1, 2>(g, s);
  }
}

}  // namespace
}  // namespace nv

using namespace nv;

extern "C" int32_t nv_op_linear8(const void* x, int64_t ldx, const uint8_t* xs, const void* w,
                                 int64_t ldw, const uint8_t* ws, const float* bias,
                                 const void* residual, int64_t ldr, void* out, int64_t ldo,
                                 int32_t dtype, int64_t M, int32_t N, int32_t K, void* stream) {
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
  const int form = linear8_form(M, N, K);
  if ((double)ceil_div(M, L8_FORMS[form].bm) * (double)ceil_div(N, L8_FORMS[form].bn) > 8388607.0) {
    set_error("more output tiles than a grid holds");
    return NV_ERR_UNSUPPORTED;
  }
  Linear8Args g{};
  g.x = (const uint8_t*)x, g.w = (const uint8_t*)w, g.xs = xs, g.ws = ws;
  g.ldx = ldx, g.ldw = ldw, g.ldr = ldr, g.ldo = ldo;
  g.bias = bias, g.residual = residual, g.out = out;
  g.M = M, g.N = N, g.K = K;
  const hipStream_t s = (hipStream_t)stream;
  NV_HIP_TRY(dtype == NV_F16 ? launch<_Float16>(g, form, s) : launch<__bf16>(g, form, s));
  return NV_OK;
}
