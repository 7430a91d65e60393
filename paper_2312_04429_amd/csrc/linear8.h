// The 8-bit matrix product: arguments of its kernels and which of them a size takes (host only;
// no HIP in this file).
#pragma once
#include <cstdint>

namespace nv {

struct Linear8Args {
  const uint8_t *x, *w, *xs, *ws;   // codes [M][ldx], [N][ldw]; scale bytes [M][KB], [N / 128][KB]
  int64_t ldx, ldw, ldr, ldo;
  const float* bias;                // [N] or null
  const void* residual;             // [M][ldr] or null
  void* out;                        // [M][ldo]
  int64_t M;
  int N, K;
};

constexpr int S8_TILES = 48;  // 128-deep tiles whose scale bytes sit in LDS at a time

// Forms and their cost in us: a launch costs 3, a single round of tiles f1 + s1 per 128-deep tile
// of K, each of several rounds f2 + s2.  A round is 256 tiles times the workgroups that fit a CU (its
// last one, if it has at most 256 tiles, costs f1 and s1).  Fitted to 330 products of 8 to 8192 rows,
// 320 to 10240 columns, K 320 to 5120 (graph-timed, operands not in L2): the choice takes 1.3 % more
// than the fastest form on average, 18 % at most; without any one of the forms the best of the rest
// takes 0.3 to 2.4 % more on average and up to 53 % at single sizes.  Shares of K on workgroups of
// their own, summed by a second kernel, were slower at every one of these sizes (5 us for that
// launch and the partial sums), so there are none.
struct Linear8Form {
  int bm, bn, per_cu, teams;
  float f1, s1, f2, s2;
};
constexpr int L8_FEW = 0;
constexpr Linear8Form L8_FORMS[] = {
    {16, 16, 3, 1, 0.13f, 0.114f, 0.22f, 0.325f},     // 0: rows in registers, eight waves share K
    {32, 32, 1, 4, 1.90f, 0.078f, 2.90f, 0.098f},     // 1: four teams of one wave
    {32, 64, 3, 1, 0.98f, 0.185f, 2.51f, 0.349f},     // 2: 2 waves of 32 x 32
    {64, 64, 2, 1, 1.20f, 0.201f, 2.74f, 0.373f},     // 3: 4 waves of 32 x 32
    {64, 128, 2, 1, 1.52f, 0.291f, 3.62f, 0.588f},    // 4: 4 waves of 64 x 32
    {128, 128, 2, 1, 2.48f, 0.521f, 5.92f, 0.856f},   // 5: 4 waves of 64 x 64
    {128, 128, 1, 1, 2.24f, 0.381f, 3.88f, 0.482f},   // 6: 8 waves of 64 x 32, four buffers
    {256, 256, 1, 1, 12.06f, 1.075f, 12.75f, 1.221f}, // 7: 4 waves of 128 x 128
};
constexpr int L8_COUNT = sizeof(L8_FORMS) / sizeof(L8_FORMS[0]);

inline float linear8_cost(const Linear8Form& f, int64_t M, int N, int K) {
  const float n = (float)((K + 127) / 128), one = f.f1 + f.s1 * n, each = f.f2 + f.s2 * n;
  const int64_t tiles = (M + f.bm - 1) / f.bm * (((int64_t)N + f.bn - 1) / f.bn);
  if (f.per_cu == 1) return 3.f + (tiles <= 256 ? one : (float)((tiles + 255) / 256) * each);
  const int64_t slots = 256 * f.per_cu, rem = tiles % slots;
  return 3.f + (float)(tiles / slots) * each + (rem == 0 ? 0.f : rem <= 256 ? one : each);
}

// The cheapest form.  The first takes at most 16 rows; teams need K in whole 16-byte chunks.
inline int linear8_form(int64_t M, int N, int K) {
  int best = -1;
  float cost = 0.f;
  for (int i = 0; i < L8_COUNT; ++i) {
    const Linear8Form& f = L8_FORMS[i];
    if ((i == L8_FEW && M > 16) || (f.teams > 1 && K % 16)) continue;
    const float c = linear8_cost(f, M, N, K);
    if (best < 0 || c < cost) best = i, cost = c;
  }
  return best;
}

}  // namespace nv
