// The 8-bit matrix product: arguments of its kernels and which of them a size takes.
#pragma once
#include <algorithm>
#include <cstdint>

namespace nv {

struct Linear8Args {
  const uint8_t *x, *w, *xs, *ws;   // codes [M][ldx], [N][ldw]; scale bytes [M][KB], [N / 128][KB]
  int64_t ldx, ldw, ldr, ldo;
  const float* bias;                // [N] or null
  const void* residual;             // [M][ldr] or null
  void* out;                        // [M][ldo]
  float* partial;                   // [splits][M][N rounded up to 4]
  int64_t M;
  int N, K;
  int vec;                          // four columns of out, residual and bias move as a vector
  int n_major;                      // tile order: columns of w outermost
};

constexpr int S8_TILES = 32;  // 128-deep tiles whose scale bytes sit in LDS at a time

struct Linear8Plan {
  int splits;  // shares of K
};

inline Linear8Plan linear8_plan(int64_t M, int N, int K) {
  const int64_t tiles = (M + 127) / 128 * ((N + 127) / 128), kb = (K + 127) / 128;
  int splits = 1;
  while (tiles * splits * 2 <= 512 && kb / (splits * 2) >= 4) splits *= 2;
  return {splits};
}

}  // namespace nv
