// The 8-bit key / value cache: arguments of its kernels, and how attention's work is shared out.
#pragma once
#include <algorithm>
#include <cstdint>

namespace nv {

struct Kv8AppendArgs {
  const uint8_t *k, *v;       // 16-bit elements
  uint8_t *kp, *vp, *ks, *vs;
  int64_t ldk, k_row, ldv, v_row, n_pages;
  const int32_t *table, *pos, *count;
  int T, heads, dh, table_w;
};

struct Kv8AttnArgs {
  const void* q;
  int64_t ldq, q_row;
  const uint8_t *kp, *vp, *ks, *vs;
  int64_t n_pages;
  const int32_t *table, *lens, *qpos;
  int table_w, rows, S, heads, kv_heads, dh;
  float scale;
  void* out;
  int64_t ldo, o_row;
  int col_tiles, splits, tall;
  float *part_o, *part_ml;    // per query and share: dh sums; (reference maximum, sum)
};

struct Kv8Plan {
  int col_tiles;  // tiles of queries of a kv head
  int splits;     // shares of a row's pages
  int tall;       // 0: tiles of 16 queries; 1, 2: of 64, 128 that share each page
};

inline Kv8Plan kv8_plan(int64_t rows, int S, int heads, int kv_heads, int table_w) {
  const int64_t cols = (int64_t)S * (heads / kv_heads), rh = rows * kv_heads;
  if (cols > 32) {
    const int tall = rh * ((cols + 127) / 128) > 256 ? 2 : 1;
    Kv8Plan p{(int)((cols + 64 * tall - 1) / (64 * tall)), 1, tall};
    const int64_t want = 512 / (rh * p.col_tiles), can = table_w / 4;
    p.splits = (int)std::max<int64_t>(1, std::min<int64_t>(std::min(want, can), 128));
    return p;
  }
  Kv8Plan p{(int)((cols + 15) / 16), 1, 0};
  const int64_t want = std::max<int64_t>(1, 1024 / (rh * p.col_tiles));
  const int64_t can = std::max(1, table_w / 8);
  p.splits = (int)std::min<int64_t>(std::min(want, can), 256);
  return p;
}

}  // namespace nv
