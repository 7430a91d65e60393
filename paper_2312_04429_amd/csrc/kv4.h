// The 4-bit key / value cache: arguments of its kernels, and how attention's work is shared out.
#pragma once
#include "kv8.h"

namespace nv {

struct Kv4AppendArgs {
  const void *k, *v;
  uint8_t *kp, *vp, *ks, *vs;
  int64_t ldk, k_row, ldv, v_row, n_pages;
  const int32_t *table, *pos, *count;
  int T, heads, dh, table_w;
};

struct Kv4ReadArgs {
  const uint8_t *kp, *vp, *ks, *vs;
  int64_t n_pages;
  const int32_t *table, *pos, *count;
  void *k, *v;
  int64_t ldk, k_row, ldv, v_row;
  int T, heads, dh, table_w;
};

typedef Kv8AttnArgs Kv4AttnArgs;  // kp, vp: bytes of two codes; ks, vs: scale bytes of blocks

inline Kv8Plan kv4_plan(int64_t rows, int S, int heads, int kv_heads, int dh, int table_w) {
  Kv8Plan p = kv8_plan(rows, S, heads, kv_heads, dh, table_w);
  if (p.tall == 0 && table_w > 16) {
    const double n = (double)(rows * kv_heads) * p.col_tiles;
    p.splits = (int)std::max(1., std::min(512. / n, table_w / 4.));
    p.splits = std::min(p.splits, KV8_MAX_SPLITS);
  }
  return p;
}

}  // namespace nv
