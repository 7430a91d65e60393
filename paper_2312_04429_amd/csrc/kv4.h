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

constexpr int KV4_FEW_COLS = 256;  // queries a kv head that tiles of 16 are tried for

// us of a head's queries in tiles of 16 (tall 0: a workgroup's waves take pages of their own), 64 or 128 (tall
// 1, 2: they share each page), with their pages in `splits` shares.  A page takes a workgroup longer the
// more channels it has and when two share a compute unit (LDS: not past 128 channels); shares end in partial
// results, written and read once, and a second launch.
inline double kv4_cost(double rh, int64_t cols, int dh, int table_w, int tall, int splits) {
  const double base[3] = {3.5, 2.2, 2.5}, one[3] = {1.7, 1.3, 1.8}, two[3] = {2.2, 1.8, 2.5};
  const int64_t tile = tall ? 64 * tall : 16;
  const double wgs = rh * ((cols + tile - 1) / tile) * splits;
  const int pages = std::max(std::min(table_w, KV8_SHARE), (table_w + splits - 1) / splits);
  const double size = tall ? 0.36 + 0.64 * dh / 128 : 0.17 + 0.83 * dh / 128,
               steps = (tall ? pages : (pages + 3) / 4) * size;
  double us;
  if (wgs <= 256.) us = base[tall] + steps * one[tall];
  else if (dh > 128) us = std::ceil(wgs / 256.) * (base[tall] + steps * one[tall]);
  else us = std::max(1., wgs / 512.) * (base[tall] + steps * two[tall]);
  return splits == 1 ? us : us + 4.9 + rh * cols * splits * dh * 8. / 4.3e6;
}

// The cheapest of the three tiles and of 1, 2, 4 .. shares of at least four pages each, by the cost
// above.  Of 98 sizes (1 to 8192 queries a kv head, 2 to 1024 heads, 2 to 1024 pages, 64 and 128 channels,
// full rows) it takes 1.5 % more than the best measured choice on average, 15 % at most (one query over 65536
// tokens of 8 heads of 128: 345 us in one piece, 32 in 16 shares, 23 in 64; 256 queries over 4096: 20.3 in
// tiles of 16 with four shares, 22.8 in tiles of 64 with eight, 26 of 128 with sixteen).  Of 56 sizes of 32, 40,
// 80 and 160 channels, which it was not fitted to, 0.9 and 8 %; of 14 of 16 channels 4.5 %, 11 % at most but for
// one of 39 % (2 rows of 8 heads, 96 queries a head, 64 pages: 16.9 us in one piece, 12.2 in four shares).  A
// causal limit is not priced: every tile counts as the longest.  Shares stay within 1024 workgroups, and so do
// the partial results (84 MB).
inline Kv8Plan kv4_plan(int64_t rows, int S, int heads, int kv_heads, int dh, int table_w) {
  // products of three sizes are taken in float64: they may pass 64 bits before they are refused
  const int64_t cols = (int64_t)S * (heads / kv_heads);
  const double rh = (double)(rows * kv_heads);
  Kv8Plan p{0, 1, 0};
  double best = -1.;
  for (int tall = cols <= KV4_FEW_COLS ? 0 : 1; tall <= (cols <= 16 ? 0 : 2); ++tall) {
    const int64_t tile = tall ? 64 * tall : 16;
    for (int s = 1; s == 1 || (s <= KV8_MAX_SPLITS && s <= table_w / KV8_SHARE &&
                               rh * ((cols + tile - 1) / tile) * s <= 1024.); s *= 2) {
      const double c = kv4_cost(rh, cols, dh, table_w, tall, s);
      if (best < 0. || c < best) best = c, p.tall = tall, p.splits = s;
    }
  }
  const int64_t tile = p.tall ? 64 * p.tall : 16;
  p.col_tiles = (int)std::min<int64_t>((cols + tile - 1) / tile, 0x7FFFFFFF);
  return p;
}

}  // namespace nv
