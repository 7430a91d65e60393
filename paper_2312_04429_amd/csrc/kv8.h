// The 8-bit key / value cache: arguments of its kernels, and how attention's work is shared out.
#pragma once
#include <algorithm>
#include <cmath>
#include <cstdint>

namespace nv {

struct Kv8AppendArgs {
  const void *k, *v;
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
  int col_tiles, splits, tall;  // as in Kv8Plan
  float *part_o, *part_ml;    // per query and share: dh means; (reference maximum, sum)
};

constexpr int KV8_MAX_SPLITS = 256, KV8_FEW = 8;  // shares at most; joined by a thread up to
constexpr int KV8_SHARE = 4;                      // pages that a share has at least

struct Kv8Plan {
  int col_tiles;  // tiles of queries of a kv head
  int splits;     // shares of a row's pages
  int tall;       // 0: tiles of 16 queries; 1, 2: of 64, 128 that share each page
};

// us of a head's tiles of 64 * tall queries with their pages in `splits` shares.  A page takes a
// workgroup longer the more channels it has and when two share a compute unit (LDS: not past 128
// channels); shares end in partial results, written and read once, and a second launch.
inline double kv8_tall_cost(double rh, int64_t cols, int dh, int table_w, int tall, int splits) {
  const double wgs = rh * ((cols + 64 * tall - 1) / (64 * tall)) * splits;
  const int pages = std::max(std::min(table_w, KV8_SHARE), (table_w + splits - 1) / splits);
  const double size = 0.5 + 0.5 * dh / 128, one = pages * size * (tall == 1 ? 1.7 : 2.4),
               two = pages * size * (tall == 1 ? 2.0 : 2.6);
  double us;
  if (wgs <= 256.) us = 2. + one;
  else if (dh > 128) us = std::ceil(wgs / 256.) * (2. + one);
  else if (wgs <= 512.) us = 2. + two;
  else us = (wgs / 512. + 0.1) * (2. + two);
  return splits == 1 ? us : us + 3.5 + rh * cols * splits * dh * 8. / 3.5e6;
}

// Up to 32 queries a kv head, tiles of 16: their kernel's waves take pages of their own, and at most
// 16 of those are not worth a second launch; longer rows are shared out down to a page a wave until
// every compute unit has a workgroup, or two if the tiles alone are more than half as many: rows of
// differing length even out (one query over 200000 tokens of 8 heads of 128: 1271 us in one piece, 78
// in 32 shares, 84 in 128; 16 rows of 2048 to 8192: 38 with one, 41 with two a unit; 24 rows of
// as many, 8 heads of 64: 41 and 32; 16 rows of 1000: 12.2 in one piece, 13.2 in two).  Beyond
// that, of the tiles whose queries share a page (8 x 16 queries of 4 heads each, 4096 tokens: 34 us,
// tiles of 16 48; 24 queries of 100000 tokens 66, tiles of 16 49), the cheaper by the cost above: of
// 105 sizes (77 to 20000 tokens, dh 40 to 160) it takes 1.7 % more than the best measured choice on
// average, 16 % at most (of 30 with up to 32 queries 2.8 %, 16 % at most).  Shares stay within 1024
// workgroups, and so do the partial results (84 MB).
inline Kv8Plan kv8_plan(int64_t rows, int S, int heads, int kv_heads, int dh, int table_w) {
  // products of three sizes are taken in float64: they may pass 64 bits before they are refused
  const int64_t cols = (int64_t)S * (heads / kv_heads);
  const double rh = (double)(rows * kv_heads);
  Kv8Plan p{0, 1, 0};
  if (cols <= 32) {
    const double n = rh * ((cols + 15) / 16);
    if (table_w > 16)
      p.splits = (int)std::max(1., std::min((n <= 128. ? 256. : 512.) / n, table_w / 4.));
    p.splits = std::min(p.splits, KV8_MAX_SPLITS);
  } else {
    double best = 0.;
    for (int tall = 1; tall <= 2; ++tall)
      for (int s = 1; s == 1 || (s <= 128 && s <= table_w / 2 &&
                                 rh * ((cols + 64 * tall - 1) / (64 * tall)) * s <= 1024.); s *= 2) {
        const double c = kv8_tall_cost(rh, cols, dh, table_w, tall, s);
        if (p.tall == 0 || c < best) best = c, p.tall = tall, p.splits = s;
      }
  }
  const int64_t tile = p.tall ? 64 * p.tall : 16;
  p.col_tiles = (int)std::min<int64_t>((cols + tile - 1) / tile, 0x7FFFFFFF);
  return p;
}

}  // namespace nv
