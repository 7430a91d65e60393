// The 8-bit key / value cache: arguments of its kernels, and how attention's work is shared out.
#pragma once
#include <algorithm>
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
  float *part_o, *part_ml;    // per query and share: dh sums; (reference maximum, sum)
};

constexpr int KV8_MAX_SPLITS = 256, KV8_FEW = 8;  // shares at most; joined by a thread up to
constexpr int KV8_SHARE = 4;                      // pages that a share has at least

struct Kv8Plan {
  int col_tiles;  // tiles of queries of a kv head
  int splits;     // shares of a row's pages
  int tall;       // 0: tiles of 16 queries; 1, 2: of 64, 128 that share each page
};

// Tiles of 16 queries up to 32 queries a kv head (64: 1 to 4 % slower or equal either way), beyond
// that tiles of 128, or of 64 where 128 would leave compute units without a workgroup (1 x 2048
// queries, 16 heads of 128 over 4096 tokens, causal: 116 us against 131).  Pages are shared out until
// the chip has two workgroups a compute unit, where the table has 8 pages a share (4 for the larger
// tiles, whose pages take longer): 1 x 128 queries over 20000 tokens 505 -> 45 us, one query over
// 200000 tokens of 8 heads 84 us with 512 workgroups, 89 with 1024, 97 with 2048 (every share ends in
// a merge and a partial result).
inline Kv8Plan kv8_plan(int64_t rows, int S, int heads, int kv_heads, int table_w) {
  // products of three sizes are taken in float64: they may pass 64 bits before they are refused
  const int64_t cols = (int64_t)S * (heads / kv_heads), rh = rows * kv_heads;
  Kv8Plan p{};
  if (cols > 32) p.tall = (double)rh * ((cols + 127) / 128) > 256. ? 2 : 1;
  const int64_t tile = p.tall ? 64 * p.tall : 16, tiles = (cols + tile - 1) / tile;
  p.col_tiles = (int)std::min<int64_t>(tiles, 0x7FFFFFFF);
  const int64_t want = (int64_t)(512. / ((double)rh * tiles)), can = table_w / (p.tall ? 4 : 8);
  p.splits = (int)std::max<int64_t>(1, std::min<int64_t>(std::min(want, can), KV8_MAX_SPLITS));
  return p;
}

}  // namespace nv
