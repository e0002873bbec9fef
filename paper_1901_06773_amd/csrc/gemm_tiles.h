// The order of a launch's tiles and which tiles the bf16 products of gemm_bf16.h are cut in.
#pragma once
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "sizes.h"

namespace acc {

// Tile `at` of a launch: every XCD takes a contiguous range (neighbours share operand rows in its L2), rows innermost.
__device__ __forceinline__ int xcd_tile(int blocks) { return ((int)blockIdx.x & 7) * (blocks >> 3) + ((int)blockIdx.x >> 3); }

// Which tile: columns in blocks of four, within a block row by row, so that the workgroups of an XCD that run at the same time (thirty-two) stand eight by
// four and share operand rows both ways.
struct TileAt { int m, n; };
__device__ __forceinline__ TileAt tile_at(int at, int tiles_m, int tiles) {
  const int block = at / (4 * tiles_m), in = at - block * 4 * tiles_m, left = tiles / tiles_m - 4 * block, width = left < 4 ? left : 4, m = in / width;
  return TileAt{m, 4 * block + in - m * width};
}

// Which tiles: the ones with the smallest predicted time, microseconds, from the tiles of the busiest compute unit and the steps of 64 values of k
// (times the parts of A).  256 x 256 has a compute unit to itself, of the others two workgroups share one.  Constants from eleven shapes (41 to 8000 rows, widths
// 256 to 4096, 1000 to 50001 classes), every tile on each; measured, 256 / 128 / 64: logits and sums, 777 x 1160 x 50001 154 / 145 / 234, 1000 x 2048 x 1000
// 46 / 26 / 12, 4096 x 1024 x 8192 68 / 73 / 152; dw, 2000 x 512 x 20000 127 / 168 / 261, 41 x 2048 x 1000 10.9 / 6.4 / 4.8.
struct TileCost {
  double first, first_step, next, next_step;
};
enum { RowsByRows = 0, ByColumns };            // both operands along k, in steps of 64; B in rows of k, steps of 32 (dx, dw)
inline constexpr TileCost kCost[2][3] = {{{4.0, 1.28, 8.0, 1.60}, {3.0, 0.62, 3.2, 0.50}, {1.5, 0.31, 1.7, 0.205}},
                                  {{4.0, 1.30, 12.0, 1.50}, {3.0, 0.62, 5.0, 0.55}, {1.5, 0.31, 1.0, 0.28}}};
inline constexpr int kTiles[3] = {256, 128, 64};
inline double tile_us(int kind, int t, long tiles, double steps) {
  const long most = ceil_div(tiles, 256);
  const TileCost& c = kCost[kind][t];
  const double first = c.first + c.first_step * steps, next = c.next + c.next_step * steps;
  if (t == 0) return 3.0 + first + (most - 1) * next;
  auto round = [&](long r) { return r == 0 ? 0.0 : first > r * next ? first : r * next; };
  return 3.0 + (most / 2) * round(2) + round(most % 2);
}
// Tiles and, for a product whose sum over k may be cut, parts of `step` values of k or more, whose sums cost writing and reading
struct Choice {
  int tile, splits, k;           // k: values of it in one part
  double us;                     // predicted
};
inline Choice choose(int kind, long m, long n, long k, int parts, long most_sums, long step, int first = 0) {
  Choice best{256, 1, (int)up(k, 64), 0.0};
  double us = 0;
  for (int t = first; t < 3; ++t) {
    const long tiles = ceil_div(m, kTiles[t]) * ceil_div(n, kTiles[t]);
    // cuts in one to sixty-four, and those that fill the compute units once, twice and four times
    for (int i = 0; i < 10; ++i) {
      const long s = i < 7 ? 1L << i : (256L << (i - 7)) / tiles;
      if (s < 1) continue;
      const long each = up(ceil_div(k, s), 64), splits = ceil_div(k, each);
      if (s > 1 && (each < step || splits * m * n > most_sums)) continue;
      const double sums = splits > 1 ? (first ? 5.0 : 2.0) + (double)splits * m * n * 8 / 6e6 : 0.0;      // (5: a launch for them alone)
      const double v = tile_us(kind, t, tiles * splits, each / 64.0 * parts) + sums;
      if (us == 0 || v < us) {
        us = v;
        best = Choice{kTiles[t], (int)splits, (int)each, v};
      }
    }
  }
  return best;
}

}  // namespace acc
