// How a product of 8-bit matrices is divided: plain C++ on sizes, so that it can
// be checked without a GPU.
#pragma once

#include <stdint.h>

#include <algorithm>

namespace sphinx {

// Tiles of outputs: 256x256 and 192x256 in eight waves, one per CU; 128x128 and
// 128x64 (two per CU) and 64x64 (four) in four waves.
enum Q8Tile { kQ8Tile256, kQ8Tile192, kQ8Tile128, kQ8Tile128x64, kQ8Tile64 };

struct Q8Plan {
  Q8Tile tile;
  int pieces;  // the contraction is cut into so many, which a second kernel adds up
};

constexpr int kQ8Cus = 256;

struct Q8TileCost {
  int rows, cols, per_cu;
  double start, block;  // us of a round of tiles: start + blocks of 128 of the contraction
  double alone;         // `block` where a CU has one tile
};

// Fitted on products of M 64 to 32256, N 64 to 8192 and K 200 to 32256, each in
// a stream of equal launches.
inline const Q8TileCost& q8_tile_cost(bool f32, int tile) {
  static const Q8TileCost bf16[] = {{256, 256, 1, 6.6, 1.52, 1.35}, {192, 256, 1, 7.4, 1.04, 1.02},
                                    {128, 128, 2, 4.7, 0.86, 0.60}, {128, 64, 2, 4.0, 0.62, 0.42},
                                    {64, 64, 4, 3.5, 0.88, 0.22}};
  static const Q8TileCost wide[] = {{256, 256, 1, 1e9, 0, 0},       {192, 256, 1, 9.0, 2.1, 2.1},
                                    {128, 128, 2, 6.5, 1.62, 0.92}, {128, 64, 2, 5.0, 0.95, 0.58},
                                    {64, 64, 4, 4.5, 1.15, 0.33}};
  return f32 ? wide[tile] : bf16[tile];
}

inline Q8Plan plan_q8_matmul(bool f32, int M, int N, int KB) {
  Q8Plan best = {kQ8Tile64, 1};
  double us = 1e30;
  for (int t = 0; t < 5; ++t) {
    const Q8TileCost& c = q8_tile_cost(f32, t);
    const int64_t tiles = (int64_t)((M + c.rows - 1) / c.rows) * ((N + c.cols - 1) / c.cols);
    for (int pieces = 1; pieces <= 16; pieces *= 2) {
      const int per = ((KB + pieces - 1) / pieces + 3) / 4 * 4;
      if (pieces > 1 && ((pieces - 1) * per >= KB || per < 8)) break;  // no empty piece
      const int64_t slots = (int64_t)kQ8Cus * c.per_cu, n = tiles * pieces;
      const int64_t full = n / slots, rem = n % slots;
      // a last round of one tile per CU runs faster than a full one
      const double whole = c.start + per * c.block, lone = c.start + per * c.alone;
      const double last = rem == 0 ? 0.0 : rem <= kQ8Cus ? lone : lone + (whole - lone) * (double)(rem - kQ8Cus) / (slots - kQ8Cus);
      double cost = full * whole + last;
      // the pieces' sums are written and read back (4 TB/s), in a launch of its own
      if (pieces > 1) cost += 4.0 + (double)pieces * M * N * 8.0 / 4e6;
      if (cost < us) {
        us = cost;
        best = Q8Plan{(Q8Tile)t, pieces};
      }
    }
  }
  return best;
}

}  // namespace sphinx
