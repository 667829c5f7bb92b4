// How a product of 8-bit matrices is divided: plain C++ on sizes, so that it can
// be checked without a GPU.
#pragma once

#include <stdint.h>

#include <algorithm>

namespace sphinx {

// Tiles of outputs: 256x256 and 192x256 in eight waves, one per CU; 128x128 and
// 128x64 (two per CU) and 64x64 (four) in four waves; up to 16 rows by 16
// columns.
enum Q8Tile { kQ8Tile256, kQ8Tile192, kQ8Tile128, kQ8Tile128x64, kQ8Tile64, kQ8Few };

// What becomes of the outputs: bf16 or fp32 values, an fp32 residual that they
// are added to through a gate, or a matrix in 8 bits.
enum Q8Kind { kQ8Bf16, kQ8F32, kQ8Gated, kQ8Bytes };

struct Q8Plan {
  Q8Tile tile;
  int pieces;  // the contraction is cut into so many, which a second kernel adds up
};

constexpr int kQ8Cus = 256;

struct Q8TileCost {
  int rows, cols, per_cu;
  double start, gelu;  // us of a round of tiles: start (and GELU) + blocks of 128 of the contraction
  double block, alone;  // a block where every slot, and where one of a CU, has a tile
};

// Fitted on 24 products (17 where the kind asks for whole blocks of columns) of
// M 64 to 32256, N 64 to 8192 and K 200 to 32256 with a bias, each in a stream of
// equal launches: 5 to 15 % rms.  The choice by them costs 1 % on average against
// the fastest of the tiles, and 15 % at most (fp32, 4800 x 1152 x 1152: 23 us, 20).
inline const Q8TileCost& q8_tile_cost(Q8Kind kind, int tile) {
  static const Q8TileCost cost[4][5] = {
      {{256, 256, 1, 9.1, 2.8, 1.35, 1.09}, {192, 256, 1, 7.7, 2.0, 1.10, 0.87}, {128, 128, 2, 5.5, 0.9, 0.86, 0.50},
       {128, 64, 2, 4.4, 0.4, 0.67, 0.42}, {64, 64, 4, 4.1, 0.3, 0.84, 0.30}},
      {{}, {192, 256, 1, 11.1, 1.6, 2.01, 1.61}, {128, 128, 2, 7.8, 1.1, 1.44, 0.71},
       {128, 64, 2, 5.0, 0.7, 0.89, 0.48}, {64, 64, 4, 4.4, 0.5, 1.06, 0.36}},
      {{256, 256, 1, 15.5, 2.8, 2.54, 1.10}, {192, 256, 1, 12.6, 2.0, 1.55, 0.89}, {128, 128, 2, 8.0, 0.9, 1.13, 0.55},
       {128, 64, 2, 4.5, 0.4, 0.74, 0.51}, {64, 64, 4, 3.4, 0.3, 0.94, 0.37}},
      {{256, 256, 1, 10.4, 2.8, 1.54, 1.14}, {192, 256, 1, 8.8, 2.0, 1.13, 0.93}, {128, 128, 2, 5.0, 0.9, 0.95, 0.57},
       {}, {}}};
  return cost[kind][tile];
}

// fp32 outputs have no 256x256, whose fragments in bf16 would spill; outputs in 8 bits
// need tiles of whole blocks of 128 columns; few rows have a kernel for values only.
constexpr bool q8_has_tile(Q8Kind kind, Q8Tile t) {
  if (t == kQ8Few) return kind == kQ8Bf16 || kind == kQ8F32;
  return kind == kQ8F32 ? t != kQ8Tile256 : kind != kQ8Bytes || t <= kQ8Tile128;
}

// Only bf16 and fp32 outputs have a second kernel that joins pieces.  whole: there is
// no workspace for them (the refinement step's QKV product, whose contraction of up to
// 16 blocks is not worth cutting: with a workspace the plan would be the same).
inline Q8Plan plan_q8_matmul(Q8Kind kind, bool gelu, int M, int N, int KB, bool whole = false) {
  const bool values = kind == kQ8Bf16 || kind == kQ8F32, whole_k = whole || !values;
  Q8Plan best = {kQ8Tile128, 1};
  if (values && M <= 16 && N <= (1 << 22)) return Q8Plan{kQ8Few, 1};
  double us = 1e30;
  for (int t = 0; t < 5; ++t) {
    if (!q8_has_tile(kind, (Q8Tile)t)) continue;
    const Q8TileCost& c = q8_tile_cost(kind, t);
    const int64_t tiles = (int64_t)((M + c.rows - 1) / c.rows) * ((N + c.cols - 1) / c.cols);
    if (tiles >= (1 << 23)) continue;  // more threads than a launch can have
    for (int pieces = 1; pieces <= (whole_k ? 1 : 16); pieces *= 2) {
      const int per = pieces == 1 ? KB : ((KB + pieces - 1) / pieces + 3) / 4 * 4;
      if (pieces > 1 && ((pieces - 1) * per >= KB || per < 8)) break;  // no empty piece
      const int64_t slots = (int64_t)kQ8Cus * c.per_cu, n = tiles * pieces;
      const int64_t full = n / slots, rem = n % slots;
      // a last round of one tile per CU runs faster than a full one
      const double start = c.start + (gelu && pieces == 1 ? c.gelu : 0.0);
      const double whole = start + per * c.block, lone = start + per * c.alone;
      const double last = rem == 0 ? 0.0 : rem <= kQ8Cus ? lone : lone + (whole - lone) * (double)(rem - kQ8Cus) / (slots - kQ8Cus);
      double cost = full * whole + last;
      // the pieces' sums are written and read back (5 TB/s), in a launch of its own
      if (pieces > 1) cost += 3.0 + (double)pieces * M * N * 8.0 / 5e6;
      if (cost < us) {
        us = cost;
        best = Q8Plan{(Q8Tile)t, pieces};
      }
    }
  }
  return best;
}

}  // namespace sphinx
