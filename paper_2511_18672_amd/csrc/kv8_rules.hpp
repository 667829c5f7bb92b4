// How an attention call over the 8-bit cache is divided: plain C++ on sizes, so
// that it can be checked without a GPU.
#pragma once

#include <stdint.h>

#include <algorithm>

#include "sphinx.h"

namespace sphinx {

// The keys of a segment are cut into chunks of `chunk` blocks; a workgroup takes
// one chunk of one row tile and key/value head.  Segments of more than one chunk
// leave partial results, which a second kernel joins.
struct Kv8Plan {
  int tile;                                  // rows per workgroup, 32 or 128
  int chunk;                                 // blocks per chunk
  int chunks[SPHINX_MAX_REQUESTS];           // of a segment, at least 1
  int item[SPHINX_MAX_REQUESTS + 1];         // work items of the segments before (one head)
  int row[SPHINX_MAX_REQUESTS + 1];          // rows to join of the segments before (one head)
  int64_t part[SPHINX_MAX_REQUESTS + 1];     // partial rows of the segments before (all heads)
};

// Workgroups that a call is cut into where its keys allow, and the blocks that a
// chunk holds at least.  32-row tiles: four workgroups per CU, a block for each of
// their waves.  128-row tiles: as many workgroups as run at once, three per CU (two
// at head_dim 72), and eight blocks for the work around a chunk.
constexpr int kKv8ItemsRows = 1024, kKv8MinChunkRows = 4;
constexpr int kKv8ItemsTiles = 768, kKv8ItemsTiles72 = 512, kKv8MinChunkTiles = 8;

inline int kv8_tiles(int64_t rows, int tile) { return (int)((rows + tile - 1) / tile); }
inline int kv8_blocks(int tokens) { return (int)(((int64_t)tokens + 63) / 64); }

// rows[i]: queries times group of segment i; klen[i]: its tokens that count.
inline Kv8Plan plan_kv8(bool bf16, int kv_heads, int head_dim, int nseg, const int64_t* rows, const int* klen) {
  Kv8Plan p = {};
  int64_t small = 0, tall = 0;  // blocks times tiles of 32 and of 128 rows
  for (int i = 0; i < nseg; ++i) {
    small += (int64_t)kv8_tiles(rows[i], 32) * kv8_blocks(klen[i]);
    tall += (int64_t)kv8_tiles(rows[i], 128) * kv8_blocks(klen[i]);
  }
  // a 128-row tile takes about 2.4 times a 32-row tile's time
  p.tile = bf16 && 5 * small > 12 * tall ? 128 : 32;
  const int64_t work = (p.tile == 128 ? tall : small) * kv_heads;
  const int items = p.tile == 32 ? kKv8ItemsRows : head_dim == 64 ? kKv8ItemsTiles : kKv8ItemsTiles72;
  const int least = p.tile == 32 ? kKv8MinChunkRows : kKv8MinChunkTiles;
  // no segment has 2^26 blocks
  p.chunk = (int)std::clamp<int64_t>((work + items - 1) / items, least, 1 << 26);
  for (int i = 0; i < nseg; ++i) {
    p.chunks[i] = std::max(1, (kv8_blocks(klen[i]) + p.chunk - 1) / p.chunk);
    const bool split = p.chunks[i] > 1;
    p.item[i + 1] = p.item[i] + kv8_tiles(rows[i], p.tile) * p.chunks[i];
    p.row[i + 1] = p.row[i] + (split ? (int)rows[i] : 0);
    p.part[i + 1] = p.part[i] + (split ? rows[i] * kv_heads * p.chunks[i] : 0);
  }
  return p;
}

// Partial rows that no plan for these segments passes, with any klen up to the
// given one.  A chunk holds four blocks at least; and only segments of more than
// `chunk` blocks are cut, into fewer than 2 blocks / chunk pieces, so that at
// most twice the items above leave partial rows, one tile each.
inline int64_t kv8_most_parts(int kv_heads, int nseg, const int64_t* rows, const int* klen) {
  int64_t by_chunk = 0, by_item = 0;
  for (int i = 0; i < nseg; ++i) {
    by_item = std::max(by_item, std::max(2 * kKv8ItemsRows * std::min<int64_t>(rows[i], 32),
                                         2 * kKv8ItemsTiles * std::min<int64_t>(rows[i], 128)));
    const int64_t chunks = (kv8_blocks(klen[i]) + kKv8MinChunkRows - 1) / kKv8MinChunkRows;
    if (chunks > 1) by_chunk += rows[i] * kv_heads * chunks;
  }
  return std::min(by_chunk, by_item);
}

}  // namespace sphinx
