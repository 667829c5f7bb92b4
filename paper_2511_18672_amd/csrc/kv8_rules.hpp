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
  int chunk;                                 // blocks per chunk
  int chunks[SPHINX_MAX_REQUESTS];           // of a segment, at least 1
  int item[SPHINX_MAX_REQUESTS + 1];         // work items of the segments before (one head)
  int row[SPHINX_MAX_REQUESTS + 1];          // rows to join of the segments before (one head)
  int64_t part[SPHINX_MAX_REQUESTS + 1];     // partial rows of the segments before (all heads)
};

constexpr int kKv8RowTile = 32;     // rows per workgroup
constexpr int kKv8Items = 1024;     // workgroups that a call is cut into where its keys allow
constexpr int kKv8MinChunk = 4;     // blocks: one for each wave of a workgroup

inline int kv8_tiles(int64_t rows) { return (int)((rows + kKv8RowTile - 1) / kKv8RowTile); }
inline int kv8_blocks(int tokens) { return (int)(((int64_t)tokens + 63) / 64); }

// rows[i]: queries times group of segment i; klen[i]: its tokens that count.
inline Kv8Plan plan_kv8(int kv_heads, int nseg, const int64_t* rows, const int* klen) {
  Kv8Plan p = {};
  int64_t work = 0;
  for (int i = 0; i < nseg; ++i) work += (int64_t)kv8_tiles(rows[i]) * kv8_blocks(klen[i]) * kv_heads;
  // no segment has 2^26 blocks
  p.chunk = (int)std::clamp<int64_t>((work + kKv8Items - 1) / kKv8Items, kKv8MinChunk, 1 << 26);
  for (int i = 0; i < nseg; ++i) {
    p.chunks[i] = std::max(1, (kv8_blocks(klen[i]) + p.chunk - 1) / p.chunk);
    const bool split = p.chunks[i] > 1;
    p.item[i + 1] = p.item[i] + kv8_tiles(rows[i]) * p.chunks[i];
    p.row[i + 1] = p.row[i] + (split ? (int)rows[i] : 0);
    p.part[i + 1] = p.part[i] + (split ? rows[i] * kv_heads * p.chunks[i] : 0);
  }
  return p;
}

// Partial rows that no plan for these segments passes, with any klen up to the
// given one.  A chunk holds kKv8MinChunk blocks at least; and only segments of
// more than `chunk` blocks are cut, into fewer than 2 blocks / chunk pieces, so
// that at most 2 kKv8Items work items leave partial rows, one tile each.
inline int64_t kv8_most_parts(int kv_heads, int nseg, const int64_t* rows, const int* klen) {
  int64_t by_chunk = 0, tall = 0;
  for (int i = 0; i < nseg; ++i) {
    tall = std::max(tall, std::min<int64_t>(rows[i], kKv8RowTile));
    const int64_t chunks = (kv8_blocks(klen[i]) + kKv8MinChunk - 1) / kKv8MinChunk;
    if (chunks > 1) by_chunk += rows[i] * kv_heads * chunks;
  }
  return std::min(by_chunk, 2 * (int64_t)kKv8Items * tall);
}

}  // namespace sphinx
