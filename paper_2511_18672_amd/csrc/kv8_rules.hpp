// How an attention call over the 8-bit cache is divided: plain C++ on sizes, so
// that it can be checked without a GPU.
#pragma once

#include <stdint.h>

#include <algorithm>

#include "sphinx.h"

namespace sphinx {

// The keys of segment i are cut into chunks[i] chunks of size[i] blocks (the last
// may hold fewer); a workgroup takes one chunk of one row tile and key/value
// head.  Segments of more than one chunk leave partial results, which a second
// kernel joins.
struct Kv8Plan {
  int tile;                                  // rows per workgroup, 32 or 128
  int waves;                                 // of a workgroup of a 32-row tile, 4 or 8
  int chunks[SPHINX_MAX_REQUESTS];           // at least 1
  int size[SPHINX_MAX_REQUESTS];             // blocks, at least 1
  int item[SPHINX_MAX_REQUESTS + 1];         // work items of the segments before (one head)
  int row[SPHINX_MAX_REQUESTS + 1];          // rows to join of the segments before (one head)
  int64_t part[SPHINX_MAX_REQUESTS + 1];     // partial rows of the segments before (all heads)
};

constexpr int kKv8Cus = 256;
// 32-row tiles: as many workgroups as run at once (three per CU at bf16 and
// head_dim 64, two else).  Chunks are evened out below their limit, which is four
// blocks at least, one for each wave: a segment's chunks (but its last) hold more
// than half of the limit, so three blocks at least.
constexpr int kKv8ItemsRows = 3 * kKv8Cus, kKv8MinChunkRows = 4;
// 128-row tiles: cut into this many workgroups at most, with a limit of eight blocks
// at least, so that a segment's chunks (but its last) hold five at least.
constexpr int kKv8ItemsTiles = 6 * kKv8Cus, kKv8MinChunkTiles = 8;

inline int kv8_tiles(int64_t rows, int tile) { return (int)((rows + tile - 1) / tile); }
inline int kv8_blocks(int tokens) { return (int)(((int64_t)tokens + 63) / 64); }

// Cuts every segment into chunks of at most `most` blocks.
inline void cut_kv8(Kv8Plan& p, int kv_heads, int nseg, const int64_t* rows, const int* klen, int64_t most) {
  for (int i = 0; i < nseg; ++i) {
    const int nb = std::max(1, kv8_blocks(klen[i]));
    p.chunks[i] = (int)((nb + most - 1) / most);
    p.size[i] = (nb + p.chunks[i] - 1) / p.chunks[i];
    p.chunks[i] = (nb + p.size[i] - 1) / p.size[i];  // no empty chunk
    const bool split = p.chunks[i] > 1;
    p.item[i + 1] = p.item[i] + kv8_tiles(rows[i], p.tile) * p.chunks[i];
    p.row[i + 1] = p.row[i] + (split ? (int)rows[i] : 0);
    p.part[i + 1] = p.part[i] + (split ? rows[i] * kv_heads * p.chunks[i] : 0);
  }
}

// rows[i]: queries times group of segment i; klen[i]: its tokens that count.
inline Kv8Plan plan_kv8(bool bf16, int kv_heads, int head_dim, int nseg, const int64_t* rows, const int* klen) {
  Kv8Plan p = {};
  int64_t small = 0, tall = 0;  // blocks times tiles of 32 and of 128 rows
  int longest = 1;
  for (int i = 0; i < nseg; ++i) {
    small += (int64_t)kv8_tiles(rows[i], 32) * kv8_blocks(klen[i]);
    tall += (int64_t)kv8_tiles(rows[i], 128) * kv8_blocks(klen[i]);
    longest = std::max(longest, kv8_blocks(klen[i]));
  }
  // a 128-row tile takes about 2.4 times a 32-row tile's time
  p.tile = bf16 && 5 * small > 12 * tall ? 128 : 32;
  p.waves = 4;
  if (p.tile == 32) {
    int64_t units = 0;
    for (int i = 0; i < nseg; ++i) units += (int64_t)kv8_tiles(rows[i], 32) * kv_heads;
    // Small calls: eight waves take up to three blocks each, at about 1.7 us a block,
    // in one launch instead of two.  One query of 8 heads, calls in a stream, whole
    // and cut: 1100 keys 8.8 us and 10.6, 1500 keys 9.9 and 10.7, 2048 keys 11.3 and
    // 10.6; the kernels of a captured graph, without the caller's time for a second
    // launch: 7.9 and 7.3, 9.1 and 7.8, 10.5 and 8.1.
    if (bf16 && units <= kKv8Cus && longest <= 24) {
      p.waves = 8;
      cut_kv8(p, kv_heads, nseg, rows, klen, longest);
      return p;
    }
    // Chunks of equal work for all workgroups that run at once, counting that cutting
    // leaves half a chunk per tile on average.  fp32: where tiles fill the chip, one
    // workgroup per CU, a cut for a second one gains less than its join costs (1024
    // queries against 2048 keys of 8 heads, 256 tiles: 50 us in two chunks, 48 us whole).
    const int64_t slots = bf16 && head_dim == 64 ? kKv8ItemsRows : !bf16 && units >= kKv8Cus ? kKv8Cus : 2 * kKv8Cus;
    const int64_t pieces = bf16 ? std::max(slots - units / 2, slots / 2) : slots;
    cut_kv8(p, kv_heads, nseg, rows, klen,
            std::max<int64_t>((small * kv_heads + pieces - 1) / pieces, kKv8MinChunkRows));
    return p;
  }
  // The number of chunks of the longest segment with the least estimated time, in
  // blocks of one workgroup: a CU gets through its workgroups' blocks one after
  // the other, those of equal chunks come in whole numbers per CU, and the last
  // one alone does not fill it (16 heads against 504 blocks: 324, 550, 760, 988 us
  // for 1, 2, 3, 4 workgroups per CU); three blocks' time goes by around a chunk.
  // Joining moves each partial row twice, at about 4 TB/s, after a launch of 3 us.
  const double block_us = head_dim == 64 ? 0.47 : 0.63;
  Kv8Plan best = p;
  double least = 0.0;
  for (int k = 1; k <= longest; k += k < 6 ? 1 : k / 3) {
    const int most = std::max(kKv8MinChunkTiles, (longest + k - 1) / k);
    Kv8Plan q = p;
    cut_kv8(q, kv_heads, nseg, rows, klen, most);
    double total = 0.0;
    int64_t cut = 0;
    for (int i = 0; i < nseg; ++i) {
      const int64_t n = (int64_t)(q.item[i + 1] - q.item[i]) * kv_heads;
      total += (double)n * (q.size[i] + 3);
      if (q.chunks[i] > 1) cut += n;
    }
    if (cut > kKv8ItemsTiles) break;
    const int64_t rounds = (int64_t)(total / ((double)kKv8Cus * (most + 3)) + 0.999);
    const double join = q.part[nseg] == 0 ? 0.0 : 3.0 + (double)q.part[nseg] * (head_dim * 4 + 8) * 2.0 / 4e6;
    const double us = ((double)rounds + 0.36) * (most + 3) * block_us + join;
    if (k == 1 || us < least) {
      least = us;
      best = q;
    }
    if (most == kKv8MinChunkTiles) break;
  }
  return best;
}

// Partial rows that no plan for these segments passes, with any klen up to the
// given one.  No limit of a chunk is below four blocks, so a segment has no more
// chunks than fours of blocks.  32-row tiles: a cut segment has less than twice
// its blocks over the limit as chunks, so less than twice the items leave partial
// rows; each item leaves one tile's.
inline int64_t kv8_most_parts(int kv_heads, int nseg, const int64_t* rows, const int* klen) {
  int64_t by_chunk = 0, by_item = 0;
  for (int i = 0; i < nseg; ++i) {
    by_item = std::max(by_item, std::max(2 * kKv8ItemsRows * std::min<int64_t>(rows[i], 32),
                                         kKv8ItemsTiles * std::min<int64_t>(rows[i], 128)));
    const int64_t chunks = (kv8_blocks(klen[i]) + kKv8MinChunkRows - 1) / kKv8MinChunkRows;
    if (chunks > 1) by_chunk += rows[i] * kv_heads * chunks;
  }
  return std::min(by_chunk, by_item);
}

}  // namespace sphinx
