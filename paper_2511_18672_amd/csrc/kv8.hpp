// The 8-bit key/value cache: its layout and the launchers of its kernels.
//
// A slice holds the keys and values of one denoiser block: kv_heads heads of d
// dims (64 or 72) for the tokens of up to SPHINX_MAX_REQUESTS segments.  The
// tokens of a segment are grouped in blocks of 64 from its first one, so a
// block never holds two segments' tokens and what a segment's part of the cache
// holds does not depend on what it is packed with.  (How an attention call is
// divided does, and so the order of its sums: kv8_rules.hpp.)  Block b of head h is a tile of 64 d bytes of keys
// and one of 64 d bytes of values at (h nblk + b) 2 64 d; behind all tiles,
// from a 256-byte boundary, one byte per (head, block, keys | values) holds the
// block's scale 2^(byte - 127).  A zeroed slice holds zeros.
//
// Bytes stand in the operand order of the 32-row matrix instructions, so that
// a wave loads a fragment as consecutive 16-byte chunks, one per lane
// (lane l = 32 g + r):
//   keys    chunk (2 rb + hf) 64 + l: row 32 rb + r, dims 32 g + 16 hf .. + 15
//           head_dim 72: behind these, row by row, dims 64 .. 71
//   values  chunk (2 db + kb) 64 + l: dim 32 db + r, byte 8 hf + j the key
//           32 kb + 16 hf + 8 (j / 4) + 4 g + j % 4, which is where score
//           register 8 hf + j of a 32x32 tile of K Q^T has its key
//           head_dim 72: behind these, chunk (2 kb + g) 8 + i: dim 64 + i
#pragma once

#include "common.hpp"

namespace sphinx {

constexpr int kKv8Block = 64;

// Segments of a slice: first token and first block of each.
struct Kv8Segs {
  int nseg;
  int tok[SPHINX_MAX_REQUESTS + 1];
  int blk[SPHINX_MAX_REQUESTS + 1];
};

struct Kv8Slice {
  unsigned char* tiles;
  unsigned char* scales;
  int kv_heads;
  int64_t nblk;
};

inline size_t kv8_scale_offset(int kv_heads, int head_dim, int64_t nblk) {
  const size_t tiles = (size_t)kv_heads * (size_t)nblk * 2 * kKv8Block * (size_t)head_dim;
  return (tiles + 255) & ~(size_t)255;
}
inline size_t kv8_slice_bytes(int kv_heads, int head_dim, int64_t nblk) {
  return kv8_scale_offset(kv_heads, head_dim, nblk) + (((size_t)kv_heads * (size_t)nblk * 2 + 255) & ~(size_t)255);
}

// Rows of k and v: row j at element j ld, head h at dims h d (both operands).
struct Kv8Rows {
  const int32_t* idx;  // token of each row, ascending, or NULL: row j is token j
  int n;
  int64_t ld;
};

// kv8_cache.hip
hipError_t launch_kv8_store(sphinx_dtype dt, int head_dim, const Kv8Segs& S, const Kv8Slice& c, const Kv8Rows& rows,
                            const void* k, const void* v, hipStream_t s);
hipError_t launch_kv8_load(sphinx_dtype dt, int head_dim, const Kv8Segs& S, const Kv8Slice& c, const Kv8Rows& rows,
                           void* k, void* v, hipStream_t s);

// One attention call: segment i (of those with queries, most keys first) has
// queries [q0[i], q0[i] + nq[i]), which attend to the first klen[i] tokens of
// the slice's segment that starts at block blk[i].  A row is a query of one of
// the `group` query heads that share a key/value head.
struct Kv8Attn {
  const void* q;
  void* o;
  int64_t ldq, ldo;
  int group;  // query heads per key/value head
  int nseg;
  int q0[SPHINX_MAX_REQUESTS];
  int nq[SPHINX_MAX_REQUESTS];
  int klen[SPHINX_MAX_REQUESTS];
  int blk[SPHINX_MAX_REQUESTS];
};

// kv8_attention.hip
// Workspace of a call with these segments, whatever part of their tokens counts
// (klen up to the given ones).
size_t kv8_attention_ws_bytes(int kv_heads, int head_dim, int group, int nseg, const int* nq, const int* klen);
hipError_t launch_kv8_attention(sphinx_dtype dt, int head_dim, const Kv8Attn& A, const Kv8Slice& c, void* ws,
                                hipStream_t s);

}  // namespace sphinx
