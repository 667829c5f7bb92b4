// Attention over the 8-bit key/value cache (layout: kv8.hpp): per segment and
// query head o = sum_t 2^(q.k_t) v_t / sum_t 2^(q.k_t) over the segment's cached
// tokens, keys and values being the numbers that the cache's bytes stand for.

#include <cfloat>

#include <algorithm>
#include <type_traits>

#include "kv8.hpp"
#include "kv8_rules.hpp"

namespace sphinx {

namespace {
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
constexpr int kTPB = 256;
constexpr int kRows = 32;  // rows (queries of the heads that share a key/value head) per workgroup

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// Largest of 32 scores of a lane and of the lane 32 further (its row's other keys).
__device__ __forceinline__ float row_max(const f32x16& a, const f32x16& b) {
  float x = fmaxf(a[0], b[0]);
#pragma unroll
  for (int i = 1; i < 16; ++i) x = fmaxf(x, fmaxf(a[i], b[i]));
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// Segment of a work item or of a row to join: the last whose first one (of the
// prefix sums `first`) is not behind it.
__device__ __forceinline__ int find_segment(const int* first, int nseg, int at) {
  int lo = 0, hi = nseg - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (first[mid] <= at) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// Partial results: row r of head h, chunk j of segment i is number
// part[i] + (h rows_i + r) chunks_i + j: its running maximum and sum, and O.
struct Parts {
  float2* ml;
  float* o;  // [number][head_dim]
};

// A cleared block has byte 0 and holds zeros, at any scale.
__device__ __forceinline__ float byte_scale(int b) { return __uint_as_float((uint32_t)max(b, 1) << 23); }

// Sixteen stored bytes as operands: two bf16 fragments of eight, which hold the
// scaled values exactly (the scale is a power of two), or 16 floats.
__device__ __forceinline__ void operand(const uint4& b, float scale, bf16x8 (&f)[2]) {
  const uint32_t w[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], scale, false);
    const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], scale, true);
    f[i >> 1][4 * (i & 1)] = lo[0];
    f[i >> 1][4 * (i & 1) + 1] = lo[1];
    f[i >> 1][4 * (i & 1) + 2] = hi[0];
    f[i >> 1][4 * (i & 1) + 3] = hi[1];
  }
}
__device__ __forceinline__ void operand(const uint4& b, float (&f)[16]) {  // without the scale
  const uint32_t w[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], false);
    const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], true);
    f[4 * i] = lo[0];
    f[4 * i + 1] = lo[1];
    f[4 * i + 2] = hi[0];
    f[4 * i + 3] = hi[1];
  }
}

// One workgroup = 32 rows of one segment and key/value head against one chunk of
// the segment's keys; its four or eight waves take the chunk's blocks in turn and merge
// (m, l, O) through LDS.  A wave reads a block's bytes straight into the operand
// layouts, the next block's while it works on this one's:
//  * S^T = K Q^T in two 32-key tiles: lane l = 32 g + r has key r and dims
//    32 g .. + 31 (two chunks), for the queries the same dims of row r;
//  * P^T needs no move: score register 8 hf + j of tile kb belongs to the key
//    that byte 8 hf + j of the values' chunk (db, kb) holds;
//  * O^T = V^T P^T leaves the row on the lane.
// bf16: 32x32x16 products, P as the sum of two bf16 numbers, which is off by at most
// 2^-15 of it, so that o's own rounding is all that a result shows.  (One bf16 number
// costs errors of 1.2e-3 to 1.5e-3 beside o's 1.7e-3 and saves half of the V^T P^T
// products and the splitting, next to which the bytes come: one query against 2^20
// keys 102.5 instead of 105.2 us, 32 queries of 16 heads against 32256 keys 22.9
// instead of 24.3, one against 1500 8.7 instead of 9.8.)
// f32: 32x32x2 products of the unscaled bytes, nothing rounded (the keys' scale goes
// into the exponent, the values' into P: a product per byte between its conversion
// and its matrix instruction kept the two from overlapping).
// bf16 is bound by the cache's bytes: one query against 2^20 keys of 4 heads takes
// 95 us (5.6 TB/s), 48 sequences of 32 heads on 4 73 us.  f32 is bound by the matrix
// instructions and what stands between them in the one wave of a SIMD: 1024 queries
// against 2048 keys of 8 heads take 44 us, the matrix cores busy for 52 % of it, 4000
// against 4000 296 us (111 TFLOP/s).
template <typename T, int HD, int WAVES>
__global__ __launch_bounds__(64 * WAVES, sizeof(T) == 2 && HD == 64 && WAVES == 4 ? 3 : 2) void k_kv8_attn_rows(Kv8Attn A, Kv8Slice c, Kv8Plan P, Parts part, int first) {
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int DB = (HD + 31) / 32;
  __shared__ float sO[WAVES][kRows][DB * 32 + 1];
  __shared__ float sM[WAVES][kRows], sL[WAVES][kRows];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 5, r32 = lane & 31;
  const int unit = first + (int)blockIdx.x, h = unit % c.kv_heads, item = unit / c.kv_heads;
  const int s = find_segment(P.item, A.nseg, item);
  const int chunks = P.chunks[s], tile = (item - P.item[s]) / chunks, chunk = item - P.item[s] - tile * chunks;
  const int row0 = tile * kRows, nrows = A.nq[s] * A.group;
  const int L = A.klen[s], b0 = chunk * P.size[s], nb = min((L + kKv8Block - 1) / kKv8Block, b0 + P.size[s]);
  auto row_of = [&](int row, int64_t ld) -> int64_t {  // element of a row in q or o
    const int q = row / A.group;
    return (A.q0[s] + (int64_t)q) * ld + (int64_t)(h * A.group + row - q * A.group) * HD;
  };
  const T* Q = static_cast<const T*>(A.q) + row_of(min(row0 + r32, nrows - 1), A.ldq);
  T qf[32];  // dims 32 g .. + 31
#pragma unroll
  for (int i = 0; i < 32; ++i) qf[i] = Q[32 * g + i];
  s16x4 q4 = {};  // head_dim 72: dims 64 + 4 g .. + 3
  if constexpr (HD == 72) q4 = *reinterpret_cast<const s16x4*>(Q + 64 + 4 * g);
  f32x16 oacc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) oacc[db] = f32x16{};
  float m = -INFINITY, l = 0.0f;
  const unsigned char* base = c.tiles + ((int64_t)h * c.nblk + A.blk[s]) * 2 * kKv8Block * HD;
  const unsigned char* scales = c.scales + ((int64_t)h * c.nblk + A.blk[s]) * 2;
  uint4 kc[2][2], vc[DB][2], kn[2][2], vn[DB][2];
  uint32_t kt8[2], kn8[2];  // head_dim 72: dims 64 + 4 g .. + 3 of the two key rows
  float ks = 0.0f, vs = 0.0f, ksn = 0.0f, vsn = 0.0f;
  auto fetch = [&](int b) {
    const unsigned char* kt = base + (int64_t)b * 2 * kKv8Block * HD;
    const unsigned char* vt = kt + kKv8Block * HD;
    ksn = byte_scale(scales[2 * (int64_t)b]);
    vsn = byte_scale(scales[2 * (int64_t)b + 1]);
#pragma unroll
    for (int rb = 0; rb < 2; ++rb) {
#pragma unroll
      for (int hf = 0; hf < 2; ++hf)
        kn[rb][hf] = *reinterpret_cast<const uint4*>(kt + ((rb * 2 + hf) * 64 + lane) * 16);
      if constexpr (HD == 72) kn8[rb] = *reinterpret_cast<const uint32_t*>(kt + 4096 + (32 * rb + r32) * 8 + 4 * g);
    }
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
        vn[db][kb] = *reinterpret_cast<const uint4*>(
            vt + (db < 2 ? ((db * 2 + kb) * 64 + lane) * 16 : 4096 + ((kb * 2 + g) * 8 + (r32 & 7)) * 16));
  };
  if (b0 + wave < nb) fetch(b0 + wave);
  for (int b = b0 + wave; b < nb; b += WAVES) {
    const int left = L - b * kKv8Block;  // keys from this block on
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int j = 0; j < 2; ++j) kc[i][j] = kn[i][j];
      kt8[i] = kn8[i];
    }
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) vc[i][j] = vn[i][j];
    ks = ksn;
    vs = vsn;
    if (b + WAVES < nb) fetch(b + WAVES);
    // The products of the two key blocks alternate, so that none waits for the one before.
    f32x16 sc[2] = {f32x16{}, f32x16{}};
    if constexpr (F32) {
      // two sums of 32 dims: a score's roundings are what an f32 result is off by
      f32x16 more[2] = {f32x16{}, f32x16{}};
      float k0[16], k1[16], k2[16], k3[16];
      operand(kc[0][0], k0);
      operand(kc[1][0], k1);
      operand(kc[0][1], k2);
      operand(kc[1][1], k3);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        sc[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(k0[i], qf[i], sc[0], 0, 0, 0);
        sc[1] = __builtin_amdgcn_mfma_f32_32x32x2f32(k1[i], qf[i], sc[1], 0, 0, 0);
        more[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(k2[i], qf[16 + i], more[0], 0, 0, 0);
        more[1] = __builtin_amdgcn_mfma_f32_32x32x2f32(k3[i], qf[16 + i], more[1], 0, 0, 0);
      }
      sc[0] += more[0];
      sc[1] += more[1];
    } else {
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        bf16x8 k0[2], k1[2];
        operand(kc[0][hf], ks, k0);
        operand(kc[1][hf], ks, k1);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          bf16x8 qv;
#pragma unroll
          for (int i = 0; i < 8; ++i) qv[i] = qf[16 * hf + 8 * e + i];
          sc[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k0[e], qv, sc[0], 0, 0, 0);
          sc[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k1[e], qv, sc[1], 0, 0, 0);
        }
      }
    }
    if constexpr (HD == 72) {
#pragma unroll
      for (int rb = 0; rb < 2; ++rb) {
        const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(kt8[rb], ks, false);
        const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(kt8[rb], ks, true);
        const bf16x4 kv = {lo[0], lo[1], hi[0], hi[1]};
        sc[rb] = __builtin_amdgcn_mfma_f32_32x32x8bf16_1k(__builtin_bit_cast(s16x4, kv), q4, sc[rb], 0, 0, 0);
      }
    }
    if (left < kKv8Block) {  // the segment's last, partial block: what lies behind it may hold anything
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (32 * kb + 8 * (r >> 2) + 4 * g + (r & 3) >= left) sc[kb][r] = -INFINITY;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
          uint32_t* w = reinterpret_cast<uint32_t*>(&vc[db][kb]);
#pragma unroll
          for (int i = 0; i < 4; ++i) {  // keys 32 kb + 8 i + 4 g .. + 3
            const int n = min(max(left - (32 * kb + 8 * i + 4 * g), 0), 4);
            w[i] &= n == 4 ? ~0u : (1u << (8 * n)) - 1u;
          }
        }
    }
    const float kscale = F32 ? ks : 1.0f;  // f32: the scores are of unscaled keys so far
    const float mx = row_max(sc[0], sc[1]) * kscale;
    // while every score is -inf the base is 0: such keys weigh nothing
    const float mn = fmaxf(m, mx), at = mn == -INFINITY ? 0.0f : mn;
    if (__ballot(mn > m) != 0) {
      const float corr = fast_exp2(m - at);
#pragma unroll
      for (int db = 0; db < DB; ++db) oacc[db] *= corr;
      l *= corr;
      m = mn;
    }
    float ps = 0.0f;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      if constexpr (F32) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          sc[kb][r] = fast_exp2(fmaf(sc[kb][r], kscale, -at));
          ps += sc[kb][r];
          sc[kb][r] *= vs;
        }
        float v0[16], v1[16];
        operand(vc[0][kb], v0);
        operand(vc[1][kb], v1);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          oacc[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(v0[r], sc[kb][r], oacc[0], 0, 0, 0);
          oacc[1] = __builtin_amdgcn_mfma_f32_32x32x2f32(v1[r], sc[kb][r], oacc[1], 0, 0, 0);
        }
      } else {
        // p in two parts: its upper 16 bits, and the rest rounded to bf16
        bf16x8 pf[2], pl[2];
#pragma unroll
        for (int r = 0; r < 16; r += 2) {
          const float p0 = fast_exp2(sc[kb][r] - at), p1 = fast_exp2(sc[kb][r + 1] - at);
          const uint32_t u0 = __float_as_uint(p0), u1 = __float_as_uint(p1);
          const bf16x2 hi = __builtin_bit_cast(bf16x2, __builtin_amdgcn_perm(u1, u0, 0x07060302));
          pf[r >> 3][r & 7] = hi[0];
          pf[r >> 3][(r & 7) + 1] = hi[1];
          pl[r >> 3][r & 7] = (bf16)(p0 - __uint_as_float(u0 & 0xffff0000u));
          pl[r >> 3][(r & 7) + 1] = (bf16)(p1 - __uint_as_float(u1 & 0xffff0000u));
          ps += p0;
          ps += p1;
        }
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          bf16x8 vf[2];
          operand(vc[db][kb], vs, vf);
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            oacc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[hf], pf[hf], oacc[db], 0, 0, 0);
            oacc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[hf], pl[hf], oacc[db], 0, 0, 0);
          }
        }
      }
    }
    l += ps;  // this lane's half of the keys
  }
  l += __shfl_xor(l, 32, kWave);
  if (g == 0) {
    sM[wave][r32] = m;
    sL[wave][r32] = l;
  }
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) sO[wave][r32][32 * db + 8 * (r >> 2) + 4 * g + (r & 3)] = oacc[db][r];
  __syncthreads();
  const int64_t part0 = P.part[s] + ((int64_t)h * nrows + row0) * chunks + chunk;
  for (int i = tid; i < kRows * HD; i += 64 * WAVES) {
    const int row = i / HD, d = i - row * HD;
    if (row0 + row >= nrows) break;
    float mm = sM[0][row];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) mm = fmaxf(mm, sM[w][row]);
    const float at = mm == -INFINITY ? 0.0f : mm;
    float num = 0.0f, den = 0.0f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {  // a wave without a block has m = -inf and weighs 0
      const float f = fast_exp2(sM[w][row] - at);
      num = fmaf(sO[w][row][d], f, num);
      den = fmaf(sL[w][row], f, den);
    }
    if (chunks == 1) {
      static_cast<T*>(A.o)[row_of(row0 + row, A.ldo) + d] = L > 0 ? (T)(num / den) : (T)0.0f;
    } else {
      const int64_t at_part = part0 + (int64_t)row * chunks;
      part.o[at_part * HD + d] = num;
      if (d == 0) part.ml[at_part] = make_float2(mm, den);
    }
  }
}

// ---------------------------------------------------------------------------
// Many rows: one workgroup = 128 rows of one segment and key/value head against
// one chunk of its keys, four waves of 32 rows.  The matrix cores set the floor
// (bf16 products: 256 cycles a wave for K Q^T of 64 keys at head_dim 64 and as
// many for V^T P^T), next to the exponentials; so bytes become bf16 once per
// workgroup, not once per wave:
//  * thread t takes chunk t of a block's key tile and of its value tile (copied
//    straight to LDS, issued half an iteration ahead), turns them into two
//    fragments each and writes these to LDS in the order in which a wave reads
//    them (fragment f at 1024 f, 16 bytes a lane), so that writes and reads
//    are consecutive and free of bank conflicts, with constant offsets;
//  * iteration t does K Q^T of block t + 1 and V^T P^T of block t - 1 next to the
//    softmax of block t, none of which waits on another, as one straight run of
//    steps: a product, two exponentials, the rounding and the sum of a pair of
//    probabilities, and a conversion of the staged bytes;
//  * LDS holds two blocks of keys and two of values: in iteration t the keys
//    t + 1 and the values t - 1 are read, the keys t + 2 and the values t
//    written, and one barrier ends it;
//  * no maximum is taken per block: probabilities are 2^(score - m) with m fixed
//    at 0 (or at the first block's maximum, if that is not in [-24, 24]) until
//    a block's probabilities sum past 2^32; then m moves to that block's
//    maximum, O and l are rescaled and the block's probabilities are made again
//    from its bytes;
//  * P is rounded to bf16, once for the product and for the row sum: in two parts,
//    as the 32-row tiles take it, half as many products again would bound the
//    kernel.  Against 64 bits o is off by 2.2e-3 of its size (rms); its own
//    rounding gives 1.7e-3.
// Bound by the chip's power: 9677 queries against 32256 keys of 16 heads take 1.23 ms
// (1040 TFLOP/s) at 1.70 GHz, matrix cores busy for 51 % of the cycles; 645 queries
// 103 us at 2.1 GHz and 38 %; head_dim 72 runs at 1.9 GHz and 53 %, a fifth of its
// products on padding.
template <int HD>
struct TileGeo {
  static constexpr int DB = (HD + 31) / 32;   // 32-row blocks of O^T (head_dim 72: of the third, 8 rows count)
  static constexpr int NPV = 4 * DB, NQK = HD == 72 ? 10 : 8;
  static constexpr int SLOT = 8192 + (HD == 72 ? 1088 : 0);  // one block's keys, or its values, as bf16
  static constexpr int TILE = kKv8Block * HD;                // the same as bytes
};
template <int HD>
struct TileSmem {
  unsigned char k[2][TileGeo<HD>::SLOT];
  unsigned char v[2][TileGeo<HD>::SLOT];
  unsigned char rk[4096];  // one block's bytes, as they came
  unsigned char rv[4096];
};
constexpr float kPsumMax = 4294967296.0f;  // 2^32

__device__ __forceinline__ bf16x2 cvt2(uint32_t w, float scale, bool hi) {
  return hi ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true)
            : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false);
}
__device__ __forceinline__ uint32_t keep_keys(uint32_t w, int left) {  // the first `left` of four bytes
  const int n = min(max(left, 0), 4);
  return w & (n == 4 ? ~0u : (1u << (8 * n)) - 1u);
}

template <int HD>
__global__ __launch_bounds__(kTPB, 3) void k_kv8_attn_tiles(Kv8Attn A, Kv8Slice c, Kv8Plan P,
                                                                            Parts part, int first, int total) {
  typedef TileGeo<HD> G;
  constexpr int DB = G::DB, NPV = G::NPV, NSTEP = G::NPV + G::NQK;
  __shared__ __attribute__((aligned(16))) TileSmem<HD> sm;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 5, r32 = lane & 31;
  // whole heads per XCD, and within a head the row tiles of a chunk side by side:
  // they read the same bytes
  const int unit = xcd_tile(first + (int)blockIdx.x, total), items = P.item[A.nseg];
  const int h = unit / items, item = unit - h * items;
  const int s = find_segment(P.item, A.nseg, item);
  const int chunks = P.chunks[s], tiles = (P.item[s + 1] - P.item[s]) / chunks;
  const int chunk = (item - P.item[s]) / tiles, tile = item - P.item[s] - chunk * tiles;
  const int nrows = A.nq[s] * A.group;
  const int L = A.klen[s], b0 = chunk * P.size[s], nkt = min((L + kKv8Block - 1) / kKv8Block - b0, P.size[s]);
  const int row = tile * 128 + wave * 32 + r32;
  const bool active = tile * 128 + wave * 32 < nrows;  // a wave without rows only stages bytes
  auto row_of = [&](int64_t ld) -> int64_t {
    const int q = row / A.group;
    return (A.q0[s] + (int64_t)q) * ld + (int64_t)(h * A.group + row - q * A.group) * HD;
  };
  const bf16x8 zero8 = {};
  bf16x8 qf[4];
  s16x4 q4 = {};
#pragma unroll
  for (int ks = 0; ks < 4; ++ks) qf[ks] = zero8;
  if (row < nrows) {
    const bf16* Q = static_cast<const bf16*>(A.q) + row_of(A.ldq);
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) qf[ks] = *reinterpret_cast<const bf16x8*>(Q + 32 * g + 8 * ks);
    if constexpr (HD == 72) q4 = *reinterpret_cast<const s16x4*>(Q + 64 + 4 * g);
  }
  const unsigned char* base = c.tiles + ((int64_t)h * c.nblk + A.blk[s] + b0) * 2 * G::TILE;
  const unsigned char* scales = c.scales + ((int64_t)h * c.nblk + A.blk[s] + b0) * 2;
  const int last = L - (b0 + nkt - 1) * kKv8Block;  // keys of the chunk's last block (64 and more: whole)

  // Bytes of a block on their way: chunk `tid` of its key tile and of its value
  // tile, copied straight into LDS by the wave that will convert them, which
  // holds no registers meanwhile; head_dim 72: also four of the bytes behind the
  // chunks, the keys' in waves 0 and 1, the values' in waves 2 and 3 (so that no
  // wave branches in the run of steps).
  uint4 sk, sv;
  uint32_t st = 0;
  float ksc, vsc;
  auto fetch_k = [&](int t) {
    const unsigned char* p = base + (int64_t)t * 2 * G::TILE;
    lds_dma16_at(p, tid * 16, sm.rk + wave * 1024);
    ksc = byte_scale(scales[2 * (int64_t)t]);
  };
  auto fetch_v = [&](int t) {
    const unsigned char* p = base + (int64_t)t * 2 * G::TILE + G::TILE;
    lds_dma16_at(p, tid * 16, sm.rv + wave * 1024);
    vsc = byte_scale(scales[2 * (int64_t)t + 1]);
  };
  const bool vtail = wave >= 2;
  auto fetch_tail = [&](int tk, int tv) {
    const unsigned char* p = base + (int64_t)(vtail ? tv : tk) * 2 * G::TILE + (vtail ? G::TILE : 0) + 4096;
    st = *reinterpret_cast<const uint32_t*>(p + (tid & 127) * 4);
  };
  // This wave's copies have landed (only it reads them).
  auto landed = [&]() {
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
    asm volatile("" ::: "memory");
  };
  auto take_k = [&]() {
    sk = *reinterpret_cast<const uint4*>(sm.rk + tid * 16);
  };
  auto take_v = [&]() {
    sv = *reinterpret_cast<const uint4*>(sm.rv + tid * 16);
  };
  // What was taken is in registers, so that its place may be filled again.
  auto taken = [&]() {
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
    asm volatile("" ::: "memory");
  };
  // what lies behind the segment's last key may hold anything: its values become zero
  auto trim_v = [&]() {
    const int kb = wave & 1;
    uint32_t* w = reinterpret_cast<uint32_t*>(&sv);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = keep_keys(w[i], last - (32 * kb + 8 * i + 4 * g));
    // word w = tid - 128 behind the value chunks: keys 32 (w / 64) + 8 (w % 4) + 4 (w / 32 % 2) .. + 3
    if (HD == 72 && vtail) st = keep_keys(st, last - (32 * ((tid >> 6) & 1) + 8 * (tid & 3) + 4 * ((tid >> 5) & 1)));
  };
  auto put = [&](unsigned char* slot, int e, const uint4& b, float scale) {  // half e of a chunk: fragment 2 wave + e
    const uint32_t w0 = e ? b.z : b.x, w1 = e ? b.w : b.y;
    bf16x8 f;
    const bf16x2 a0 = cvt2(w0, scale, false), a1 = cvt2(w0, scale, true);
    const bf16x2 a2 = cvt2(w1, scale, false), a3 = cvt2(w1, scale, true);
    f[0] = a0[0]; f[1] = a0[1]; f[2] = a1[0]; f[3] = a1[1];
    f[4] = a2[0]; f[5] = a2[1]; f[6] = a3[0]; f[7] = a3[1];
    *reinterpret_cast<bf16x8*>(slot + (2 * wave + e) * 1024 + lane * 16) = f;
  };
  // The four bytes behind the chunks, in the slots of parity par.
  // keys: dims 64 .. 71 as [32-row block][half of the dims][row] eight bytes
  // values: [32-key block][half]: [g][dim] sixteen bytes, then sixteen zeros, which
  // stand for the dims 72 .. 95 of the third block (zeros cost the matrix cores less
  // power, and so the chip less clock, than any other bytes)
  const int tail_at = vtail ? (int)(sm.v[0] - sm.k[0]) + 8192 + (((tid >> 6) & 1) * 2 + ((tid >> 1) & 1)) * 272 +
                                  ((tid >> 2) & 15) * 16 + (tid & 1) * 8
                            : 8192 + (tid >> 6) * 512 + (tid & 1) * 256 + ((tid >> 1) & 31) * 8;
  auto put_tail = [&](int par) {
    const float scale = vtail ? vsc : ksc;
    const bf16x2 a0 = cvt2(st, scale, false), a1 = cvt2(st, scale, true);
    const bf16x4 f = {a0[0], a0[1], a1[0], a1[1]};
    *reinterpret_cast<bf16x4*>(sm.k[0] + tail_at + par * G::SLOT) = f;
  };
  // Fragment reads.  keys: 32-row block rb, k-step ks; values: key block kb, half hf, dim block db
  auto key_frag = [&](const unsigned char* slot, int rb, int ks) -> bf16x8 {
    return *reinterpret_cast<const bf16x8*>(slot + (rb * 4 + ks) * 1024 + lane * 16);
  };
  auto key_tail = [&](const unsigned char* slot, int rb) -> s16x4 {
    return *reinterpret_cast<const s16x4*>(slot + 8192 + rb * 512 + lane * 8);
  };
  const int third = r32 < 8 ? g * 128 + r32 * 16 : 256;
  auto val_frag = [&](const unsigned char* slot, int kb, int hf, int db) -> bf16x8 {
    if (db < 2) return *reinterpret_cast<const bf16x8*>(slot + ((db * 2 + kb) * 2 + hf) * 1024 + lane * 16);
    return *reinterpret_cast<const bf16x8*>(slot + 8192 + (kb * 2 + hf) * 272 + third);
  };
  auto qk = [&](const unsigned char* slot, f32x16& s0, f32x16& s1) {
    s0 = f32x16{};
    s1 = f32x16{};
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      s0 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(key_frag(slot, 0, ks), qf[ks], s0, 0, 0, 0);
      s1 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(key_frag(slot, 1, ks), qf[ks], s1, 0, 0, 0);
    }
    if constexpr (HD == 72) {
      s0 = __builtin_amdgcn_mfma_f32_32x32x8bf16_1k(key_tail(slot, 0), q4, s0, 0, 0, 0);
      s1 = __builtin_amdgcn_mfma_f32_32x32x8bf16_1k(key_tail(slot, 1), q4, s1, 0, 0, 0);
    }
  };
  auto mask_tail = [&](f32x16& s0, f32x16& s1) {  // of the chunk's last block
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int key = (r >> 2) * 8 + g * 4 + (r & 3);
      if (key >= last) s0[r] = -INFINITY;
      if (key + 32 >= last) s1[r] = -INFINITY;
    }
  };

  f32x16 oacc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) oacc[db] = f32x16{};
  float m_run = 0.0f, l_run = 0.0f;
  bool shifted = false;  // wave-uniform: m_run is subtracted from the scores

  // Scores of 32 keys of a block once more, from its bytes (rare).
  auto rescore = [&](int t, int rb) -> f32x16 {
    const unsigned char* p = base + (int64_t)t * 2 * G::TILE;
    const float scale = byte_scale(scales[2 * (int64_t)t]);
    f32x16 a = f32x16{};
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      bf16x8 f[2];
      operand(*reinterpret_cast<const uint4*>(p + ((rb * 2 + hf) * 64 + lane) * 16), scale, f);
#pragma unroll
      for (int e = 0; e < 2; ++e) a = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[e], qf[2 * hf + e], a, 0, 0, 0);
    }
    if constexpr (HD == 72) {
      const uint32_t w = *reinterpret_cast<const uint32_t*>(p + 4096 + (32 * rb + r32) * 8 + 4 * g);
      const bf16x2 a0 = cvt2(w, scale, false), a1 = cvt2(w, scale, true);
      bf16x4 f;
      f[0] = a0[0]; f[1] = a0[1]; f[2] = a1[0]; f[3] = a1[1];
      a = __builtin_amdgcn_mfma_f32_32x32x8bf16_1k(__builtin_bit_cast(s16x4, f), q4, a, 0, 0, 0);
    }
#pragma unroll
    for (int r = 0; r < 16; ++r)
      a[r] = t == nkt - 1 && 32 * rb + (r >> 2) * 8 + g * 4 + (r & 3) >= last ? -INFINITY : a[r];
    return a;
  };
  // Moves the maximum to block t's where that is larger; O holds the blocks up to t - 1.
  auto rebase = [&](int t, bf16x8 (&pf)[2][2]) -> float {
    float mx = -INFINITY;
#pragma unroll 1
    for (int rb = 0; rb < 2; ++rb) {
      const f32x16 a = rescore(t, rb);
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, a[r]);
    }
    mx = fmaxf(mx, __shfl_xor(mx, 32, kWave));
    const float to = fmaxf(m_run, mx), alpha = fast_exp2(m_run - to);
#pragma unroll
    for (int db = 0; db < DB; ++db) oacc[db] *= alpha;
    l_run *= alpha;
    m_run = to;
    shifted = true;
    float psum = 0.0f;
    bf16x8 q0[2], q1[2];
#pragma unroll 1
    for (int rb = 0; rb < 2; ++rb) {
      const f32x16 a = rescore(t, rb);
      bf16x8 x[2];
#pragma unroll
      for (int r = 0; r < 16; r += 2) {
        bf16x2 pr;
        pr[0] = (bf16)fast_exp2(a[r] - to);
        pr[1] = (bf16)fast_exp2(a[r + 1] - to);
        psum = add_pair(psum, pr);
        x[r >> 3][r & 7] = pr[0];
        x[r >> 3][(r & 7) + 1] = pr[1];
      }
      if (rb == 0) {
        q0[0] = x[0];
        q0[1] = x[1];
      } else {
        q1[0] = x[0];
        q1[1] = x[1];
      }
    }
    pf[0][0] = q0[0];
    pf[0][1] = q0[1];
    pf[1][0] = q1[0];
    pf[1][1] = q1[1];
    return pair_sum(psum);
  };
  auto settle = [&](f32x16& a, f32x16& b) {
    if (shifted)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        a[r] -= m_run;
        b[r] -= m_run;
      }
  };
  auto barrier = [&]() {
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): this wave's LDS writes; loads stay in flight
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  // Product step st: V^T P^T first (its probabilities die while new ones are made), then K Q^T
  auto frag = [&](const unsigned char* ks_, const unsigned char* vs_, int st_) -> bf16x8 {
    if (st_ < NPV) return val_frag(vs_, st_ / (2 * DB), (st_ / DB) & 1, st_ % DB);
    const int ks = (st_ - NPV) >> 1, rb = (st_ - NPV) & 1;
    if (HD == 72 && ks == 4) {
      const s16x4 x = key_tail(ks_, rb);
      const s16x4 r[2] = {x, x};
      return *reinterpret_cast<const bf16x8*>(r);
    }
    return key_frag(ks_, rb, ks);
  };
  // loads of iteration t: keys t + 3, values t + 1
  auto fetch = [&](int t) {
    fetch_k(min(t + 3, nkt - 1));
    fetch_v(t + 1);
    if constexpr (HD == 72) fetch_tail(min(t + 3, nkt - 1), t + 1);
  };
  // Iteration t; PAR = t % 2.  c: scores of block t, n: of block t + 1; pp: probabilities of block t - 1, pn: of t.
  auto iter = [&](int t, auto PAR, f32x16& c0, f32x16& c1, f32x16& n0, f32x16& n1, bf16x8 (&pp)[2][2],
                  bf16x8 (&pn)[2][2]) {
    constexpr int par = decltype(PAR)::value;
    const unsigned char* kr = sm.k[par ^ 1];
    const unsigned char* vr = sm.v[par ^ 1];
    unsigned char* kw = sm.k[par];
    unsigned char* vw = sm.v[par];
    settle(c0, c1);
    bf16x8 fr[3];
    fr[0] = frag(kr, vr, 0);
    fr[1] = frag(kr, vr, 1);
    auto score = [&](int i, int e) -> float {  // pair i of the block's 16 pairs a lane
      const int r = (i >> 3) * 8 + 2 * ((i >> 1) & 3) + e;
      return (i & 1) ? c1[r] : c0[r];
    };
    float ex[16][2];
#pragma unroll
    for (int e = 0; e < 2; ++e) ex[0][e] = fast_exp2(score(0, e));
    __builtin_amdgcn_sched_barrier(0);
    float psum = 0.0f;
    const f32x16 zero16 = {};
#pragma unroll
    for (int i = 0; i < NSTEP; ++i) {
      if (i + 2 < NSTEP) fr[(i + 2) % 3] = frag(kr, vr, i + 2);
      if (i < NPV) {
        oacc[i % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[i % 3], pp[i / (2 * DB)][(i / DB) & 1], oacc[i % DB],
                                                                0, 0, 0);
      } else {
        const int ks = (i - NPV) >> 1;
        f32x16& n = ((i - NPV) & 1) ? n1 : n0;
        if (HD == 72 && ks == 4)
          n = __builtin_amdgcn_mfma_f32_32x32x8bf16_1k(*reinterpret_cast<const s16x4*>(&fr[i % 3]), q4, n, 0, 0, 0);
        else
          n = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[i % 3], qf[ks], ks == 0 ? zero16 : n, 0, 0, 0);
      }
      if (i + 1 < 16)
#pragma unroll
        for (int e = 0; e < 2; ++e) ex[i + 1][e] = fast_exp2(score(i + 1, e));
      if (i < 16) {
        const int hf = i >> 3, j = (i >> 1) & 3, w = i & 1;
        bf16x2 pr;
        pr[0] = (bf16)ex[i][0];
        pr[1] = (bf16)ex[i][1];
        psum = add_pair(psum, pr);
        pn[w][hf][2 * j] = pr[0];
        pn[w][hf][2 * j + 1] = pr[1];
      }
      // the staged bytes: keys t + 2, values t; then the next copies (every step ends
      // in a fence, so that what was taken has been converted by then)
      if (i == 0) {
        landed();
        take_k();
      }
      if (i == 6) take_v();
      if (i == 2) put(kw, 0, sk, ksc);
      if (i == 4) put(kw, 1, sk, ksc);
      if (i == 8) put(vw, 0, sv, vsc);
      if (i == 10) put(vw, 1, sv, vsc);
      if (HD == 72 && i == 11) put_tail(par);
      if (i == 12) fetch(t);
      __builtin_amdgcn_sched_barrier(0);
    }
    // the probabilities are made here, not after the next branch
#pragma unroll
    for (int w = 0; w < 2; ++w)
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) asm volatile("" : "+v"(pn[w][hf]));
    psum = pair_sum(psum);
    if (__ballot(!(psum <= kPsumMax)) != 0) psum = rebase(t, pn);
    l_run += psum;
    barrier();
  };

  if (nkt > 0) {
    // values of "block -1": zeros, times zero probabilities (and the zeros that stay)
    for (int i = tid; i < G::SLOT / 16; i += kTPB) reinterpret_cast<bf16x8*>(sm.v[1])[i] = zero8;
    if (HD == 72 && tid < 4) *reinterpret_cast<bf16x8*>(sm.v[0] + 8192 + tid * 272 + 256) = zero8;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      fetch_k(min(t, nkt - 1));
      if constexpr (HD == 72) fetch_tail(min(t, nkt - 1), 0);
      landed();
      take_k();
      taken();
      put(sm.k[t], 0, sk, ksc);
      put(sm.k[t], 1, sk, ksc);
      if (HD == 72 && !vtail) put_tail(t);
    }
    fetch_k(min(2, nkt - 1));
    fetch_v(0);
    if constexpr (HD == 72) fetch_tail(min(2, nkt - 1), 0);
    barrier();
    if (!active) {
      barrier();
      int t = 0;
      for (; t < nkt; ++t) {  // at the last block only its values are left to stage
        unsigned char* vw = sm.v[t & 1];
        landed();
        take_v();
        if (t + 1 == nkt && last < kKv8Block) trim_v();
        put(vw, 0, sv, vsc);
        put(vw, 1, sv, vsc);
        if (HD == 72 && (vtail || t + 1 < nkt)) put_tail(t & 1);
        if (t + 1 < nkt) {
          unsigned char* kw = sm.k[t & 1];
          take_k();
          put(kw, 0, sk, ksc);
          put(kw, 1, sk, ksc);
          taken();
          fetch(t);
        }
        barrier();
      }
      return;
    }
    f32x16 a0, a1, d0, d1;
    qk(sm.k[0], a0, a1);
    if (nkt == 1 && last < kKv8Block) mask_tail(a0, a1);
    {
      const float mx = row_max(a0, a1);
      shifted = __ballot(!(mx >= -24.0f && mx <= 24.0f)) != 0;
      m_run = !shifted ? 0.0f : mx > -INFINITY ? mx : -FLT_MAX;  // any score above it moves it
    }
    barrier();  // every wave is done with keys 0, whose slot takes keys 2
    bf16x8 pa[2][2] = {{zero8, zero8}, {zero8, zero8}}, pb[2][2];
    using Even = std::integral_constant<int, 0>;
    using Odd = std::integral_constant<int, 1>;
    int t = 0;
    for (; t + 2 < nkt; t += 2) {
      iter(t, Even{}, a0, a1, d0, d1, pa, pb);
      iter(t + 1, Odd{}, d0, d1, a0, a1, pb, pa);
    }
    if (t + 1 < nkt) {
      iter(t, Even{}, a0, a1, d0, d1, pa, pb);
      a0 = d0;
      a1 = d1;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) pa[kb][hf] = pb[kb][hf];
      ++t;
    }
    // the last block
    unsigned char* vw = sm.v[t & 1];
    const unsigned char* vr = sm.v[(t & 1) ^ 1];
    landed();
    take_v();
    if (last < kKv8Block) trim_v();
    put(vw, 0, sv, vsc);
    put(vw, 1, sv, vsc);
    if (HD == 72 && vtail) put_tail(t & 1);
    auto pv = [&](const unsigned char* slot, const bf16x8 (&p)[2][2]) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int hf = 0; hf < 2; ++hf)
#pragma unroll
          for (int db = 0; db < DB; ++db)
            oacc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(val_frag(slot, kb, hf, db), p[kb][hf], oacc[db], 0, 0, 0);
    };
    settle(a0, a1);
    if (last < kKv8Block) mask_tail(a0, a1);
    float psum = 0.0f;
#pragma unroll
    for (int r = 0; r < 16; r += 2) {
      bf16x2 x, y;
      x[0] = (bf16)fast_exp2(a0[r]);
      x[1] = (bf16)fast_exp2(a0[r + 1]);
      y[0] = (bf16)fast_exp2(a1[r]);
      y[1] = (bf16)fast_exp2(a1[r + 1]);
      psum = add_pair(add_pair(psum, x), y);
      pb[0][r >> 3][r & 7] = x[0];
      pb[0][r >> 3][(r & 7) + 1] = x[1];
      pb[1][r >> 3][r & 7] = y[0];
      pb[1][r >> 3][(r & 7) + 1] = y[1];
    }
    psum = pair_sum(psum);
    pv(vr, pa);
    if (__ballot(!(psum <= kPsumMax)) != 0) psum = rebase(t, pb);
    l_run += psum;
    barrier();
    pv(vw, pb);
    l_run += __shfl_xor(l_run, 32, kWave);
  }
  if (row >= nrows) return;
  if (chunks == 1) {
    const float inv = L > 0 ? 1.0f / l_run : 0.0f;
    bf16* o = static_cast<bf16*>(A.o) + row_of(A.ldo);
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int rr = 0; rr < 4; ++rr)
        if (db * 32 + rr * 8 < HD) {
          bf16x4 v;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = (bf16)(oacc[db][rr * 4 + e] * inv);
          *reinterpret_cast<bf16x4*>(o + db * 32 + rr * 8 + g * 4) = v;
        }
  } else {
    const int64_t at = P.part[s] + ((int64_t)h * nrows + row) * chunks + chunk;
    float* o = part.o + at * HD;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int rr = 0; rr < 4; ++rr)
        if (db * 32 + rr * 8 < HD) {
          f32x4 v;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = oacc[db][rr * 4 + e];
          *reinterpret_cast<f32x4*>(o + db * 32 + rr * 8 + g * 4) = v;
        }
    if (g == 0) part.ml[at] = make_float2(m_run, l_run);
  }
}

// Joins the chunks of a row and head: one wave per row and head, or (few rows of
// many chunks) a workgroup of 16 waves, wave w taking chunks w (mod 16).  A
// lane has one dim; at head_dim 72 eight lanes have a second one.  Bound by the
// latency of the loads: a wave asks for the maxima, sums and values of eight
// chunks at once and joins them as it goes.  645 queries of 16 heads in eight chunks
// take 9 us (42 MB moved, mostly through the last-level cache).
template <typename T, int HD, int WAVES>
__global__ __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES) void k_kv8_attn_join(Kv8Attn A, int kv_heads, Kv8Plan P, Parts part, int rows) {
  __shared__ float sO[WAVES][HD], sL[WAVES], sM[WAVES];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int unit = WAVES == 1 ? (int)blockIdx.x * 4 + wave : (int)blockIdx.x;  // row * kv_heads + head
  if (unit >= rows * kv_heads) return;  // only with one wave per row, which has no barrier
  const int h = unit % kv_heads, at = unit / kv_heads;
  const int s = find_segment(P.row, A.nseg, at);
  const int row = at - P.row[s], chunks = P.chunks[s], nrows = A.nq[s] * A.group;
  const int64_t first = P.part[s] + ((int64_t)h * nrows + row) * chunks;
  float m = -INFINITY, num = 0.0f, num2 = 0.0f, den = 0.0f;
  constexpr int U = 8;
  for (int j0 = WAVES == 1 ? 0 : wave; j0 < chunks; j0 += WAVES * U) {
    float2 ml[U];
    float o[U], o2[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t j = first + min(j0 + u * WAVES, chunks - 1);
      ml[u] = part.ml[j];
      o[u] = part.o[j * HD + lane];
      o2[u] = HD == 72 ? part.o[j * HD + 64 + (lane & 7)] : 0.0f;
    }
    float mn = m;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (j0 + u * WAVES >= chunks) ml[u] = make_float2(-INFINITY, 0.0f);
      mn = fmaxf(mn, ml[u].x);
    }
    const float base = mn == -INFINITY ? 0.0f : mn, f0 = fast_exp2(m - base);
    num *= f0;
    num2 *= f0;
    den *= f0;
    m = mn;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (j0 + u * WAVES >= chunks) break;
      const float f = fast_exp2(ml[u].x - base);
      num = fmaf(o[u], f, num);
      num2 = fmaf(o2[u], f, num2);
      den = fmaf(ml[u].y, f, den);
    }
  }
  if constexpr (WAVES > 1) {
    sO[wave][lane] = num;
    if (HD == 72 && lane < 8) sO[wave][64 + lane] = num2;
    if (lane == 0) {
      sL[wave] = den;
      sM[wave] = m;
    }
    __syncthreads();
    if (wave != 0) return;
    m = sM[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) m = fmaxf(m, sM[w]);
    const float base = m == -INFINITY ? 0.0f : m;
    num = num2 = den = 0.0f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {  // a wave without a chunk has m = -inf and weighs 0
      const float f = fast_exp2(sM[w] - base);
      num = fmaf(sO[w][lane], f, num);
      if (HD == 72) num2 = fmaf(sO[w][64 + (lane & 7)], f, num2);
      den = fmaf(sL[w], f, den);
    }
  }
  const int q = row / A.group;
  T* o = static_cast<T*>(A.o) + (A.q0[s] + (int64_t)q) * A.ldo + (int64_t)(h * A.group + row - q * A.group) * HD;
  const float inv = 1.0f / den;
  o[lane] = (T)(num * inv);
  if (HD == 72 && lane < 8) o[64 + lane] = (T)(num2 * inv);
}
}  // namespace

size_t kv8_attention_ws_bytes(int kv_heads, int head_dim, int group, int nseg, const int* nq, const int* klen) {
  int64_t rows[SPHINX_MAX_REQUESTS];
  for (int i = 0; i < nseg; ++i) rows[i] = (int64_t)nq[i] * group;
  const size_t parts = (size_t)kv8_most_parts(kv_heads, nseg, rows, klen);
  return 256 + ((parts * 8 + 255) & ~(size_t)255) + parts * (size_t)head_dim * 4;
}

hipError_t launch_kv8_attention(sphinx_dtype dt, int head_dim, const Kv8Attn& A, const Kv8Slice& c, void* ws,
                                hipStream_t s) {
  int64_t rows[SPHINX_MAX_REQUESTS];
  for (int i = 0; i < A.nseg; ++i) rows[i] = (int64_t)A.nq[i] * A.group;
  const Kv8Plan P = plan_kv8(dt == SPHINX_BF16, c.kv_heads, head_dim, A.nseg, rows, A.klen);
  const size_t parts = (size_t)P.part[A.nseg];
  const Parts part{static_cast<float2*>(ws),
                   reinterpret_cast<float*>(static_cast<unsigned char*>(ws) + ((parts * 8 + 255) & ~(size_t)255))};
  // at most 2^31 / 32 tiles; a launch holds 2^32 threads, so 2^23 workgroups at a time
  const int total = P.item[A.nseg] * c.kv_heads, most_wg = 1 << 23;
  auto go = [&](auto t, auto hd) {
    using T = decltype(t);
    constexpr int HD = decltype(hd)::value;
    for (int first = 0; first < total; first += most_wg) {
      if constexpr (sizeof(T) == 2) {
        if (P.tile == 128) {
          k_kv8_attn_tiles<HD><<<std::min(most_wg, total - first), kTPB, 0, s>>>(A, c, P, part, first, total);
          continue;
        }
        if (P.waves == 8) {
          k_kv8_attn_rows<T, HD, 8><<<std::min(most_wg, total - first), 512, 0, s>>>(A, c, P, part, first);
          continue;
        }
      }
      k_kv8_attn_rows<T, HD, 4><<<std::min(most_wg, total - first), kTPB, 0, s>>>(A, c, P, part, first);
    }
    if (parts == 0) return;
    const int join = P.row[A.nseg];
    int most = 0;
    for (int i = 0; i < A.nseg; ++i) most = std::max(most, P.chunks[i]);
    // a wave per row where a wave's first eight loads see all chunks, or rows fill the chip
    const int units = join * c.kv_heads;
    if (most <= 8 || units >= 1024)
      k_kv8_attn_join<T, HD, 1><<<(units + 3) / 4, 256, 0, s>>>(A, c.kv_heads, P, part, join);
    else
      k_kv8_attn_join<T, HD, 16><<<units, 1024, 0, s>>>(A, c.kv_heads, P, part, join);
  };
  if (dt == SPHINX_F32)
    go(float{}, std::integral_constant<int, 64>{});
  else if (head_dim == 64)
    go(bf16{}, std::integral_constant<int, 64>{});
  else
    go(bf16{}, std::integral_constant<int, 72>{});
  return hipGetLastError();
}

}  // namespace sphinx
