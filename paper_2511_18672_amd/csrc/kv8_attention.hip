// Attention over the 8-bit key/value cache (layout: kv8.hpp): per segment and
// query head o = sum_t 2^(q.k_t) v_t / sum_t 2^(q.k_t) over the segment's cached
// tokens, keys and values being the numbers that the cache's bytes stand for.

#include <algorithm>
#include <type_traits>

#include "kv8.hpp"

namespace sphinx {

namespace {
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
constexpr int kTPB = 256;
constexpr int kRows = 32;  // rows (queries of the heads that share a key/value head) per workgroup

__device__ __forceinline__ float byte_scale(int b) { return __uint_as_float((uint32_t)b << 23); }

// Sixteen stored bytes as operands: two bf16 fragments of eight, or 16 floats.
// The scale is a power of two, so both forms hold the values exactly.
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
__device__ __forceinline__ void operand(const uint4& b, float scale, float (&f)[16]) {
  const uint32_t w[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], false);
    const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], true);
    f[4 * i] = lo[0] * scale;
    f[4 * i + 1] = lo[1] * scale;
    f[4 * i + 2] = hi[0] * scale;
    f[4 * i + 3] = hi[1] * scale;
  }
}

// One workgroup = 32 rows of one segment and key/value head; its four waves take
// the blocks b = wave (mod 4) and merge (m, l, O) through LDS.  A wave reads a
// block's bytes straight into the operand layouts:
//  * S^T = K Q^T in two 32-key tiles: lane l = 32 g + r has key r and dims
//    32 g .. + 31 (two chunks), for the queries the same dims of row r;
//  * P^T needs no move: score register 8 hf + j of tile kb belongs to the key
//    that byte 8 hf + j of the values' chunk (db, kb) holds;
//  * O^T = V^T P^T leaves the row on the lane.
// bf16: 32x32x16 products, P rounded to bf16 for the product, the row sum adding
// the same rounded values; f32: 32x32x2 products, nothing rounded.
template <typename T, int HD>
__global__ __launch_bounds__(kTPB) void k_kv8_attn_rows(Kv8Attn A, Kv8Slice c) {
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int DB = (HD + 31) / 32;
  __shared__ float sO[4][kRows][DB * 32 + 1];
  __shared__ float sM[4][kRows], sL[4][kRows];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 5, r32 = lane & 31;
  const int h = (int)blockIdx.x % c.kv_heads, tile = (int)blockIdx.x / c.kv_heads;
  int s = 0;
  while (s + 1 < A.nseg && A.tile_prefix[s + 1] <= tile) ++s;
  const int row0 = (tile - A.tile_prefix[s]) * kRows, nrows = A.nq[s] * A.group;
  const int L = A.klen[s], nb = (L + kKv8Block - 1) / kKv8Block;
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
  for (int b = wave; b < nb; b += 4) {
    const unsigned char* kt = base + (int64_t)b * 2 * kKv8Block * HD;
    const unsigned char* vt = kt + kKv8Block * HD;
    const float ks = byte_scale(scales[2 * (int64_t)b]), vs = byte_scale(scales[2 * (int64_t)b + 1]);
    const int left = L - b * kKv8Block;  // keys from this block on
    uint4 kc[2][2], vc[DB][2];
#pragma unroll
    for (int rb = 0; rb < 2; ++rb)
#pragma unroll
      for (int hf = 0; hf < 2; ++hf)
        kc[rb][hf] = *reinterpret_cast<const uint4*>(kt + ((rb * 2 + hf) * 64 + lane) * 16);
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
        vc[db][kb] = *reinterpret_cast<const uint4*>(
            vt + (db < 2 ? ((db * 2 + kb) * 64 + lane) * 16 : 4096 + ((kb * 2 + g) * 8 + (r32 & 7)) * 16));
    f32x16 sc[2];
#pragma unroll
    for (int rb = 0; rb < 2; ++rb) {
      sc[rb] = f32x16{};
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        if constexpr (F32) {
          float kf[16];
          operand(kc[rb][hf], ks, kf);
#pragma unroll
          for (int i = 0; i < 16; ++i)
            sc[rb] = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[i], qf[16 * hf + i], sc[rb], 0, 0, 0);
        } else {
          bf16x8 kf[2];
          operand(kc[rb][hf], ks, kf);
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            bf16x8 qv;
#pragma unroll
            for (int i = 0; i < 8; ++i) qv[i] = qf[16 * hf + 8 * e + i];
            sc[rb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[e], qv, sc[rb], 0, 0, 0);
          }
        }
      }
      if constexpr (HD == 72) {
        const uint32_t w = *reinterpret_cast<const uint32_t*>(kt + 4096 + (32 * rb + r32) * 8 + 4 * g);
        bf16x4 kv;
        const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, ks, false);
        const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, ks, true);
        kv[0] = lo[0];
        kv[1] = lo[1];
        kv[2] = hi[0];
        kv[3] = hi[1];
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
    float mx = -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; ++r) mx = fmaxf(mx, fmaxf(sc[0][r], sc[1][r]));
    mx = fmaxf(mx, __shfl_xor(mx, 32, kWave));
    // while every score is -inf the base is 0: such keys weigh nothing
    const float mn = fmaxf(m, mx), at = mn == -INFINITY ? 0.0f : mn, corr = exp2f(m - at);
    m = mn;
    float ps = 0.0f;
#pragma unroll
    for (int db = 0; db < DB; ++db) oacc[db] *= corr;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      if constexpr (F32) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          sc[kb][r] = exp2f(sc[kb][r] - at);
          ps += sc[kb][r];
        }
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          float vf[16];
          operand(vc[db][kb], vs, vf);
#pragma unroll
          for (int r = 0; r < 16; ++r)
            oacc[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(vf[r], sc[kb][r], oacc[db], 0, 0, 0);
        }
      } else {
        bf16x8 pf[2];
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          pf[r >> 3][r & 7] = (bf16)exp2f(sc[kb][r] - at);
          ps += (float)pf[r >> 3][r & 7];
        }
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          bf16x8 vf[2];
          operand(vc[db][kb], vs, vf);
#pragma unroll
          for (int hf = 0; hf < 2; ++hf)
            oacc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[hf], pf[hf], oacc[db], 0, 0, 0);
        }
      }
    }
    l = fmaf(l, corr, ps);  // this lane's half of the keys
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
  for (int i = tid; i < kRows * HD; i += kTPB) {
    const int row = i / HD, d = i - row * HD;
    if (row0 + row >= nrows) break;
    const float mm = fmaxf(fmaxf(sM[0][row], sM[1][row]), fmaxf(sM[2][row], sM[3][row]));
    float num = 0.0f, den = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {  // a wave without a block has m = -inf and weighs 0
      const float f = sM[w][row] == -INFINITY && mm == -INFINITY ? 1.0f : exp2f(sM[w][row] - mm);
      num = fmaf(sO[w][row][d], f, num);
      den = fmaf(sL[w][row], f, den);
    }
    static_cast<T*>(A.o)[row_of(row0 + row, A.ldo) + d] = L > 0 ? (T)(num / den) : (T)0.0f;
  }
}
}  // namespace

hipError_t launch_kv8_attention(sphinx_dtype dt, int head_dim, const Kv8Attn& A0, const Kv8Slice& c, hipStream_t s) {
  Kv8Attn A = A0;
  A.tile_prefix[0] = 0;
  for (int i = 0; i < A.nseg; ++i)
    A.tile_prefix[i + 1] = A.tile_prefix[i] + (int)(((int64_t)A.nq[i] * A.group + kRows - 1) / kRows);
  const unsigned grid = (unsigned)A.tile_prefix[A.nseg] * (unsigned)c.kv_heads;
  if (dt == SPHINX_F32)
    k_kv8_attn_rows<float, 64><<<grid, kTPB, 0, s>>>(A, c);
  else if (head_dim == 64)
    k_kv8_attn_rows<bf16, 64><<<grid, kTPB, 0, s>>>(A, c);
  else
    k_kv8_attn_rows<bf16, 72><<<grid, kTPB, 0, s>>>(A, c);
  return hipGetLastError();
}

}  // namespace sphinx
