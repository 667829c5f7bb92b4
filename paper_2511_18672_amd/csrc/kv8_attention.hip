// Attention over the 8-bit key/value cache (layout: kv8.hpp): per segment and
// query head o = sum_t 2^(q.k_t) v_t / sum_t 2^(q.k_t) over the segment's cached
// tokens, keys and values being the numbers that the cache's bytes stand for.

#include <algorithm>
#include <type_traits>

#include "kv8.hpp"
#include "kv8_rules.hpp"

namespace sphinx {

namespace {
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
constexpr int kTPB = 256;
constexpr int kRows = kKv8RowTile;  // rows (queries of the heads that share a key/value head) per workgroup

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// Partial results: row r of head h, chunk j of segment i is number
// part[i] + (h rows_i + r) chunks_i + j: its running maximum and sum, and O.
struct Parts {
  float2* ml;
  float* o;  // [number][head_dim]
};

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

// One workgroup = 32 rows of one segment and key/value head against one chunk of
// the segment's keys; its four waves take the chunk's blocks in turn and merge
// (m, l, O) through LDS.  A wave reads a block's bytes straight into the operand
// layouts, the next block's while it works on this one's:
//  * S^T = K Q^T in two 32-key tiles: lane l = 32 g + r has key r and dims
//    32 g .. + 31 (two chunks), for the queries the same dims of row r;
//  * P^T needs no move: score register 8 hf + j of tile kb belongs to the key
//    that byte 8 hf + j of the values' chunk (db, kb) holds;
//  * O^T = V^T P^T leaves the row on the lane.
// bf16: 32x32x16 products, P rounded to bf16 for the product, the row sum adding
// the same rounded values; f32: 32x32x2 products, nothing rounded.
template <typename T, int HD>
__global__ __launch_bounds__(kTPB, 2) void k_kv8_attn_rows(Kv8Attn A, Kv8Slice c, Kv8Plan P, Parts part, int first) {
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int DB = (HD + 31) / 32;
  __shared__ float sO[4][kRows][DB * 32 + 1];
  __shared__ float sM[4][kRows], sL[4][kRows];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 5, r32 = lane & 31;
  const int unit = first + (int)blockIdx.x, h = unit % c.kv_heads, item = unit / c.kv_heads;
  int s = 0;
  while (s + 1 < A.nseg && P.item[s + 1] <= item) ++s;
  const int chunks = P.chunks[s], tile = (item - P.item[s]) / chunks, chunk = item - P.item[s] - tile * chunks;
  const int row0 = tile * kRows, nrows = A.nq[s] * A.group;
  const int L = A.klen[s], b0 = chunk * P.chunk, nb = min((L + kKv8Block - 1) / kKv8Block, b0 + P.chunk);
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
  for (int b = b0 + wave; b < nb; b += 4) {
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
    if (b + 4 < nb) fetch(b + 4);
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
        const uint32_t w = kt8[rb];
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
          sc[kb][r] = fast_exp2(sc[kb][r] - at);
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
          pf[r >> 3][r & 7] = (bf16)fast_exp2(sc[kb][r] - at);
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
  for (int i = tid; i < kRows * HD; i += kTPB) {
    const int row = i / HD, d = i - row * HD;
    if (row0 + row >= nrows) break;
    const float mm = fmaxf(fmaxf(sM[0][row], sM[1][row]), fmaxf(sM[2][row], sM[3][row]));
    const float at = mm == -INFINITY ? 0.0f : mm;
    float num = 0.0f, den = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {  // a wave without a block has m = -inf and weighs 0
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

// Joins the chunks of a row: one workgroup of eight waves per row and head, wave
// w taking chunks w (mod 8), or (few chunks) one wave per row.  A lane has one
// dim; at head_dim 72 eight lanes have a second one.
template <typename T, int HD, int WAVES>
__global__ __launch_bounds__(512) void k_kv8_attn_join(Kv8Attn A, int kv_heads, Kv8Plan P, Parts part, int rows) {
  __shared__ float sO[WAVES][HD], sL[WAVES], sM[WAVES];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int unit = WAVES == 1 ? (int)blockIdx.x * 8 + wave : (int)blockIdx.x;  // row * kv_heads + head
  if (unit >= rows * kv_heads) return;  // only with one wave per row, which has no barrier
  const int h = unit % kv_heads, at = unit / kv_heads;
  int s = 0;
  while (s + 1 < A.nseg && P.row[s + 1] <= at) ++s;
  const int row = at - P.row[s], chunks = P.chunks[s], nrows = A.nq[s] * A.group;
  const int64_t first = P.part[s] + ((int64_t)h * nrows + row) * chunks;
  const int w0 = WAVES == 1 ? 0 : wave;
  float m = -INFINITY;
  for (int j = lane; j < chunks; j += kWave) m = fmaxf(m, part.ml[first + j].x);
  m = wave_max(m);
  const float base = m == -INFINITY ? 0.0f : m;
  float num = 0.0f, num2 = 0.0f, den = 0.0f;
  constexpr int U = 8;
  for (int j0 = w0; j0 < chunks; j0 += WAVES * U) {
    float2 ml[U];
    float o[U], o2[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t j = first + min(j0 + u * WAVES, chunks - 1);
      ml[u] = part.ml[j];
      o[u] = part.o[j * HD + lane];
      o2[u] = HD == 72 ? part.o[j * HD + 64 + (lane & 7)] : 0.0f;
    }
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
    if (lane == 0) sL[wave] = den;
    __syncthreads();
    if (wave != 0) return;
    num = num2 = den = 0.0f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      num += sO[w][lane];
      if (HD == 72) num2 += sO[w][64 + (lane & 7)];
      den += sL[w];
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
  const Kv8Plan P = plan_kv8(c.kv_heads, A.nseg, rows, A.klen);
  const size_t parts = (size_t)P.part[A.nseg];
  const Parts part{static_cast<float2*>(ws),
                   reinterpret_cast<float*>(static_cast<unsigned char*>(ws) + ((parts * 8 + 255) & ~(size_t)255))};
  // at most 2^31 / 32 tiles; a launch holds 2^32 threads, so 2^23 workgroups at a time
  const int total = P.item[A.nseg] * c.kv_heads, most_wg = 1 << 23;
  auto go = [&](auto t, auto hd) {
    using T = decltype(t);
    constexpr int HD = decltype(hd)::value;
    for (int first = 0; first < total; first += most_wg)
      k_kv8_attn_rows<T, HD><<<std::min(most_wg, total - first), kTPB, 0, s>>>(A, c, P, part, first);
    if (parts == 0) return;
    const int join = P.row[A.nseg];
    int most = 0;
    for (int i = 0; i < A.nseg; ++i) most = std::max(most, P.chunks[i]);
    if (most <= 8)
      k_kv8_attn_join<T, HD, 1><<<(unsigned)(((int64_t)join * c.kv_heads + 7) / 8), 512, 0, s>>>(A, c.kv_heads, P,
                                                                                              part, join);
    else
      k_kv8_attn_join<T, HD, 8><<<(unsigned)join * (unsigned)c.kv_heads, 512, 0, s>>>(A, c.kv_heads, P, part, join);
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
