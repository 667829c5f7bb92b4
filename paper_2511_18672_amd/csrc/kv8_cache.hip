// Writing and reading back the 8-bit key/value cache (layout: kv8.hpp).
//
// A block of 64 tokens of one head keeps its keys, and likewise its values, as
// e4m3 numbers with one scale 2^e: with A the largest finite magnitude among
// them, e is the smallest integer with A <= 448 2^e, held in -100 .. 119, and x
// is kept as the e4m3 number nearest to x 2^-e (ties to even), NaN if it is not
// finite.  The scale is a power of two, so multiplying by it is exact, and
// rows that a write leaves alone keep their values when the scale shrinks; when
// it grows by 2^g only those below 2^(e + g - 6) lose bits.

#include <algorithm>
#include <type_traits>

#include "kv8.hpp"

namespace sphinx {

namespace {
typedef float f32x2 __attribute__((ext_vector_type(2)));
constexpr int kTPB = 256;
constexpr int kExpMin = -100, kExpMax = 119;

__device__ __forceinline__ float two_to(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Byte of the scale of a block whose largest finite magnitude is `top`.
__device__ __forceinline__ int scale_byte(float top) {
  const uint32_t b = __float_as_uint(top);
  int e = (int)(b >> 23) - 127 - ((b & 0x7fffffu) <= 0x600000u ? 8 : 7);  // 448 = 1.75 2^8
  if (b < 0x00800000u) e = kExpMin;  // zero or subnormal
  return min(max(e, kExpMin), kExpMax) + 127;
}

__device__ __forceinline__ float finite_abs(float x) {
  const float a = fabsf(x);
  return a < INFINITY ? a : 0.0f;  // NaN compares false
}

// Two values scaled and rounded into half `hi` of `old`.  The hardware rounds to
// nearest even and turns what is past 464, infinities and NaN into NaN; finite
// values past 448, which the largest scale leaves, saturate.
template <bool HI>
__device__ __forceinline__ uint32_t pack2(float a, float b, float inv, uint32_t old) {
  float x = a * inv, y = b * inv;
  if (fabsf(a) < INFINITY) x = fminf(fmaxf(x, -448.0f), 448.0f);
  if (fabsf(b) < INFINITY) y = fminf(fmaxf(y, -448.0f), 448.0f);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x, y, (int)old, HI);
}
__device__ __forceinline__ uint32_t pack4(const float* x, float inv) {
  return pack2<true>(x[2], x[3], inv, pack2<false>(x[0], x[1], inv, 0u));
}

// The values of four stored bytes.
__device__ __forceinline__ void unpack4(uint32_t w, float scale, float* x) {
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  x[0] = a[0] * scale;
  x[1] = a[1] * scale;
  x[2] = b[0] * scale;
  x[3] = b[1] * scale;
}

// n (a multiple of 4) consecutive elements as floats, and back.
template <int N>
__device__ __forceinline__ void load_row(const bf16* p, float* x) {
  constexpr int W = N % 8 == 0 ? 8 : 4;
  typedef __bf16 vec __attribute__((ext_vector_type(W)));
#pragma unroll
  for (int i = 0; i < N; i += W) {
    const vec v = *reinterpret_cast<const vec*>(p + i);
#pragma unroll
    for (int e = 0; e < W; ++e) x[i + e] = (float)v[e];
  }
}
template <int N>
__device__ __forceinline__ void load_row(const float* p, float* x) {
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    const f32x4 v = *reinterpret_cast<const f32x4*>(p + i);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[i + e] = v[e];
  }
}
template <int N>
__device__ __forceinline__ void store_row(bf16* p, const float* x) {
#pragma unroll
  for (int i = 0; i < N; i += 8) {
    bf16x8 v;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (bf16)x[i + e];  // exact: e4m3 times a power of two
    *reinterpret_cast<bf16x8*>(p + i) = v;
  }
}
template <int N>
__device__ __forceinline__ void store_row(float* p, const float* x) {
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    const f32x4 v = {x[i], x[i + 1], x[i + 2], x[i + 3]};
    *reinterpret_cast<f32x4*>(p + i) = v;
  }
}

// Byte offsets inside a tile.
// keys: dims 16 p .. + 15 of a row (p = 4: the eight behind them)
__device__ __forceinline__ int key_off(int row, int p) {
  if (p == 4) return 64 * 64 + row * 8;
  return ((((row >> 5) * 2 + (p & 1)) << 6) + (p >> 1) * 32 + (row & 31)) * 16;
}
// values: keys 4 a .. 4 a + 3 of a dim, four consecutive bytes
__device__ __forceinline__ int val_off(int a, int dim) {
  const int kb = a >> 3, hf = (a >> 2) & 1, j4 = (a >> 1) & 1, g = a & 1;
  const int chunk = dim < 64 ? ((dim >> 5) * 2 + kb) * 64 + g * 32 + (dim & 31) : 256 + (kb * 2 + g) * 8 + (dim - 64);
  return chunk * 16 + hf * 8 + j4 * 4;
}

__device__ __forceinline__ int segment_of(const Kv8Segs& S, int t) {
  int lo = 0, hi = S.nseg - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (S.tok[mid] <= t) lo = mid; else hi = mid - 1;
  }
  return lo;
}
// Block of token t, and its row there; -1 for a token outside the slice.
__device__ __forceinline__ int block_of(const Kv8Segs& S, int t, int* row) {
  if (t < 0 || t >= S.tok[S.nseg]) return -1;
  const int s = segment_of(S, t), at = t - S.tok[s];
  *row = at & (kKv8Block - 1);
  return S.blk[s] + (at >> 6);
}

// The rows of a call fall into runs, one per block, since listed tokens ascend.
// A workgroup looks at `group` rows (of one head) and does the runs that start
// among them; without listed tokens it does block `unit`.  body(block, first row).
template <typename F>
__device__ __forceinline__ void for_each_run(const Kv8Segs& S, const Kv8Rows& rows, int group, int unit, const F& body) {
  if (rows.idx == nullptr) {
    int lo = 0, hi = S.nseg - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (S.blk[mid] <= unit) lo = mid; else hi = mid - 1;
    }
    const int first = S.tok[lo] + (unit - S.blk[lo]) * kKv8Block;
    if (first < rows.n) body(unit, first);
    return;
  }
  const int lane = lane_id();
  const int64_t j = (int64_t)unit * group + lane;
  const bool in = lane < group && j < rows.n;
  int at, block = in ? block_of(S, rows.idx[j], &at) : -1;
  const int before = in && j > 0 ? block_of(S, rows.idx[j - 1], &at) : -1;
  uint64_t starts = __ballot(block >= 0 && block != before);  // the same in every wave
  while (starts != 0) {
    const int l = __builtin_ctzll(starts);
    starts &= starts - 1;
    body(__builtin_amdgcn_readlane(block, l), unit * group + l);
  }
}

// The units of all heads over the workgroups: neighbouring heads of a unit on
// one XCD, one after the other, since a head's piece of a row (144 bytes at
// head_dim 72) shares cache lines with the next head's.
template <typename F>
__device__ __forceinline__ void for_each_unit(const Kv8Segs& S, const Kv8Rows& rows, int kv_heads, int group, int units,
                                              const F& body) {
  const int total = units * kv_heads;
  for (int64_t b = blockIdx.x; b < total; b += gridDim.x) {
    const int u = xcd_tile((int)b, total), unit = u / kv_heads, h = u - unit * kv_heads;
    for_each_run(S, rows, group, unit, [&](int block, int first) { body(h, block, first); });
  }
}

// Row of the call for each row of a block, -1 where none names it; by one wave.
// A token listed more than once takes its last row.
__device__ __forceinline__ void map_rows(const Kv8Segs& S, const Kv8Rows& rows, int block, int first, int* row_at) {
  const int lane = lane_id();
  if (rows.idx == nullptr) {
    const int s = segment_of(S, first), j = first + lane;
    row_at[lane] = j < min(S.tok[s + 1], rows.n) ? j : -1;
    return;
  }
  row_at[lane] = -1;
  for (int64_t j = first + lane;; j += kWave) {
    int at = 0;
    const bool in = j < rows.n && block_of(S, rows.idx[j], &at) == block;
    if (in) atomicMax(&row_at[at], (int)j);
    if (~__ballot(in) != 0) break;  // the run ends here
  }
}

// One workgroup writes one block of one head at a time: the rows of the call and
// the kept rows come together in registers as floats, give the new scales, and
// are rounded once.  A thread has 16 dims of one key row (neighbouring threads
// the same row's next dims, so that a row of a head is read in one piece) and
// four dims of four value rows; head_dim 72: 64 threads more key dims, 32 threads
// more value dims.  Four keys of a dim are four neighbouring bytes of the value
// tile, which is put together in LDS, so that its old bytes come in and its new
// ones go out as consecutive 16-byte pieces.
// Bound by bytes: a full step's rows in and tiles out, in a partial step also
// the old tiles in.
template <typename T, int HD>
__global__ __launch_bounds__(kTPB) void k_kv8_store(Kv8Segs S, Kv8Slice c, Kv8Rows rows, const T* __restrict__ k,
                                                    const T* __restrict__ v, int group, int units) {
  constexpr int NV = kKv8Block * HD / 16;  // 16-byte pieces of a tile
  __shared__ __attribute__((aligned(16))) uint4 image[NV];  // the value tile
  __shared__ int row_at[kKv8Block];
  __shared__ float sh[4][2];
  const int tid = threadIdx.x;
  const int kr = tid >> 2, kp = tid & 3, va = tid >> 4, vd = (tid & 15) * 4;
  unsigned char* img = reinterpret_cast<unsigned char*>(image);
  auto body = [&](int h, int block, int first) {
    unsigned char* kt = c.tiles + ((int64_t)h * c.nblk + block) * 2 * kKv8Block * HD;
    unsigned char* vt = kt + kKv8Block * HD;
    unsigned char* sc = c.scales + ((int64_t)h * c.nblk + block) * 2;
    __syncthreads();  // the block before is done with LDS
    const float ks = __uint_as_float((uint32_t)sc[0] << 23), vs = __uint_as_float((uint32_t)sc[1] << 23);
    const bool whole = rows.idx == nullptr && first + kKv8Block <= rows.n;  // no row is kept, or only padding
    uint4 old = make_uint4(0u, 0u, 0u, 0u);
    uint2 old2 = make_uint2(0u, 0u);
    if (!whole) {
      old = *reinterpret_cast<const uint4*>(kt + key_off(kr, kp));
      if (HD == 72 && tid < 64) old2 = *reinterpret_cast<const uint2*>(kt + key_off(tid, 4));
      for (int i = tid; i < NV; i += kTPB) image[i] = reinterpret_cast<const uint4*>(vt)[i];
    }
    if (tid < kWave) map_rows(S, rows, block, first, row_at);
    __syncthreads();
    float kx[16], vx[4][4], kx2[8], vx2[4][4];
    float ka = 0.0f, vm = 0.0f;
    const int j = row_at[kr];
    if (j >= 0) {
      load_row<16>(k + j * rows.ld + h * HD + kp * 16, kx);
    } else {
      unpack4(old.x, ks, kx);
      unpack4(old.y, ks, kx + 4);
      unpack4(old.z, ks, kx + 8);
      unpack4(old.w, ks, kx + 12);
    }
    // values [dim][key]
    auto gather_v = [&](int a, int d0, float (&x)[4][4]) {
      const int4 at = *reinterpret_cast<const int4*>(row_at + 4 * a);
      const int js[4] = {at.x, at.y, at.z, at.w};
      if (min(min(js[0], js[1]), min(js[2], js[3])) < 0)
#pragma unroll
        for (int e = 0; e < 4; ++e) unpack4(*reinterpret_cast<const uint32_t*>(img + val_off(a, d0 + e)), vs, x[e]);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        if (js[r] < 0) continue;
        float t[4];
        load_row<4>(v + js[r] * rows.ld + h * HD + d0, t);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e][r] = t[e];
      }
    };
    auto top_v = [&](const float (&x)[4][4]) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int r = 0; r < 4; ++r) vm = fmaxf(vm, finite_abs(x[e][r]));
    };
    gather_v(va, vd, vx);
    if constexpr (HD == 72) {
      if (tid < 64) {
        const int j2 = row_at[tid];
        if (j2 >= 0) {
          load_row<8>(k + j2 * rows.ld + h * HD + 64, kx2);
        } else {
          unpack4(old2.x, ks, kx2);
          unpack4(old2.y, ks, kx2 + 4);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) ka = fmaxf(ka, finite_abs(kx2[i]));
      } else if (tid < 96) {
        gather_v((tid - 64) >> 1, 64 + 4 * (tid & 1), vx2);
        top_v(vx2);
      }
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) ka = fmaxf(ka, finite_abs(kx[i]));
    top_v(vx);
    ka = wave_max(ka);
    vm = wave_max(vm);
    if (lane_id() == 0) {
      sh[tid >> 6][0] = ka;
      sh[tid >> 6][1] = vm;
    }
    __syncthreads();
    const int kb = scale_byte(fmaxf(fmaxf(sh[0][0], sh[1][0]), fmaxf(sh[2][0], sh[3][0])));
    const int vb = scale_byte(fmaxf(fmaxf(sh[0][1], sh[1][1]), fmaxf(sh[2][1], sh[3][1])));
    const float ki = two_to(127 - kb), vi = two_to(127 - vb);
    *reinterpret_cast<uint4*>(kt + key_off(kr, kp)) =
        make_uint4(pack4(kx, ki), pack4(kx + 4, ki), pack4(kx + 8, ki), pack4(kx + 12, ki));
#pragma unroll
    for (int e = 0; e < 4; ++e) *reinterpret_cast<uint32_t*>(img + val_off(va, vd + e)) = pack4(vx[e], vi);
    if constexpr (HD == 72) {
      if (tid < 64)
        *reinterpret_cast<uint2*>(kt + key_off(tid, 4)) = make_uint2(pack4(kx2, ki), pack4(kx2 + 4, ki));
      else if (tid < 96)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          *reinterpret_cast<uint32_t*>(img + val_off((tid - 64) >> 1, 64 + 4 * (tid & 1) + e)) = pack4(vx2[e], vi);
    }
    if (tid == 0) {
      sc[0] = (unsigned char)kb;
      sc[1] = (unsigned char)vb;
    }
    __syncthreads();
    for (int i = tid; i < NV; i += kTPB) reinterpret_cast<uint4*>(vt)[i] = image[i];
  };
  for_each_unit(S, rows, c.kv_heads, group, units, body);
}

// One workgroup reads the listed rows of one block of one head at a time.
template <typename T, int HD>
__global__ __launch_bounds__(kTPB) void k_kv8_load(Kv8Segs S, Kv8Slice c, Kv8Rows rows, T* __restrict__ k,
                                                   T* __restrict__ v, int group, int units) {
  __shared__ __attribute__((aligned(16))) unsigned char sv[kKv8Block * HD];
  constexpr int NP = HD / 8;  // pieces of eight dims
  const int tid = threadIdx.x;
  auto body = [&](int h, int block, int first) {
    const unsigned char* kt = c.tiles + ((int64_t)h * c.nblk + block) * 2 * kKv8Block * HD;
    const unsigned char* vt = kt + kKv8Block * HD;
    const unsigned char* sc = c.scales + ((int64_t)h * c.nblk + block) * 2;
    __syncthreads();  // the block before is done with LDS
    for (int i = tid; i < kKv8Block * HD / 16; i += kTPB)
      reinterpret_cast<uint4*>(sv)[i] = reinterpret_cast<const uint4*>(vt)[i];
    const float ks = __uint_as_float((uint32_t)sc[0] << 23), vs = __uint_as_float((uint32_t)sc[1] << 23);
    __syncthreads();
    const int end = rows.idx == nullptr ? min(rows.n, S.tok[segment_of(S, first) + 1]) : rows.n;
    for (int i = tid;; i += kTPB) {
      const int64_t j = (int64_t)first + i / NP;
      const int p = i % NP;
      if (j >= end) break;
      int at = (int)(j - first);
      if (rows.idx == nullptr ? at >= kKv8Block : block_of(S, rows.idx[j], &at) != block) break;
      float x[8];
      const int off = p < 8 ? key_off(at, p >> 1) + 8 * (p & 1) : key_off(at, 4);
      const uint2 b = *reinterpret_cast<const uint2*>(kt + off);
      unpack4(b.x, ks, x);
      unpack4(b.y, ks, x + 4);
      store_row<8>(k + j * rows.ld + h * HD + p * 8, x);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        x[e] = __builtin_amdgcn_cvt_pk_f32_fp8((int)sv[val_off(at >> 2, p * 8 + e) + (at & 3)], false)[0] * vs;
      store_row<8>(v + j * rows.ld + h * HD + p * 8, x);
    }
  };
  for_each_unit(S, rows, c.kv_heads, group, units, body);
}

template <typename F>
hipError_t by_type(sphinx_dtype dt, int head_dim, const F& go) {
  if (dt == SPHINX_BF16 && head_dim == 64) go(bf16{}, std::integral_constant<int, 64>{});
  else if (dt == SPHINX_BF16) go(bf16{}, std::integral_constant<int, 72>{});
  else if (head_dim == 64) go(float{}, std::integral_constant<int, 64>{});
  else go(float{}, std::integral_constant<int, 72>{});
  return hipGetLastError();
}

// Rows that a workgroup looks at: one workgroup per row and head where that makes
// no more than about 8192 (four rounds of a full chip); with many rows several of
// them share a block anyway.
struct Split {
  int group, units;
  unsigned grid;
};
Split split(const Kv8Slice& c, const Kv8Rows& rows) {
  Split p;
  p.group = (int)std::clamp<int64_t>((int64_t)rows.n * c.kv_heads / 8192, 1, 16);
  p.units = rows.idx ? (int)(((int64_t)rows.n + p.group - 1) / p.group) : (int)c.nblk;
  p.grid = (unsigned)std::min<int64_t>((int64_t)p.units * c.kv_heads, 1 << 20);  // each then takes several
  return p;
}
}  // namespace

hipError_t launch_kv8_store(sphinx_dtype dt, int head_dim, const Kv8Segs& S, const Kv8Slice& c, const Kv8Rows& rows,
                            const void* k, const void* v, hipStream_t s) {
  const Split p = split(c, rows);
  return by_type(dt, head_dim, [&](auto t, auto hd) {
    using T = decltype(t);
    k_kv8_store<T, decltype(hd)::value><<<p.grid, kTPB, 0, s>>>(S, c, rows, static_cast<const T*>(k),
                                                                static_cast<const T*>(v), p.group, p.units);
  });
}

hipError_t launch_kv8_load(sphinx_dtype dt, int head_dim, const Kv8Segs& S, const Kv8Slice& c, const Kv8Rows& rows,
                           void* k, void* v, hipStream_t s) {
  const Split p = split(c, rows);
  return by_type(dt, head_dim, [&](auto t, auto hd) {
    using T = decltype(t);
    k_kv8_load<T, decltype(hd)::value>
        <<<p.grid, kTPB, 0, s>>>(S, c, rows, static_cast<T*>(k), static_cast<T*>(v), p.group, p.units);
  });
}

}  // namespace sphinx
