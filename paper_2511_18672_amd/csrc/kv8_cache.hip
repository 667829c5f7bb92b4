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
  static_assert(N % 4 == 0, "whole 8-byte pieces");
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    const bf16x4 v = *reinterpret_cast<const bf16x4*>(p + i);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[i + e] = (float)v[e];
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
  for (int i = 0; i < N; i += 4) {
    bf16x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = (bf16)x[i + e];  // exact: e4m3 times a power of two
    *reinterpret_cast<bf16x4*>(p + i) = v;
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

// The rows of a call that fall into one block: rows [first, first + count) of
// the call.  Work unit w of a call with listed tokens is row w, and only the
// first row of a run of rows in one block has work; without listed tokens unit w
// is block w.
struct Run {
  int block, first, count;
};
__device__ __forceinline__ bool find_run(const Kv8Segs& S, const Kv8Rows& rows, int w, Run* run) {
  int at;
  if (rows.idx == nullptr) {
    int lo = 0, hi = S.nseg - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (S.blk[mid] <= w) lo = mid; else hi = mid - 1;
    }
    run->block = w;
    run->first = S.tok[lo] + (w - S.blk[lo]) * kKv8Block;
    run->count = min(min(kKv8Block, S.tok[lo + 1] - run->first), rows.n - run->first);
    return run->count > 0;
  }
  run->block = block_of(S, rows.idx[w], &at);
  if (run->block < 0 || (w > 0 && block_of(S, rows.idx[w - 1], &at) == run->block)) return false;
  run->first = w;
  const int lane = lane_id();
  int n = 0;
  for (;;) {  // lanes look 64 rows ahead
    const int j = w + n + lane;
    const bool in = j < rows.n && block_of(S, rows.idx[j], &at) == run->block;
    const uint64_t out = ~__ballot(in);
    if (out != 0) {
      n += __builtin_ctzll(out);
      break;
    }
    n += kWave;
  }
  run->count = n;
  return true;
}

// Largest value over the workgroup, in every thread (two at once).
__device__ __forceinline__ void block_max(float& a, float& b, float (*sh)[2]) {
  a = wave_max(a);
  b = wave_max(b);
  __syncthreads();
  if (lane_id() == 0) {
    sh[threadIdx.x >> 6][0] = a;
    sh[threadIdx.x >> 6][1] = b;
  }
  __syncthreads();
  a = fmaxf(fmaxf(sh[0][0], sh[1][0]), fmaxf(sh[2][0], sh[3][0]));
  b = fmaxf(fmaxf(sh[0][1], sh[1][1]), fmaxf(sh[2][1], sh[3][1]));
}

// One workgroup writes one block of one head: the rows of the call and the kept
// rows of the block come together in registers as floats, give the new scales,
// and are rounded once.  A thread has 16 dims of one key row and four dims of
// four value rows (then four keys of a dim are one 4-byte store); head_dim 72:
// one wave more key dims, half a wave more value dims.
template <typename T, int HD>
__global__ __launch_bounds__(kTPB) void k_kv8_store(Kv8Segs S, Kv8Slice c, Kv8Rows rows, const T* __restrict__ k,
                                                    const T* __restrict__ v, int64_t units) {
  __shared__ int row_at[kKv8Block];  // row of the call for each row of the block, -1: kept
  __shared__ float sh[4][2];
  const int tid = threadIdx.x;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int h = (int)(u % c.kv_heads), w = (int)(u / c.kv_heads);
    Run run;
    if (!find_run(S, rows, w, &run)) continue;  // the same for all threads
    __syncthreads();
    if (tid < kKv8Block) row_at[tid] = -1;
    __syncthreads();
    for (int i = tid; i < run.count; i += kTPB) {
      int at = i;
      if (rows.idx != nullptr) block_of(S, rows.idx[run.first + i], &at);
      atomicMax(&row_at[at], run.first + i);  // a token listed twice takes its last row
    }
    __syncthreads();
    unsigned char* kt = c.tiles + ((int64_t)h * c.nblk + run.block) * 2 * kKv8Block * HD;
    unsigned char* vt = kt + kKv8Block * HD;
    unsigned char* sc = c.scales + ((int64_t)h * c.nblk + run.block) * 2;
    const float ks = __uint_as_float((uint32_t)sc[0] << 23), vs = __uint_as_float((uint32_t)sc[1] << 23);
    const int kr = tid >> 2, kp = tid & 3, va = tid >> 4, vd = (tid & 15) * 4;
    float kx[16], vx[4][4], kx2[8], vx2[4][4];
    float ka = 0.0f, vm = 0.0f;
    {
      const int j = row_at[kr];
      if (j >= 0) {
        load_row<16>(k + j * rows.ld + h * HD + kp * 16, kx);
      } else {
        const uint4 b = *reinterpret_cast<const uint4*>(kt + key_off(kr, kp));
        unpack4(b.x, ks, kx);
        unpack4(b.y, ks, kx + 4);
        unpack4(b.z, ks, kx + 8);
        unpack4(b.w, ks, kx + 12);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) ka = fmaxf(ka, finite_abs(kx[i]));
    }
    // values [dim][key]
    auto gather_v = [&](int a, int d0, float (&x)[4][4]) {
      bool kept = false;
#pragma unroll
      for (int r = 0; r < 4; ++r) kept |= row_at[4 * a + r] < 0;
      if (kept)
#pragma unroll
        for (int e = 0; e < 4; ++e) unpack4(*reinterpret_cast<const uint32_t*>(vt + val_off(a, d0 + e)), vs, x[e]);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int j = row_at[4 * a + r];
        if (j < 0) continue;
        float t[4];
        load_row<4>(v + j * rows.ld + h * HD + d0, t);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e][r] = t[e];
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int r = 0; r < 4; ++r) vm = fmaxf(vm, finite_abs(x[e][r]));
    };
    gather_v(va, vd, vx);
    if constexpr (HD == 72) {
      if (tid < 64) {
        const int j = row_at[tid];
        if (j >= 0) {
          load_row<8>(k + j * rows.ld + h * HD + 64, kx2);
        } else {
          const uint2 b = *reinterpret_cast<const uint2*>(kt + key_off(tid, 4));
          unpack4(b.x, ks, kx2);
          unpack4(b.y, ks, kx2 + 4);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) ka = fmaxf(ka, finite_abs(kx2[i]));
      } else if (tid < 96) {
        gather_v((tid - 64) >> 1, 64 + 4 * (tid & 1), vx2);
      }
    }
    block_max(ka, vm, sh);
    const int kb = scale_byte(ka), vb = scale_byte(vm);
    const float ki = two_to(127 - kb), vi = two_to(127 - vb);
    *reinterpret_cast<uint4*>(kt + key_off(kr, kp)) =
        make_uint4(pack4(kx, ki), pack4(kx + 4, ki), pack4(kx + 8, ki), pack4(kx + 12, ki));
#pragma unroll
    for (int e = 0; e < 4; ++e) *reinterpret_cast<uint32_t*>(vt + val_off(va, vd + e)) = pack4(vx[e], vi);
    if constexpr (HD == 72) {
      if (tid < 64)
        *reinterpret_cast<uint2*>(kt + key_off(tid, 4)) = make_uint2(pack4(kx2, ki), pack4(kx2 + 4, ki));
      else if (tid < 96)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          *reinterpret_cast<uint32_t*>(vt + val_off((tid - 64) >> 1, 64 + 4 * (tid & 1) + e)) = pack4(vx2[e], vi);
    }
    if (tid == 0) {
      sc[0] = (unsigned char)kb;
      sc[1] = (unsigned char)vb;
    }
  }
}

// One workgroup reads the listed rows of one block of one head.
template <typename T, int HD>
__global__ __launch_bounds__(kTPB) void k_kv8_load(Kv8Segs S, Kv8Slice c, Kv8Rows rows, T* __restrict__ k,
                                                   T* __restrict__ v, int64_t units) {
  __shared__ __attribute__((aligned(16))) unsigned char sv[kKv8Block * HD];
  const int tid = threadIdx.x;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int h = (int)(u % c.kv_heads), w = (int)(u / c.kv_heads);
    Run run;
    if (!find_run(S, rows, w, &run)) continue;  // the same for all threads
    const unsigned char* kt = c.tiles + ((int64_t)h * c.nblk + run.block) * 2 * kKv8Block * HD;
    const unsigned char* vt = kt + kKv8Block * HD;
    const unsigned char* sc = c.scales + ((int64_t)h * c.nblk + run.block) * 2;
    const float ks = __uint_as_float((uint32_t)sc[0] << 23), vs = __uint_as_float((uint32_t)sc[1] << 23);
    __syncthreads();
    for (int i = tid; i < kKv8Block * HD / 16; i += kTPB)
      reinterpret_cast<uint4*>(sv)[i] = reinterpret_cast<const uint4*>(vt)[i];
    __syncthreads();
    constexpr int NP = HD / 8;  // pieces of eight dims
    for (int i = tid; i < run.count * NP; i += kTPB) {
      const int j = run.first + i / NP, p = i % NP;
      int at = j - run.first;
      if (rows.idx != nullptr) block_of(S, rows.idx[j], &at);
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
  }
}

template <typename F>
hipError_t by_type(sphinx_dtype dt, int head_dim, const F& go) {
  if (dt == SPHINX_BF16 && head_dim == 64) go(bf16{}, std::integral_constant<int, 64>{});
  else if (dt == SPHINX_BF16) go(bf16{}, std::integral_constant<int, 72>{});
  else if (head_dim == 64) go(float{}, std::integral_constant<int, 64>{});
  else go(float{}, std::integral_constant<int, 72>{});
  return hipGetLastError();
}
// workgroups of a launch: one per unit, at most 2^20 (each then takes several)
unsigned unit_grid(int64_t units) { return (unsigned)std::min<int64_t>(units, 1 << 20); }
}  // namespace

hipError_t launch_kv8_store(sphinx_dtype dt, int head_dim, const Kv8Segs& S, const Kv8Slice& c, const Kv8Rows& rows,
                            const void* k, const void* v, hipStream_t s) {
  const int64_t units = (rows.idx ? (int64_t)rows.n : c.nblk) * c.kv_heads;
  return by_type(dt, head_dim, [&](auto t, auto hd) {
    using T = decltype(t);
    k_kv8_store<T, decltype(hd)::value><<<unit_grid(units), kTPB, 0, s>>>(
        S, c, rows, static_cast<const T*>(k), static_cast<const T*>(v), units);
  });
}

hipError_t launch_kv8_load(sphinx_dtype dt, int head_dim, const Kv8Segs& S, const Kv8Slice& c, const Kv8Rows& rows,
                           void* k, void* v, hipStream_t s) {
  const int64_t units = (rows.idx ? (int64_t)rows.n : c.nblk) * c.kv_heads;
  return by_type(dt, head_dim, [&](auto t, auto hd) {
    using T = decltype(t);
    k_kv8_load<T, decltype(hd)::value>
        <<<unit_grid(units), kTPB, 0, s>>>(S, c, rows, static_cast<T*>(k), static_cast<T*>(v), units);
  });
}

}  // namespace sphinx
