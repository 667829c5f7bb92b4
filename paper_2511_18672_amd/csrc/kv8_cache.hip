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

// Four values scaled and rounded.  The hardware rounds to nearest even and turns
// what is past 464, infinities and NaN into NaN.
__device__ __forceinline__ uint32_t pack4(float x0, float x1, float x2, float x3, float inv) {
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(x0 * inv, x1 * inv, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x2 * inv, x3 * inv, lo, true);
}

// The values of four stored bytes.
__device__ __forceinline__ void unpack4(uint32_t w, float scale, float* x) {
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  x[0] = a[0] * scale;
  x[1] = a[1] * scale;
  x[2] = b[0] * scale;
  x[3] = b[1] * scale;
}

// n consecutive floats as elements.
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

// Block of token t, and its row there; -1 for a token outside the slice.  Every
// lane looks at every segment, whose bounds come through scalar loads; a search
// by lanes would be a chain of vector loads from the kernel's arguments.
__device__ __forceinline__ int block_of(const Kv8Segs& S, int t, int* row) {
  int tok = 0, blk = 0;
  for (int s = 1; s < S.nseg; ++s) {
    const bool behind = t >= S.tok[s];
    tok = behind ? S.tok[s] : tok;
    blk = behind ? S.blk[s] : blk;
  }
  const int at = t - tok;
  *row = at & (kKv8Block - 1);
  return t < 0 || t >= S.tok[S.nseg] ? -1 : blk + (at >> 6);
}

// Largest number over a wave.
__device__ __forceinline__ uint32_t wave_top(uint32_t v) {
  auto other = [&](auto ctrl) {
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, decltype(ctrl)::value, 0xf, 0xf, false);
  };
  v = max(v, other(std::integral_constant<int, 0xB1>{}));   // lane ^ 1
  v = max(v, other(std::integral_constant<int, 0x4E>{}));   // lane ^ 2
  v = max(v, other(std::integral_constant<int, 0x141>{}));  // the other quad of the 8-lane half
  v = max(v, other(std::integral_constant<int, 0x140>{}));  // the other half of the row
  const auto r16 = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = max((uint32_t)r16[0], (uint32_t)r16[1]);
  const auto r32 = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return max((uint32_t)r32[0], (uint32_t)r32[1]);
}

// LDS operations of a wave are done in order; this keeps the compiler from moving
// them across.
__device__ __forceinline__ void lds_order() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_wave_barrier();
}

// The rows of a call fall into runs, one per block, since listed tokens ascend.
// A wave (or every wave of a workgroup alike) looks at `group` rows and does the
// runs that start among them; without listed tokens it does block `unit`.
struct Run {
  int block, first;  // the run's block and its first row of the call
  int count;         // rows of the block, from its first, that rows `first` and on fill; -1: some listed tokens
  int from, at, lane_block;  // listed tokens: row of the call, row and block of this lane's token (rows from .. + 63)
};
template <bool WHOLE, typename F>
__device__ __forceinline__ void for_each_run(const Kv8Segs& S, const Kv8Rows& rows, int group, int unit, const F& body) {
  if (rows.idx == nullptr) {
    int lo = 0, hi = S.nseg - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (S.blk[mid] <= unit) lo = mid; else hi = mid - 1;
    }
    const int first = S.tok[lo] + (unit - S.blk[lo]) * kKv8Block;
    const int count = min(min(kKv8Block, S.tok[lo + 1] - first), rows.n - first);
    if (count > 0) body(Run{unit, first, count, 0, 0, 0});
    return;
  }
  const int lane = lane_id(), from = unit * group;
  const int64_t j = (int64_t)from + lane;
  const int prev = from > 0 ? rows.idx[from - 1] : -1;
  const int token = j < rows.n ? rows.idx[j] : -1, further = WHOLE && j + kWave < rows.n ? rows.idx[j + kWave] : -1;
  int at, before_at;
  const int block = block_of(S, token, &at);
  int before = __shfl_up(block, 1, kWave);
  if (lane == 0) before = block_of(S, prev, &before_at);
  uint64_t starts = __ballot(lane < group && block >= 0 && block != before);  // the same in every wave
  while (starts != 0) {
    const int l = __builtin_ctzll(starts);
    starts &= starts - 1;
    // WHOLE: looks for runs of all 64 tokens of a block, one row each (the row behind
    // them is another block's), which keep no row.
    const int run_block = __builtin_amdgcn_readlane(block, l);
    const int t0 = __builtin_amdgcn_readlane(token, l), row0 = __builtin_amdgcn_readlane(at, l);
    const bool next = lane >= l ? token == t0 + lane - l : further == t0 + kWave + lane - l;
    const bool whole = WHOLE && row0 == 0 && __ballot(next) == ~0ull &&
                       block_of(S, t0 + kKv8Block - 1, &before_at) == run_block &&
                       block_of(S, __builtin_amdgcn_readlane(further, l), &before_at) != run_block;
    body(Run{run_block, from + l, whole ? kKv8Block : -1, from, at, block});
  }
}

// The units of all heads over the workgroups: neighbouring heads of a unit on
// one XCD, one after the other, since a head's piece of a row (144 bytes at
// head_dim 72) shares cache lines with the next head's.  `per`: units that a
// workgroup does at a time, this is its `mine`-th.
template <bool WHOLE, typename F>
__device__ __forceinline__ void for_each_unit(const Kv8Segs& S, const Kv8Rows& rows, int heads, int group, int units,
                                              int per, int mine, const F& body) {
  const int total = units * heads, groups = (total + per - 1) / per;
  for (int64_t b = blockIdx.x; b < groups; b += gridDim.x) {
    const int u = xcd_tile((int)b, groups) * per + mine;
    if (u >= total) continue;
    const int unit = u / heads, h = u - unit * heads;
    for_each_run<WHOLE>(S, rows, group, unit, [&](const Run& run) { body(h, run); });
  }
}

// Row of the call for each row of a run's block, -1 where none names it, in LDS;
// by one wave.  A token listed more than once takes its last row.
__device__ __forceinline__ void map_rows(const Kv8Segs& S, const Kv8Rows& rows, const Run& run, int* row_at) {
  const int lane = lane_id();
  if (run.count >= 0) {
    row_at[lane] = lane < run.count ? run.first + lane : -1;
    return;
  }
  row_at[lane] = -1;
  lds_order();
  const bool here = run.from + lane >= run.first && run.lane_block == run.block;
  if (here) atomicMax(&row_at[run.at], run.from + lane);
  if ((__ballot(here) >> 63) == 0) return;  // the run ends among the lanes' tokens
  for (int64_t j = (int64_t)run.from + kWave + lane;; j += kWave) {
    int at = 0;
    const bool in = block_of(S, j < rows.n ? rows.idx[j] : -1, &at) == run.block;
    if (in) atomicMax(&row_at[at], (int)j);
    if (~__ballot(in) != 0) return;
  }
}

// Eight elements of a row as they came.  peak: the largest magnitude, as the bits
// of a float.  set: values of stored bytes, which both types hold exactly.
template <typename T>
struct Piece;
template <>
struct Piece<bf16> {
  uint32_t w[4];
  __device__ __forceinline__ void load(const bf16* p) {
    const uint4 x = *reinterpret_cast<const uint4*>(p);
    w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
  }
  __device__ __forceinline__ float get(int i) const {
    return __uint_as_float((i & 1) ? (w[i >> 1] & 0xffff0000u) : (w[i >> 1] << 16));
  }
  __device__ __forceinline__ void set2(int i, float a, float b) {
    bf16x2 v;
    v[0] = (bf16)a;
    v[1] = (bf16)b;
    w[i >> 1] = __builtin_bit_cast(uint32_t, v);
  }
  __device__ __forceinline__ uint32_t peak() const {
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    u16x2 m = __builtin_bit_cast(u16x2, w[0] & 0x7fff7fffu);
#pragma unroll
    for (int i = 1; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w[i] & 0x7fff7fffu));
    return (uint32_t)max(m[0], m[1]) << 16;
  }
};
template <>
struct Piece<float> {
  float x[8];
  __device__ __forceinline__ void load(const float* p) {
    const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = a[i];
      x[4 + i] = b[i];
    }
  }
  __device__ __forceinline__ float get(int i) const { return x[i]; }
  __device__ __forceinline__ void set2(int i, float a, float b) {
    x[i] = a;
    x[i + 1] = b;
  }
  __device__ __forceinline__ uint32_t peak() const {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);
    return m;
  }
};
template <typename T>
__device__ __forceinline__ uint32_t finite_peak(const Piece<T>& p) {  // the same of the finite ones
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t b = __float_as_uint(p.get(i)) & 0x7fffffffu;
    m = b < 0x7f800000u ? max(m, b) : m;
  }
  return m;
}

// Keeps what follows from being computed before here, where it would be held in
// twice the registers.
__device__ __forceinline__ void hold(Piece<bf16>& p) {
#pragma unroll
  for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(p.w[i]));
}
__device__ __forceinline__ void hold(Piece<float>&) {}
template <typename T>
__device__ __forceinline__ void saturate(Piece<T>& p) {  // finite ones to 448 times the largest scale
  const float lim = 448.0f * two_to(kExpMax);
  auto of = [&](float x) { return fabsf(x) < INFINITY ? fminf(fmaxf(x, -lim), lim) : x; };
#pragma unroll
  for (int i = 0; i < 8; i += 2) p.set2(i, of(p.get(i)), of(p.get(i + 1)));
}

// One wave writes the keys or the values of one block of one head at a time:
// lane (a, c) = (l / 8, l % 8) has dims 8 c .. + 7 of rows 8 a .. + 7, so that
// eight loads bring the 64 rows, eight whole rows each; head_dim 72: lane l also
// has the last eight dims of row l.  Rows that are kept are made from the old
// tile, which comes into LDS in consecutive 16-byte pieces, and are then treated
// like new ones.  The largest magnitude is one reduction over the wave; the
// rounded bytes are put in the tile's order in LDS and leave in 16-byte pieces.
// Bound by bytes: a full step's rows in and tiles out, in a partial step also the
// old tiles in.  A wave and not a workgroup per tile: a workgroup spends the way
// of a row to its bytes on barriers.  bf16 has to fit 128 registers, so that four
// waves per SIMD wait for memory at once: 9677 listed of 32256 tokens, 16 heads
// of 64, caches not at hand, 56 -> 50 us, and 44 since the old tile goes to LDS past
// the registers; all of them 55 -> 48.
template <typename T, int HD>
__global__ __launch_bounds__(kTPB, sizeof(T) == 2 ? 4 : 2)
void k_kv8_store(Kv8Segs S, Kv8Slice c, Kv8Rows rows, const T* __restrict__ k, const T* __restrict__ v, int group,
                 int units) {
  constexpr int NV = kKv8Block * HD / 16;  // 16-byte pieces of a tile
  __shared__ __attribute__((aligned(16))) uint4 images[4][NV];
  __shared__ __attribute__((aligned(16))) int maps[4][kKv8Block];
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  unsigned char* img = reinterpret_cast<unsigned char*>(images[wave]);
  int* row_at = maps[wave];
  const int a = lane >> 3, cc = lane & 7;
  // Offsets in the tile, from which the others are constants further: 16 r of row
  // 8 a + r, 512 g + 16 e of keys 8 a + 4 g .. + 3 of dim 8 c + e.
  const int key0 = key_off(8 * a, cc >> 1) + 8 * (cc & 1), val0 = val_off(2 * a, 8 * cc);
  const int key_tail = key_off(lane, 4), val_tail = val_off(lane >> 2, 64) + (lane & 3);
  auto body = [&](int hh, const Run& run) {
    const int h = hh >> 1;
    const bool values = (hh & 1) != 0;  // the same for the whole wave
    unsigned char* tile = c.tiles + (((int64_t)h * c.nblk + run.block) * 2 + (values ? 1 : 0)) * kKv8Block * HD;
    unsigned char* sc = c.scales + ((int64_t)h * c.nblk + run.block) * 2 + (values ? 1 : 0);
    const T* src = (values ? v : k) + h * HD;
    Piece<T> p[8], pt;
    lds_order();  // the tile before has left LDS
    if (run.count == kKv8Block) {  // no row is kept
      const T* row = src + (run.first + 8 * a) * rows.ld + 8 * cc;
#pragma unroll
      for (int r = 0; r < 8; ++r) p[r].load(row + r * rows.ld);
      if constexpr (HD == 72) pt.load(src + (run.first + lane) * rows.ld + 64);
    } else {
      // the old tile goes straight to LDS while the rows are looked for
#pragma unroll
      for (int i = 0; i < NV; i += kWave)
        if (i + kWave <= NV || lane < NV - i)
          lds_dma16_at(tile, (uint32_t)(i + lane) * 16, &images[wave][i]);
      const float old = __uint_as_float((uint32_t)*sc << 23);
      map_rows(S, rows, run, row_at);
      lds_order();
      const int4 x = *reinterpret_cast<const int4*>(row_at + 8 * a), y = *reinterpret_cast<const int4*>(row_at + 8 * a + 4);
      const int js[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
      // the kept rows' loads are of row 0 of the call and are replaced
#pragma unroll
      for (int r = 0; r < 8; ++r) p[r].load(src + max(js[r], 0) * rows.ld + 8 * cc);
      const int jt = row_at[lane];
      if constexpr (HD == 72) pt.load(src + max(jt, 0) * rows.ld + 64);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the old tile is in LDS
      if (__ballot(jt < 0) != 0) {
        if (!values) {
#pragma unroll
          for (int r = 0; r < 8; ++r) {
            const uint2 w = *reinterpret_cast<const uint2*>(img + key0 + 16 * r);
            float t[8];
            unpack4(w.x, old, t);
            unpack4(w.y, old, t + 4);
            if (js[r] < 0)
#pragma unroll
              for (int e = 0; e < 8; e += 2) p[r].set2(e, t[e], t[e + 1]);
          }
          if constexpr (HD == 72) {
            const uint2 w = *reinterpret_cast<const uint2*>(img + key_tail);
            float t[8];
            unpack4(w.x, old, t);
            unpack4(w.y, old, t + 4);
            if (jt < 0)
#pragma unroll
              for (int e = 0; e < 8; e += 2) pt.set2(e, t[e], t[e + 1]);
          }
        } else {
#pragma unroll
          for (int e = 0; e < 8; e += 2)
#pragma unroll
            for (int g = 0; g < 2; ++g) {  // keys 8 a + 4 g .. + 3 of dims 8 c + e and the next
              float t[4], u[4];
              unpack4(*reinterpret_cast<const uint32_t*>(img + val0 + 512 * g + 16 * e), old, t);
              unpack4(*reinterpret_cast<const uint32_t*>(img + val0 + 512 * g + 16 * e + 16), old, u);
#pragma unroll
              for (int r = 0; r < 4; ++r)
                if (js[4 * g + r] < 0) p[4 * g + r].set2(e, t[r], u[r]);
            }
          if constexpr (HD == 72) {
            if (jt < 0) {
              float t[8];
#pragma unroll
              for (int e = 0; e < 8; ++e)
                t[e] = __builtin_amdgcn_cvt_pk_f32_fp8((int)img[val_tail + 16 * e], false)[0] * old;
#pragma unroll
              for (int e = 0; e < 8; e += 2) pt.set2(e, t[e], t[e + 1]);
            }
          }
        }
      }
    }
    uint32_t top = p[0].peak();
#pragma unroll
    for (int r = 1; r < 8; ++r) top = max(top, p[r].peak());
    if constexpr (HD == 72) top = max(top, pt.peak());
    top = wave_top(top);
    if (top >= 0x7f800000u) {  // infinities or NaN among them (rare)
      top = 0;
#pragma unroll
      for (int r = 0; r < 8; ++r) top = max(top, finite_peak(p[r]));
      if constexpr (HD == 72) top = max(top, finite_peak(pt));
      top = wave_top(top);
    }
    const int b = scale_byte(__uint_as_float(top));
    const float inv = two_to(127 - b);
    if (lane == 0) *sc = (unsigned char)b;
    if (b == kExpMax + 127) {  // only this scale leaves finite values past 448 (rare)
#pragma unroll
      for (int r = 0; r < 8; ++r) saturate(p[r]);
      if constexpr (HD == 72) saturate(pt);
    }
    auto pack = [&](float x0, float x1, float x2, float x3) { return pack4(x0, x1, x2, x3, inv); };
    auto put_key = [&](int off, const Piece<T>& q) {
      *reinterpret_cast<uint2*>(img + off) = make_uint2(pack(q.get(0), q.get(1), q.get(2), q.get(3)),
                                                        pack(q.get(4), q.get(5), q.get(6), q.get(7)));
    };
    lds_order();
    if (!values) {
#pragma unroll
      for (int r = 0; r < 8; ++r) hold(p[r]);
#pragma unroll
      for (int r = 0; r < 8; ++r) put_key(key0 + 16 * r, p[r]);
      if constexpr (HD == 72) put_key(key_tail, pt);
    } else {
#pragma unroll
      for (int r = 0; r < 8; ++r) hold(p[r]);
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int g = 0; g < 2; ++g)
          *reinterpret_cast<uint32_t*>(img + val0 + 512 * g + 16 * e) =
              pack(p[4 * g].get(e), p[4 * g + 1].get(e), p[4 * g + 2].get(e), p[4 * g + 3].get(e));
      if constexpr (HD == 72)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          img[val_tail + 16 * e] = (unsigned char)pack(pt.get(e), 0.0f, 0.0f, 0.0f);
    }
    lds_order();
    for (int i = lane; i < NV; i += kWave) reinterpret_cast<uint4*>(tile)[i] = images[wave][i];
  };
  for_each_unit<true>(S, rows, 2 * c.kv_heads, group, units, 4, wave, body);
}

// One workgroup reads the listed rows of one block of one head at a time: the
// value tile comes into LDS in consecutive 16-byte pieces, a thread takes eight
// dims of a row.  Bound by bytes: 32256 tokens of 16 heads of 64 take 30 us (198 MB,
// 6.6 TB/s, part of it in the last-level cache).  (A wave per tile, as in the store, was no
// faster: all of 32256 tokens of 16 heads 45 us against 42, 1905 rows 22 us
// against 17.)
template <typename T, int HD>
__global__ __launch_bounds__(kTPB) void k_kv8_load(Kv8Segs S, Kv8Slice c, Kv8Rows rows, T* __restrict__ k,
                                                   T* __restrict__ v, int group, int units) {
  __shared__ __attribute__((aligned(16))) unsigned char sv[kKv8Block * HD];
  __shared__ int listed[kWave];  // listed tokens: rows of the block of the run's first rows, -1 behind them
  constexpr int NP = HD / 8;     // pieces of eight dims
  const int tid = threadIdx.x;
  auto body = [&](int h, const Run& run) {
    const unsigned char* kt = c.tiles + ((int64_t)h * c.nblk + run.block) * 2 * kKv8Block * HD;
    const unsigned char* vt = kt + kKv8Block * HD;
    const unsigned char* sc = c.scales + ((int64_t)h * c.nblk + run.block) * 2;
    __syncthreads();  // the block before is done with LDS
    for (int i = tid; i < kKv8Block * HD / 16; i += kTPB)
      reinterpret_cast<uint4*>(sv)[i] = reinterpret_cast<const uint4*>(vt)[i];
    const float ks = __uint_as_float((uint32_t)sc[0] << 23), vs = __uint_as_float((uint32_t)sc[1] << 23);
    const int known = run.count >= 0 ? 0 : kWave - (run.first - run.from);  // rows of the run that lanes look at
    if (run.count < 0 && tid < kWave && tid >= kWave - known)
      listed[tid - (kWave - known)] = run.lane_block == run.block ? run.at : -1;
    __syncthreads();
    for (int i = tid;; i += kTPB) {
      const int r = i / NP, p = i % NP;
      const int64_t j = (int64_t)run.first + r;
      int at = r;
      if (run.count >= 0) {
        if (r >= run.count) break;
      } else if (r < known) {
        at = listed[r];
        if (at < 0) break;
      } else if (block_of(S, j < rows.n ? rows.idx[j] : -1, &at) != run.block) {
        break;
      }
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
  for_each_unit<false>(S, rows, c.kv_heads, group, units, 1, 0, body);
}

template <typename F>
hipError_t by_type(sphinx_dtype dt, int head_dim, const F& go) {
  if (dt == SPHINX_BF16 && head_dim == 64) go(bf16{}, std::integral_constant<int, 64>{});
  else if (dt == SPHINX_BF16) go(bf16{}, std::integral_constant<int, 72>{});
  else if (head_dim == 64) go(float{}, std::integral_constant<int, 64>{});
  else go(float{}, std::integral_constant<int, 72>{});
  return hipGetLastError();
}

// Rows that a worker looks at (a wave when storing, a workgroup when reading
// back): as many as leave `workers` of them, at most `most`.  Listed rows mostly
// come in runs, and a worker without a run's first row has nothing to do; one
// with several does them one after the other.  16 heads of 64, bf16, 32256 tokens:
// storing 3 % in runs of 16 takes 14.3 us with 16384 workers, 8.7 with 4096 and
// 8.3 with 2048, which take 39.8 instead of 31.5 where the 3 % are scattered; 90 %
// in runs of 64 take 34.1 us with 16 rows each, 29.2 with 32, 30 % in runs of 8
// 32.9, 33.7, and 36.9 with 64.  Reading back those 90 % takes 49.4 us with 16 rows
// each, 39.4 with 32, 35.4 with 64, scattered 3 % 12.0 us with 2048 workers and
// 17.1 with 8192.
struct Split {
  int group, units;
  unsigned grid;
};
Split split(int parts, int64_t nblk, const Kv8Rows& rows, int workers, int most,
            int per) {  // parts: tiles or heads of a block
  Split p;
  p.group = (int)std::clamp<int64_t>((int64_t)rows.n * parts / workers, 1, most);
  p.units = rows.idx ? (int)(((int64_t)rows.n + p.group - 1) / p.group) : (int)nblk;
  p.grid = (unsigned)std::min<int64_t>(((int64_t)p.units * parts + per - 1) / per, 1 << 20);  // each then takes several
  return p;
}
}  // namespace

hipError_t launch_kv8_store(sphinx_dtype dt, int head_dim, const Kv8Segs& S, const Kv8Slice& c, const Kv8Rows& rows,
                            const void* k, const void* v, hipStream_t s) {
  const Split p = split(2 * c.kv_heads, c.nblk, rows, 4096, 32, 4);
  return by_type(dt, head_dim, [&](auto t, auto hd) {
    using T = decltype(t);
    k_kv8_store<T, decltype(hd)::value><<<p.grid, kTPB, 0, s>>>(S, c, rows, static_cast<const T*>(k),
                                                                static_cast<const T*>(v), p.group, p.units);
  });
}

hipError_t launch_kv8_load(sphinx_dtype dt, int head_dim, const Kv8Segs& S, const Kv8Slice& c, const Kv8Rows& rows,
                           void* k, void* v, hipStream_t s) {
  const Split p = split(c.kv_heads, c.nblk, rows, 2048, 64, 1);
  return by_type(dt, head_dim, [&](auto t, auto hd) {
    using T = decltype(t);
    k_kv8_load<T, decltype(hd)::value>
        <<<p.grid, kTPB, 0, s>>>(S, c, rows, static_cast<T*>(k), static_cast<T*>(v), p.group, p.units);
  });
}

}  // namespace sphinx
