// Quantisation in blocks of 128 (q8.hpp has the layout): along the rows, along
// the columns into a transposed copy, or in squares, in one pass over x, with
// the column sums on the way.  A tile of 128 x 128 values sits in the registers
// of a workgroup, four rows of eight columns each thread; the transposed bytes
// go through LDS.  Bound by HBM: rows alone 5.4-5.8 TB/s (32256 x 4096 in bf16
// 71-73 us); 9677 x 4096 in bf16 both ways 32.7 us, the transposed copy alone 25.0
// (4.9 and 4.8 TB/s; the columns' magnitudes have to be known before the first
// byte of a tile leaves it, so a tile's loads and stores overlap only with those
// of the other workgroups of its CU).
#include "q8.hpp"

namespace sphinx {

namespace {
constexpr int kNT = 256;
// Rows of eight columns that a thread of a tile holds, and a tile's threads.  With
// eight rows the chain of a thread's work shows where there are few tiles: 1333 x
// 1152 in bf16 both ways 8.5 us, 6.2 with four (7.4 with two), 9677 x 4096 34.2 and
// 32.7 (45.5).
constexpr int kTileR = 4, kTileNT = kQ8Block * kQ8Block / (8 * kTileR);

// The rows of a matrix alone: 16 lanes hold a block of 128 columns.
template <typename T>
__global__ __launch_bounds__(kNT) void k_q8_rows(const T* __restrict__ x, int64_t ldx, int rows, int cols, int wide,
                                                 uint8_t* __restrict__ q, uint8_t* __restrict__ s) {
  const int64_t at = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * (kNT / 16) + (threadIdx.x >> 4);  // block of 128
  const int64_t row = at / wide;
  const int t = (int)threadIdx.x & 15, k = (int)(at - row * wide), c = k * kQ8Block + 8 * t;
  float v[8];
  load8(x + min(row, (int64_t)rows - 1) * ldx + c, cols - c, v);
  const int sb = q8_scale_byte(row_max(finite_top(v)));
  if (row >= rows) return;
  *reinterpret_cast<uint2*>(q + row * wide * kQ8Block + c) = q8_pack8(v, sb);
  if (t == 0) s[row * q8_scale_row(wide) + k] = (uint8_t)sb;
}

// Place of 16-byte chunk b of row r in the transposed tile: neighbouring columns
// of a thread's eight and the sixteen threads of a row fall on all banks, when
// they are written (4 bytes a lane, rows 8 apart) and when they are read (whole
// rows).
__device__ __forceinline__ int tr_at(int r, int b) { return (r + (r >> 6)) * kQ8Block + ((b ^ (r >> 3 & 7)) << 4); }

// Sums over all rows for 32 of the columns, eight rows in flight.  The last ones'
// workgroup overlaps the one before, so that all loads are whole.
template <typename T>
__device__ __forceinline__ void q8_column_sums(const T* __restrict__ x, int64_t ldx, int rows, int cols, int first,
                                               float* __restrict__ sums, float* buf) {
  constexpr int U = 8, S = kTileNT / 4;
  const int c0 = min(first, cols - 32);
  const T* p = x + c0 + 8 * ((int)threadIdx.x & 3);
  float sum[8] = {};
  for (int row = (int)threadIdx.x >> 2; row < rows; row += S * U) {
    float v[U][8];
#pragma unroll
    for (int u = 0; u < U; ++u) load8(p + (int64_t)min(row + S * u, rows - 1) * ldx, 8, v[u]);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (row + S * u < rows) {
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] += v[u][e];
      }
    }
  }
  const float v = join_slices<kTileNT>(sum, buf);
  const int col = c0 + (int)threadIdx.x;
  if ((int)threadIdx.x < 32 && col >= first) sums[col] = v;
}

// The first sum_blocks workgroups sum 32 columns each into sums; the others have a
// tile each, and leave its columns' sums in part, if it is given.
template <typename T, bool SQUARE>
__global__ __launch_bounds__(kTileNT) void k_q8_tile(const T* __restrict__ x, int64_t ldx, int rows, int cols,
                                                 uint8_t* __restrict__ q, uint8_t* __restrict__ s,
                                                 uint8_t* __restrict__ qt, uint8_t* __restrict__ st,
                                                 float* __restrict__ part, float* __restrict__ sums,
                                                 int sum_blocks) {
  constexpr int R = kTileR, W = kTileNT / 64;
  __shared__ __attribute__((aligned(16))) float red[2][W][kQ8Block];  // sums, magnitudes: of a wave's 4 R rows
  __shared__ __attribute__((aligned(16))) unsigned char tr[(kQ8Block + 1) * kQ8Block];
  const int t = (int)threadIdx.x & 15, g = (int)threadIdx.x >> 4;  // columns 8 t .. + 7, rows R g .. + R - 1 of the tile
  const int wave = (int)threadIdx.x >> 6;
  const int wide = (cols + kQ8Block - 1) / kQ8Block, tall = (rows + kQ8Block - 1) / kQ8Block;
  int at = (int)(blockIdx.y * gridDim.x + blockIdx.x);  // of less than 2^24 tiles
  if (at < sum_blocks) {
    q8_column_sums(x, ldx, rows, cols, 32 * at, sums, reinterpret_cast<float*>(tr));
    return;
  }
  at -= sum_blocks;
  if (at >= wide * tall) return;
  const int tm = at / wide, tn = at % wide;
  const int m0 = tm * kQ8Block, c = tn * kQ8Block + 8 * t;
  float v[R][8];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int m = m0 + R * g + i;
    load8(x + (int64_t)min(m, rows - 1) * ldx + c, m < rows ? cols - c : 0, v[i]);
  }
  // columns: their sums and largest magnitudes over the wave's rows
  if (part != nullptr) {
    float sum[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      sum[e] = v[0][e];
#pragma unroll
      for (int i = 1; i < R; ++i) sum[e] += v[i][e];
      sum[e] = rows4_sum(sum[e]);
    }
    if ((g & 3) == 0) __builtin_memcpy(__builtin_assume_aligned(&red[0][wave][8 * t], 16), sum, 32);
  }
  if (SQUARE || qt != nullptr) {
    float top[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float col[R];
#pragma unroll
      for (int i = 0; i < R; ++i) col[i] = v[i][e];
      top[e] = rows4_max(finite_top(col));
    }
    if ((g & 3) == 0) __builtin_memcpy(__builtin_assume_aligned(&red[1][wave][8 * t], 16), top, 32);
  }
  __syncthreads();
  if (part != nullptr && (int)threadIdx.x < kQ8Block && tn * kQ8Block + (int)threadIdx.x < cols) {
    const int k = (int)threadIdx.x;
    float sum = red[0][0][k] + red[0][1][k];
#pragma unroll
    for (int w = 2; w < W; w += 2) sum += red[0][w][k] + red[0][w + 1][k];
    part[(int64_t)tm * cols + tn * kQ8Block + k] = sum;
  }
  int sb[8];  // scales of the thread's columns
  if (SQUARE || qt != nullptr) {
    float top[8] = {};
#pragma unroll
    for (int w = 0; w < W; ++w)
#pragma unroll
      for (int e = 0; e < 8; ++e) top[e] = fmaxf(top[e], red[1][w][8 * t + e]);
    if constexpr (SQUARE) {
      const int one = q8_scale_byte(row_max(finite_top(top)));
#pragma unroll
      for (int e = 0; e < 8; ++e) sb[e] = one;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) sb[e] = q8_scale_byte(top[e]);
    }
  }
  if (q != nullptr) {
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int rb = SQUARE ? sb[0] : q8_scale_byte(row_max(finite_top(v[i])));
      const int64_t m = m0 + R * g + i;
      if (m < rows) {
        *reinterpret_cast<uint2*>(q + m * wide * kQ8Block + c) = q8_pack8(v[i], rb);
        if (t == 0) s[m * q8_scale_row(wide) + tn] = (uint8_t)rb;
      }
    }
  }
  if (qt == nullptr) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float col[R];
    uint32_t w[1];
#pragma unroll
    for (int i = 0; i < R; ++i) col[i] = v[i][e];
    q8_pack(col, sb[e], w);
    *reinterpret_cast<uint32_t*>(tr + tr_at(8 * t + e, g >> 2) + 4 * (g & 3)) = w[0];
    if (g == 0 && c + e < cols) st[(int64_t)(c + e) * q8_scale_row(tall) + tm] = (uint8_t)sb[e];
  }
  __syncthreads();
#pragma unroll
  for (int p = 0; p < R / 2; ++p) {
    const int r = p * (kTileNT / 8) + ((int)threadIdx.x >> 3), b = (int)threadIdx.x & 7;
    const int64_t n = (int64_t)tn * kQ8Block + r;
    if (n < cols)
      *reinterpret_cast<uint4*>(qt + n * tall * kQ8Block + m0 + 16 * b) =
          *reinterpret_cast<const uint4*>(tr + tr_at(r, b));
  }
}
}  // namespace

hipError_t launch_q8_quantise(sphinx_dtype dt, const void* x, int64_t ldx, int rows, int cols, bool square, uint8_t* q,
                              uint8_t* s, uint8_t* qt, uint8_t* st, float* sums, float* ws, hipStream_t stream) {
  const int wide = (cols + kQ8Block - 1) / kQ8Block, tall = (rows + kQ8Block - 1) / kQ8Block;
  // A second launch joins the tiles' sums, except where one tile's are the sums, and where small inputs are read again
  // for them beside the tiles: 1333 x 840 in bf16 10.5 -> 7.0 us a call (10.2 -> 7.3 from HBM), 2000 x 1024 10.4 -> 7.1
  // (fp32 from HBM 10.3 -> 8.2).  It loses to the join where they do not stay in the caches (2048 x 4096 in bf16 12.2 ->
  // 15.0) and where a workgroup has many rows to add (4096 x 1024 from HBM 10.5 -> 12.4).
  const bool beside = sums != nullptr && tall > 1 && cols >= 32 && rows <= 2048 &&
                      (int64_t)rows * cols * (dt == SPHINX_BF16 ? 2 : 4) <= (8 << 20);
  const bool join = sums != nullptr && tall != 1 && !beside;
  if (rows > 0) {
    auto go = [&](auto t) {
      typedef decltype(t) T;
      const T* in = static_cast<const T*>(x);
      const int sum_blocks = beside ? (cols + 31) / 32 : 0;
      const dim3 tiles = long_grid((int64_t)wide * tall + sum_blocks);
      float* part = join ? ws : beside ? nullptr : sums;
      if (!square && qt == nullptr && sums == nullptr) {
        const int64_t grid = ((int64_t)rows * wide + kNT / 16 - 1) / (kNT / 16);
        k_q8_rows<T><<<long_grid(grid), kNT, 0, stream>>>(in, ldx, rows, cols, wide, q, s);
      } else if (square) {
        k_q8_tile<T, true><<<tiles, kTileNT, 0, stream>>>(in, ldx, rows, cols, q, s, qt, st, part, sums, sum_blocks);
      } else {
        k_q8_tile<T, false><<<tiles, kTileNT, 0, stream>>>(in, ldx, rows, cols, q, s, qt, st, part, sums, sum_blocks);
      }
    };
    if (dt == SPHINX_BF16) go(bf16{});
    else go(float{});
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (!join) return hipSuccess;
  PartBounds P;
  P.nseg = 1;
  P.first[0] = 0;
  P.first[1] = tall;
  return launch_join_parts(ws, cols, cols, P, sums, nullptr, cols, stream);
}

}  // namespace sphinx
