// Quantisation in blocks of 128 (q8.hpp has the layout): along the rows, along
// the columns into a transposed copy, or in squares, in one pass over x, with
// the column sums on the way.  A tile of 128 x 128 values sits in the registers
// of a workgroup, eight rows of eight columns each thread; the transposed bytes
// go through LDS.  Bound by HBM.
#include "q8.hpp"

namespace sphinx {

namespace {
constexpr int kNT = 256;

// The rows of a matrix alone: 16 lanes hold a block of 128 columns.
template <typename T>
__global__ __launch_bounds__(kNT) void k_q8_rows(const T* __restrict__ x, int64_t ldx, int rows, int cols, int wide,
                                                 uint8_t* __restrict__ q, uint8_t* __restrict__ s) {
  const int64_t at = (int64_t)blockIdx.x * (kNT / 16) + (threadIdx.x >> 4);  // block of the matrix
  const int64_t row = at / wide;
  const int t = (int)threadIdx.x & 15, k = (int)(at - row * wide), c = k * kQ8Block + 8 * t;
  float v[8];
  load8(x + min(row, (int64_t)rows - 1) * ldx + c, cols - c, v);
  float top = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = fmaxf(top, finite_abs(v[e]));
  const int sb = q8_scale_byte(row_max(top));
  if (row >= rows) return;
  *reinterpret_cast<uint2*>(q + row * wide * kQ8Block + c) = q8_pack8(v, sb);
  if (t == 0) s[row * q8_scale_row(wide) + k] = (uint8_t)sb;
}

template <typename T, bool SQUARE>
__global__ __launch_bounds__(kNT) void k_q8_tile(const T* __restrict__ x, int64_t ldx, int rows, int cols,
                                                 uint8_t* __restrict__ q, uint8_t* __restrict__ s,
                                                 uint8_t* __restrict__ qt, uint8_t* __restrict__ st,
                                                 float* __restrict__ part) {
  __shared__ float red[16][kQ8Block];
  __shared__ __attribute__((aligned(16))) unsigned char tr[kQ8Block][kQ8Block + 16];
  const int t = (int)threadIdx.x & 15, g = (int)threadIdx.x >> 4;  // columns 8 t .. + 7, rows 8 g .. + 7 of the tile
  const int wide = (cols + kQ8Block - 1) / kQ8Block, tall = (rows + kQ8Block - 1) / kQ8Block;
  const int tm = (int)blockIdx.x / wide, tn = (int)blockIdx.x % wide;
  const int m0 = tm * kQ8Block, c = tn * kQ8Block + 8 * t;
  float v[8][8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int m = m0 + 8 * g + i;
    load8(x + (int64_t)min(m, rows - 1) * ldx + c, m < rows ? cols - c : 0, v[i]);
  }
  int square = 0;
  if constexpr (SQUARE) {
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) top = fmaxf(top, finite_abs(v[i][e]));
    top = row_max(top);
    if (t == 0) red[g][0] = top;
    __syncthreads();
    top = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) top = fmaxf(top, red[i][0]);
    square = q8_scale_byte(top);
    __syncthreads();
  }
  if (q != nullptr) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      int sb = square;
      if constexpr (!SQUARE) {
        float top = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) top = fmaxf(top, finite_abs(v[i][e]));
        sb = q8_scale_byte(row_max(top));
      }
      const int64_t m = m0 + 8 * g + i;
      if (m < rows) {
        *reinterpret_cast<uint2*>(q + m * wide * kQ8Block + c) = q8_pack8(v[i], sb);
        if (t == 0) s[m * q8_scale_row(wide) + tn] = (uint8_t)sb;
      }
    }
  }
  if (part != nullptr) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += v[i][e];
      red[g][8 * t + e] = sum;
    }
    __syncthreads();
    if ((int)threadIdx.x < kQ8Block && tn * kQ8Block + (int)threadIdx.x < cols) {
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < 16; ++i) sum += red[i][threadIdx.x];
      part[(int64_t)tm * cols + tn * kQ8Block + threadIdx.x] = sum;
    }
    __syncthreads();
  }
  if (qt == nullptr) return;
  if constexpr (!SQUARE) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float top = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) top = fmaxf(top, finite_abs(v[i][e]));
      red[g][8 * t + e] = top;
    }
    __syncthreads();
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    int sb = square;
    if constexpr (!SQUARE) {
      float top = 0.0f;
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, red[i][8 * t + e]);
      sb = q8_scale_byte(top);
    }
    float col[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) col[i] = v[i][e];
    *reinterpret_cast<uint2*>(&tr[8 * t + e][8 * g]) = q8_pack8(col, sb);
    if (g == 0 && c + e < cols) st[(int64_t)(c + e) * q8_scale_row(tall) + tm] = (uint8_t)sb;
  }
  __syncthreads();
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    const int r = p * 32 + ((int)threadIdx.x >> 3), b = 16 * ((int)threadIdx.x & 7);
    const int64_t n = (int64_t)tn * kQ8Block + r;
    if (n < cols)
      *reinterpret_cast<uint4*>(qt + n * tall * kQ8Block + m0 + b) = *reinterpret_cast<const uint4*>(&tr[r][b]);
  }
}
}  // namespace

hipError_t launch_q8_quantise(sphinx_dtype dt, const void* x, int64_t ldx, int rows, int cols, bool square, uint8_t* q,
                              uint8_t* s, uint8_t* qt, uint8_t* st, float* sums, float* ws, hipStream_t stream) {
  const int wide = (cols + kQ8Block - 1) / kQ8Block, tall = (rows + kQ8Block - 1) / kQ8Block;
  if (rows > 0) {
    auto go = [&](auto t) {
      typedef decltype(t) T;
      const T* in = static_cast<const T*>(x);
      if (!square && qt == nullptr && sums == nullptr) {
        const int64_t grid = ((int64_t)rows * wide + kNT / 16 - 1) / (kNT / 16);
        k_q8_rows<T><<<(unsigned)grid, kNT, 0, stream>>>(in, ldx, rows, cols, wide, q, s);
      } else if (square) {
        k_q8_tile<T, true><<<(unsigned)(wide * tall), kNT, 0, stream>>>(in, ldx, rows, cols, q, s, qt, st,
                                                                        sums != nullptr ? ws : nullptr);
      } else {
        k_q8_tile<T, false><<<(unsigned)(wide * tall), kNT, 0, stream>>>(in, ldx, rows, cols, q, s, qt, st,
                                                                         sums != nullptr ? ws : nullptr);
      }
    };
    if (dt == SPHINX_BF16) go(bf16{});
    else go(float{});
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (sums == nullptr) return hipSuccess;
  PartBounds P;
  P.nseg = 1;
  P.first[0] = 0;
  P.first[1] = tall;
  return launch_join_parts(ws, cols, cols, P, sums, nullptr, cols, stream);
}

}  // namespace sphinx
