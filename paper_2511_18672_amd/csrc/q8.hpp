// Matrices in 8 bits with a scale for each block of 128, and the layer norm:
// launchers (callers validate every argument first) and device helpers.
//
// A matrix [rows][cols] in 8 bits is rows of Kp = 128 ceil(cols / 128) e4m3
// bytes (zeros behind cols), and rows of scale bytes, one for each 128 columns,
// padded to a multiple of sixteen (a row's scales of sixteen blocks are one 16-byte
// copy): byte b stands for 2^(b - 127).  Scales are
// powers of two, so that the matrix cores apply them by themselves and exactly;
// any other scale would cost a multiply-add of every partial sum of 128
// products, 16 vector instructions beside 128 cycles of a 32x32x64 product.
#pragma once

#include "kernels.hpp"
#include "q8_rules.hpp"

namespace sphinx {

constexpr int kQ8Block = 128;
constexpr int kQ8MaxCols = 1 << 23;  // a tile's rows are addressed with 32-bit byte offsets
constexpr int kLnMaxCols = 16384;

inline int64_t q8_row_bytes(int64_t cols) { return (cols + kQ8Block - 1) / kQ8Block * kQ8Block; }
// Bytes of a row's scales, from its number of blocks.
__host__ __device__ inline int q8_scale_row(int blocks) { return (blocks + 15) & ~15; }
inline int64_t q8_scale_bytes(int64_t cols) { return q8_scale_row((int)((cols + kQ8Block - 1) / kQ8Block)); }

// A grid of n workgroups or more, numbered y * gridDim.x + x: a dimension has less than 2^32 threads.
inline dim3 long_grid(int64_t n) {
  const int64_t wide = 1 << 20;
  return n <= wide ? dim3((unsigned)n) : dim3((unsigned)wide, (unsigned)((n + wide - 1) / wide));
}

// Rows [cu[i], cu[i+1]) belong to segment i.
struct LnSegs {
  int nseg;
  int cu[SPHINX_MAX_REQUESTS + 1];
};

struct LnArgs {
  const void* x;
  int64_t ldx;
  const void* w;  // NULL: ones (plus_one: zeros)
  const void* b;  // NULL: zeros
  int64_t ldw;
  bool w_bf16, plus_one;
  int cols;
  float eps;
  const int32_t* row_of;  // row of w and b that each row takes, instead of its segment's (forward only), or NULL
};

// layer_norm.hip.  One of y (rows at ldy) and q/s is given; stats may be NULL.
hipError_t launch_layer_norm(sphinx_dtype xdt, sphinx_dtype ydt, const LnArgs& a, const LnSegs& S, void* y,
                             int64_t ldy, uint8_t* q, uint8_t* s, float* stats, hipStream_t st);
size_t layer_norm_backward_ws_bytes(int cols, const LnSegs& S);
hipError_t launch_layer_norm_backward(sphinx_dtype xdt, sphinx_dtype gdt, const LnArgs& a, const LnSegs& S,
                                      const float* stats, const void* dy, int64_t lddy, void* dx, int64_t lddx,
                                      float* dw, float* db, int64_t ldg, float* ws, hipStream_t st);
// Sums over parts: out0[i][c] = sum over parts p in [first[i], first[i+1]) of part[p * stride + c], c < cols, and out1
// likewise of the cols behind them; one output row per segment, in a fixed order.  Either may be NULL.
struct PartBounds {
  int nseg;
  int first[SPHINX_MAX_REQUESTS + 1];
};
hipError_t launch_join_parts(const float* part, int64_t stride, int cols, const PartBounds& P, float* out0,
                             float* out1, int64_t ldo, hipStream_t st);

// q8_quantise.hip
hipError_t launch_q8_quantise(sphinx_dtype dt, const void* x, int64_t ldx, int rows, int cols, bool square, uint8_t* q,
                              uint8_t* s, uint8_t* qt, uint8_t* st, float* sums, float* ws, hipStream_t stream);

// q8_matmul.hip: C[M][N] = A[M][K] B[N][K]^T + bias
enum { Q8_EPI_STORE = 0, Q8_EPI_GELU = 1, Q8_EPI_ADD = 2 };
struct Q8Mat {
  const uint8_t* q;
  const uint8_t* s;
};
struct Q8Epi {
  int epi;
  const void* bias;  // NULL: none
  bool bias_bf16;
  void* out;         // outputs of the given type; kQ8Gated: the fp32 residual; kQ8Bytes: rows of e4m3 bytes
  int64_t ldo;
  uint8_t* scales;      // kQ8Bytes: its scales
  const float* gate;    // kQ8Gated: out += (1 + gate[row_of[m]][n]) C, rows of gate at ldg
  int64_t ldg;
  const int32_t* row_of;
  int qcols;            // kQ8Bf16 stored: columns [0, qcols) are multiplied by qscale (qcols a multiple of 32, which a
                        // tile's epilogue takes at a time); the contraction is not cut
  float qscale;
};
size_t q8_matmul_ws_bytes(sphinx_dtype odt, int M, int N, int K);
// ws: q8_matmul_ws_bytes for kQ8Bf16 and kQ8F32; NULL: the contraction is not cut.  The other kinds never are.
hipError_t launch_q8_matmul(Q8Kind kind, int M, int N, int K, const Q8Mat& a, const Q8Mat& b, const Q8Epi& e,
                            float* ws, hipStream_t stream);

// ---------------------------------------------------------------------------
// device helpers
// ---------------------------------------------------------------------------
__device__ __forceinline__ float two_to(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Scale byte of a group whose largest finite magnitude is `top`: 127 + the
// smallest e with top <= 448 2^e, held in -100 .. 119.
__device__ __forceinline__ int q8_scale_byte(float top) {
  const uint32_t b = __float_as_uint(top);
  int e = (int)(b >> 23) - 127 - ((b & 0x7fffffu) <= 0x600000u ? 8 : 7);  // 448 = 1.75 2^8
  if (b < 0x00800000u) e = -100;  // zero or subnormal
  return min(max(e, -100), 119) + 127;
}

// Largest finite magnitude of N numbers.  The maximum passes over NaN by itself;
// only where it meets an infinity (or nothing but NaN) are they looked at one by
// one.
template <int N>
__device__ __forceinline__ float finite_top(const float (&x)[N]) {
  const float inf = __uint_as_float(0x7f800000u);
  float top = 0.0f;
#pragma unroll
  for (int i = 0; i < N; ++i) top = fmaxf(top, fabsf(x[i]));
  if (__builtin_expect(!(top < inf), 0)) {  // a branch: taken along, it costs as much as the rest
    top = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) top = fabsf(x[i]) < inf ? fmaxf(top, fabsf(x[i])) : top;
  }
  return top;
}

// N values (4 or 8) times 2^-e in e4m3, rounded to nearest even; infinities and
// NaN become NaN.  At the largest scale finite values may lie past 448, where the
// hardware would give NaN: they saturate.
template <int N>
__device__ __forceinline__ void q8_pack(const float (&x)[N], int sbyte, uint32_t (&w)[N / 4]) {
  const float inv = two_to(127 - sbyte);
  float v[N];
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = x[i] * inv;
  if (sbyte == 119 + 127) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (fabsf(v[i]) < __uint_as_float(0x7f800000u)) v[i] = fminf(fmaxf(v[i], -448.0f), 448.0f);
  }
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    const int k = __builtin_amdgcn_cvt_pk_fp8_f32(v[i], v[i + 1], 0, false);
    w[i / 4] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[i + 2], v[i + 3], k, true);
  }
}
__device__ __forceinline__ uint2 q8_pack8(const float (&x)[8], int sbyte) {
  uint32_t w[2];
  q8_pack(x, sbyte, w);
  return make_uint2(w[0], w[1]);
}

// Elements p[0 .. n) as floats, zeros behind them (n may be past 8 or below 1).
// Whole groups are read at once whatever their alignment: a row of an odd
// number of elements starts anywhere, and global loads take any address.
__device__ __forceinline__ void load8(const float* p, int n, float (&v)[8]) {
  if (n >= 8) {
    __builtin_memcpy(v, p, 32);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? p[i] : 0.0f;
  }
}
__device__ __forceinline__ void load8(const bf16* p, int n, float (&v)[8]) {
  if (n >= 8) {
    bf16x8 t;
    __builtin_memcpy(&t, p, 16);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)t[i];
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? (float)p[i] : 0.0f;
  }
}
__device__ __forceinline__ void store8(float* p, int n, const float (&v)[8]) {
  if (n >= 8) {
    __builtin_memcpy(p, v, 32);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = v[i];
  }
}
__device__ __forceinline__ void store8(bf16* p, int n, const float (&v)[8]) {
  if (n >= 8) {
    bf16x8 t;
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = (bf16)v[i];
    __builtin_memcpy(p, &t, 16);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = (bf16)v[i];
  }
}

// Sum and maximum over the 16 lanes of a row, in every lane of it, and over the
// lanes at the same place of a wave's four rows.
__device__ __forceinline__ float row_sum(float v) {
  v += dpp_f<0xB1>(v);
  v += dpp_f<0x4E>(v);
  v += dpp_f<0x141>(v);
  return v + dpp_f<0x140>(v);
}
__device__ __forceinline__ float row_max(float v) {
  v = fmaxf(v, dpp_f<0xB1>(v));
  v = fmaxf(v, dpp_f<0x4E>(v));
  v = fmaxf(v, dpp_f<0x141>(v));
  return fmaxf(v, dpp_f<0x140>(v));
}

__device__ __forceinline__ float rows4_sum(float v) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
__device__ __forceinline__ float rows4_max(float v) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// Sums over slices of rows: thread t of NT holds columns 8 (t % 4) .. + 7 of slice t / 4; the first 32 threads get the
// column of their number, added in a fixed order.  buf: 8 floats a thread.
template <int NT>
__device__ __forceinline__ float join_slices(const float (&sum)[8], float* buf) {
  const int t = (int)threadIdx.x;
  __syncthreads();
  __builtin_memcpy(__builtin_assume_aligned(buf + 8 * t, 16), sum, 32);
  __syncthreads();
  float v = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) v += buf[32 * (8 * (t >> 5) + i) + (t & 31)];
  __syncthreads();
  buf[t] = v;
  __syncthreads();
  v = 0.0f;
  if (t < 32)
#pragma unroll
    for (int i = 0; i < NT / 32; ++i) v += buf[32 * i + t];
  return v;
}

}  // namespace sphinx
