// Layer norm over rows in segments, forward and backward:
//   m = mean(x), r = 1 / sqrt(mean((x - m)^2) + eps), xh = (x - m) r
//   y = xh w' + b                                  w' = w or 1 + w, per segment
//   g = dy w', dx = r (g - mean(g) - xh mean(g xh)), dw = sum dy xh, db = sum dy
//
// A row lives in the registers of LPR lanes (16, 64, 256 or 512), eight
// consecutive columns each and NI such groups, so HBM is read once and both
// passes of the variance run over registers.  Everything is in fp32; y and dx
// are rounded once.  Both directions are bound by HBM: 32256 x 1024 in fp32 to
// bf16 takes 30 us (6.6 TB/s, part of it from the caches), to 8 bits 25.5; backward
// in bf16 37.5 (5.3 TB/s) and 4 for the sums over the rows.  One row takes 2.6 us,
// the latency of its loads and of two sums.
#include <algorithm>

#include "q8.hpp"

namespace sphinx {

namespace {
// Threads of a workgroup, and rows that it holds at a time.
template <int LPR>
struct LnCfg {
  static constexpr int NT = LPR > 256 ? LPR : 256, ROWS = NT / LPR;
};

// Sum over the LPR lanes of a row, in each of them; every lane of the workgroup
// calls it where LPR > 64 (red: one float per wave, two sets used in turn).
template <int LPR>
__device__ __forceinline__ float ln_sum(float v, float* red) {
  if constexpr (LPR == 16) return row_sum(v);
  v = wave_sum(v);
  if constexpr (LPR > 64) {
    constexpr int NW = LPR / 64;
    if (lane_id() == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0f;
#pragma unroll
    for (int i = 0; i < NW; ++i) v += red[i];
  }
  return v;
}

__device__ __forceinline__ int ln_segment(const LnSegs& S, int row) {
  int lo = 0, hi = S.nseg - 1;
  while (lo < hi) {  // the last segment that starts at or before the row (empty ones start there as well)
    const int mid = (lo + hi + 1) >> 1;
    if (S.cu[mid] <= row) lo = mid; else hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ void ln_load_w(const void* w, bool is_bf16, int64_t at, int n, float none, float (&v)[8]) {
  if (w == nullptr) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = none;
  } else if (is_bf16) {
    load8(static_cast<const bf16*>(w) + at, n, v);
  } else {
    load8(static_cast<const float*>(w) + at, n, v);
  }
}

struct Q8Out {
  uint8_t* q;
  uint8_t* s;
};

// OUT: bf16, float, or Q8Out for rows in 8 bits (16 lanes hold a block of 128 columns).
template <typename XT, typename OUT, int LPR, int NI>
__global__ __launch_bounds__(LnCfg<LPR>::NT) void k_layer_norm(LnArgs a, LnSegs S, OUT* y, int64_t ldy,
                                                               Q8Out qo, float* __restrict__ stats) {
  typedef LnCfg<LPR> C;
  __shared__ float red[2][16];
  const int t = (int)threadIdx.x % LPR, rows = S.cu[S.nseg], cols = a.cols;
  const int64_t row0 = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * C::ROWS + (int)threadIdx.x / LPR;
  const bool live = row0 < rows;
  const int row = live ? (int)row0 : rows - 1;  // lanes past the end repeat the last row and store nothing
  const XT* x = static_cast<const XT*>(a.x) + (int64_t)row * a.ldx;
  // short rows: everything that they need is on its way before the first sum is waited for.  Longer ones would pay for
  // it with waves (3000 x 8192 in bf16 21.3 -> 23.3 us)
  constexpr bool kEarly = NI <= 2 && LPR <= 64;
  constexpr int kFull = LPR > 64 && NI == 4 ? 2 : NI - 1;  // groups of columns that by_cols fills
  auto left = [&](int i) { return i < kFull ? 8 : cols - 8 * (i * LPR + t); };
  float v[NI][8], w[NI][8], b[NI][8];
#pragma unroll
  for (int i = 0; i < NI; ++i) load8(x + 8 * (i * LPR + t), left(i), v[i]);
  const int64_t wr = (int64_t)(a.row_of != nullptr ? a.row_of[row] : ln_segment(S, row)) * a.ldw;
  const float one = a.plus_one ? 1.0f : 0.0f;
  auto weights = [&](int i) {
    const int c = 8 * (i * LPR + t);
    ln_load_w(a.w, a.w_bf16, wr + c, left(i), 1.0f - one, w[i]);
    ln_load_w(a.b, a.w_bf16, wr + c, left(i), 0.0f, b[i]);
  };
  if constexpr (kEarly)
#pragma unroll
    for (int i = 0; i < NI; ++i) weights(i);
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) s += v[i][e];
  const float mean = ln_sum<LPR>(s, red[0]) / (float)cols;
  s = 0.0f;
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int n = left(i);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[i][e] = e < n ? v[i][e] - mean : 0.0f;
      s = fmaf(v[i][e], v[i][e], s);
    }
  }
  const float var = ln_sum<LPR>(s, red[1]) / (float)cols, inf = __uint_as_float(0x7f800000u);
  const uint64_t far_rows = __ballot(!(var < inf));
  const bool near = live && var < inf;
  auto keep = [&](bool store, int to, float m, float r) {
    if (stats != nullptr && store) {
      stats[2 * (int64_t)to] = m;
      stats[2 * (int64_t)to + 1] = r;
    }
  };
  // columns c .. c + 7 from their differences from the mean
  auto put = [&](bool store, int to, int c, int n, const float (&d)[8], float r, const float (&wc)[8], const float (&bc)[8]) {
    float o[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = fmaf(d[e] * r, wc[e] + one, bc[e]);
    if constexpr (std::is_same_v<OUT, Q8Out>) {
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = e < n ? o[e] : 0.0f;
      const int sb = q8_scale_byte(row_max(finite_top(o)));
      const uint2 p = q8_pack8(o, sb);
      const int64_t ld = (cols + kQ8Block - 1) / kQ8Block * (int64_t)kQ8Block;
      if (store && c < ld) {
        *reinterpret_cast<uint2*>(qo.q + to * ld + c) = p;
        if (c % 128 == 0) qo.s[to * (int64_t)q8_scale_row((int)(ld >> 7)) + (c >> 7)] = (uint8_t)sb;
      }
    } else {
      if (store) store8(y + (int64_t)to * ldy + c, n, o);
    }
  };
  const float rstd = 1.0f / sqrtf(var + a.eps);
  keep(near && t == 0, row, mean, rstd);
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    if constexpr (!kEarly) weights(i);
    put(near, row, 8 * (i * LPR + t), left(i), v[i], rstd, w[i], b[i]);
  }
  if (far_rows == 0) return;
  // A row whose sum, or that of its squares, passes fp32's largest (or that holds an infinity or a NaN, which stay NaN) is
  // taken again from memory in units of 2^80: its numbers are below 2^48 then, and their squares' sum below 2^110.  All
  // lanes of the row come here, behind the rest, so that other rows neither wait nor keep registers for it (as a branch
  // before the stores, 32256 x 1152 in fp32 to bf16 43.4 us instead of 42.4, 3000 x 16384 to 8 bits 58 instead of 53).
  const float down = two_to(-80), up = two_to(80);
  int tid = (int)threadIdx.x;
  asm volatile("" : "+v"(tid));  // all else is found again
  if ((far_rows >> (tid & 63) & 1) == 0) return;
  const int64_t r0 = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * C::ROWS + tid / LPR;
  const bool alive = r0 < rows;
  const int again = alive ? (int)r0 : rows - 1, first = 8 * (tid % LPR);
  const XT* xa = static_cast<const XT*>(a.x) + (int64_t)again * a.ldx;
  auto each = [&](float m, auto f) {
#pragma unroll 1
    for (int i = 0; i < NI; ++i) {
      const int c = 8 * LPR * i + first, n = cols - c;
      float u[8];
      load8(xa + c, n, u);
#pragma unroll
      for (int e = 0; e < 8; ++e) u[e] = e < n ? u[e] * down - m : 0.0f;
      f(c, u);
    }
  };
  s = 0.0f;
  each(0.0f, [&](int, const float (&u)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) s += u[e];
  });
  const float m = ln_sum<LPR>(s, red[0]) / (float)cols;
  s = 0.0f;
  each(m, [&](int, const float (&u)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fmaf(u[e], u[e], s);
  });
  const float far = ln_sum<LPR>(s, red[1]) / (float)cols, whole = far * up * up;
  // where only a sum was too large, the variance is taken back; where that is below 2^-96, no difference is left here
  const float r = whole < inf ? fminf(up / sqrtf(whole + a.eps), 0x1p127f) : 1.0f / sqrtf(far + a.eps * down * down);
  keep(alive && first == 0, again, m * up, whole < inf ? 1.0f / sqrtf(whole + a.eps) : r * down);
  const int64_t wa = (int64_t)(a.row_of != nullptr ? a.row_of[again] : ln_segment(S, again)) * a.ldw;
  each(m, [&](int c, const float (&u)[8]) {
    float wc[8], bc[8];
    ln_load_w(a.w, a.w_bf16, wa + c, cols - c, 1.0f - one, wc);
    ln_load_w(a.b, a.w_bf16, wa + c, cols - c, 0.0f, bc);
    put(alive, again, c, cols - c, u, r, wc, bc);
  });
}

// Rows of a chunk: a workgroup walks over one chunk of one segment's rows and
// keeps the sums of its columns in registers; the chunks' sums are joined by
// k_join_parts in a fixed order, so a call repeats bit for bit.
struct LnChunks {
  int rows;                             // of a chunk (the segment's last may hold fewer)
  int first[SPHINX_MAX_REQUESTS + 1];   // chunks of the segments before
};

struct LnSums {
  float* dw;  // rows of weight and bias gradients per segment, at ld; either may be NULL
  float* db;
  int64_t ld;
  int blocks;  // workgroups that sum columns
};

// Eight elements as they are in memory, zeros behind n.
template <typename T>
struct Raw8 {
  T v[8];
  __device__ __forceinline__ void load(const T* p, int n) {
    if (n >= 8) {
      __builtin_memcpy(v, p, sizeof(v));
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = i < n ? p[i] : (T)0.0f;
    }
  }
};

// Sums over all rows of a segment for 32 of its columns, from the statistics of
// the forward pass alone: 4 lanes of eight columns, 64 slices of the rows, eight
// rows in flight, joined in a fixed order.  buf: 8 floats a thread.  At least 32
// columns: the last ones' workgroup overlaps the one before, so that all loads are
// whole.
template <typename XT, typename GT>
__device__ __forceinline__ void ln_column_sums(const LnArgs& a, int r0, int r1, int c0,
                                               const float* __restrict__ stats, const GT* dy, int64_t lddy,
                                               float* dw, float* db, float* buf) {
  constexpr int NT = 256, U = 8;
  const int first = c0;
  c0 = min(c0, a.cols - 32);
  const int c = c0 + 8 * ((int)threadIdx.x & 3), slice = (int)threadIdx.x >> 2;
  const XT* x = static_cast<const XT*>(a.x) + c;
  float sum[2][8] = {};
  for (int row = r0 + slice; row < r1; row += NT / 4 * U) {
    Raw8<XT> rx[U];
    Raw8<GT> rg[U];
    float2 st[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t at = min(row + NT / 4 * u, r1 - 1);
      st[u] = *reinterpret_cast<const float2*>(stats + 2 * at);
      rx[u].load(x + at * a.ldx, 8);
      rg[u].load(dy + at * lddy + c, 8);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (row + NT / 4 * u < r1) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float d = (float)rg[u].v[e];
          sum[0][e] = fmaf(d, ((float)rx[u].v[e] - st[u].x) * st[u].y, sum[0][e]);
          sum[1][e] += d;
        }
      }
    }
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    float* out = k == 0 ? dw : db;
    if (out == nullptr) continue;
    const float v = join_slices<NT>(sum[k], buf);
    const int col = c0 + (int)threadIdx.x;
    if ((int)threadIdx.x < 32 && col >= first) out[col] = v;
  }
}

// The next row's loads are issued before this row's arithmetic (also where dx
// is dy: they are other rows).  Columns behind the last one hold x = 0 and dy = 0,
// which add nothing to a sum over the row while mean * rstd is finite; where it is
// not, they are left out.  The widest rows read their weights from
// LDS each time, since the registers do not hold them (3000 x 10000 148 -> 74 us).
// ONE: the first to.blocks workgroups sum columns into to.dw and to.db, and the
// others, a chunk each, leave the sums alone (part is not used).
template <typename XT, typename GT, int LPR, int NI, bool ONE>
__global__ __launch_bounds__(LnCfg<LPR>::NT) void k_layer_norm_backward(LnArgs a, LnSegs S, LnChunks P,
                                                                        const float* __restrict__ stats,
                                                                        const GT* dy, int64_t lddy,
                                                                        GT* dx, int64_t lddx,
                                                                        float* __restrict__ part, LnSums to) {
  typedef LnCfg<LPR> C;
  __shared__ float red[4][16];
  constexpr bool kWeightsInLds = LPR == 512;
  __shared__ __attribute__((aligned(16))) float sums[C::ROWS > 1 ? C::NT * NI * 8 : kWeightsInLds ? LPR * NI * 8 : 1];
  const int t = (int)threadIdx.x % LPR, grp = (int)threadIdx.x / LPR, cols = a.cols;
  int chunk = (int)blockIdx.x;
  if constexpr (ONE) {
    static_assert(C::NT == 256 && C::ROWS > 1, "sums hold eight floats of 256 threads");
    if (chunk < to.blocks) {
      const int groups = (cols + 31) / 32, of = chunk / groups;
      ln_column_sums<XT, GT>(a, S.cu[of], S.cu[of + 1], 32 * (chunk - of * groups), stats, dy, lddy,
                             to.dw == nullptr ? nullptr : to.dw + of * to.ld,
                             to.db == nullptr ? nullptr : to.db + of * to.ld, sums);
      return;
    }
    chunk -= to.blocks;
  }
  int seg = 0;
  {
    int lo = 0, hi = S.nseg - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (P.first[mid] <= chunk) lo = mid; else hi = mid - 1;
    }
    seg = lo;
  }
  const int r0 = S.cu[seg] + (chunk - P.first[seg]) * P.rows, r1 = min(r0 + P.rows, S.cu[seg + 1]);
  const float one = a.plus_one ? 1.0f : 0.0f;
  float w[kWeightsInLds ? 1 : NI][8], sw[NI][8], sb[NI][8];
  Raw8<XT> rx[NI];
  Raw8<GT> rg[NI];
  float mean, rstd;
  auto fetch = [&](int row) {
    const XT* xr = static_cast<const XT*>(a.x) + (int64_t)row * a.ldx;
    const GT* gr = dy + (int64_t)row * lddy;
    mean = stats[2 * (int64_t)row];
    rstd = stats[2 * (int64_t)row + 1];
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int c = 8 * (i * LPR + t);
      rx[i].load(xr + c, cols - c);
      rg[i].load(gr + c, cols - c);
    }
  };
  fetch(min(r0 + grp, r1 - 1));
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int c = 8 * (i * LPR + t);
    float (&wi)[8] = w[kWeightsInLds ? 0 : i];
    ln_load_w(a.w, a.w_bf16, seg * a.ldw + c, cols - c, 1.0f - one, wi);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      wi[e] += one;
      sw[i][e] = sb[i][e] = 0.0f;
    }
    if constexpr (kWeightsInLds) __builtin_memcpy(__builtin_assume_aligned(sums + c, 16), wi, 32);  // read by this lane
  }
  for (int row = r0 + grp; row < r1; row += C::ROWS) {
    float xh[NI][8], g[NI][8];
    float s1 = 0.0f, s2 = 0.0f;
    const float r = rstd;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      float (&wi)[8] = w[kWeightsInLds ? 0 : i];
      if constexpr (kWeightsInLds) __builtin_memcpy(wi, __builtin_assume_aligned(sums + 8 * (i * LPR + t), 16), 32);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        xh[i][e] = ((float)rx[i].v[e] - mean) * r;
        const float d = (float)rg[i].v[e];
        if constexpr (!ONE) {
          sw[i][e] = fmaf(d, xh[i][e], sw[i][e]);
          sb[i][e] += d;
        }
        g[i][e] = d * wi[e];
        s1 += g[i][e];
        s2 = fmaf(g[i][e], xh[i][e], s2);
      }
    }
    // rare, and cheaper than a selection per number; behind the loads, but where the registers do not hold both
    const bool far = !(fabsf(mean * r) < __uint_as_float(0x7f800000u));
    auto inside = [&]() {
      s2 = 0.0f;
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) s2 = 8 * (i * LPR + t) + e < cols ? fmaf(g[i][e], xh[i][e], s2) : s2;
    };
    if (kWeightsInLds && far) inside();
    fetch(min(row + C::ROWS, r1 - 1));
    if (dx != nullptr) {
      if (!kWeightsInLds && far) inside();
      const int par = LPR > 64 ? 2 * ((row - r0) & 1) : 0;
      s1 = ln_sum<LPR>(s1, red[par]) / (float)cols;
      s2 = ln_sum<LPR>(s2, red[par + 1]) / (float)cols;
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const int c = 8 * (i * LPR + t);
        float o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = r * (g[i][e] - s1 - xh[i][e] * s2);
        store8(dx + (int64_t)row * lddx + c, cols - c, o);
      }
    }
  }
  if (ONE || part == nullptr) return;
  float* out = part + (int64_t)blockIdx.x * 2 * cols;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    if constexpr (C::ROWS == 1) {
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const int c = 8 * (i * LPR + t);
        store8(out + k * cols + c, cols - c, k == 0 ? sw[i] : sb[i]);
      }
    } else {  // the row groups' sums through LDS
      __syncthreads();
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) sums[grp * (LPR * NI * 8) + 8 * (i * LPR + t) + e] = k == 0 ? sw[i][e] : sb[i][e];
      __syncthreads();
      for (int c = (int)threadIdx.x; c < cols; c += C::NT) {
        float v = 0.0f;
#pragma unroll
        for (int j = 0; j < C::ROWS; ++j) v += sums[j * (LPR * NI * 8) + c];
        out[k * cols + c] = v;
      }
    }
  }
}

// 64 columns x 16 slices of the parts per workgroup; out1 takes the columns from
// `cols` on (a part holds two rows of them), and either may be NULL.
__global__ __launch_bounds__(1024) void k_join_parts(const float* __restrict__ part, int64_t stride, int cols,
                                                     PartBounds P, float* __restrict__ out0, float* __restrict__ out1,
                                                     int64_t ldo) {
  __shared__ float red[16][64];
  const int lane = (int)threadIdx.x & 63, slice = (int)threadIdx.x >> 6;
  const int c = (int)blockIdx.x * 64 + lane, seg = (int)blockIdx.y;
  const bool second = blockIdx.z == 1 || out0 == nullptr;
  const float* p = part + (second ? cols : 0) + c;
  float v[4] = {};
  if (c < cols) {
    const int end = P.first[seg + 1];
    int i = P.first[seg] + slice;
    for (; i + 48 < end; i += 64) {  // four sums, so that four loads are in flight
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] += p[(int64_t)(i + 16 * k) * stride];
    }
    for (; i < end; i += 16) v[0] += p[(int64_t)i * stride];
  }
  red[slice][lane] = (v[0] + v[1]) + (v[2] + v[3]);
  __syncthreads();
  if (slice == 0 && c < cols) {
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) sum += red[i][lane];
    (second ? out1 : out0)[seg * ldo + c] = sum;
  }
}

// Calls f with the lanes per row and groups of eight columns per lane as constants.
// `sums`: the columns' sums take registers as well (backward), so that four groups of columns per lane would leave one
// wave per SIMD.  All groups but the last (of 256 and 512 lanes with four, the last two) are full.
template <typename F>
void by_cols(int cols, bool sums, F&& f) {
  typedef std::integral_constant<int, 16> L16;
  typedef std::integral_constant<int, 64> L64;
  typedef std::integral_constant<int, 256> L256;
  typedef std::integral_constant<int, 512> L512;
  typedef std::integral_constant<int, 1> N1;
  typedef std::integral_constant<int, 2> N2;
  typedef std::integral_constant<int, 3> N3;
  typedef std::integral_constant<int, 4> N4;
  const int g = (cols + 7) / 8;
  if (g <= 16) f(L16{}, N1{});
  else if (g <= 64) f(L64{}, N1{});
  else if (g <= 128) f(L64{}, N2{});
  else if (g <= 192) f(L64{}, N3{});
  else if (sums && g <= 256) f(L256{}, N1{});
  else if (g <= 256) f(L64{}, N4{});
  else if (g <= 512) f(L256{}, N2{});
  else if (g <= 1024) f(L256{}, N4{});
  else f(L512{}, N4{});
}

LnChunks ln_chunks(int cols, const LnSegs& S) {
  // about 512 workgroups, two per CU, of at least one turn each (1024: 32256 x 1024 in bf16 38 -> 43 us, 9677 x 1024
  // 17 -> 20, since twice as many sums are written and joined)
  const int per = cols <= 128 ? 16 : cols <= 1536 ? 4 : 1;  // rows of a turn
  const int64_t rows = S.cu[S.nseg];
  LnChunks P;
  P.rows = (int)std::max<int64_t>(per, (rows + 511) / 512);
  P.rows = (P.rows + per - 1) / per * per;
  P.first[0] = 0;
  for (int i = 0; i < S.nseg; ++i)
    P.first[i + 1] = P.first[i] + (int)(((int64_t)S.cu[i + 1] - S.cu[i] + P.rows - 1) / P.rows);
  return P;
}
}  // namespace

hipError_t launch_join_parts(const float* part, int64_t stride, int cols, const PartBounds& P, float* out0,
                             float* out1, int64_t ldo, hipStream_t st) {
  const dim3 grid((unsigned)((cols + 63) / 64), (unsigned)P.nseg, out0 != nullptr && out1 != nullptr ? 2 : 1);
  k_join_parts<<<grid, 1024, 0, st>>>(part, stride, cols, P, out0, out1, ldo);
  return hipGetLastError();
}

hipError_t launch_layer_norm(sphinx_dtype xdt, sphinx_dtype ydt, const LnArgs& a, const LnSegs& S, void* y,
                             int64_t ldy, uint8_t* q, uint8_t* s, float* stats, hipStream_t st) {
  by_cols(a.cols, false, [&](auto L, auto N) {
    constexpr int LPR = decltype(L)::value, NI = decltype(N)::value;
    typedef LnCfg<LPR> C;
    const dim3 grid = long_grid(((int64_t)S.cu[S.nseg] + C::ROWS - 1) / C::ROWS);
    auto go = [&](auto xt, auto* out) {
      typedef decltype(xt) XT;
      typedef std::remove_pointer_t<decltype(out)> OT;
      k_layer_norm<XT, OT, LPR, NI><<<grid, C::NT, 0, st>>>(a, S, out, ldy, Q8Out{q, s}, stats);
    };
    auto by_out = [&](auto xt) {
      if (q != nullptr) go(xt, (Q8Out*)nullptr);
      else if (ydt == SPHINX_BF16) go(xt, (bf16*)y);
      else go(xt, (float*)y);
    };
    if (xdt == SPHINX_BF16) by_out(bf16{});
    else by_out(float{});
  });
  return hipGetLastError();
}

size_t layer_norm_backward_ws_bytes(int cols, const LnSegs& S) {
  return (size_t)ln_chunks(cols, S).first[S.nseg] * 2 * cols * 4;
}

hipError_t launch_layer_norm_backward(sphinx_dtype xdt, sphinx_dtype gdt, const LnArgs& a, const LnSegs& S,
                                      const float* stats, const void* dy, int64_t lddy, void* dx, int64_t lddx,
                                      float* dw, float* db, int64_t ldg, float* ws, hipStream_t st) {
  const LnChunks P = ln_chunks(a.cols, S);
  const int grid = P.first[S.nseg];
  float* part = dw != nullptr || db != nullptr ? ws : nullptr;
  // Small calls sum the columns beside the rows, in workgroups of their own that read x and dy again, instead of
  // joining chunks in a second launch: 1000 x 1024 in bf16 11.7 -> 8.6 us a call (12.3 -> 9.2 where x and dy come from
  // HBM), 2048 x 1024 in eight segments 11.4 -> 8.4 (11.9 -> 8.5).  A workgroup's share is a segment's rows (1500 x 333
  // in fp32 from HBM 12.6 -> 13.6, 2000 x 1024 from the caches 14.0 -> 15.4), and the second reading has to find them in
  // the caches (4000 x 1024 in bf16 in four segments, 16.4 MB, 11.4 -> 12.3).
  const int64_t rows = S.cu[S.nseg];
  int longest = 0;
  for (int i = 0; i < S.nseg; ++i) longest = std::max(longest, S.cu[i + 1] - S.cu[i]);
  const int xb = xdt == SPHINX_BF16 ? 2 : 4, gb = gdt == SPHINX_BF16 ? 2 : 4;
  if ((dw != nullptr || db != nullptr) && a.cols >= 32 && a.cols <= 1536 && longest <= 1024 &&
      rows * a.cols * (xb + gb) <= (12 << 20)) {
    // rows that dx overlaps are summed before it is written
    auto apart = [&](const void* p, int64_t ld, int bytes) {
      auto end = [&](const void* q, int64_t l, int b) { return (uintptr_t)q + ((rows - 1) * l + a.cols) * b; };
      return dx == nullptr || rows == 0 || end(p, ld, bytes) <= (uintptr_t)dx || end(dx, lddx, gb) <= (uintptr_t)p;
    };
    const bool one = apart(a.x, a.ldx, xb) && apart(dy, lddy, gb);
    by_cols(a.cols, true, [&](auto L, auto N) {
      constexpr int LPR = decltype(L)::value, NI = decltype(N)::value;
      if constexpr (LPR <= 64 && NI <= 3) {
        auto go = [&](auto xt, auto gt) {
          typedef decltype(xt) XT;
          typedef decltype(gt) GT;
          auto launch = [&](int blocks, int chunks) {
            k_layer_norm_backward<XT, GT, LPR, NI, true><<<(unsigned)(blocks + chunks), LnCfg<LPR>::NT, 0, st>>>(
                a, S, P, stats, (const GT*)dy, lddy, (GT*)dx, lddx, nullptr, LnSums{dw, db, ldg, blocks});
          };
          const int blocks = (a.cols + 31) / 32 * S.nseg, chunks = dx != nullptr ? grid : 0;
          launch(blocks, one ? chunks : 0);
          if (!one && chunks > 0) launch(0, chunks);
        };
        auto by_g = [&](auto xt) {
          if (gdt == SPHINX_BF16) go(xt, bf16{});
          else go(xt, float{});
        };
        if (xdt == SPHINX_BF16) by_g(bf16{});
        else by_g(float{});
      }
    });
    return hipGetLastError();
  }
  if (grid > 0) {
    by_cols(a.cols, true, [&](auto L, auto N) {
      constexpr int LPR = decltype(L)::value, NI = decltype(N)::value;
      auto go = [&](auto xt, auto gt) {
        typedef decltype(xt) XT;
        typedef decltype(gt) GT;
        k_layer_norm_backward<XT, GT, LPR, NI, false><<<grid, LnCfg<LPR>::NT, 0, st>>>(
            a, S, P, stats, (const GT*)dy, lddy, (GT*)dx, lddx, part, LnSums{});
      };
      auto by_g = [&](auto xt) {
        if (gdt == SPHINX_BF16) go(xt, bf16{});
        else go(xt, float{});
      };
      if (xdt == SPHINX_BF16) by_g(bf16{});
      else by_g(float{});
    });
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (dw == nullptr && db == nullptr) return hipSuccess;
  PartBounds B;
  B.nseg = S.nseg;
  for (int i = 0; i <= S.nseg; ++i) B.first[i] = P.first[i];
  return launch_join_parts(ws, 2 * (int64_t)a.cols, a.cols, B, dw, db, ldg, st);
}

}  // namespace sphinx
