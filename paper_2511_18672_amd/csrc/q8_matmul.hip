// Product of two matrices in 8 bits with power-of-two scales per block of 128
// (q8.hpp has the layout): out[M][N] = sum_k A[m][k] B[n][k], + bias, GELU, added
// to out, or left in 8 bits.  A workgroup computes a tile of 64 x 64 to 256 x 256
// outputs in four or eight waves (q8_rules.hpp chooses).  K steps of 128 bytes are
// copied straight to LDS into one of two stages, the next one's while this one is
// read; a wave's fragments of the next 64 bytes are read between its products, and
// one barrier a step frees a stage.  16-byte chunk c of row r sits at
// c ^ ((r >> 1) & 7), so that the 16 rows of a pass of a 16-byte LDS read fall on
// all banks.
//
// bf16 outputs: v_mfma_scale_f32_32x32x64_f8f6f4 on the bytes, the scales in the
// instruction.  Its sums are fp32, but inside a group of eight products what lies
// 2^-13 below the largest is dropped: 2e-5 of the result on products of random
// e4m3 numbers (5e-5 where their exponents are uniform), a hundredth of the
// rounding of a bf16 output.
// fp32 outputs: the numbers are made bf16 with their scale, which is exact
// (v_cvt_scalef32_pk_bf16_fp8), and go through v_mfma_f32_32x32x16_bf16, whose
// products are exact and sums fp32 (1e-7).
//
// 8192 x 8192 x 8192: 410-418 us, 2630-2690 TFLOP/s (a loop of the instruction on
// registers alone 3300-3850, by the power that the numbers take); fp32 outputs
// 850-880 us, 1250-1290 (the same loop of bf16 products 1410 in a library product).
// Short contractions are bound by what a tile costs besides its steps: 9677 x 4096
// x 1024 into bf16 takes 56 us in a stream of such calls, of which 40 are left
// without the epilogue's LDS rounds and stores (62 behind a norm, with GELU, with
// the matrix cores busy 27 % of them);
// 32256 x 4608 x 1152 takes 220, of which 58 would be the store alone at 5 TB/s.
#include <algorithm>
#include <type_traits>

#include "q8.hpp"

namespace sphinx {

namespace {
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x8_16 __attribute__((ext_vector_type(8), aligned(16)));  // in memory
typedef int i32x4 __attribute__((ext_vector_type(4)));

// s_waitcnt immediate: vmcnt(vm) lgkmcnt(0)
constexpr int wait_vm(int vm) { return 0x0070 | (vm & 15) | ((vm >> 4) << 14); }

// What follows the sums (they start at the bias): nothing, GELU, or the scale of
// the columns before qcols.  A constant, so that the epilogue has no branches.
enum { Q8_THEN_NOTHING = 0, Q8_THEN_GELU = 1, Q8_THEN_SCALE = 2 };

template <int THEN>
__device__ __forceinline__ void q8_finish(const Q8Epi& e, int n, float (&v)[8]) {
  if constexpr (THEN == Q8_THEN_GELU) {
#pragma unroll
    for (int t = 0; t < 8; ++t) v[t] = gelu_tanh(v[t]);
  }
  if constexpr (THEN == Q8_THEN_SCALE) {
    const float qs = n < e.qcols ? e.qscale : 1.0f;
#pragma unroll
    for (int t = 0; t < 8; ++t) v[t] *= qs;
  }
}

// Biases of four columns from n0 + 8 k + n on, for each k (zeros without one), as
// they are in memory until value() is asked for: all loads are on their way
// before the first is waited for.
template <int C>
struct Q8Bias {
  f32x4 raw[C] = {};
  bool is_bf16 = false;
  __device__ __forceinline__ void load(const Q8Epi& e, int n, int N) {
    if (e.bias == nullptr) return;
    const bf16* h = static_cast<const bf16*>(e.bias);
    const float* f = static_cast<const float*>(e.bias);
    // across the last column: one by one, and the last one's for those behind it, which are not stored
    const bool whole = __ballot(n + 8 * (C - 1) + 4 <= N) == ~0ull;
    is_bf16 = e.bias_bf16;
#pragma unroll
    for (int k = 0; k < C; ++k) {
      if (whole) {
        if (is_bf16) __builtin_memcpy(&raw[k], h + n + 8 * k, 8);
        else __builtin_memcpy(&raw[k], f + n + 8 * k, 16);
      } else if (is_bf16) {
        bf16x4 v;
#pragma unroll
        for (int t = 0; t < 4; ++t) v[t] = h[min(n + 8 * k + t, N - 1)];
        __builtin_memcpy(&raw[k], &v, 8);
      } else {
#pragma unroll
        for (int t = 0; t < 4; ++t) raw[k][t] = f[min(n + 8 * k + t, N - 1)];
      }
    }
  }
  __device__ __forceinline__ f32x4 value(int k) const {
    if (!is_bf16) return raw[k];
    bf16x4 h;
    __builtin_memcpy(&h, &raw[k], 8);
    return f32x4{(float)h[0], (float)h[1], (float)h[2], (float)h[3]};
  }
};

// Finished columns n .. n + 7 of row m.
template <typename OT>
__device__ __forceinline__ void q8_store8(const Q8Epi& e, int64_t m, int n, int N, float (&v)[8]) {
  if (n >= N) return;
  OT* o = static_cast<OT*>(e.out) + m * e.ldo + n;
  if (e.epi == Q8_EPI_ADD) {
    float b[8];
    load8(o, N - n, b);
#pragma unroll
    for (int t = 0; t < 8; ++t) v[t] += b[t];
  }
  store8(o, N - n, v);
}

__device__ __forceinline__ bf16x8 q8_widen(int lo, int hi, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Waves in WM x WN, each 32 TI x 32 TJ outputs.
template <int TI, int TJ, int WM, int WN>
struct Q8Cfg {
  static constexpr int NW = WM * WN, NT = 64 * NW, BM = 32 * TI * WM, BN = 32 * TJ * WN;
  static constexpr int STAGE = (BM + BN) * 128, SCALES = 64 * NW * 16, SMEM = 2 * (STAGE + SCALES);
  static constexpr int COPIES = (BM + BN) / 8 / NW;  // 8-row copies per wave and stage
  static_assert(COPIES * 8 * NW == BM + BN, "every wave copies as many rows");
  static_assert(BM % 64 == 0 && BM + BN <= 64 * NW, "one copy of 64 rows' scales per wave, of one operand");
};

// Outputs as a matrix in 8 bits, quantised from fp32: a block of 128 columns is
// two waves' (TJ = 2), which tell each other their rows' largest magnitudes.
template <int TI, int TJ, int WN, int THEN, typename A, typename F>
__device__ __forceinline__ void q8_rows_in_8_bits(A& acc, F& eight, const Q8Epi& e, unsigned char* smem, int m0, int n0,
                                                  int M, int N, int wave) {
  static_assert(TJ == 2 && WN % 2 == 0, "64 columns a wave");
  const int lane = (int)threadIdx.x & 63, g = lane >> 5, r32 = lane & 31;
  const int Np = (N + kQ8Block - 1) / kQ8Block * kQ8Block;
  constexpr int PITCH = 64 + 16;
  unsigned char* mine = smem + wave * 32 * PITCH;
  float* tops = reinterpret_cast<float*>(smem + 16 * 32 * PITCH) + wave * 32 * TI;
  const float* other = tops + ((wave & 1) != 0 ? -32 * TI : 32 * TI);
  float top[TI];
#pragma unroll
  for (int i = 0; i < TI; ++i) {
    float all[32];
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int q = 0; q < 4; q += 2) {
        float v[8];
        const int n = n0 + 32 * j + 8 * (q + g);
        eight(i, j, q, v);
        q8_finish<THEN>(e, n, v);
#pragma unroll
        for (int t = 0; t < 8; ++t) {
          v[t] = n + t < N ? v[t] : 0.0f;
          all[16 * j + 4 * q + t] = acc[i][j][4 * q + t] = v[t];
        }
      }
    top[i] = finite_top(all);
    const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(top[i]), __float_as_uint(top[i]), false, false);
    top[i] = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
    if (g == 0) tops[32 * i + r32] = top[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < TI; ++i) {
    const int sb = q8_scale_byte(fmaxf(top[i], other[32 * i + r32]));
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int q = 0; q < 4; q += 2) {
        float v[8];
#pragma unroll
        for (int t = 0; t < 8; ++t) v[t] = acc[i][j][4 * q + t];
        *reinterpret_cast<uint2*>(mine + r32 * PITCH + 32 * j + 8 * (q + g)) = q8_pack8(v, sb);
      }
    const int m = m0 + 32 * i + r32;
    if ((wave & 1) == 0 && g == 0 && m < M && n0 < Np)
      e.scales[(int64_t)m * q8_scale_row(Np / kQ8Block) + n0 / kQ8Block] = (uint8_t)sb;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const int r = 16 * p + (lane >> 2), c = 16 * (lane & 3), row = m0 + 32 * i + r;
      const uint4 w = *reinterpret_cast<const uint4*>(mine + r * PITCH + c);
      if (row < M && n0 < Np) *reinterpret_cast<uint4*>(static_cast<uint8_t*>(e.out) + (int64_t)row * Np + n0 + c) = w;
    }
  }
}

// out += (1 + gate) C on an fp32 residual whose N is a multiple of 4.  Rows of the
// residual are read one set of 32 ahead of their use; a wave's rows mostly have
// one row of gates, which is then read once.
template <int TI, int TJ, typename A, typename F>
__device__ __forceinline__ void q8_rows_gated(A& acc, F& eight, const Q8Epi& e, unsigned char* smem, int m0, int n0,
                                              int M, int N, int wave) {
  constexpr int PITCH = 32 * TJ * 4 + 16, LPW = 8 * TJ, RPP = 64 / LPW, P = 32 / RPP;
  const int lane = (int)threadIdx.x & 63, g = lane >> 5, r32 = lane & 31;
  unsigned char* mine = smem + wave * 32 * PITCH;
  const int c = lane % LPW * 4, n = min(n0 + c, N - 4), sub = lane / LPW;
  const bool in = n0 + c < N;
  float* out = static_cast<float*>(e.out) + n;
  f32x4 h[2][P];
  auto load = [&](int i) {
#pragma unroll
    for (int p = 0; p < P; ++p)
      h[i & 1][p] = *reinterpret_cast<const f32x4*>(out + (int64_t)min(m0 + 32 * i + p * RPP + sub, M - 1) * e.ldo);
  };
  load(0);
  const int first = e.row_of[min(m0, M - 1)];
  bool same = true;
#pragma unroll
  for (int i = 0; i < TI; ++i) same = same && e.row_of[min(m0 + 32 * i + r32, M - 1)] == first;
  auto rows = [&](auto SAME) {
    f32x4 gate;
    if constexpr (decltype(SAME)::value) gate = *reinterpret_cast<const f32x4*>(e.gate + first * e.ldg + n);
#pragma unroll
    for (int i = 0; i < TI; ++i) {
      if (i + 1 < TI) load(i + 1);
#pragma unroll
      for (int j = 0; j < TJ; ++j)
#pragma unroll
        for (int q = 0; q < 4; q += 2) {
          float v[8];
          eight(i, j, q, v);
          __builtin_memcpy(__builtin_assume_aligned(mine + r32 * PITCH + (32 * j + 8 * (q + g)) * 4, 16), v, 32);
        }
#pragma unroll
      for (int p = 0; p < P; ++p) {
        const int r = p * RPP + sub, m = m0 + 32 * i + r;
        const f32x4 v = *reinterpret_cast<const f32x4*>(mine + r * PITCH + c * 4);
        if constexpr (!decltype(SAME)::value)
          gate = *reinterpret_cast<const f32x4*>(e.gate + e.row_of[min(m, M - 1)] * e.ldg + n);
        f32x4 o;
#pragma unroll
        for (int t = 0; t < 4; ++t) o[t] = fmaf(1.0f + gate[t], v[t], h[i & 1][p][t]);
        if (in && m < M) *reinterpret_cast<f32x4*>(out + (int64_t)m * e.ldo) = o;
      }
    }
  };
  if (__ballot(same) == ~0ull) rows(std::true_type{});
  else rows(std::false_type{});
}

// Tile (m0, n0) over the blocks k0 .. k1 - 1 of the contraction (k0 a multiple
// of 4); part != NULL: the sums go there, [M][N], as they are.
template <Q8Kind KIND, int TI, int TJ, int WM, int WN>
__device__ __forceinline__ void q8_tile(const uint8_t* __restrict__ A, const uint8_t* __restrict__ sA,
                                        const uint8_t* __restrict__ B, const uint8_t* __restrict__ sB, int M, int N,
                                        int KB, const Q8Epi& e, unsigned char* smem, int m0, int n0, int k0, int k1,
                                        float* part) {
  typedef Q8Cfg<TI, TJ, WM, WN> C;
  constexpr bool kWide = KIND == kQ8F32;
  typedef std::conditional_t<KIND == kQ8Bf16, bf16, float> OT;
  constexpr int BM = C::BM, STAGE = C::STAGE, COPIES = C::COPIES, NW = C::NW;
  const int tid = (int)threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WN, wn = wave % WN, g = lane >> 5, r32 = lane & 31;
  const int64_t ld = (int64_t)KB * kQ8Block;
  const int lds = q8_scale_row(KB);
  // copy c of this wave fills rows 8q .. 8q+7 of the stage (A rows, then B rows), q = NW c + wave
  const uint8_t* src[COPIES];
  uint32_t voff[COPIES];
#pragma unroll
  for (int c = 0; c < COPIES; ++c) {
    const int q = NW * c + wave, row = 8 * q + (lane >> 3);
    const int ch = (lane & 7) ^ ((row >> 1) & 7);
    const bool is_a = 8 * q < BM;
    src[c] = is_a ? A + m0 * ld : B + n0 * ld;  // rows past the end repeat the last one
    voff[c] = (uint32_t)((is_a ? min(row, M - 1 - m0) : min(row - BM, N - 1 - n0)) * ld + 16 * ch);
  }
  auto copy = [&](int kt, int slot, int c) {
    lds_dma16_at(src[c] + (int64_t)kt * kQ8Block, voff[c], smem + slot * STAGE + (NW * c + wave) * 1024);
  };
  const int a0 = wm * 32 * TI, b0 = wn * 32 * TJ;
  // Scales: 16 bytes of a row are 16 steps; rows of the tile in order (A, then B), two such sets used in turn.  A
  // lane takes the bytes of four steps at a time, a dword for each row of a fragment.
  unsigned char* ssm = smem + 2 * STAGE;
  const uint8_t* ssrc;
  {
    const int row = 64 * wave;  // of lane 0; a wave's 64 rows are of one operand (past the tile: of none)
    const bool is_a = row < BM;
    const int at = is_a ? min(m0 + row + lane, M - 1) : min(n0 + row - BM + lane, N - 1);
    ssrc = (is_a ? sA : sB) + (int64_t)at * lds;
  }
  auto copy_scales = [&](int chunk) {
    lds_dma16(ssrc + 16 * min(chunk, lds / 16 - 1), ssm + (chunk & 1) * C::SCALES + wave * 1024);
  };
  int sc[TI + TJ], sn[TI + TJ];
  auto read_scales = [&](int kt) {
    const unsigned char* p = ssm + (kt >> 4 & 1) * C::SCALES + (kt >> 2 & 3) * 4 + r32 * 16;
#pragma unroll
    for (int i = 0; i < TI; ++i) sn[i] = *reinterpret_cast<const int*>(p + (a0 + 32 * i) * 16);
#pragma unroll
    for (int j = 0; j < TJ; ++j) sn[TI + j] = *reinterpret_cast<const int*>(p + (BM + b0 + 32 * j) * 16);
  };
  int foff[2][2];
#pragma unroll
  for (int ks = 0; ks < 2; ++ks)
#pragma unroll
    for (int h = 0; h < 2; ++h) foff[ks][h] = r32 * 128 + (((4 * ks + 2 * g + h) ^ ((r32 >> 1) & 7)) << 4);

  // transposed blocks: lane l holds row l % 32 and, in registers 4q .. 4q+3, columns 8q + 4 (l / 32) .. + 3.  The sums
  // start at the bias (of pieces, where they are joined).
  Q8Bias<4 * TJ> bias;
  if (part == nullptr) bias.load(e, n0 + b0 + 4 * g, N);
  if (k1 > k0) {
    copy_scales(k0 >> 4);
#pragma unroll
    for (int st = 0; st < 2; ++st)
#pragma unroll
      for (int c = 0; c < COPIES; ++c) copy(min(k0 + st, k1 - 1), st, c);
    __builtin_amdgcn_s_waitcnt(wait_vm(COPIES));  // stage 0 must land
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    read_scales(k0);
#pragma unroll
    for (int i = 0; i < TI + TJ; ++i) sc[i] = sn[i];
  }
  f32x16 acc[TI][TJ];
#pragma unroll
  for (int j = 0; j < TJ; ++j)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const f32x4 v = bias.value(4 * j + q);
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < TI; ++i) acc[i][j][4 * q + t] = v[t];
    }
  i32x8 fa[2][TI], fb[2][TJ];
  // fragment r of a k-step: the TJ of B first, then the TI of A
  auto read = [&](int slot, int ks, int r) {
    const unsigned char* st = smem + slot * STAGE + (r < TJ ? BM + b0 + 32 * r : a0 + 32 * (r - TJ)) * 128;
    const i32x4 lo = *reinterpret_cast<const i32x4*>(st + foff[ks][0]);
    const i32x4 hi = *reinterpret_cast<const i32x4*>(st + foff[ks][1]);
    const i32x8 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    if (r < TJ) fb[ks][r] = v; else fa[ks][r - TJ] = v;
  };
  bf16x8 wb[TJ][4];
  // a row of a k-step: its TJ products
  auto row = [&](int ks, int i, auto U) {
    constexpr int u = decltype(U)::value;
    if constexpr (!kWide) {
#pragma unroll
      for (int j = 0; j < TJ; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fb[ks][j], fa[ks][i], acc[i][j], 0, 0, u,
                                                                    sc[TI + j], u, sc[i]);
    } else {
      // eight bytes of a lane at a time: the order of the contraction is free, and the same on both sides
      const float s = __int_as_float((int)(((uint32_t)sc[i] >> (8 * u) & 255u) << 23));
      if (i == 0) {
#pragma unroll
        for (int j = 0; j < TJ; ++j) {
          const float t = __int_as_float((int)(((uint32_t)sc[TI + j] >> (8 * u) & 255u) << 23));
#pragma unroll
          for (int p = 0; p < 4; ++p) wb[j][p] = q8_widen(fb[ks][j][2 * p], fb[ks][j][2 * p + 1], t);
        }
      }
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        const bf16x8 wa = q8_widen(fa[ks][i][2 * p], fa[ks][i][2 * p + 1], s);
#pragma unroll
        for (int j = 0; j < TJ; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wb[j][p], wa, acc[i][j], 0, 0, 0);
      }
    }
    // the products stay here: without this the compiler sinks them past the copies and the barrier into the next
    // block, and spills the fragments that they wait with
#pragma unroll
    for (int j = 0; j < TJ; ++j) asm volatile("" : "+v"(acc[i][j]));
    __builtin_amdgcn_sched_barrier(0);
  };
  constexpr int LAST = TJ + TI - 1;       // A fragment TI - 1, read at the start of its own k-step
  constexpr int BR = TI >= 3 ? 1 : 0;     // rows of the second k-step before the barrier
  constexpr int RR = TI - BR;             // and after it
  auto step = [&](int kt, auto U) {
    constexpr int u = decltype(U)::value, s = u & 1;
#pragma unroll
    for (int i = 0; i < TI; ++i) {
      if (i == 0) read(s, 0, LAST);
      if (i < TJ) read(s, 1, i);
      if (i >= 1) read(s, 1, TJ + i - 1);
      if (TI < TJ && i + 1 == TI) read(s, 1, TJ - 1);
      row(0, i, U);
    }
#pragma unroll
    for (int i = 0; i < TI; ++i) {
      if (i == 0) read(s, 1, LAST);
      if (i == BR) {
        // stage kt+1 has landed, and every wave has read all of stage kt
        __builtin_amdgcn_s_waitcnt(wait_vm(0));
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
      }
      if (i >= BR) {
        // the last stages are refilled with the last one, which is not read again
        constexpr int CR = RR > 1 ? RR - 1 : 1;
#pragma unroll
        for (int c = 0; c < COPIES; ++c)
          if (c * CR / COPIES == i - BR) copy(min(kt + 2, k1 - 1), s, c);
        // the next 16 steps' scales, four times over: that costs less than a branch
        if (u == 1 && i == BR) copy_scales((kt >> 4) + 1);
        if (u == 3 && i + 1 == TI) read_scales(kt + 1);
        // the next stage's first k-step over the rows left; fa[r] not before row r + 1
#pragma unroll
        for (int r = 0; r < LAST; ++r) {
          const int even = r * RR / LAST, after = r - TJ + 1 - BR;
          if ((even > after ? even : after) == i - BR) read(s ^ 1, 0, r);
        }
      }
      row(1, i, U);
    }
    if constexpr (u == 3) {
#pragma unroll
      for (int i = 0; i < TI + TJ; ++i) sc[i] = sn[i];
    }
  };
  if (k1 > k0) {
#pragma unroll
    for (int r = 0; r < LAST; ++r) read(0, 0, r);
    typedef std::integral_constant<int, 0> U0;
    typedef std::integral_constant<int, 1> U1;
    typedef std::integral_constant<int, 2> U2;
    typedef std::integral_constant<int, 3> U3;
    int kt = k0;
    for (; kt + 4 <= k1; kt += 4) {
      step(kt, U0{});
      step(kt + 1, U1{});
      step(kt + 2, U2{});
      step(kt + 3, U3{});
    }
    if (kt < k1) step(kt, U0{});
    if (kt + 1 < k1) step(kt + 1, U1{});
    if (kt + 2 < k1) step(kt + 2, U2{});
  }
  // the refills of the last stages must land while the workgroup holds its LDS
  __builtin_amdgcn_s_waitcnt(wait_vm(0));
  asm volatile("" ::: "memory");
  // the two halves of the wave swap so that each lane has eight neighbouring columns, n0 + b0 + 32 j + 8 (q + g)
  auto eight = [&](int i, int j, int q, float (&v)[8]) {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(acc[i][j][4 * q + t]),
                                                      __float_as_uint(acc[i][j][4 * q + 4 + t]), false, false);
      v[t] = __uint_as_float(x[0]);
      v[4 + t] = __uint_as_float(x[1]);
    }
  };
  // bf16 outputs that are added to: the sum is rounded once, so it does not go through LDS in bf16
  if (KIND == kQ8Bf16 && part == nullptr && e.epi == Q8_EPI_ADD) {
#pragma unroll
    for (int i = 0; i < TI; ++i) {
      const int m = m0 + a0 + 32 * i + r32;
#pragma unroll
      for (int j = 0; j < TJ; ++j)
#pragma unroll
        for (int q = 0; q < 4; q += 2) {
          float v[8];
          eight(i, j, q, v);
          if (m < M) q8_store8<OT>(e, m, n0 + b0 + 32 * j + 8 * (q + g), N, v);
        }
    }
    return;
  }
  // Rows go out through LDS, 32 at a time in a region of the wave's own, so that a store writes whole lines, which then
  // bypass the caches (stores of 16-byte pieces of 32 rows, joined in L2, push the operands out of it: M 32256, N 4608,
  // K 1152 195 us instead of 174; whole lines through L2 209).  Rows that start inside a line, and half lines, go
  // through L2.
  __builtin_amdgcn_s_barrier();  // every wave has read its last stage
  asm volatile("" ::: "memory");
  if constexpr (KIND == kQ8Gated) {
    q8_rows_gated<TI, TJ>(acc, eight, e, smem, m0 + a0, n0 + b0, M, N, wave);
    return;
  }
  if constexpr (KIND == kQ8Bytes) {
    if (e.epi == Q8_EPI_GELU)
      q8_rows_in_8_bits<TI, TJ, WN, Q8_THEN_GELU>(acc, eight, e, smem, m0 + a0, n0 + b0, M, N, wave);
    else
      q8_rows_in_8_bits<TI, TJ, WN, Q8_THEN_NOTHING>(acc, eight, e, smem, m0 + a0, n0 + b0, M, N, wave);
    return;
  }
  auto rows_out = [&](auto* out, int64_t ldo, auto then, auto add) {
    typedef std::remove_pointer_t<decltype(out)> ST;
    constexpr int THEN = decltype(then)::value;
    constexpr bool ADD = decltype(add)::value;
    constexpr int V = 16 / (int)sizeof(ST), PITCH = 32 * TJ * (int)sizeof(ST) + 16;  // values of a piece; bytes of a row
    constexpr int LPW = 32 * TJ / V, RPP = 64 / LPW;                                // lanes of a row; rows of a store
    unsigned char* mine = smem + wave * 32 * PITCH;
    const int c = lane % LPW * V, n = n0 + b0 + c, left = N - n;
    const bool lines = 32 * TJ * sizeof(ST) >= 128 && (((uintptr_t)out | (uint64_t)ldo * sizeof(ST)) & 127) == 0;
#pragma unroll
    for (int i = 0; i < TI; ++i) {
#pragma unroll
      for (int j = 0; j < TJ; ++j)
#pragma unroll
        for (int q = 0; q < 4; q += 2) {
          float v[8];
          eight(i, j, q, v);
          q8_finish<THEN>(e, n0 + b0 + 32 * j, v);  // 32 columns are all before qcols or none
          ST w[8];
#pragma unroll
          for (int t = 0; t < 8; ++t) w[t] = (ST)v[t];
          __builtin_memcpy(__builtin_assume_aligned(mine + r32 * PITCH + (32 * j + 8 * (q + g)) * sizeof(ST), 16), w,
                           8 * sizeof(ST));
        }
#pragma unroll
      for (int p = 0; p < 32 / RPP; ++p) {
        const int r = p * RPP + lane / LPW, m = m0 + a0 + 32 * i + r;
        ST w[V];
        __builtin_memcpy(w, __builtin_assume_aligned(mine + r * PITCH + c * sizeof(ST), 16), 16);
        if (m >= M) continue;
        ST* o = out + m * ldo + n;
        if (left >= V) {
          if constexpr (ADD) {
            ST old[V];
            __builtin_memcpy(old, o, 16);
#pragma unroll
            for (int t = 0; t < V; ++t) w[t] = (ST)((float)w[t] + (float)old[t]);
          }
          if (lines) {
            f32x4 z;
            __builtin_memcpy(&z, w, 16);
            __builtin_nontemporal_store(z, reinterpret_cast<f32x4*>(o));
          } else {
            __builtin_memcpy(o, w, 16);
          }
        } else {
#pragma unroll
          for (int t = 0; t < V; ++t)
            if (t < left) o[t] = ADD ? (ST)((float)w[t] + (float)o[t]) : w[t];
        }
      }
    }
  };
  typedef std::integral_constant<int, Q8_THEN_NOTHING> Nothing;
  OT* out = static_cast<OT*>(e.out);
  if (part != nullptr) rows_out(part, N, Nothing{}, std::false_type{});
  else if (e.epi == Q8_EPI_GELU) rows_out(out, e.ldo, std::integral_constant<int, Q8_THEN_GELU>{}, std::false_type{});
  else if (kWide && e.epi == Q8_EPI_ADD) rows_out(out, e.ldo, Nothing{}, std::bool_constant<kWide>{});
  else if (!kWide && e.qcols > 0) rows_out(out, e.ldo, std::integral_constant<int, Q8_THEN_SCALE>{}, std::false_type{});
  else rows_out(out, e.ldo, Nothing{}, std::false_type{});
}

// Tiles are dealt to the XCDs in contiguous ranges of panels four row tiles
// high, column by column inside a panel, so that the tiles an XCD runs at a
// time share few rows of A and B in its L2.  With part != NULL the contraction
// is cut into gridDim.y pieces of `per` blocks.
template <Q8Kind KIND, int TI, int TJ, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN, 2) void k_q8_matmul(
    const uint8_t* __restrict__ A, const uint8_t* __restrict__ sA, const uint8_t* __restrict__ B,
    const uint8_t* __restrict__ sB, int M, int N, int KB, Q8Epi e, int per, float* __restrict__ part) {
  typedef Q8Cfg<TI, TJ, WM, WN> C;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[C::SMEM];
  const int nt = (N + C::BN - 1) / C::BN, rt = (M + C::BM - 1) / C::BM;
  const int tile = xcd_tile((int)blockIdx.x, rt * nt);
  const int panel = tile / (4 * nt), rem = tile - panel * 4 * nt, ph = min(4, rt - 4 * panel);
  const int k0 = (int)blockIdx.y * per;
  q8_tile<KIND, TI, TJ, WM, WN>(A, sA, B, sB, M, N, KB, e, smem, (4 * panel + rem % ph) * C::BM, (rem / ph) * C::BN, k0,
                              min(KB, k0 + per), part == nullptr ? nullptr : part + (int64_t)blockIdx.y * M * N);
}

// The pieces of a cut contraction added in order, and the epilogue.
template <typename OT>
__global__ __launch_bounds__(256) void k_q8_join(const float* __restrict__ part, int pieces, int M, int N, Q8Epi e) {
  const int wide = (N + 7) / 8;
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x, m = at / wide;
  if (m >= M) return;
  const int n = (int)(at - m * wide) * 8;
  const float* p = part + m * N + n;
  float v[8];
  load8(p, N - n, v);
  for (int i = 1; i < pieces; ++i) {
    float w[8];
    load8(p + (int64_t)i * M * N, N - n, w);
#pragma unroll
    for (int t = 0; t < 8; ++t) v[t] += w[t];
  }
  if (e.bias != nullptr) {
    float b[8];
    if (e.bias_bf16) load8(static_cast<const bf16*>(e.bias) + n, N - n, b);
    else load8(static_cast<const float*>(e.bias) + n, N - n, b);
#pragma unroll
    for (int t = 0; t < 8; ++t) v[t] += b[t];
  }
  if (e.epi == Q8_EPI_GELU) q8_finish<Q8_THEN_GELU>(e, n, v);
  q8_store8<OT>(e, m, n, N, v);
}

// Few rows (M <= 16): what is read is B, once.  A workgroup has 16 columns; its
// eight waves take every eighth block of the contraction, straight from memory
// to the matrix cores (lane l holds bytes 32 (l / 16) .. + 31 of a block of row
// l % 16, whole lines in all), and add their sums through LDS.  One row through
// N = K = 8192: 16.2 us, 4.1 TB/s, where tiles of 64 x 64 take 30.5; 16 rows 24
// (every workgroup reads A as well).  The same for 32 rows takes 35, tiles 31.
template <Q8Kind KIND>
__global__ __launch_bounds__(512) void k_q8_matmul_few(const uint8_t* __restrict__ A, const uint8_t* __restrict__ sA,
                                                       const uint8_t* __restrict__ B, const uint8_t* __restrict__ sB,
                                                       int M, int N, int KB, Q8Epi e) {
  typedef std::conditional_t<KIND == kQ8Bf16, bf16, float> OT;
  constexpr int U = 4;  // blocks whose loads are in flight at a time
  __shared__ __attribute__((aligned(16))) f32x4 sums[8][64];
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int r = lane & 15, g = lane >> 4, n0 = (int)blockIdx.x * 16;
  const int64_t ld = (int64_t)KB * kQ8Block;
  const int lds = q8_scale_row(KB);
  const int rb = min(n0 + r, N - 1), ra = min(r, M - 1);  // rows past the end repeat the last one
  const uint8_t* b = B + rb * ld + 32 * g;
  const uint8_t* sb = sB + (int64_t)rb * lds;
  const uint8_t* a = A + ra * ld + 32 * g;
  const uint8_t* sa = sA + (int64_t)ra * lds;
  f32x4 acc = {};
  for (int k0 = wave; k0 < KB; k0 += 8 * U) {
    i32x8 fb[U], fa[U];
    int xb[U], xa[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = min(k0 + 8 * u, KB - 1);  // past the end: a block that is not used
      fb[u] = *reinterpret_cast<const i32x8_16*>(b + (int64_t)k * kQ8Block);
      fa[u] = *reinterpret_cast<const i32x8_16*>(a + (int64_t)k * kQ8Block);
      xb[u] = sb[k];
      xa[u] = sa[k];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (k0 + 8 * u >= KB) break;
      if constexpr (KIND == kQ8Bf16) {
        acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb[u], fa[u], acc, 0, 0, 0, xb[u], 0, xa[u]);
      } else {
#pragma unroll
        for (int p = 0; p < 4; ++p)
          acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q8_widen(fb[u][2 * p], fb[u][2 * p + 1], two_to(xb[u] - 127)),
                                                        q8_widen(fa[u][2 * p], fa[u][2 * p + 1], two_to(xa[u] - 127)),
                                                        acc, 0, 0, 0);
      }
    }
  }
  // lane l holds row l % 16 and columns 4 (l / 16) .. + 3
  sums[wave][lane] = acc;
  __syncthreads();
  const int n = n0 + 4 * g;
  if (wave != 0 || r >= M || n >= N) return;
  f32x4 v = sums[0][lane];
#pragma unroll
  for (int w = 1; w < 8; ++w) v += sums[w][lane];
  OT* o = static_cast<OT*>(e.out) + r * e.ldo + n;
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    if (n + t >= N) break;
    if (e.bias != nullptr)
      v[t] += e.bias_bf16 ? (float)static_cast<const bf16*>(e.bias)[n + t] : static_cast<const float*>(e.bias)[n + t];
    if (e.epi == Q8_EPI_GELU) v[t] = gelu_tanh(v[t]);
    if (n + t < e.qcols) v[t] *= e.qscale;
    if (e.epi == Q8_EPI_ADD) v[t] += (float)o[t];
    o[t] = (OT)v[t];
  }
}

template <Q8Kind KIND, int TI, int TJ, int WM, int WN>
void launch_tiles(int M, int N, int KB, const Q8Mat& a, const Q8Mat& b, const Q8Epi& e, int pieces, float* ws,
                  hipStream_t stream) {
  typedef Q8Cfg<TI, TJ, WM, WN> C;
  const int64_t grid = (int64_t)((M + C::BM - 1) / C::BM) * ((N + C::BN - 1) / C::BN);
  const int per = ((KB + pieces - 1) / pieces + 3) / 4 * 4;
  k_q8_matmul<KIND, TI, TJ, WM, WN><<<dim3((unsigned)grid, (unsigned)pieces), C::NT, 0, stream>>>(
      a.q, a.s, b.q, b.s, M, N, KB, e, per, pieces > 1 ? ws : nullptr);
  if constexpr (KIND == kQ8Bf16 || KIND == kQ8F32) {
    typedef std::conditional_t<KIND == kQ8Bf16, bf16, float> OT;
    const int64_t n = (int64_t)M * ((N + 7) / 8);
    if (pieces > 1) k_q8_join<OT><<<(unsigned)((n + 255) / 256), 256, 0, stream>>>(ws, pieces, M, N, e);
  }
}
}  // namespace

size_t q8_matmul_ws_bytes(sphinx_dtype odt, int M, int N, int K) {
  const int KB = (K + kQ8Block - 1) / kQ8Block;
  const Q8Kind kind = odt == SPHINX_F32 ? kQ8F32 : kQ8Bf16;
  int pieces = 1;  // of whichever epilogue
  for (bool gelu : {false, true}) pieces = std::max(pieces, plan_q8_matmul(kind, gelu, M, N, KB).pieces);
  return pieces > 1 ? (size_t)pieces * M * N * 4 : 0;
}

hipError_t launch_q8_matmul(Q8Kind kind, int M, int N, int K, const Q8Mat& a, const Q8Mat& b, const Q8Epi& e,
                            float* ws, hipStream_t stream) {
  const int KB = (K + kQ8Block - 1) / kQ8Block;
  if (e.qcols % 32 != 0 || (e.qcols > 0 && (kind != kQ8Bf16 || e.epi != Q8_EPI_STORE))) return hipErrorInvalidValue;
  const Q8Plan p = plan_q8_matmul(kind, e.epi == Q8_EPI_GELU, M, N, KB, ws == nullptr || e.qcols > 0);
  bool launched = false;
  auto go = [&](auto k) {
    constexpr Q8Kind KIND = decltype(k)::value;
    auto tiles = [&](auto tile, auto ti, auto tj, auto wn) {  // waves 2 x wn, each 32 ti x 32 tj outputs
      if constexpr (q8_has_tile(KIND, decltype(tile)::value)) {
        if (p.tile != decltype(tile)::value) return;
        launch_tiles<KIND, decltype(ti)::value, decltype(tj)::value, 2, decltype(wn)::value>(M, N, KB, a, b, e, p.pieces,
                                                                                             ws, stream);
        launched = true;
      }
    };
    if constexpr (q8_has_tile(KIND, kQ8Few)) {
      if (p.tile == kQ8Few) {
        k_q8_matmul_few<KIND><<<(unsigned)((N + 15) / 16), 512, 0, stream>>>(a.q, a.s, b.q, b.s, M, N, KB, e);
        launched = true;
      }
    }
    typedef std::integral_constant<int, 1> I1;
    typedef std::integral_constant<int, 2> I2;
    typedef std::integral_constant<int, 3> I3;
    typedef std::integral_constant<int, 4> I4;
    tiles(std::integral_constant<Q8Tile, kQ8Tile256>{}, I4{}, I2{}, I4{});
    tiles(std::integral_constant<Q8Tile, kQ8Tile192>{}, I3{}, I2{}, I4{});
    tiles(std::integral_constant<Q8Tile, kQ8Tile128>{}, I2{}, I2{}, I2{});
    tiles(std::integral_constant<Q8Tile, kQ8Tile128x64>{}, I2{}, I1{}, I2{});
    tiles(std::integral_constant<Q8Tile, kQ8Tile64>{}, I1{}, I1{}, I2{});
  };
  switch (kind) {
    case kQ8Bf16: go(std::integral_constant<Q8Kind, kQ8Bf16>{}); break;
    case kQ8F32: go(std::integral_constant<Q8Kind, kQ8F32>{}); break;
    case kQ8Gated: go(std::integral_constant<Q8Kind, kQ8Gated>{}); break;
    default: go(std::integral_constant<Q8Kind, kQ8Bytes>{});
  }
  return launched ? hipGetLastError() : hipErrorInvalidValue;
}

}  // namespace sphinx
