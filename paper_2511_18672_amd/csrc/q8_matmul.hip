// Product of two matrices in 8 bits with power-of-two scales per block of 128
// (q8.hpp has the layout): out[M][N] = sum_k A[m][k] B[n][k], + bias, GELU or
// added to out.  A workgroup computes a tile of 128 x 128 outputs in four waves
// of 64 x 64; K steps of 128 bytes are copied straight to LDS, two of them in
// flight.  16-byte chunk c of row r sits at c ^ ((r >> 1) & 7), so that the 16
// rows of a pass of a 16-byte LDS read fall on all banks.
//
// bf16 outputs: v_mfma_scale_f32_32x32x64_f8f6f4 on the bytes, the scales in the
// instruction.  Its sums are fp32, but inside a group of eight products what lies
// 2^-13 below the largest is dropped: 2e-5 of the result on products of random
// e4m3 numbers (5e-5 where their exponents are uniform), a hundredth of the
// rounding of a bf16 output.
// fp32 outputs: the numbers are made bf16 with their scale, which is exact
// (v_cvt_scalef32_pk_bf16_fp8), and go through v_mfma_f32_32x32x16_bf16, whose
// products are exact and sums fp32.
#include <algorithm>
#include <type_traits>

#include "q8.hpp"

namespace sphinx {

namespace {
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

// s_waitcnt immediate: vmcnt(vm) lgkmcnt(0)
constexpr int wait_vm(int vm) { return 0x0070 | (vm & 15) | ((vm >> 4) << 14); }

template <typename OT>
__device__ __forceinline__ void q8_store4(const Q8Epi& e, int64_t m, int n, int N, f32x4 v) {
  OT* o = static_cast<OT*>(e.out) + m * e.ldo + n;
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    if (e.bias != nullptr && n + t < N)
      v[t] += e.bias_bf16 ? (float)static_cast<const bf16*>(e.bias)[n + t] : static_cast<const float*>(e.bias)[n + t];
    if (e.epi == Q8_EPI_GELU) v[t] = gelu_tanh(v[t]);
  }
#pragma unroll
  for (int t = 0; t < 4; ++t)
    if (n + t < N) o[t] = (OT)(e.epi == Q8_EPI_ADD ? (float)o[t] + v[t] : v[t]);
}

template <typename OT>
__global__ __launch_bounds__(256, 2) void k_q8_matmul(const uint8_t* __restrict__ A, const uint8_t* __restrict__ sA,
                                                      const uint8_t* __restrict__ B, const uint8_t* __restrict__ sB,
                                                      int M, int N, int KB, Q8Epi e) {
  constexpr bool kWide = std::is_same_v<OT, float>;  // fp32 outputs
  constexpr int BM = 128, BN = 128, STAGE = (BM + BN) * 128, COPIES = (BM + BN) / 8 / 4;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[2 * STAGE];
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int r32 = lane & 31, g = lane >> 5;
  const int nt = (N + BN - 1) / BN;
  const int tile = xcd_tile((int)blockIdx.x, (int)gridDim.x);
  const int m0 = tile / nt * BM, n0 = tile % nt * BN;
  const int64_t ld = (int64_t)KB * kQ8Block;
  const int lds = (KB + 3) & ~3;
  const uint8_t* src[COPIES];
  uint32_t voff[COPIES];
#pragma unroll
  for (int i = 0; i < COPIES; ++i) {
    const int qd = wave * COPIES + i, row = 8 * qd + (lane >> 3);
    const int c = (lane & 7) ^ ((row >> 1) & 7);
    const bool is_a = 8 * qd < BM;
    src[i] = is_a ? A + m0 * ld : B + n0 * ld;  // rows past the end repeat the last one
    voff[i] = (uint32_t)((is_a ? min(row, M - 1 - m0) : min(row - BM, N - 1 - n0)) * ld + 16 * c);
  }
  auto copy = [&](int kb) {
    unsigned char* base = smem + (kb & 1) * STAGE;
#pragma unroll
    for (int i = 0; i < COPIES; ++i)
      lds_dma16_at(src[i] + (int64_t)kb * kQ8Block, voff[i], base + (wave * COPIES + i) * 1024);
  };
  const int a0 = (wave >> 1) * 64, b0 = (wave & 1) * 64;
  const uint8_t* sa[2];
  const uint8_t* sb[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    sa[i] = sA + (int64_t)min(m0 + a0 + 32 * i + r32, M - 1) * lds;
    sb[i] = sB + (int64_t)min(n0 + b0 + 32 * i + r32, N - 1) * lds;
  }
  f32x16 acc[2][2] = {};
  if (KB > 0) copy(0);
  for (int kb = 0; kb < KB; ++kb) {
    const int xa[2] = {sa[0][kb], sa[1][kb]}, xb[2] = {sb[0][kb], sb[1][kb]};
    __builtin_amdgcn_s_waitcnt(wait_vm(0));  // step kb has landed, and every wave has read step kb - 1
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (kb + 1 < KB) copy(kb + 1);
    const unsigned char* st = smem + (kb & 1) * STAGE;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      i32x4 fa[2][2], fb[2][2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int off = r32 * 128 + (((4 * ks + 2 * g + h) ^ ((r32 >> 1) & 7)) << 4);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          fa[i][h] = *reinterpret_cast<const i32x4*>(st + (a0 + 32 * i) * 128 + off);
          fb[i][h] = *reinterpret_cast<const i32x4*>(st + (BM + b0 + 32 * i) * 128 + off);
        }
      }
      if constexpr (!kWide) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
                __builtin_shufflevector(fb[j][0], fb[j][1], 0, 1, 2, 3, 4, 5, 6, 7),
                __builtin_shufflevector(fa[i][0], fa[i][1], 0, 1, 2, 3, 4, 5, 6, 7), acc[i][j], 0, 0, 0, xb[j], 0, xa[i]);
      } else {
        // eight bytes of a lane at a time: the order of the contraction is free, and the same on both sides
        auto wide = [](int lo, int hi, float scale) {
          const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
          const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
          const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
          const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
          return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
        };
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          bf16x8 wa[2], wb[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            wa[i] = wide(fa[i][u >> 1][2 * (u & 1)], fa[i][u >> 1][2 * (u & 1) + 1], two_to(xa[i] - 127));
            wb[i] = wide(fb[i][u >> 1][2 * (u & 1)], fb[i][u >> 1][2 * (u & 1) + 1], two_to(xb[i] - 127));
          }
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
              acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wb[j], wa[i], acc[i][j], 0, 0, 0);
        }
      }
    }
  }
  // transposed blocks: lane l holds row l % 32 and, in registers 4q .. 4q+3, columns 8q + 4 (l / 32) .. + 3
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int m = m0 + a0 + 32 * i + r32;
    if (m >= M) continue;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        q8_store4<OT>(e, m, n0 + b0 + 32 * j + 8 * q + 4 * g, N,
                      f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]});
  }
}
}  // namespace

size_t q8_matmul_ws_bytes(sphinx_dtype odt, int M, int N, int K) { return 0; }

hipError_t launch_q8_matmul(sphinx_dtype odt, int M, int N, int K, const Q8Mat& a, const Q8Mat& b, const Q8Epi& e,
                            float* ws, hipStream_t stream) {
  const int KB = (K + kQ8Block - 1) / kQ8Block;
  const int64_t grid = (int64_t)((M + 127) / 128) * ((N + 127) / 128);
  if (odt == SPHINX_BF16) k_q8_matmul<bf16><<<(unsigned)grid, 256, 0, stream>>>(a.q, a.s, b.q, b.s, M, N, KB, e);
  else k_q8_matmul<float><<<(unsigned)grid, 256, 0, stream>>>(a.q, a.s, b.q, b.s, M, N, KB, e);
  return hipGetLastError();
}

}  // namespace sphinx
