// C ABI of the layer norm and of the matrices in 8 bits (declared in
// include/sphinx.h).  Host code only: arguments are validated before any HIP
// call.
#include <algorithm>

#include "q8.hpp"

using namespace sphinx;

namespace {
inline bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }
inline bool valid_dtype(sphinx_dtype d) { return d == SPHINX_F32 || d == SPHINX_BF16; }
inline sphinx_status hip_status(hipError_t e) { return e == hipSuccess ? SPHINX_OK : SPHINX_E_HIP; }

sphinx_status ln_segs(int32_t cols, const int32_t* cu, int32_t nseg, LnSegs* S) {
  if (cols < 1 || cu == nullptr || nseg < 1 || cu[0] != 0) return SPHINX_E_INVALID;
  if (cols > kLnMaxCols || nseg > SPHINX_MAX_REQUESTS) return SPHINX_E_UNSUPPORTED;
  S->nseg = nseg;
  S->cu[0] = 0;
  for (int i = 0; i < nseg; ++i) {
    if (cu[i + 1] < cu[i]) return SPHINX_E_INVALID;
    S->cu[i + 1] = cu[i + 1];
  }
  if (cu[nseg] > (1 << 30)) return SPHINX_E_UNSUPPORTED;  // rows are stepped over in 32 bits
  return SPHINX_OK;
}

// What both directions share; *todo: there are rows.
sphinx_status ln_check(sphinx_dtype xdt, sphinx_dtype wdt, int32_t cols, const void* x, int64_t ldx, const void* w,
                       const void* b, int64_t ldw, int32_t plus_one, const int32_t* cu, int32_t nseg, LnSegs* S) {
  if (!valid_dtype(xdt) || !valid_dtype(wdt)) return SPHINX_E_UNSUPPORTED;
  const sphinx_status st = ln_segs(cols, cu, nseg, S);
  if (st != SPHINX_OK) return st;
  if (ldx < cols || (plus_one != 0 && plus_one != 1)) return SPHINX_E_INVALID;
  if ((w != nullptr || b != nullptr) && ldw < cols) return SPHINX_E_INVALID;
  if (!aligned(x, 16) || !aligned(w, 16) || !aligned(b, 16)) return SPHINX_E_INVALID;
  if (S->cu[nseg] > 0 && x == nullptr) return SPHINX_E_INVALID;
  return SPHINX_OK;
}

sphinx_status q8_size_check(int32_t rows, int32_t cols) {
  if (rows < 0 || cols < 0) return SPHINX_E_INVALID;
  // a launch has less than 2^32 threads (2^24 tiles of 128 x 128 hold 256 GB)
  const int64_t wide = ((int64_t)cols + 127) / 128, tall = ((int64_t)rows + 127) / 128;
  if (cols > kQ8MaxCols || rows > (1 << 28) || wide * tall >= (1 << 24)) return SPHINX_E_UNSUPPORTED;
  return SPHINX_OK;
}
// Outputs of a product, whose columns may be as many as B's rows.
sphinx_status q8_outputs_check(int32_t M, int32_t N) {
  return (((int64_t)M + 127) / 128) * (((int64_t)N + 127) / 128) < (1 << 24) ? SPHINX_OK : SPHINX_E_UNSUPPORTED;
}
}  // namespace

extern "C" {

sphinx_status sphinx_layer_norm(sphinx_dtype xdt, sphinx_dtype wdt, sphinx_dtype ydt, int32_t cols, float eps,
                                const void* x, int64_t ldx, const void* w, const void* b, int64_t ldw,
                                int32_t plus_one, const int32_t* cu, int32_t nseg, void* y, int64_t ldy, float* stats,
                                void* stream) {
  LnSegs S;
  if (!valid_dtype(ydt)) return SPHINX_E_UNSUPPORTED;
  const sphinx_status st = ln_check(xdt, wdt, cols, x, ldx, w, b, ldw, plus_one, cu, nseg, &S);
  if (st != SPHINX_OK) return st;
  if (!(eps >= 0.0f) || ldy < cols || !aligned(y, 16) || !aligned(stats, 16)) return SPHINX_E_INVALID;
  if (S.cu[nseg] == 0) return SPHINX_OK;
  if (y == nullptr) return SPHINX_E_INVALID;
  const LnArgs a{x, ldx, w, b, ldw, wdt == SPHINX_BF16, plus_one != 0, cols, eps, nullptr};
  return hip_status(launch_layer_norm(xdt, ydt, a, S, y, ldy, nullptr, nullptr, stats, (hipStream_t)stream));
}

sphinx_status sphinx_layer_norm_q8(sphinx_dtype xdt, sphinx_dtype wdt, int32_t cols, float eps, const void* x,
                                   int64_t ldx, const void* w, const void* b, int64_t ldw, int32_t plus_one,
                                   const int32_t* cu, int32_t nseg, uint8_t* q, uint8_t* s, float* stats,
                                   void* stream) {
  LnSegs S;
  const sphinx_status st = ln_check(xdt, wdt, cols, x, ldx, w, b, ldw, plus_one, cu, nseg, &S);
  if (st != SPHINX_OK) return st;
  if (!(eps >= 0.0f) || !aligned(q, 16) || !aligned(s, 16) || !aligned(stats, 16)) return SPHINX_E_INVALID;
  if (S.cu[nseg] == 0) return SPHINX_OK;
  if (q == nullptr || s == nullptr) return SPHINX_E_INVALID;
  const LnArgs a{x, ldx, w, b, ldw, wdt == SPHINX_BF16, plus_one != 0, cols, eps, nullptr};
  return hip_status(launch_layer_norm(xdt, SPHINX_BF16, a, S, nullptr, 0, q, s, stats, (hipStream_t)stream));
}

sphinx_status sphinx_layer_norm_backward_workspace_bytes(int32_t cols, const int32_t* cu, int32_t nseg,
                                                         size_t* bytes) {
  LnSegs S;
  const sphinx_status st = ln_segs(cols, cu, nseg, &S);
  if (st != SPHINX_OK) return st;
  if (bytes == nullptr) return SPHINX_E_INVALID;
  *bytes = layer_norm_backward_ws_bytes(cols, S);
  return SPHINX_OK;
}

sphinx_status sphinx_layer_norm_backward(sphinx_dtype xdt, sphinx_dtype wdt, sphinx_dtype gdt, int32_t cols,
                                         const void* x, int64_t ldx, const float* stats, const void* w, int64_t ldw,
                                         int32_t plus_one, const int32_t* cu, int32_t nseg, const void* dy,
                                         int64_t lddy, void* dx, int64_t lddx, float* dw, float* db, int64_t ldg,
                                         void* ws, size_t ws_bytes, void* stream) {
  LnSegs S;
  if (!valid_dtype(gdt)) return SPHINX_E_UNSUPPORTED;
  const sphinx_status st = ln_check(xdt, wdt, cols, x, ldx, w, nullptr, ldw, plus_one, cu, nseg, &S);
  if (st != SPHINX_OK) return st;
  const bool sums = dw != nullptr || db != nullptr;
  if (lddy < cols || (dx != nullptr && lddx < cols) || (sums && ldg < cols)) return SPHINX_E_INVALID;
  if (!aligned(stats, 16) || !aligned(dy, 16) || !aligned(dx, 16) || !aligned(dw, 16) || !aligned(db, 16) ||
      !aligned(ws, 256))
    return SPHINX_E_INVALID;
  if (S.cu[nseg] > 0 && (stats == nullptr || dy == nullptr)) return SPHINX_E_INVALID;
  if (!sums && (dx == nullptr || S.cu[nseg] == 0)) return SPHINX_OK;
  if (sums) {
    const size_t need = layer_norm_backward_ws_bytes(cols, S);
    if (need > 0 && ws == nullptr) return SPHINX_E_INVALID;
    if (ws_bytes < need) return SPHINX_E_WORKSPACE;
  }
  const LnArgs a{x, ldx, w, nullptr, ldw, wdt == SPHINX_BF16, plus_one != 0, cols, 0.0f, nullptr};
  return hip_status(launch_layer_norm_backward(xdt, gdt, a, S, stats, dy, lddy, dx, lddx, dw, db, ldg,
                                               static_cast<float*>(ws), (hipStream_t)stream));
}

sphinx_status sphinx_q8_bytes(int32_t rows, int32_t cols, size_t* q_bytes, size_t* s_bytes) {
  const sphinx_status st = q8_size_check(rows, cols);
  if (st != SPHINX_OK) return st;
  if (q_bytes == nullptr || s_bytes == nullptr) return SPHINX_E_INVALID;
  *q_bytes = (size_t)rows * (size_t)q8_row_bytes(cols);
  *s_bytes = (size_t)rows * (size_t)q8_scale_bytes(cols);
  return SPHINX_OK;
}

sphinx_status sphinx_q8_quantise_workspace_bytes(int32_t rows, int32_t cols, size_t* bytes) {
  const sphinx_status st = q8_size_check(rows, cols);
  if (st != SPHINX_OK) return st;
  if (bytes == nullptr) return SPHINX_E_INVALID;
  *bytes = ((size_t)rows + 127) / 128 * (size_t)cols * 4;
  return SPHINX_OK;
}

sphinx_status sphinx_q8_quantise(sphinx_dtype dtype, const void* x, int64_t ldx, int32_t rows, int32_t cols,
                                 int32_t square, uint8_t* q, uint8_t* s, uint8_t* qt, uint8_t* st, float* sums,
                                 void* ws, size_t ws_bytes, void* stream) {
  if (!valid_dtype(dtype)) return SPHINX_E_UNSUPPORTED;
  sphinx_status r = q8_size_check(rows, cols);
  if (r == SPHINX_OK && qt != nullptr) r = q8_size_check(cols, rows);
  if (r != SPHINX_OK) return r;
  if (ldx < cols || (square != 0 && square != 1)) return SPHINX_E_INVALID;
  if (!aligned(x, 16) || !aligned(q, 16) || !aligned(s, 16) || !aligned(qt, 16) || !aligned(st, 16) ||
      !aligned(sums, 16) || !aligned(ws, 256))
    return SPHINX_E_INVALID;
  if ((q == nullptr && qt == nullptr && sums == nullptr) || (q != nullptr && s == nullptr) ||
      (qt != nullptr && st == nullptr))
    return cols == 0 || (rows == 0 && sums == nullptr) ? SPHINX_OK : SPHINX_E_INVALID;
  if (cols == 0 || (rows == 0 && sums == nullptr)) return SPHINX_OK;
  if (rows > 0 && x == nullptr) return SPHINX_E_INVALID;
  if (sums != nullptr) {
    const size_t need = ((size_t)rows + 127) / 128 * (size_t)cols * 4;
    if (need > 0 && ws == nullptr) return SPHINX_E_INVALID;
    if (ws_bytes < need) return SPHINX_E_WORKSPACE;
  }
  return hip_status(launch_q8_quantise(dtype, x, ldx, rows, cols, square != 0, q, s, qt, st, sums,
                                       static_cast<float*>(ws), (hipStream_t)stream));
}

sphinx_status sphinx_q8_matmul_workspace_bytes(sphinx_dtype odt, int32_t M, int32_t N, int32_t K, size_t* bytes) {
  if (!valid_dtype(odt)) return SPHINX_E_UNSUPPORTED;
  sphinx_status st = q8_size_check(M, K);
  if (st == SPHINX_OK) st = q8_size_check(N, K);
  if (st == SPHINX_OK) st = q8_outputs_check(M, N);
  if (st != SPHINX_OK) return st;
  if (bytes == nullptr) return SPHINX_E_INVALID;
  *bytes = M == 0 || N == 0 ? 0 : q8_matmul_ws_bytes(odt, M, N, K);
  return SPHINX_OK;
}

sphinx_status sphinx_q8_matmul(sphinx_dtype odt, int32_t M, int32_t N, int32_t K, const uint8_t* a, const uint8_t* sa,
                               const uint8_t* b, const uint8_t* sb, sphinx_dtype bdt, const void* bias,
                               sphinx_q8_epilogue epilogue, void* out, int64_t ldo, void* ws, size_t ws_bytes,
                               void* stream) {
  if (!valid_dtype(bdt)) return SPHINX_E_UNSUPPORTED;
  size_t need;
  const sphinx_status st = sphinx_q8_matmul_workspace_bytes(odt, M, N, K, &need);
  if (st != SPHINX_OK) return st;
  if (epilogue < SPHINX_Q8_STORE || epilogue > SPHINX_Q8_ADD || ldo < N) return SPHINX_E_INVALID;
  if (!aligned(a, 16) || !aligned(sa, 16) || !aligned(b, 16) || !aligned(sb, 16) || !aligned(bias, 16) ||
      !aligned(out, 16) || !aligned(ws, 256))
    return SPHINX_E_INVALID;
  if (M == 0 || N == 0) return SPHINX_OK;
  if (out == nullptr || (K > 0 && (!a || !sa || !b || !sb)) || (need > 0 && ws == nullptr)) return SPHINX_E_INVALID;
  if (ws_bytes < need) return SPHINX_E_WORKSPACE;
  const Q8Epi e{(int)epilogue, bias, bdt == SPHINX_BF16, out, ldo};
  return hip_status(launch_q8_matmul(odt == SPHINX_F32 ? kQ8F32 : kQ8Bf16, M, N, K, Q8Mat{a, sa}, Q8Mat{b, sb}, e, static_cast<float*>(ws),
                                     (hipStream_t)stream));
}

sphinx_status sphinx_q8_matmul_q8(int32_t M, int32_t N, int32_t K, const uint8_t* a, const uint8_t* sa,
                                  const uint8_t* b, const uint8_t* sb, sphinx_dtype bdt, const void* bias,
                                  sphinx_q8_epilogue epilogue, uint8_t* q, uint8_t* s, void* stream) {
  if (!valid_dtype(bdt)) return SPHINX_E_UNSUPPORTED;
  sphinx_status st = q8_size_check(M, K);
  if (st == SPHINX_OK) st = q8_size_check(N, K);
  if (st == SPHINX_OK) st = q8_size_check(M, N);
  if (st != SPHINX_OK) return st;
  if (epilogue != SPHINX_Q8_STORE && epilogue != SPHINX_Q8_GELU) return SPHINX_E_INVALID;
  if (!aligned(a, 16) || !aligned(sa, 16) || !aligned(b, 16) || !aligned(sb, 16) || !aligned(bias, 16) ||
      !aligned(q, 16) || !aligned(s, 16))
    return SPHINX_E_INVALID;
  if (M == 0 || N == 0) return SPHINX_OK;
  if (!q || !s || (K > 0 && (!a || !sa || !b || !sb))) return SPHINX_E_INVALID;
  Q8Epi e{(int)epilogue, bias, bdt == SPHINX_BF16, q, 0};
  e.scales = s;
  return hip_status(launch_q8_matmul(kQ8Bytes, M, N, K, Q8Mat{a, sa}, Q8Mat{b, sb}, e, nullptr, (hipStream_t)stream));
}

}  // extern "C"
