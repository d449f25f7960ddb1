// Entry points of the 8-bit integer operators: checks of the arguments and the launches.
#include "../../include/int8.h"
#include "int8_internal.h"

using namespace dit;

namespace {
inline bool off16(const void* p) { return ((uintptr_t)p & 15) != 0; }
inline bool off4(const void* p) { return ((uintptr_t)p & 3) != 0; }
inline int rup128(int n) { return (n + 127) / 128 * 128; }
inline dit_status launched() { return hipGetLastError() == hipSuccess ? DIT_OK : DIT_EDEVICE; }

// (tiles and shares are counted in 32 bits)
inline bool countable(int M, int N) { return M <= (1 << 30) && N <= (1 << 30) && (M + 127LL) / 128 * ((N + 15LL) / 16) < (1LL << 26); }

// (a tile's results are stored at 32-bit byte offsets from its first row: up to 15 rows of bf16 or 7 of float32)
constexpr int MAX_LDC = 1 << 26;

// what the three forms of the product have in common
dit_status check_product(const void* A, int lda, const float* a_scale, const void* W, int ldw, const float* w_scale, int M, int N, int K,
                         const void* out, const void* work) {
  if (!A || !a_scale || !W || !w_scale || !out) return DIT_EINVAL;
  if (M < 0 || N < 0 || K <= 0 || K % 128 || K > DIT_I8_MAX_K || lda < K || ldw < K || lda % 16 || ldw % 16) return DIT_ESHAPE;
  if (lda >= (1 << 22) || ldw >= (1 << 22)) return DIT_ESHAPE;                       // 32-bit offsets inside a tile
  if (!countable(M, N)) return DIT_ESHAPE;
  if (off16(A) || off16(W) || off16(out) || off16(work) || off4(a_scale) || off4(w_scale)) return DIT_ESHAPE;
  return DIT_OK;
}

GemmI8 product(const void* A, int lda, const float* a_scale, const void* W, int ldw, const float* w_scale, const float* bias, int M, int N,
               int K, int kind, void* out, int ldc, void* work, size_t work_bytes) {
  GemmI8 p = {};
  p.A = (const int8_t*)A; p.lda = lda; p.sa = a_scale;
  p.W = (const int8_t*)W; p.ldw = ldw; p.sw = w_scale; p.bias = bias;
  p.M = M; p.N = N; p.K = K; p.kind = kind; p.out = out; p.ldc = ldc; p.vt_from = N;
  p.partial = (int*)work; p.partial_bytes = work ? work_bytes : 0;
  return p;
}
}  // namespace

extern "C" {

dit_status dit_op_quantize_i8(void* stream, const void* x, int x_kind, int ldx, int M, int d, void* codes, int ldq, float* scale) {
  if (!x || !codes || !scale || (x_kind != DIT_X_BF16 && x_kind != DIT_X_F32)) return DIT_EINVAL;
  if (M < 0 || M > DIT_I8_MAX_ROWS || d < 1 || d > DIT_I8_MAX_ROW || ldx < d || ldx % (x_kind == DIT_X_F32 ? 4 : 8) || ldq < rup128(d) || ldq % 16) return DIT_ESHAPE;
  if (off16(x) || off16(codes) || off4(scale)) return DIT_ESHAPE;
  if (M == 0) return DIT_OK;
  launch_quantize_i8((hipStream_t)stream, x, x_kind == DIT_X_F32, ldx, M, d, (int8_t*)codes, ldq, scale);
  return launched();
}

dit_status dit_op_rmsnorm_i8(void* stream, const float* x, int ldx, const void* delta, int delta_kind, int ldd, const float* gain,
                             float eps, int M, int d, float* x_out, int ldo, void* codes, int ldq, float* scale) {
  if (!x || !gain || !codes || !scale) return DIT_EINVAL;
  if (delta && delta_kind != DIT_X_BF16 && delta_kind != DIT_X_F32) return DIT_EINVAL;
  if (!(eps > 0.f) || eps > 1e30f) return DIT_EINVAL;
  if (M < 0 || M > DIT_I8_MAX_ROWS || d < 1 || d > DIT_I8_MAX_ROW || ldx < d || ldx % 4 || ldq < rup128(d) || ldq % 16) return DIT_ESHAPE;
  if (delta && (ldd < d || ldd % (delta_kind == DIT_X_F32 ? 4 : 8) || off16(delta))) return DIT_ESHAPE;
  if (x_out && (ldo < d || ldo % 4 || off16(x_out) || (x_out == x && ldo != ldx))) return DIT_ESHAPE;
  if (off16(x) || off16(codes) || off16(gain) || off4(scale)) return DIT_ESHAPE;
  if (M == 0) return DIT_OK;
  launch_rmsnorm_i8((hipStream_t)stream, x, ldx, delta, delta_kind == DIT_X_F32, ldd, gain, eps, M, d, x_out, ldo, (int8_t*)codes, ldq, scale);
  return launched();
}

dit_status dit_op_gemm_i8(void* stream, const void* A, int lda, const float* a_scale, const void* W, int ldw, const float* w_scale,
                          const float* bias, int M, int N, int K, int out_kind, void* out, int ldc, const float* gate,
                          int gate_stride, const int* row_req, void* work, size_t work_bytes) {
  const dit_status st = check_product(A, lda, a_scale, W, ldw, w_scale, M, N, K, out, work);
  if (st != DIT_OK) return st;
  if (out_kind < OUT_BF16 || out_kind > OUT_RESID_F32) return DIT_EINVAL;
  if (ldc < N || ldc >= MAX_LDC || ldc % (out_kind == OUT_F32 || out_kind == OUT_RESID_F32 ? 4 : 8) || off4(bias)) return DIT_ESHAPE;
  if (out_kind == OUT_RESID_F32 && (off4(gate) || off4(row_req))) return DIT_ESHAPE;
  if (M == 0 || N == 0) return DIT_OK;
  GemmI8 p = product(A, lda, a_scale, W, ldw, w_scale, bias, M, N, K, out_kind, out, ldc, work, work_bytes);
  if (out_kind == OUT_RESID_F32) { p.gate = gate; p.gate_stride = gate_stride; p.row_req = row_req; }
  return launch_gemm_i8((hipStream_t)stream, p) ? launched() : DIT_ESHAPE;
}

dit_status dit_op_gemm_i8_geglu(void* stream, const void* A, int lda, const float* a_scale, const void* W_gate, const float* gate_scale,
                                const void* W_up, const float* up_scale, int ldw, int M, int N, int K, void* out, int ldc,
                                void* work, size_t work_bytes) {
  const dit_status st = check_product(A, lda, a_scale, W_gate, ldw, gate_scale, M, N, K, out, work);
  if (st != DIT_OK) return st;
  if (!W_up || !up_scale) return DIT_EINVAL;
  if (ldc < N || ldc >= MAX_LDC || ldc % 8 || off16(W_up) || off4(up_scale)) return DIT_ESHAPE;
  if (M == 0 || N == 0) return DIT_OK;
  GemmI8 p = product(A, lda, a_scale, W_gate, ldw, gate_scale, nullptr, M, N, K, OUT_BF16, out, ldc, work, work_bytes);
  p.W2 = (const int8_t*)W_up; p.sw2 = up_scale;
  return launch_gemm_i8((hipStream_t)stream, p) ? launched() : DIT_ESHAPE;
}

dit_status dit_op_gemm_i8_transposed(void* stream, const void* A, int lda, const float* a_scale, const void* W, int ldw,
                                     const float* w_scale, const float* bias, int M, int N, int K, void* out, int ldo,
                                     const int* col, void* work, size_t work_bytes) {
  const dit_status st = check_product(A, lda, a_scale, W, ldw, w_scale, M, N, K, out, work);
  if (st != DIT_OK) return st;
  if (!col) return DIT_EINVAL;
  if (ldo < M || ldo % 8 || off4(bias) || off4(col)) return DIT_ESHAPE;
  if (M == 0 || N == 0) return DIT_OK;
  GemmI8 p = product(A, lda, a_scale, W, ldw, w_scale, bias, M, N, K, OUT_BF16, nullptr, 0, work, work_bytes);
  p.vt = (bf16_t*)out; p.ldvt = ldo; p.vt_col = col; p.vt_from = 0;
  return launch_gemm_i8((hipStream_t)stream, p) ? launched() : DIT_ESHAPE;
}

static bool sizes_ok(int M, int N, int K) { return M > 0 && N > 0 && K > 0 && K % 128 == 0 && K <= DIT_I8_MAX_K && countable(M, N); }

size_t dit_op_gemm_i8_work_bytes(int M, int N, int K, int pair) { return sizes_ok(M, N, K) ? gemm_i8_work_bytes(M, N, K, pair != 0) : 0; }

int dit_op_gemm_i8_tile(int M, int N, int K, int pair, size_t work_bytes, int* plan) {
  if (!sizes_ok(M, N, K)) return -1;
  int p[3];
  const int tile = gemm_i8_plan(M, N, K, pair != 0, work_bytes, p);
  for (int i = 0; plan && i < 3; ++i) plan[i] = p[i];
  return tile;
}

}  // extern "C"
