// Internal declarations of the 8-bit integer operators.  Not part of the C ABI.
#pragma once
#include "dit_internal.h"

namespace dit {

// Rows to codes: scale = max(max|row| / 127, 2^-126), code = value / scale to nearest even; columns d .. rup(d, 128) - 1 get code 0.
void launch_quantize_i8(hipStream_t s, const void* x, bool f32, int ldx, int M, int d, int8_t* codes, int ldq, float* scale);
// x_out (optional) = x + delta (delta optional); codes and scales of its RMS norm times gain
void launch_rmsnorm_i8(hipStream_t s, const float* x, int ldx, const void* delta, bool delta_f32, int ldd, const float* gain, float eps,
                       int M, int d, float* x_out, int ldo, int8_t* codes, int ldq, float* scale);

// One product of codes.  Columns from vt_from on leave transposed (vt[(n - vt_from) * ldvt + vt_col[m]], bf16), vt_from = N:
// none; vt_from is 0, N or a multiple of 256.  W2 != null: a gated pair, W the gate, N the columns of each.
struct GemmI8 {
  const int8_t* A; int lda; const float* sa;
  const int8_t* W; int ldw; const float* sw;
  const int8_t* W2; const float* sw2;
  const float* bias;
  int M, N, K, kind;                  // kind: OUT_BF16, OUT_F32, OUT_GELU_BF16, OUT_RESID_F32
  void* out; int ldc;
  const float* gate; int gate_stride; const int* row_req;
  bf16_t* vt; int ldvt; const int* vt_col; int vt_from;
  int* partial; size_t partial_bytes; // scratch for the sums of a product split along K, or null
  int tiles_m, tiles_n, splits;       // filled by the launcher
};
bool launch_gemm_i8(hipStream_t s, GemmI8& p);                  // false: its choice is no variant, and the result not all written
size_t gemm_i8_work_bytes(int M, int N, int K, bool pair);      // scratch of its choice
// its choice of tile with so much scratch (host only): the tile; out: shares of K (of the rest where there is one), columns of a first
// launch (0: one launch for all), and the tile of the rest
int gemm_i8_plan(int M, int N, int K, bool pair, size_t scratch, int (&out)[3]);
// a launch with a given tile and p.splits (false: no such variant)
bool launch_gemm_i8_variant(hipStream_t s, GemmI8& p, int variant);

}  // namespace dit
