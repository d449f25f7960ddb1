/* C ABI of the 8-bit integer operators, and of the Encode stage that runs its products on them.
 *
 * A tensor in 8 bits is a matrix of codes, dev int8, with a float32 scale per row: code c of row r stands for
 * c * scale[r].  Rows are tokens (activations) or output channels (weights, stored [out][in] as everywhere in this
 * library), so that a product of the two needs one factor per result.  Codes lie in -127 .. 127:
 *     scale = max(max|row| / 127, 2^-126)     (float32, rounded to nearest)
 *     code  = value / scale                   (rounded to nearest, ties to even, of the exact quotient)
 * A row of zeros has codes 0.  A row that holds an infinity or a NaN has codes 0 and the scale NaN: what is computed
 * from it is NaN, and other rows are not touched.
 *
 * Conventions are those of dit.h: status codes, caller-owned device buffers, nothing allocated, arguments
 * checked before anything is launched, launches only (no copies, no waiting: every dit_op_* call here may be captured into a HIP
 * graph), on `stream` (NULL = default stream) of the current device.  Buffers and matrix rows start at multiples of 16 bytes
 * (scales, gains, biases, gates and maps: at their element's size).  Buffers of one call do not overlap unless it says so.
 */
#ifndef DIT_INT8_H
#define DIT_INT8_H

#include "encoder.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { DIT_X_BF16 = 0, DIT_X_F32 = 1 };
enum { DIT_I8_MAX_ROW = 16384, /* columns of a row that gets codes */
       DIT_I8_MAX_ROWS = 1 << 23, /* rows of one such call */
       DIT_I8_MAX_K = 131072 - 128 /* K of a product: its sums stay inside 32 bits */ };

/* Codes and scales of the rows of x [M][ldx], d columns each (1..DIT_I8_MAX_ROW, any number), x_kind DIT_X_*.
 * codes: [M][ldq], ldq at least d rounded up to 128: the columns from d to there are set to 0, which makes the row an
 * operand of a product with K = d rounded up to 128. */
dit_status dit_op_quantize_i8(void* stream, const void* x, int x_kind, int ldx, int M, int d, void* codes, int ldq, float* scale);

/* RMS norm with the residual's addition, leaving codes:
 *     x' = x + delta;   y = x' / sqrt(mean(x'^2) + eps) * gain;   codes and scales of the rows y (never rounded before).
 * x: dev float32 [M][ldx]; delta: [M][ldd], delta_kind DIT_X_*, NULL = none; x_out: dev float32 [M][ldo] receives x', may be x
 * itself (with ldo == ldx) or NULL; gain: dev float32 [d], 16-byte aligned; 0 < eps <= 1e30; codes and columns past d as above.  Everything behind x' is held
 * in 64 bits: a scale is the formula's or, where that lies within 2^-46 of itself of the middle of two float32 numbers, its neighbour, and a code is off by
 * one at most where the quotient lies within 2^-39 of the border of two.  A row gets the same codes and scale, bit for bit, among any others. */
dit_status dit_op_rmsnorm_i8(void* stream, const float* x, int ldx, const void* delta, int delta_kind, int ldd, const float* gain,
                             float eps, int M, int d, float* x_out, int ldo, void* codes, int ldq, float* scale);

/* C[m][n] = a_scale[m] * w_scale[n] * sum_k A[m][k] W[n][k] (+ bias[n]) on the 8-bit matrix cores; the sum is exact.
 * A: codes [M][lda]; W: codes [N][ldw] (no padding rows needed); a_scale: dev float32 [M]; w_scale: dev float32 [N]; bias: dev float32
 * [N] or NULL; K a multiple of 128, at most DIT_I8_MAX_K; lda, ldw multiples of 16 below 2^22; ldc below 2^26.  out_kind, out, ldc, gate, gate_stride and row_req
 * as for dit_op_gemm (0 bf16, 1 float32, 2 bf16 of tanh-GELU, 3 float32 out += gate * C); any code -128..127 is
 * taken.  Scales are at least 2^-126; a result may be any float32 number, whatever the product of its scales is alone.  (Save beside rows with an a_scale
 * above 2^96: rows with one below 2^-94 may lose digits there, and the other rows' results of columns with a w_scale above 2^96 be too small.)  The result does not depend on how the product is cut up: it is the same, bit for bit, alone or among other rows.
 * work: dev scratch for the shares of a product that is split along K between workgroups (dit_op_gemm_i8_work_bytes says how much the
 * library's choice takes, for most sizes nothing); with NULL or less another tile is taken.  Its contents carry nothing between
 * calls; calls that may overlap need one each. */
dit_status dit_op_gemm_i8(void* stream, const void* A, int lda, const float* a_scale, const void* W, int ldw, const float* w_scale,
                          const float* bias, int M, int N, int K, int out_kind, void* out, int ldc, const float* gate,
                          int gate_stride, const int* row_req, void* work, size_t work_bytes);

/* bf16 of tanh-GELU(product with W_gate) * (product with W_up), both [N][ldw]; ldc below 2^26. */
dit_status dit_op_gemm_i8_geglu(void* stream, const void* A, int lda, const float* a_scale, const void* W_gate, const float* gate_scale,
                                const void* W_up, const float* up_scale, int ldw, int M, int N, int K, void* out, int ldc,
                                void* work, size_t work_bytes);

/* bf16 of the product (+ bias), element (m, n) to out[n*ldo + col[m]]; col: dev int32 [M], every one above the one before, below ldo; columns that no
 * row maps to are left alone. */
dit_status dit_op_gemm_i8_transposed(void* stream, const void* A, int lda, const float* a_scale, const void* W, int ldw,
                                     const float* w_scale, const float* bias, int M, int N, int K, void* out, int ldo,
                                     const int* col, void* work, size_t work_bytes);

/* Scratch that the library's choice for a product uses (pair != 0: dit_op_gemm_i8_geglu), and the tile that it takes given so much:
 * 100 * row tiles + column tiles, of 16, of a workgroup whose waves share K, or rows * 1000 + columns of an 8-wave one.  plan (may be
 * NULL) receives three numbers: the shares of K, where there are two launches those of the second (the first has none); the columns that a first
 * launch takes where the rest has a tile of its own, else 0; that tile.  Host only; 0 and -1 for sizes that the products refuse. */
size_t dit_op_gemm_i8_work_bytes(int M, int N, int K, int pair);
int dit_op_gemm_i8_tile(int M, int N, int K, int pair, size_t work_bytes, int* plan);

/* ---- the Encode stage in 8 bits ------------------------------------------------------- */

/* enc_forward (encoder.h) with its matrix products on codes: weights with a scale per output channel, their inputs with one per token.
 * The residual stream is float32 as there; the statistics of the layers' norms are held in 64 bits, of the final one in float32; attention runs on
 * bf16; a branch is rounded to bf16 before the next norm adds it to the stream (the last one is added in float32), where enc_forward adds float32 sums.
 *
 * enc_i8_quantize writes the codes of every matrix of the bound weight arena to dev_codes (256-byte aligned, enc_i8_weight_bytes), which the
 * context refers to from then on.  The codes come on top of the arena, which stays bound and in use (embedding, bias table, gains): this form
 * reads half the bytes a pass and holds half as many again.  It has to be called again after
 * enc_init_weights, enc_set_tensor of a matrix and a bind of another arena, after which enc_i8_forward refuses with DIT_EINVAL, and after the
 * arena has been written by other means.
 * DIT_EUNSUPPORTED for matrices with more than DIT_I8_MAX_ROW inputs.
 * enc_i8_forward: arguments, results and streams of enc_forward; the workspace bound with enc_bind must have
 * enc_i8_workspace_bytes.  Capture points: those of enc_set_tap but "l<i>.ln1", which is never reached.
 * A sequence's result is the same, bit for bit, whatever it is packed with. */
size_t enc_i8_weight_bytes(const enc_ctx* ctx);
size_t enc_i8_workspace_bytes(const enc_ctx* ctx, int n_seq, const int* lens);
dit_status enc_i8_quantize(enc_ctx* ctx, void* dev_codes, size_t bytes);
dit_status enc_i8_forward(enc_ctx* ctx, int n_seq, const int* lens, const int* dev_tokens, void* dev_out_bf16, float* dev_out_f32);

#ifdef __cplusplus
}
#endif
#endif
