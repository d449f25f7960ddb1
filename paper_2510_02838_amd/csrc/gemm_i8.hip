// Product of 8-bit codes on the gfx950 matrix cores:  C[m][n] = sa[m] sw[n] sum_k A[m][k] W[n][k]  (+ epilogue).
//
// The sum is held in 32-bit integers, exact for K < 2^17, so no way of cutting the product up changes a bit of the result; the
// epilogue's float arithmetic is written with explicit fused operations, the same in every kernel.
#include "int8_internal.h"

namespace dit {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

namespace {

__device__ __forceinline__ uint16_t bf(float f) {
  uint32_t u = __float_as_uint(f);
  if ((u & 0x7FFFFFFFu) > 0x7F800000u) return 0x7FC0;    // (rounding would carry some NaN over to -0)
  u += 0x7FFFu + ((u >> 16) & 1u);
  return (uint16_t)(u >> 16);
}
// 0.5 x (1 + tanh(u)) = x / (1 + 2^(-2 log2(e) u)), u = sqrt(2/pi) (x + 0.044715 x^3)
__device__ __forceinline__ float gelu(float x) {
  const float t = x * __builtin_fmaf(0.035677408136300125f * x, x, 0.7978845608028654f);
  const float e = __builtin_amdgcn_exp2f(-2.8853900817779268f * t);
  return x * __builtin_amdgcn_rcpf(1.0f + e);
}
__device__ __forceinline__ float value(int acc, float sa, float sw, float bias) { return __builtin_fmaf((float)acc, sa * sw, bias); }

// one result to its place
__device__ __forceinline__ void put(const GemmI8& P, int m, int n, int acc) {
  if (m >= P.M || n >= P.N) return;
  float v = value(acc, P.sa[m], P.sw[n], P.bias ? P.bias[n] : 0.f);
  if (n >= P.vt_from) { P.vt[(size_t)(n - P.vt_from) * P.ldvt + P.vt_col[m]] = bf(v); return; }
  const size_t o = (size_t)m * P.ldc + n;
  if (P.kind == OUT_F32) ((float*)P.out)[o] = v;
  else if (P.kind == OUT_RESID_F32) {
    const float g = P.gate ? P.gate[(size_t)(P.row_req ? P.row_req[m] : 0) * P.gate_stride + n] : 1.f;
    ((float*)P.out)[o] = __builtin_fmaf(g, v, ((float*)P.out)[o]);
  } else ((bf16_t*)P.out)[o] = bf(P.kind == OUT_GELU_BF16 ? gelu(v) : v);
}
__device__ __forceinline__ void put_pair(const GemmI8& P, int m, int n, int gate, int up) {
  if (m >= P.M || n >= P.N) return;
  const float sa = P.sa[m];
  ((bf16_t*)P.out)[(size_t)m * P.ldc + n] = bf(gelu(value(gate, sa, P.sw[n], 0.f)) * value(up, sa, P.sw2[n], 0.f));
}

}  // namespace

// 64x64 tile, 4 waves of 32x32, operand fragments straight from memory: lane l holds 16 codes of row l % 16 from k = 16 (l / 16) on.
template <bool PAIR>
__global__ __launch_bounds__(256) void gemm_i8_simple_kernel(const GemmI8 P) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, kq = lane >> 4;
  const int m0 = blockIdx.y * 64 + (wave >> 1) * 32, n0 = blockIdx.x * 64 + (wave & 1) * 32;
  i32x4 acc[2][2] = {}, acc2[2][2] = {};
  const int8_t *a[2], *b[2], *b2[2];
  for (int i = 0; i < 2; ++i) {
    const int m = m0 + i * 16 + l16, n = n0 + i * 16 + l16;     // rows past the end repeat the last one and are not stored
    a[i] = P.A + (size_t)(m < P.M ? m : P.M - 1) * P.lda + kq * 16;
    b[i] = P.W + (size_t)(n < P.N ? n : P.N - 1) * P.ldw + kq * 16;
    b2[i] = PAIR ? P.W2 + (size_t)(n < P.N ? n : P.N - 1) * P.ldw + kq * 16 : b[i];
  }
  for (int k = 0; k < P.K; k += 64) {
    i32x4 fa[2], fb[2], fc[2];
    for (int i = 0; i < 2; ++i) {
      fa[i] = *(const i32x4*)(a[i] + k);
      fb[i] = *(const i32x4*)(b[i] + k);
      if (PAIR) fc[i] = *(const i32x4*)(b2[i] + k);
    }
    for (int i = 0; i < 2; ++i)
      for (int j = 0; j < 2; ++j) {
        acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fa[i], fb[j], acc[i][j], 0, 0, 0);
        if (PAIR) acc2[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fa[i], fc[j], acc2[i][j], 0, 0, 0);
      }
  }
  for (int i = 0; i < 2; ++i)
    for (int j = 0; j < 2; ++j)
      for (int e = 0; e < 4; ++e) {
        const int m = m0 + i * 16 + kq * 4 + e, n = n0 + j * 16 + l16;
        if (PAIR) put_pair(P, m, n, acc[i][j][e], acc2[i][j][e]);
        else put(P, m, n, acc[i][j][e]);
      }
}

size_t gemm_i8_work_bytes(int, int, int, bool) { return 0; }

void launch_gemm_i8(hipStream_t s, GemmI8& p) {
  const dim3 grid((p.N + 63) / 64, (p.M + 63) / 64);
  if (p.W2) hipLaunchKernelGGL(gemm_i8_simple_kernel<true>, grid, dim3(256), 0, s, p);
  else hipLaunchKernelGGL(gemm_i8_simple_kernel<false>, grid, dim3(256), 0, s, p);
}

}  // namespace dit
