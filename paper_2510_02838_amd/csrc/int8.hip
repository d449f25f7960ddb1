// Rows to 8-bit codes: the row quantiser and the RMS norm with the residual's addition.
//
//   scale = max(max|row| / 127, 2^-126),  code = rint(row / scale)
//   norm:   x' = x + delta,  row = x' / sqrt(mean(x'^2) + eps) * gain
//
// One pass: a row stays in registers between its reductions and its codes.  Up to 1024 columns a wave owns a row, above a
// workgroup does.  Bound: memory.
#include "int8_internal.h"

namespace dit {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

// maximum and sum over a wave, maxima of bit patterns: for values without a sign these order as the numbers do, with
// infinities and NaN on top, which a floating maximum would drop.
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) { const uint32_t w = __shfl_xor(v, o); v = w > v ? w : v; }
  return v;
}
__device__ __forceinline__ unsigned long long wave_max(unsigned long long v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) { const unsigned long long w = __shfl_xor(v, o); v = w > v ? w : v; }
  return v;
}
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}
// over the row's threads: one wave, or the workgroup's four through LDS
template <int T, class V>
__device__ __forceinline__ V row_max(V v, V* part) {
  v = wave_max(v);
  if constexpr (T == 256) {
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w) v = part[w] > v ? part[w] : v;
  }
  return v;
}

__device__ __forceinline__ float scale_of(float amax_over_127) { return fmaxf(amax_over_127, 0x1p-126f); }

// Four codes.  TIES: the quotient of two float32 numbers, times 1/scale in 64 bits, is off by at most 2^-45; a quotient that is no
// half-integer is at least 2^-25 from one, so rounding to multiples of 2^-38 first (adding and taking off 1.5 * 2^14)
// puts exact ties back on the half-integer and moves nothing else across one.
template <bool TIES>
__device__ __forceinline__ int code_of(double v, double inv) {
  double t = v * inv;
  if constexpr (TIES) {
    constexpr double GRID = 24576.0;
    t = (t + GRID) - GRID;
  }
  return (int)__builtin_rint(t);
}
__device__ __forceinline__ uint32_t pack4(int a, int b, int c, int d) {
  return (uint32_t)(a & 255) | (uint32_t)(b & 255) << 8 | (uint32_t)(c & 255) << 16 | (uint32_t)d << 24;
}
__device__ __forceinline__ float bf2f(uint32_t h) { return __uint_as_float(h << 16); }

// four columns from c on, those at or past d are 0 (rows start at multiples of 16 bytes, c is a multiple of 4)
__device__ __forceinline__ f32x4 load4(const float* p, int c, int d) {
  if (c + 4 <= d) return *(const f32x4*)(p + c);
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < 3; ++k)
    if (c + k < d) v[k] = p[c + k];
  return v;
}
__device__ __forceinline__ f32x4 load4(const bf16_t* p, int c, int d) {
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  if (c + 4 <= d) {
    const uint2 w = *(const uint2*)(p + c);
    v = f32x4{bf2f(w.x & 0xFFFF), bf2f(w.x >> 16), bf2f(w.y & 0xFFFF), bf2f(w.y >> 16)};
  } else {
#pragma unroll
    for (int k = 0; k < 3; ++k)
      if (c + k < d) v[k] = bf2f(p[c + k]);
  }
  return v;
}

}  // namespace

template <class X, int T, int V>
__global__ __launch_bounds__(256) void quantize_i8_kernel(const X* __restrict__ x, int ldx, int M, int d, int8_t* __restrict__ codes,
                                                          int ldq, float* __restrict__ scale) {
  __shared__ uint32_t part[4];
  const int row = blockIdx.x * (256 / T) + threadIdx.x / T, t = threadIdx.x % T;
  if (row >= M) return;                                // (a whole wave, and only where no barrier follows)
  const X* xr = x + (size_t)row * ldx;
  f32x4 v[V];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = load4(xr, (i * T + t) * 4, d);
#pragma unroll
  for (int i = 0; i < V; ++i)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t a = __float_as_uint(v[i][k]) & 0x7FFFFFFFu;
      m = a > m ? a : m;
    }
  m = row_max<T>(m, part);
  const bool bad = m >= 0x7F800000u;
  const float s = scale_of(__uint_as_float(m) / 127.0f);
  const double inv = bad ? 0.0 : 1.0 / (double)s;
  const int dq = (d + 127) & ~127;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int c = (i * T + t) * 4;
    if (c < dq) {
      const uint32_t w = bad ? 0u : pack4(code_of<true>(v[i][0], inv), code_of<true>(v[i][1], inv), code_of<true>(v[i][2], inv), code_of<true>(v[i][3], inv));
      *(uint32_t*)(codes + (size_t)row * ldq + c) = w;
    }
  }
  if (t == 0) scale[row] = bad ? __uint_as_float(0x7FC00000u) : s;
}

template <class D, int T, int V>
__global__ __launch_bounds__(256) void rmsnorm_i8_kernel(const float* x, int ldx, const D* delta, int ldd, const float* __restrict__ gain,
                                                         float eps, int M, int d, float* x_out, int ldo, int8_t* __restrict__ codes,
                                                         int ldq, float* __restrict__ scale) {
  __shared__ double part_q[4];
  __shared__ unsigned long long part_m[4];
  const int row = blockIdx.x * (256 / T) + threadIdx.x / T, t = threadIdx.x % T;
  if (row >= M) return;
  f32x4 v[V], g[V];
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = load4(x + (size_t)row * ldx, (i * T + t) * 4, d);
  if (delta) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const f32x4 e = load4(delta + (size_t)row * ldd, (i * T + t) * 4, d);
#pragma unroll
      for (int k = 0; k < 4; ++k) v[i][k] += e[k];
    }
  }
#pragma unroll
  for (int i = 0; i < V; ++i) g[i] = load4(gain, (i * T + t) * 4, d);
  if (x_out) {
    float* xo = x_out + (size_t)row * ldo;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int c = (i * T + t) * 4;
      if (c + 4 <= d) *(f32x4*)(xo + c) = v[i];
      else {
#pragma unroll
        for (int k = 0; k < 3; ++k)
          if (c + k < d) xo[c + k] = v[i][k];
      }
    }
  }
  double q = 0.0;
#pragma unroll
  for (int i = 0; i < V; ++i)
#pragma unroll
    for (int k = 0; k < 4; ++k) q = __builtin_fma((double)v[i][k], (double)v[i][k], q);
  q = wave_sum(q);
  if constexpr (T == 256) {
    if ((threadIdx.x & 63) == 0) part_q[threadIdx.x >> 6] = q;
    __syncthreads();
    q = (part_q[0] + part_q[1]) + (part_q[2] + part_q[3]);
  }
  const double r = 1.0 / __builtin_sqrt(q / (double)d + (double)eps);
  unsigned long long m = 0;
#pragma unroll
  for (int i = 0; i < V; ++i)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const double y = (double)v[i][k] * r * (double)g[i][k];
      const unsigned long long a = (unsigned long long)__double_as_longlong(y) & 0x7FFFFFFFFFFFFFFFull;
      m = a > m ? a : m;
    }
  m = row_max<T>(m, part_m);
  const float s = scale_of((float)(__longlong_as_double((long long)m) / 127.0));
  const bool bad = m >= 0x7FF0000000000000ull || !(s < __builtin_inff());      // (the second: a scale past float32)
  const double inv = r / (double)s;
  const int dq = (d + 127) & ~127;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int c = (i * T + t) * 4;
    if (c < dq) {
      int e[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) e[k] = bad ? 0 : code_of<false>((double)v[i][k] * (double)g[i][k], inv);
      *(uint32_t*)(codes + (size_t)row * ldq + c) = pack4(e[0], e[1], e[2], e[3]);
    }
  }
  if (t == 0) scale[row] = bad ? __uint_as_float(0x7FC00000u) : s;
}

template <class X, int T, int V>
static void launch_quantize_t(hipStream_t s, const void* x, int ldx, int M, int d, int8_t* codes, int ldq, float* scale) {
  hipLaunchKernelGGL((quantize_i8_kernel<X, T, V>), dim3((M + 256 / T - 1) / (256 / T)), dim3(256), 0, s, (const X*)x, ldx, M, d, codes, ldq, scale);
}
template <class X>
static void launch_quantize_x(hipStream_t s, const void* x, int ldx, int M, int d, int8_t* codes, int ldq, float* scale) {
  if (d <= 256) launch_quantize_t<X, 64, 1>(s, x, ldx, M, d, codes, ldq, scale);
  else if (d <= 1024) launch_quantize_t<X, 64, 4>(s, x, ldx, M, d, codes, ldq, scale);
  else if (d <= 2048) launch_quantize_t<X, 256, 2>(s, x, ldx, M, d, codes, ldq, scale);
  else if (d <= 4096) launch_quantize_t<X, 256, 4>(s, x, ldx, M, d, codes, ldq, scale);
  else if (d <= 8192) launch_quantize_t<X, 256, 8>(s, x, ldx, M, d, codes, ldq, scale);
  else launch_quantize_t<X, 256, 16>(s, x, ldx, M, d, codes, ldq, scale);
}
void launch_quantize_i8(hipStream_t s, const void* x, bool f32, int ldx, int M, int d, int8_t* codes, int ldq, float* scale) {
  if (M == 0) return;
  if (f32) launch_quantize_x<float>(s, x, ldx, M, d, codes, ldq, scale);
  else launch_quantize_x<bf16_t>(s, x, ldx, M, d, codes, ldq, scale);
}

template <class D, int T, int V>
static void launch_rmsnorm_t(hipStream_t s, const float* x, int ldx, const void* delta, int ldd, const float* gain, float eps, int M, int d,
                             float* x_out, int ldo, int8_t* codes, int ldq, float* scale) {
  hipLaunchKernelGGL((rmsnorm_i8_kernel<D, T, V>), dim3((M + 256 / T - 1) / (256 / T)), dim3(256), 0, s, x, ldx, (const D*)delta, ldd, gain, eps,
                     M, d, x_out, ldo, codes, ldq, scale);
}
template <class D>
static void launch_rmsnorm_d(hipStream_t s, const float* x, int ldx, const void* delta, int ldd, const float* gain, float eps, int M, int d,
                             float* x_out, int ldo, int8_t* codes, int ldq, float* scale) {
  if (d <= 256) launch_rmsnorm_t<D, 64, 1>(s, x, ldx, delta, ldd, gain, eps, M, d, x_out, ldo, codes, ldq, scale);
  else if (d <= 1024) launch_rmsnorm_t<D, 64, 4>(s, x, ldx, delta, ldd, gain, eps, M, d, x_out, ldo, codes, ldq, scale);
  else if (d <= 2048) launch_rmsnorm_t<D, 256, 2>(s, x, ldx, delta, ldd, gain, eps, M, d, x_out, ldo, codes, ldq, scale);
  else if (d <= 4096) launch_rmsnorm_t<D, 256, 4>(s, x, ldx, delta, ldd, gain, eps, M, d, x_out, ldo, codes, ldq, scale);
  else if (d <= 8192) launch_rmsnorm_t<D, 256, 8>(s, x, ldx, delta, ldd, gain, eps, M, d, x_out, ldo, codes, ldq, scale);
  else launch_rmsnorm_t<D, 256, 16>(s, x, ldx, delta, ldd, gain, eps, M, d, x_out, ldo, codes, ldq, scale);
}
void launch_rmsnorm_i8(hipStream_t s, const float* x, int ldx, const void* delta, bool delta_f32, int ldd, const float* gain, float eps,
                       int M, int d, float* x_out, int ldo, int8_t* codes, int ldq, float* scale) {
  if (M == 0) return;
  if (delta_f32) launch_rmsnorm_d<float>(s, x, ldx, delta, ldd, gain, eps, M, d, x_out, ldo, codes, ldq, scale);
  else launch_rmsnorm_d<bf16_t>(s, x, ldx, delta, ldd, gain, eps, M, d, x_out, ldo, codes, ldq, scale);
}

}  // namespace dit
