// Rows to 8-bit codes: the row quantiser and the RMS norm with the residual's addition.
//
//   scale = max(max|row| / 127, 2^-126),  code = rint(row / scale)
//   norm:   x' = x + delta,  row = x' / sqrt(mean(x'^2) + eps) * gain
//
// One pass: a row stays in registers between its reductions and its codes.  Up to 1024 columns a wave owns a row, above a
// workgroup does.  Bound: memory: 32000 x 10240 bf16 to codes 197 us (5.0 TB/s), 32000 x 4096 norm with a bf16 branch 263 us (5.5; a 4 GiB
// copy reaches 4.8); a launch for few rows: 32 x 4096 norm 4.6 us (with two reductions behind each other and LDS permutations 0.3 more).
#include "int8_internal.h"

namespace dit {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

// Sums and maxima over a wave and a row's threads.  Lane exchanges inside 16 lanes as DPP operands, across them as lane swaps: a
// chain of six LDS permutations would be longer than the rest of a short call.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, CTRL, 15, 15, true); }
template <int CTRL, class V>
__device__ __forceinline__ V moved(V v) {
  union { V v; uint32_t w[sizeof(V) / 4]; } u = {v};
#pragma unroll
  for (unsigned i = 0; i < sizeof(V) / 4; ++i) u.w[i] = dpp<CTRL>(u.w[i]);
  return u.v;
}
// op(lanes, lanes 16 or 32 away)
template <bool HALF, class V, class OP>
__device__ __forceinline__ V across(V v, OP op) {
  union { V v; uint32_t w[sizeof(V) / 4]; } u = {v}, a, b;
#pragma unroll
  for (unsigned i = 0; i < sizeof(V) / 4; ++i) {
    const auto r = HALF ? __builtin_amdgcn_permlane32_swap(u.w[i], u.w[i], false, false) : __builtin_amdgcn_permlane16_swap(u.w[i], u.w[i], false, false);
    a.w[i] = r[0]; b.w[i] = r[1];
  }
  return op(a.v, b.v);
}
template <class V, class OP>
__device__ __forceinline__ V over_wave(V v, OP op) {
  v = op(v, moved<0xB1>(v));           // lanes 1 apart, 2 apart, mirrored in 8, mirrored in 16
  v = op(v, moved<0x4E>(v));
  v = op(v, moved<0x141>(v));
  v = op(v, moved<0x140>(v));
  v = across<false>(v, op);
  return across<true>(v, op);
}
// Maxima are of bit patterns: for values without a sign these order as the numbers do, with infinities and NaN on top, which a
// floating maximum would drop.
struct Max { template <class V> __device__ __forceinline__ V operator()(V a, V b) const { return a > b ? a : b; } };
struct Add { template <class V> __device__ __forceinline__ V operator()(V a, V b) const { return a + b; } };

// 1 / v to about 2^-50 for a normal v (two Newton steps on the hardware's estimate)
__device__ __forceinline__ double reciprocal(double v) {
  double r = __builtin_amdgcn_rcp(v);
  r = __builtin_fma(__builtin_fma(-v, r, 1.0), r, r);
  return __builtin_fma(__builtin_fma(-v, r, 1.0), r, r);
}
__device__ __forceinline__ double inverse_root(double v) {
  double r = __builtin_amdgcn_rsq(v);
#pragma unroll
  for (int i = 0; i < 2; ++i) r = __builtin_fma(__builtin_fma(-v * r, r, 1.0), 0.5 * r, r);
  return r;
}

// max|row| / 127 as float32.  The product in 64 bits is off by 2^-52 of it; where max|row| is a float32 number the quotient is at least
// 2^-33 of itself from the middle of two float32 numbers, so the rounding is that of the exact quotient.
__device__ __forceinline__ float scale_of(double amax) { return fmaxf((float)(amax * (1.0 / 127.0)), 0x1p-126f); }

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

// E columns from c on, those at or past d are 0 (rows start at multiples of 16 bytes, c is a multiple of E)
template <int E>
__device__ __forceinline__ void load_cols(const float* p, int c, int d, float (&v)[E]) {
  static_assert(E == 4, "16 bytes");
  if (c + 4 <= d) {
    const f32x4 w = *(const f32x4*)(p + c);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = w[k];
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = c + k < d ? p[c + k] : 0.f;
  }
}
template <int E>
__device__ __forceinline__ void load_cols(const bf16_t* p, int c, int d, float (&v)[E]) {
  if (c + E <= d) {
    uint32_t w[E / 2];
    if constexpr (E == 8) *(uint4*)w = *(const uint4*)(p + c);
    else *(uint2*)w = *(const uint2*)(p + c);
#pragma unroll
    for (int k = 0; k < E; ++k) v[k] = __uint_as_float(k & 1 ? w[k >> 1] & 0xFFFF0000u : w[k >> 1] << 16);
  } else {
#pragma unroll
    for (int k = 0; k < E; ++k) v[k] = c + k < d ? bf2f(p[c + k]) : 0.f;
  }
}

constexpr uint32_t NAN32 = 0x7FC00000u;

}  // namespace

// Rows of up to 1024 columns belong to a wave (T = 64), longer ones to a workgroup (T = 256); V pieces of E columns a thread.
template <class X, int E, int T, int V>
__global__ __launch_bounds__(256) void quantize_i8_kernel(const X* __restrict__ x, int ldx, int M, int d, int8_t* __restrict__ codes,
                                                          int ldq, float* __restrict__ scale) {
  __shared__ uint32_t part[4];
  const int row = blockIdx.x * (256 / T) + threadIdx.x / T, t = threadIdx.x % T;
  if (row >= M) return;                                // (a whole wave, and only where no barrier follows)
  const X* xr = x + (size_t)row * ldx;
  float v[V][E];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < V; ++i) load_cols<E>(xr, (i * T + t) * E, d, v[i]);
#pragma unroll
  for (int i = 0; i < V; ++i)
#pragma unroll
    for (int k = 0; k < E; ++k) m = Max{}(m, __float_as_uint(v[i][k]) & 0x7FFFFFFFu);
  m = over_wave(m, Max{});
  if constexpr (T == 256) {
    if ((t & 63) == 0) part[t >> 6] = m;
    __syncthreads();
    m = Max{}(Max{}(part[0], part[1]), Max{}(part[2], part[3]));
  }
  const bool bad = m >= 0x7F800000u;
  const float s = scale_of((double)__uint_as_float(m));
  const double inv = reciprocal((double)s);
  const int dq = (d + 127) & ~127;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int c = (i * T + t) * E;
    if (c < dq) {
      uint32_t w[E / 4];
#pragma unroll
      for (int k = 0; k < E / 4; ++k)
        w[k] = bad ? 0u : pack4(code_of<true>(v[i][4 * k], inv), code_of<true>(v[i][4 * k + 1], inv), code_of<true>(v[i][4 * k + 2], inv), code_of<true>(v[i][4 * k + 3], inv));
      if constexpr (E == 8) *(uint2*)(codes + (size_t)row * ldq + c) = make_uint2(w[0], w[1]);
      else *(uint32_t*)(codes + (size_t)row * ldq + c) = w[0];
    }
  }
  if (t == 0) scale[row] = bad ? __uint_as_float(NAN32) : s;
}

// Both reductions at once: the largest |y| is r times the largest |x' gain|, a product that 64 bits hold exactly.
template <class D, int T, int V>
__global__ __launch_bounds__(256) void rmsnorm_i8_kernel(const float* x, int ldx, const D* delta, int ldd, const float* __restrict__ gain,
                                                         float eps, double inv_d, int M, int d, float* x_out, int ldo,
                                                         int8_t* __restrict__ codes, int ldq, float* __restrict__ scale) {
  __shared__ double part_q[4];
  __shared__ unsigned long long part_m[4];
  const int row = blockIdx.x * (256 / T) + threadIdx.x / T, t = threadIdx.x % T;
  if (row >= M) return;
  float v[V][4], g[V][4];
#pragma unroll
  for (int i = 0; i < V; ++i) load_cols<4>(x + (size_t)row * ldx, (i * T + t) * 4, d, v[i]);
  if (delta) {
    float e[V][4];
#pragma unroll
    for (int i = 0; i < V; ++i) load_cols<4>(delta + (size_t)row * ldd, (i * T + t) * 4, d, e[i]);
#pragma unroll
    for (int i = 0; i < V; ++i) load_cols<4>(gain, (i * T + t) * 4, d, g[i]);
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) v[i][k] += e[i][k];
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) load_cols<4>(gain, (i * T + t) * 4, d, g[i]);
  }
  if (x_out) {
    float* xo = x_out + (size_t)row * ldo;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int c = (i * T + t) * 4;
      if (c + 4 <= d) *(f32x4*)(xo + c) = f32x4{v[i][0], v[i][1], v[i][2], v[i][3]};
      else {
#pragma unroll
        for (int k = 0; k < 3; ++k)
          if (c + k < d) xo[c + k] = v[i][k];
      }
    }
  }
  double q = 0.0;
  unsigned long long m = 0;
#pragma unroll
  for (int i = 0; i < V; ++i)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      q = __builtin_fma((double)v[i][k], (double)v[i][k], q);
      m = Max{}(m, (unsigned long long)__double_as_longlong((double)v[i][k] * (double)g[i][k]) & 0x7FFFFFFFFFFFFFFFull);
    }
  q = over_wave(q, Add{});
  m = over_wave(m, Max{});
  if constexpr (T == 256) {
    if ((t & 63) == 0) { part_q[t >> 6] = q; part_m[t >> 6] = m; }
    __syncthreads();
    q = (part_q[0] + part_q[1]) + (part_q[2] + part_q[3]);
    m = Max{}(Max{}(part_m[0], part_m[1]), Max{}(part_m[2], part_m[3]));
  }
  const double r = inverse_root(__builtin_fma(q, inv_d, (double)eps));
  const float s = scale_of(__longlong_as_double((long long)m) * r);
  // (an infinity in x' makes q one, in the gain m; a scale past float32 counts as one too)
  const bool bad = m >= 0x7FF0000000000000ull || !(q < __builtin_inf()) || !(s < __builtin_inff());
  const double inv = r * reciprocal((double)s);
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
  if (t == 0) scale[row] = bad ? __uint_as_float(NAN32) : s;
}

template <class X, int E, int T, int V>
static bool quantize_t(hipStream_t s, const void* x, int ldx, int M, int d, int8_t* codes, int ldq, float* scale) {
  if (d > T * V * E) return false;
  hipLaunchKernelGGL((quantize_i8_kernel<X, E, T, V>), dim3((M + 256 / T - 1) / (256 / T)), dim3(256), 0, s, (const X*)x, ldx, M, d, codes, ldq, scale);
  return true;
}
// The first of the widths that holds the row: pieces past its end cost a row of 10240 columns a quarter of its time.
template <class X, int E, int T, int... V>
static bool quantize_any(hipStream_t s, const void* x, int ldx, int M, int d, int8_t* codes, int ldq, float* scale) {
  return (quantize_t<X, E, T, V>(s, x, ldx, M, d, codes, ldq, scale) || ...);
}
void launch_quantize_i8(hipStream_t s, const void* x, bool f32, int ldx, int M, int d, int8_t* codes, int ldq, float* scale) {
  if (M == 0) return;
  if (f32) quantize_any<float, 4, 64, 1, 2, 4>(s, x, ldx, M, d, codes, ldq, scale) || quantize_any<float, 4, 256, 2, 3, 4, 5, 6, 8, 10, 12, 16>(s, x, ldx, M, d, codes, ldq, scale);
  else quantize_any<bf16_t, 8, 64, 1, 2>(s, x, ldx, M, d, codes, ldq, scale) || quantize_any<bf16_t, 8, 256, 1, 2, 3, 4, 5, 6, 8>(s, x, ldx, M, d, codes, ldq, scale);
}

template <class D, int T, int V>
static bool rmsnorm_t(hipStream_t s, const float* x, int ldx, const void* delta, int ldd, const float* gain, float eps, int M, int d,
                      float* x_out, int ldo, int8_t* codes, int ldq, float* scale) {
  if (d > T * V * 4) return false;
  hipLaunchKernelGGL((rmsnorm_i8_kernel<D, T, V>), dim3((M + 256 / T - 1) / (256 / T)), dim3(256), 0, s, x, ldx, (const D*)delta, ldd, gain, eps,
                     1.0 / (double)d, M, d, x_out, ldo, codes, ldq, scale);
  return true;
}
template <class D, int T, int... V>
static bool rmsnorm_any(hipStream_t s, const float* x, int ldx, const void* delta, int ldd, const float* gain, float eps, int M, int d,
                        float* x_out, int ldo, int8_t* codes, int ldq, float* scale) {
  return (rmsnorm_t<D, T, V>(s, x, ldx, delta, ldd, gain, eps, M, d, x_out, ldo, codes, ldq, scale) || ...);
}
template <class D>
static void rmsnorm_d(hipStream_t s, const float* x, int ldx, const void* delta, int ldd, const float* gain, float eps, int M, int d,
                      float* x_out, int ldo, int8_t* codes, int ldq, float* scale) {
  rmsnorm_any<D, 64, 1, 2, 4>(s, x, ldx, delta, ldd, gain, eps, M, d, x_out, ldo, codes, ldq, scale) ||
      rmsnorm_any<D, 256, 2, 3, 4, 5, 6, 8, 12, 16>(s, x, ldx, delta, ldd, gain, eps, M, d, x_out, ldo, codes, ldq, scale);
}
void launch_rmsnorm_i8(hipStream_t s, const float* x, int ldx, const void* delta, bool delta_f32, int ldd, const float* gain, float eps,
                       int M, int d, float* x_out, int ldo, int8_t* codes, int ldq, float* scale) {
  if (M == 0) return;
  if (delta_f32) rmsnorm_d<float>(s, x, ldx, delta, ldd, gain, eps, M, d, x_out, ldo, codes, ldq, scale);
  else rmsnorm_d<bf16_t>(s, x, ldx, delta, ldd, gain, eps, M, d, x_out, ldo, codes, ldq, scale);
}

}  // namespace dit
