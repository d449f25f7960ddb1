// Product of 8-bit codes on the gfx950 matrix cores:  C[m][n] = sa[m] sw[n] sum_k A[m][k] W[n][k]  (+ epilogue).
//
// The sum is held in 32-bit integers, exact for K < 2^17, so no way of cutting the product up changes a bit of the result; the
// epilogue's float arithmetic is written with explicit fused operations, the same in every kernel.
#include "int8_internal.h"
#include <type_traits>

namespace dit {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) void* lptr_t;
typedef const __attribute__((address_space(4))) GemmI8 Problem;

namespace {

// round to nearest even (v_cvt_pk_bf16_f32)
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const f32x2 v = {a, b};
  const bf16x2 r = __builtin_convertvector(v, bf16x2);
  return *(const uint32_t*)&r;
}
__device__ __forceinline__ bf16_t bf(float f) { return (bf16_t)pack2(f, 0.f); }
// 0.5 x (1 + tanh(u)) = x / (1 + 2^(-2 log2(e) u)), u = sqrt(2/pi) (x + 0.044715 x^3)
__device__ __forceinline__ float gelu(float x) {
  const float t = x * __builtin_fmaf(0.035677408136300125f * x, x, 0.7978845608028654f);
  const float e = __builtin_amdgcn_exp2f(-2.8853900817779268f * t);
  return x * __builtin_amdgcn_rcpf(1.0f + e);
}
// The sum times the row's scale first: two scales of the row operators, down to 2^-126 each, leave the range of float32 when multiplied with each
// other, a sum of at least 1 times one of them does not fall below it.  (The smaller scale first costs 2 to 8 %: 8192 x 8192 x 1024 to bf16
// 76.6 -> 79.5 us, of GELU 91.7 -> 97.3.)
__device__ __forceinline__ float value(int acc, float sa, float sw, float bias) { return __builtin_fmaf((float)acc * sa, sw, bias); }
// A sum, below 2^31, times a row's scale above LARGE may be past float32 where the result is not: 2^32 is moved from such a scale to the columns'
// then, which changes no bit of a result.  (A column's scale that this takes past float32 becomes the largest number, so that a sum of 0 stays one.)
constexpr float LARGE = 0x1p96f, LARGEST = 0x1.fffffep127f;
__device__ __forceinline__ float eased_row(float sa, bool large) { return large ? sa * 0x1p-32f : sa; }
__device__ __forceinline__ float eased_col(float sw, bool large) {
  if (!large) return sw;
  const float t = sw * 0x1p32f;
  return t > LARGEST && sw <= LARGEST ? LARGEST : t;
}
__device__ __forceinline__ bool any_lane(bool b) { return __builtin_amdgcn_ballot_w64(b) != 0; }

// four neighbouring values of a vector at any place, those past the end are 0
typedef f32x4 f32x4_any __attribute__((aligned(4)));
__device__ __forceinline__ f32x4 load4(const float* p, int left) {
  if (left >= 4) return *(const f32x4_any*)p;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int c = 0; c < 3; ++c)
    if (c < left) v[c] = p[c];
  return v;
}

// What the epilogue needs for four neighbouring columns of a row (n + 3 may be past the end), fetched ahead of the sums: scales,
// second scales or bias, the row's request or column of the transposed matrix, and for a residual what is there and the gate.
struct Ahead { float sa; f32x4 sw, more, x, g; int map; };
template <bool PAIR, class P>
__device__ __forceinline__ Ahead fetch4(const P& p, int m, int n) {
  const int left = p.N - n;
  Ahead a;
  a.sa = p.sa[m];
  a.sw = load4(p.sw + n, left);
  a.more = f32x4{0.f, 0.f, 0.f, 0.f};
  if constexpr (PAIR) a.more = load4(p.sw2 + n, left);
  else {
    if (p.bias) a.more = load4(p.bias + n, left);
    const int* const map = n >= p.vt_from ? p.vt_col : p.row_req;
    a.map = map ? map[m] : 0;
    if (p.kind == OUT_RESID_F32) {
      a.x = load4((const float*)p.out + (size_t)m * p.ldc + n, left);
      a.g = f32x4{1.f, 1.f, 1.f, 1.f};
      if (p.gate) a.g = load4(p.gate + (size_t)a.map * p.gate_stride + n, left);
    }
  }
  return a;
}
template <bool PAIR>
__device__ __forceinline__ void ease4(Ahead& a) {
  const bool large = a.sa > LARGE;
  a.sa = eased_row(a.sa, large);
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    a.sw[c] = eased_col(a.sw[c], large);
    if constexpr (PAIR) a.more[c] = eased_col(a.more[c], large);
  }
}
// the four results to their places; up: the same columns of a pair's second product
template <class P>
__device__ __forceinline__ void put_row4(const P& p, int m, int n, const i32x4& acc, const Ahead& a) {
  const int left = p.N - n;
  float v[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) v[c] = value(acc[c], a.sa, a.sw[c], a.more[c]);
  if (n >= p.vt_from) {
#pragma unroll
    for (int c = 0; c < 4; ++c)
      if (c < left) p.vt[(size_t)(n + c - p.vt_from) * p.ldvt + a.map] = bf(v[c]);
    return;
  }
  const size_t o = (size_t)m * p.ldc + n;
  if (p.kind == OUT_F32 || p.kind == OUT_RESID_F32) {
    float* out = (float*)p.out + o;
    if (p.kind == OUT_RESID_F32) {
#pragma unroll
      for (int c = 0; c < 4; ++c) v[c] = __builtin_fmaf(a.g[c], v[c], a.x[c]);
    }
    if (left >= 4) *(f32x4*)out = f32x4{v[0], v[1], v[2], v[3]};
    else
      for (int c = 0; c < left; ++c) out[c] = v[c];
  } else {
    bf16_t* out = (bf16_t*)p.out + o;
    if (p.kind == OUT_GELU_BF16) {
#pragma unroll
      for (int c = 0; c < 4; ++c) v[c] = gelu(v[c]);
    }
    if (left >= 4) *(uint2*)out = make_uint2(pack2(v[0], v[1]), pack2(v[2], v[3]));
    else
      for (int c = 0; c < left; ++c) out[c] = bf(v[c]);
  }
}
template <class P>
__device__ __forceinline__ void put_pair4(const P& p, int m, int n, const i32x4& gate, const i32x4& up, const Ahead& a) {
  const int left = p.N - n;
  float v[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) v[c] = gelu(value(gate[c], a.sa, a.sw[c], 0.f)) * value(up[c], a.sa, a.more[c], 0.f);
  bf16_t* out = (bf16_t*)p.out + (size_t)m * p.ldc + n;
  if (left >= 4) *(uint2*)out = make_uint2(pack2(v[0], v[1]), pack2(v[2], v[3]));
  else
    for (int c = 0; c < left; ++c) out[c] = bf(v[c]);
}
// four neighbouring rows of a column of the transposed part (m + 3 may be past the end)
template <class P>
__device__ __forceinline__ void put_col4(const P& p, int m, int n, const i32x4& acc) {
  const float sw = p.sw[n], b = p.bias ? p.bias[n] : 0.f;
  bf16_t* dst = p.vt + (size_t)(n - p.vt_from) * p.ldvt;
  int col[4];
  bf16_t v[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const int k = m + c < p.M ? m + c : m;
    col[c] = p.vt_col[k];
    const bool large = p.sa[k] > LARGE;
    v[c] = bf(value(acc[c], eased_row(p.sa[k], large), eased_col(sw, large), b));
  }
  if (m + 4 <= p.M && col[3] == col[0] + 3 && (col[0] & 3) == 0)       // (columns rise)
    *(uint2*)(dst + col[0]) = make_uint2(v[0] | (uint32_t)v[1] << 16, v[2] | (uint32_t)v[3] << 16);
  else {
#pragma unroll
    for (int c = 0; c < 4; ++c)
      if (m + c < p.M) dst[col[c]] = v[c];
  }
}

// at most N vector-memory loads outstanding; LGKM0: LDS reads done too
template <int N, bool LGKM0>
__device__ __forceinline__ void wait_vm() {
  constexpr int imm = (N & 15) | ((N >> 4) << 14) | (7 << 4) | ((LGKM0 ? 0 : 15) << 8);
  __builtin_amdgcn_s_waitcnt(imm);
  asm volatile("" ::: "memory");
}
// barrier without the fence of __syncthreads(), which would wait for every load in flight
__device__ __forceinline__ void wg_barrier() {
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ void buffer_load_lds16(const void* base, lptr_t dst, uint32_t voff, int soff) {
  const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)base, (short)0, (int)0xFFFFFFFFu, 0x00020000);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, dst, 16, voff, soff, 0, 0);
}
// key of a slab row: 16 rows fall into 16 distinct 16-byte slots, consecutive ones and those of the permuted order below
__device__ __forceinline__ int swz_key(int r) { return ((r >> 1) & 1) | ((r >> 2) & 2) | ((r ^ (r >> 2)) & 4); }

// tile t -> (tile row, tile column): groups of 8 tile rows, column-major inside
template <class P>
__device__ __forceinline__ void tile_coords(const P& p, int t, int& tm, int& tn) {
  const int per = 8 * p.tiles_n, g = t / per, r = t - g * per, first = g * 8;
  const int gsz = p.tiles_m - first < 8 ? p.tiles_m - first : 8;
  tm = first + r % gsz;
  tn = r / gsz;
}

}  // namespace

// ---- 8-wave tiles ----------------------------------------------------------------------------------------------------
//
// A workgroup of two groups of four waves (one wave of each on every SIMD), half a phase apart: while one group does nothing
// but multiply, the other reads its next fragments from LDS and issues the loads of later slabs.  Slabs are 128 codes wide and
// go from memory straight into an NS-stage LDS ring; a workgroup stays on its CU and the slabs of its tiles (or of its shares of
// K) are one stream, so the next tile's first slabs arrive under the epilogue.
// Operands are swapped (W in the place of the MFMA's rows, its rows in the order {0-3, 8-11, ...}, {4-7, ...}), which gives a lane
// 8 neighbouring columns of one row; tiles of transposed results keep the first order with the rows of A permuted.
//   Bound: the matrix cores at the clock that the board's power leaves them.  8192^3 370 to 400 us, 2.75 to 2.95 POP/s, matrix cores busy in 87 %
// of the cycles at 1.36 to 1.54 GHz; 8000 x 12288 x 4096 300 to 310 us as bf16, 330 to 340 as fp32.  (128x128 tiles: what a CU pulls, 32 KB in 0.36 to 0.48 us.)
template <int BM, int BN, int WM, int WN, int NS>
__global__ __launch_bounds__(512) void gemm8_i8_kernel(const GemmI8) {
  Problem& P = *(Problem*)__builtin_amdgcn_kernarg_segment_ptr();
  constexpr int ROWB = 128;
  constexpr int RT = BM / WM / 16, CT = 4;             // 16-row and 16-column tiles of a wave
  constexpr int PH = NS == 2 ? 2 : 1, RP = RT / PH;    // phases per slab, row tiles per phase
  constexpr int LA = BM / 64, LB = BN / 64, LPS = LA + LB;   // loads per wave and slab
  constexpr int LAU = NS == 2 ? WM : LA;               // ... of the first part of A: 64 rows of every wave row
  constexpr int STAGE = (BM + BN) * ROWB, OFFB = BM * ROWB;
  static_assert(WM * WN == 8 && BN / WN == 64 && BM % 64 == 0 && RT % PH == 0, "two groups of four waves, 64 columns a wave");
  static_assert(NS >= 3 || (NS == 2 && RP * 16 == 64), "two stages: 64 rows a phase");
  static_assert((NS - 1) * LPS < 64, "vmcnt");
  extern __shared__ __attribute__((aligned(128))) unsigned char smem[];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WN, wn = wave % WN;
  unsigned char* const patch = smem + NS * STAGE + wave * 2048;
  const int splits = P.splits;
  const bool pair = P.W2 != nullptr;

  // my units (a tile, or one share of K of a tile): XCD x (workgroup ids are dealt round-robin) owns a contiguous range of them
  int t_first, t_count, t_step;
  {
    const int x = blockIdx.x & 7, T = P.tiles_m * P.tiles_n * splits, G = gridDim.x;
    t_first = x * (T >> 3) + (x < (T & 7) ? x : (T & 7));
    t_count = (T >> 3) + (x < (T & 7) ? 1 : 0);
    t_step = (G >> 3) + (x < (G & 7) ? 1 : 0);
  }
  auto unit = [&](int t, int& tm, int& tn, int& k0, int& k1) {
    const int u = t_first + t, tile = u / splits, sh = u - tile * splits, nk = P.K / 128;     // (sh * nk < 2^13: 4 shares, 2^10 slabs)
    tile_coords(P, tile, tm, tn);
    // (scalar by hand: divided in vector registers, as an offset of the loads they would cost a loop around each of them)
    tm = __builtin_amdgcn_readfirstlane(tm); tn = __builtin_amdgcn_readfirstlane(tn);
    k0 = __builtin_amdgcn_readfirstlane(sh * nk / splits); k1 = __builtin_amdgcn_readfirstlane((sh + 1) * nk / splits);
  };

  // ---- the stream of slabs: one load of a wave fills 8 slab rows -------------------------------------------------------
  auto row_a = [&](int i) {
    if constexpr (NS == 2) {         // A in two parts, the first 64 rows of every wave row and the rest
      const bool up = i < LAU;
      const int per = up ? 64 : RT * 16 - 64;
      const int rr = ((up ? i : i - LAU) * 8 + wave) * 8;
      return rr / per * (RT * 16) + rr % per + (up ? 0 : 64);
    } else {
      return (i * 8 + wave) * 8;
    }
  };
  uint32_t oa[LA], ob[LB];           // byte offsets of my lane's 16 codes of each load, from the tile's first row
  const int8_t *sA, *sW;
  int ld_t = blockIdx.x >> 3, ks = 0, ks_n = 0;      // unit (in my XCD's range) and slab that are fetched next, and the end of its slabs
  auto aim = [&](int t) {
    int tm, tn;
    unit(t, tm, tn, ks, ks_n);
    const int m0 = tm * BM, n0 = pair ? tn * (BN / 2) : tn * BN;
    int ln = lane;
    asm volatile("" : "+v"(ln));     // (made anew for each tile: kept, these would cost registers)
#pragma unroll
    for (int i = 0; i < LA; ++i) {
      const int r = row_a(i) + (ln >> 3), c = (ln & 7) ^ swz_key(r);
      const int m = m0 + r < P.M ? r : P.M - 1 - m0;             // clamp: rows past M are never stored
      oa[i] = (uint32_t)m * (uint32_t)P.lda + c * 16;
    }
#pragma unroll
    for (int i = 0; i < LB; ++i) {
      const int r = (i * 8 + wave) * 8 + (ln >> 3), c = (ln & 7) ^ swz_key(r);
      const int rw = pair ? (r >> 6) * 32 + (r & 31) : r;
      const int n = n0 + rw < P.N ? rw : P.N - 1 - n0;
      ob[i] = (uint32_t)n * (uint32_t)P.ldw + c * 16;
    }
    sA = P.A + (size_t)m0 * P.lda;
    sW = (pair && (wave & 4) ? P.W2 : P.W) + (size_t)n0 * P.ldw;    // (waves 4-7 load the upper half of each 64 rows)
  };
  // (behind the very last slab the same again, which keeps the number of loads per slab fixed)
  auto advance = [&]() {
    if (ks + 1 < ks_n) ++ks;
    else if (ld_t + t_step < t_count) {
      ld_t += t_step;
      aim(ld_t);
    }
  };
  auto issue_a = [&](int st, auto first, auto last) {
#pragma unroll
    for (int i = decltype(first)::value; i < decltype(last)::value; ++i)
      buffer_load_lds16(sA, (lptr_t)(smem + st * STAGE + row_a(i) * ROWB), oa[i], ks * 128);
  };
  auto issue_b = [&](int st) {
#pragma unroll
    for (int i = 0; i < LB; ++i) buffer_load_lds16(sW, (lptr_t)(smem + st * STAGE + OFFB + (i * 8 + wave) * 1024), ob[i], ks * 128);
  };
  constexpr std::integral_constant<int, 0> A_FIRST{};
  constexpr std::integral_constant<int, LAU> A_REST{};
  constexpr std::integral_constant<int, LA> A_END{};

  // ---- the loop over one unit's slabs --------------------------------------------------------------------------------
  i32x4 acc[RT][CT];
  const bool second = wave >= 4;
  int stage = 0;
  auto run = [&](auto vt_tag, int nk) {
    constexpr bool VT = decltype(vt_tag)::value;
    int ln = lane;
    asm volatile("" : "+v"(ln));
    const int l16 = ln & 15, kq = ln >> 4;
    const int row_c = l16, row_p = (l16 >> 2) * 8 + (l16 & 3);
    const int off_c = row_c * ROWB + ((kq ^ swz_key(row_c)) << 4), off_p = row_p * ROWB + ((kq ^ swz_key(row_p)) << 4);
    i32x4 fa[2][RP], fb[2][CT];
    // consecutive rows: 16-row tile i starts 16 i rows on; permuted ones: pairs of tiles 32 rows on, the odd one 4 rows on
    auto tile_off = [](bool perm, int i) { return perm ? (i >> 1) * 32 + (i & 1) * 4 : i * 16; };
    const int a0 = wm * (RT * 16) * ROWB + (VT ? off_p : off_c), b0 = OFFB + wn * 64 * ROWB + (VT ? off_c : off_p);
    auto read_a = [&](const unsigned char* st, auto phase) {
      const unsigned char* p[2] = {st + a0, st + (a0 ^ 64)};     // (odd tiles flip bit 2 of the key)
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int r = 0; r < RP; ++r) {
          const int i = decltype(phase)::value * RP + r;
          fa[k][r] = *(const i32x4*)(p[k ^ (i & 1)] + tile_off(VT, i) * ROWB);
        }
    };
    auto read_b = [&](const unsigned char* st) {
      const unsigned char* p[2] = {st + b0, st + (b0 ^ 64)};
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int c = 0; c < CT; ++c) fb[k][c] = *(const i32x4*)(p[k ^ (c & 1)] + tile_off(!VT, c) * ROWB);
    };
    auto multiply = [&](auto phase) {
      wg_barrier();
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int r = 0; r < RP; ++r)
#pragma unroll
          for (int c = 0; c < CT; ++c) {
            i32x4& d = acc[decltype(phase)::value * RP + r][c];
            if constexpr (VT) d = __builtin_amdgcn_mfma_i32_16x16x64_i8(fa[k][r], fb[k][c], d, 0, 0, 0);
            else d = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[k][c], fa[k][r], d, 0, 0, 0);
          }
      __builtin_amdgcn_s_setprio(0);
      __builtin_amdgcn_sched_barrier(0);
      wg_barrier();
    };
    constexpr std::integral_constant<int, 0> P0{};
    constexpr std::integral_constant<int, PH - 1> P1{};
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int c = 0; c < CT; ++c) acc[r][c] = i32x4{0, 0, 0, 0};
    auto slab = [&](auto same) {       // same: the stream's next slab is known to be of this unit
      const unsigned char* cur = smem + stage * STAGE;
      const int nxt = stage + 1 == NS ? 0 : stage + 1;
      if constexpr (decltype(same)::value) ++ks; else advance();
      read_b(cur);
      read_a(cur, P0);
      if constexpr (NS == 2) {
        // Phase 0 of slab s reads the first part of A and W; phase 1 the rest of A, and issues W and the first part of A
        // of slab s+2; when it is over the rest of A follows (over that of slab s, which everybody has read).
        wait_vm<LPS, true>();                          // rest of A of slab s (mine)
        multiply(P0);
        read_a(cur, P1);
        issue_b(stage); issue_a(stage, A_FIRST, A_REST);
        wait_vm<LPS, true>();                          // W and the first part of A of slab s+1 (mine)
        multiply(P1);
        issue_a(stage, A_REST, A_END);
      } else {
        // phase s reads slab s and issues slab s + NS - 1 into the stage that slab s-1 left
        const int free_st = stage == 0 ? NS - 1 : stage - 1;
        issue_a(free_st, A_FIRST, A_END); issue_b(free_st);
        wait_vm<(NS - 2) * LPS, true>();               // slab s+1 (mine)
        multiply(P0);
      }
      stage = nxt;
    };
    if (second) wg_barrier();
    int kt = 0;
    for (; kt < nk - (NS == 2 ? 2 : NS - 1); ++kt) slab(std::true_type{});
    for (; kt < nk; ++kt) slab(std::false_type{});
    if (!second) wg_barrier();
  };

  // ---- epilogues: C[16 r + l16][32 j + 8 kq + 0..7] of the wave's sub-tile in acc[r][2 j], acc[r][2 j + 1] ------------
  auto epilogue = [&](int tm, int tn, bool vt) {
    int ln = lane;
    asm volatile("" : "+v"(ln));
    const int l16 = ln & 15, kq = ln >> 4;
    const int prow = ln >> 3, pchunk = ln & 7;           // my row (and the one 8 on) and 16-byte chunk when a patch is read back
    const int mw = tm * BM + wm * (RT * 16), nw = tn * BN + wn * 64;
    const int M = P.M, N = P.N;
    const float* const bias = P.bias;
    auto patch_at = [&](int row, int chunk) { return patch + row * 128 + ((chunk ^ ((row >> 1) & 7)) << 4); };
    auto turn = [&](const u32x4& lo, const u32x4& hi, int c_lo, int c_hi, u32x4 (&out)[2]) {    // 16 rows x 128 bytes
      *(u32x4*)patch_at(l16, c_lo) = lo;
      *(u32x4*)patch_at(l16, c_hi) = hi;
      asm volatile("" ::: "memory");                     // (a wave's LDS accesses are executed in order)
      out[0] = *(const u32x4*)patch_at(prow, pchunk);
      out[1] = *(const u32x4*)patch_at(prow + 8, pchunk);
      asm volatile("" ::: "memory");
    };
    auto row_scale = [&](int m) { return P.sa[m < M ? m : M - 1]; };
    auto load_cols = [&](const float* p, int n0, int n_end, float (&v)[8]) {
      const f32x4 lo = p && n0 < n_end ? load4(p + n0, n_end - n0) : f32x4{0.f, 0.f, 0.f, 0.f};
      const f32x4 hi = p && n0 + 4 < n_end ? load4(p + n0 + 4, n_end - n0 - 4) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < 4; ++c) { v[c] = lo[c]; v[4 + c] = hi[c]; }
    };
    float sa[RT];
    auto load_sa = [&]() {
#pragma unroll
      for (int r = 0; r < RT; ++r) sa[r] = row_scale(mw + r * 16 + l16);
    };
    // (for all rows of a lane at once, which share its columns' scales)
    auto ease = [&](auto& rows, auto&... cols) {
      bool large = false;
      for (float s : rows) large |= s > LARGE;
      if (any_lane(large)) {
        for (float& s : rows) s = eased_row(s, large);
        auto of = [&](auto& c) { for (float& s : c) s = eased_col(s, large); };
        (of(cols), ...);
      }
    };
    auto plain_bf16 = [&](auto gelu_tag) {
      float sw[2][8], bv[2][8];
#pragma unroll
      for (int j = 0; j < 2; ++j) { load_cols(P.sw, nw + j * 32 + kq * 8, N, sw[j]); load_cols(bias, nw + j * 32 + kq * 8, N, bv[j]); }
      load_sa();
      const bool full = nw + pchunk * 8 + 8 <= N;
      const int ldc = P.ldc;
      bf16_t* const out = (bf16_t*)P.out;
      const uint32_t voff = (uint32_t)(prow * ldc + pchunk * 8) * 2u;
      ease(sa, sw[0], sw[1]);
      auto make = [&](int r, u32x4 (&w)[2]) {
        u32x4 p[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          float v[8];
#pragma unroll
          for (int c = 0; c < 8; ++c) {
            v[c] = value(acc[r][2 * j + (c >> 2)][c & 3], sa[r], sw[j][c], bv[j][c]);
            if constexpr (decltype(gelu_tag)::value) v[c] = gelu(v[c]);
          }
#pragma unroll
          for (int c = 0; c < 4; ++c) p[j][c] = pack2(v[2 * c], v[2 * c + 1]);
        }
        turn(p[0], p[1], kq, 4 + kq, w);
      };
      u32x4 w[2], nx[2];
      make(0, w);
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        if (r + 1 < RT) make(r + 1, nx);                 // (a unit is turned while the one before it is stored)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          char* const xp = (char*)(out + (size_t)(mw + r * 16 + h * 8) * ldc + nw) + voff;
          if (prow < M - mw - (r * 16 + h * 8)) {
            if (full) *(u32x4*)xp = w[h];
            else
              for (int c = 0; c < N - nw - pchunk * 8; ++c) ((bf16_t*)xp)[c] = (bf16_t)(w[h][c >> 1] >> (16 * (c & 1)));
          }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) w[h] = nx[h];
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    // fp32 results in units of 16 rows x 32 columns: plain, or added to what is there times the row's gate
    auto plain_f32 = [&](auto resid_tag) {
      constexpr bool RESID = decltype(resid_tag)::value;
      float sw[2][8], bv[2][8];
#pragma unroll
      for (int j = 0; j < 2; ++j) { load_cols(P.sw, nw + j * 32 + kq * 8, N, sw[j]); load_cols(bias, nw + j * 32 + kq * 8, N, bv[j]); }
      load_sa();
      const int nb = nw + pchunk * 4, ldc = P.ldc;       // my columns on the way out: nb + 32 j ... + 3
      float* const out = (float*)P.out;
      const uint32_t voff = (uint32_t)(prow * ldc + pchunk * 4) * 4u;
      auto row_at = [&](int u, int h) { return (char*)(out + (size_t)(mw + (u >> 1) * 16 + h * 8) * ldc + nw + 32 * (u & 1)) + voff; };
      auto row_in = [&](int u, int h) { return prow < M - mw - (u >> 1) * 16 - h * 8; };
      constexpr int U = RT * 2, AHEAD = 2;
      f32x4 xr[RESID ? AHEAD : 1][2], gr[RESID ? AHEAD : 1][2];
      const float* const gate = RESID ? P.gate : nullptr;
      const int* const rreq = P.row_req;
      // what is there, and the gate, AHEAD units before their use (the compiler may not move loads across the stores)
      auto load_x = [&](int u) {
        if constexpr (RESID) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            f32x4 x = {0.f, 0.f, 0.f, 0.f}, g = {1.f, 1.f, 1.f, 1.f};
            const int n = nb + 32 * (u & 1);
            if (row_in(u, h) && n < N) {
              const float* xp = (const float*)row_at(u, h);
              const float* gp = gate ? gate + (size_t)(rreq ? rreq[mw + (u >> 1) * 16 + h * 8 + prow] : 0) * P.gate_stride + n : nullptr;
              if (n + 4 <= N) {
                x = *(const f32x4*)xp;
                if (gp) g = f32x4{gp[0], gp[1], gp[2], gp[3]};
              } else {
#pragma unroll
                for (int c = 0; c < 3; ++c)
                  if (n + c < N) {
                    x[c] = xp[c];
                    if (gp) g[c] = gp[c];
                  }
              }
            }
            xr[u % AHEAD][h] = x; gr[u % AHEAD][h] = g;
          }
        }
      };
      auto make = [&](int u, u32x4 (&w)[2]) {
        union { float f[8]; u32x4 q[2]; } v;
        const int r = u >> 1, j = u & 1;
#pragma unroll
        for (int c = 0; c < 8; ++c) v.f[c] = value(acc[r][2 * j + (c >> 2)][c & 3], sa[r], sw[j][c], bv[j][c]);
        turn(v.q[0], v.q[1], 2 * kq, 2 * kq + 1, w);
      };
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) load_x(u);
      ease(sa, sw[0], sw[1]);
      u32x4 w[2], nx[2];
      make(0, w);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int n = nb + 32 * (u & 1);
        if (u + 1 < U) make(u + 1, nx);
        // (used here on every path: a load that some path leaves pending would be waited for in the next tile's loop)
        if constexpr (RESID) asm volatile("" :: "v"(xr[u % AHEAD][0]), "v"(xr[u % AHEAD][1]), "v"(gr[u % AHEAD][0]), "v"(gr[u % AHEAD][1]));
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if (row_in(u, h) && n < N) {
            f32x4 x4;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              x4[c] = __uint_as_float(w[h][c]);
              if constexpr (RESID) x4[c] = __builtin_fmaf(gr[u % AHEAD][h][c], x4[c], xr[u % AHEAD][h][c]);
            }
            float* xp = (float*)row_at(u, h);
            if (n + 4 <= N) *(f32x4*)xp = x4;
            else {
#pragma unroll
              for (int c = 0; c < 3; ++c)
                if (n + c < N) xp[c] = x4[c];
            }
          }
        }
        if (u + AHEAD < U) load_x(u + AHEAD);
#pragma unroll
        for (int h = 0; h < 2; ++h) w[h] = nx[h];
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    // Transposed columns: acc[2 i][c], acc[2 i + 1][c] hold rows 32 i + 8 kq + 0..7 of column 16 c + l16.  Units of 32 rows x 32
    // columns; a lane writes 8 rows of a column as one 16-byte piece (at any 2-byte offset: 1137 x 4096 x 4096 takes the same with every
    // start) where these are neighbours in the transposed matrix, else in pairs and single elements.
    auto transposed = [&]() {
      typedef u32x4 u32x4_any __attribute__((aligned(2)));
      const int nv0 = nw - P.vt_from, ldvt = P.ldvt;
      const int* const map = P.vt_col;
      bf16_t* const vt_out = P.vt;
      float bv[CT], sw[CT];
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        const int n = nw + c * 16 + l16;
        bv[c] = bias && n < N ? bias[n] : 0.f;
        sw[c] = n < N ? P.sw[n] : 0.f;
      }
      const int fr = ln >> 2, fc = ln & 3;               // my column (and the one 16 on) and piece when a unit is read back
      auto at = [&](int f, int chunk) { return patch + f * 64 + ((chunk ^ ((f >> 2) & 3)) << 4); };
      // All units' row scales and the columns of my pieces' rows, ahead of the stores: a load behind them waits for them to be done (pieces
      // fetched one by one where they are stored made ragged rows cost 9 us more than neighbours, so 2).
      float sr[RT * 4];
      int col[RT / 2][8];
#pragma unroll
      for (int i = 0; i < RT / 2; ++i) {
        const int mb = mw + i * 32, mp = mb + fc * 8;
#pragma unroll
        for (int e = 0; e < 8; ++e) col[i][e] = map[mp + e < M ? mp + e : M - 1];
        if (mb + 32 <= M) {
          const f32x4 lo = *(const f32x4_any*)(P.sa + mb + kq * 8), hi = *(const f32x4_any*)(P.sa + mb + kq * 8 + 4);
#pragma unroll
          for (int e = 0; e < 4; ++e) { sr[i * 8 + e] = lo[e]; sr[i * 8 + 4 + e] = hi[e]; }
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) sr[i * 8 + e] = row_scale(mb + kq * 8 + e);
        }
      }
      ease(sr, sw);
#pragma unroll
      for (int i = 0; i < RT / 2; ++i) {
        const int mp = mw + i * 32 + fc * 8;
        const bool whole = mp + 8 <= M && col[i][7] == col[i][0] + 7;    // (columns rise)
#pragma unroll
        for (int cp = 0; cp < 2; ++cp) {
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            const int c = cp * 2 + q;
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = value(acc[2 * i + (e >> 2)][c][e & 3], sr[i * 8 + e], sw[c], bv[c]);
            const u32x4 w = {pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7])};
            *(u32x4*)at(q * 16 + l16, kq) = w;
          }
          asm volatile("" ::: "memory");
          u32x4 w[2];
#pragma unroll
          for (int h = 0; h < 2; ++h) w[h] = *(const u32x4*)at(h * 16 + fr, fc);
          asm volatile("" ::: "memory");
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int f = cp * 32 + h * 16 + fr;
            if (f >= N - nw) continue;
            bf16_t* const dst = vt_out + (size_t)(nv0 + f) * ldvt;
            if (whole) *(u32x4_any*)(dst + col[i][0]) = w[h];
            else {
#pragma unroll
              for (int e = 0; e < 8; ++e)
                if (mp + e < M) dst[col[i][e]] = (bf16_t)(w[h][e >> 1] >> (16 * (e & 1)));
            }
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    };
    // gated pair: the wave's 64 columns are 32 of the gate (acc[.][0, 1]) and the same 32 of the values (acc[.][2, 3])
    auto gated = [&]() {
      const int nw2 = nw >> 1, ldc = P.ldc;
      bf16_t* const out = (bf16_t*)P.out;
      float sg[8], su[8];
      load_sa();
      load_cols(P.sw, nw2 + kq * 8, N, sg);
      load_cols(P.sw2, nw2 + kq * 8, N, su);
      const int fr = ln >> 2, fc = ln & 3;               // my row (and the one 16 on) and piece when 32 rows are read back
      auto at = [&](int f, int chunk) { return patch + f * 64 + ((chunk ^ ((f >> 2) & 3)) << 4); };
      const bool full = nw2 + fc * 8 + 8 <= N;
      const uint32_t voff = (uint32_t)(fr * ldc + fc * 8) * 2u;
      ease(sa, sg, su);
#pragma unroll
      for (int i = 0; i < RT / 2; ++i) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const int r = 2 * i + q;
          float v[8];
#pragma unroll
          for (int c = 0; c < 8; ++c)
            v[c] = gelu(value(acc[r][c >> 2][c & 3], sa[r], sg[c], 0.f)) * value(acc[r][2 + (c >> 2)][c & 3], sa[r], su[c], 0.f);
          const u32x4 w = {pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7])};
          *(u32x4*)at(q * 16 + l16, kq) = w;
        }
        asm volatile("" ::: "memory");
        u32x4 w[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) w[h] = *(const u32x4*)at(h * 16 + fr, fc);
        asm volatile("" ::: "memory");
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int k = i * 32 + h * 16;
          char* const xp = (char*)(out + (size_t)(mw + k) * ldc + nw2) + voff;
          if (fr < M - mw - k) {
            if (full) *(u32x4*)xp = w[h];
            else
              for (int c = 0; c < N - nw2 - fc * 8; ++c) ((bf16_t*)xp)[c] = (bf16_t)(w[h][c >> 1] >> (16 * (c & 1)));
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    if (pair) { gated(); return; }
    if (vt) { transposed(); return; }
    if (P.kind == OUT_GELU_BF16) plain_bf16(std::true_type{});
    else if (P.kind == OUT_BF16) plain_bf16(std::false_type{});
    else if (P.kind == OUT_F32) plain_f32(std::false_type{});
    else plain_f32(std::true_type{});
  };

  // ---- all my units ----------------------------------------------------------------------------------------------------
  aim(ld_t);
#pragma unroll
  for (int st = 0; st < (NS == 2 ? 2 : NS - 1); ++st) {
    if (st) advance();
    issue_b(st); issue_a(st, A_FIRST, A_END);
  }
  wait_vm<(NS == 2 ? 1 : NS - 2) * LPS, false>();
  wg_barrier();
  for (int t = blockIdx.x >> 3; t < t_count; t += t_step) {
    int tm, tn, k0, k1;
    unit(t, tm, tn, k0, k1);
    const bool vt = !pair && tn * BN >= P.vt_from;
    if (vt) run(std::true_type{}, k1 - k0);
    else run(std::false_type{}, k1 - k0);
    if (splits > 1) {
      // a share: the sums in register order, for the reduction
      int ln = lane;
      asm volatile("" : "+v"(ln));
      i32x4* const dst = (i32x4*)P.partial + ((size_t)(t_first + t) * 8 + wave) * (RT * CT * 64) + ln;
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int c = 0; c < CT; ++c) dst[(r * CT + c) * 64] = acc[r][c];
    } else {
      epilogue(tm, tn, vt);
    }
  }
  wait_vm<0, true>();                        // drain the redundant tail loads before LDS is released
}

// The shares of a split product added up, with the epilogue: a thread per four results.
template <int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(256) void reduce_i8_kernel(const GemmI8 P) {
  constexpr int RT = BM / WM / 16, CT = 4, CHUNK = 8 * RT * CT * 64;      // i32x4 of a share
  const bool pair = P.W2 != nullptr;
  const int per = pair ? CHUNK / 2 : CHUNK;
  const int tile = blockIdx.x / (per / 256);
  int q = (blockIdx.x % (per / 256)) * 256 + threadIdx.x;
  const int lane = q & 63, l16 = lane & 15, kq = lane >> 4;
  q >>= 6;
  const int c = pair ? q % 2 : q % CT, r = (pair ? q / 2 : q / CT) % RT, wave = (pair ? q / 2 : q / CT) / RT;
  const int wm = wave / WN, wn = wave % WN;
  int tm, tn;
  tile_coords(P, tile, tm, tn);
  const bool vt = !pair && tn * BN >= P.vt_from;
  const int mw = tm * BM + wm * (RT * 16), nw = tn * BN + wn * 64;
  int m, n;
  if (vt) { m = mw + (r >> 1) * 32 + kq * 8 + (r & 1) * 4; n = nw + c * 16 + l16; }
  else { m = mw + r * 16 + l16; n = (pair ? nw >> 1 : nw) + (c >> 1) * 32 + kq * 8 + (c & 1) * 4; }
  if (m >= P.M || n >= P.N) return;
  auto sum = [&](int cc) {
    const i32x4* p = (const i32x4*)P.partial + (size_t)tile * P.splits * CHUNK + ((wave * RT + r) * CT + cc) * 64 + lane;
    i32x4 s = p[0];
#pragma unroll 4
    for (int k = 1; k < P.splits; ++k) s += p[(size_t)k * CHUNK];
    return s;
  };
  if (pair) {
    Ahead a = fetch4<true>(P, m, n);
    ease4<true>(a);
    put_pair4(P, m, n, sum(c), sum(c + 2), a);
  } else if (vt) {
    put_col4(P, m, n, sum(c));
  } else {
    Ahead a = fetch4<false>(P, m, n);
    ease4<false>(a);
    put_row4(P, m, n, sum(c), a);
  }
}

// ---- few rows: the weights as a stream ---------------------------------------------------------------------------------
//
// A workgroup owns 16 NT columns (of a pair: 8 NT of each product) and 16 MT rows.  Its waves take every WV-th slab of
// 128 codes, so that together they read runs of WV * 128 bytes of every weight row, each exactly once.  Every wave has an LDS
// ring of its own, D slabs deep, and waits for nobody: no barrier until the waves' sums meet in LDS.  One launch, no scratch.
//   Bound: what a CU pulls through its L1, (MT + NT) 2 KB a slab at 85 GB/s, and HBM for the fewest rows.  1 x 12288 x 4096 9.4 us (5.3 TB/s of
// weights in the memory-side cache; 11.7 from HBM), 32 x 12288 x 4096 10.2 (13.0), 32 x 4096 x 10240 9.8 (14), 128 x 4096 x 4096 7.6.
//   Through LDS because a load then covers 8 rows x 128 bytes; straight into fragment order, 16 rows x 64 bytes, its addresses cost
// four times as much (32 x 4096 x 10240 15.8 us; the weights alone straight, with twice of them in flight, 10.7).
// Waves of a workgroup: as many slabs in flight as LDS holds (up to 8 for each wave); eight waves have 256 registers each, four have 512.
constexpr int stream_waves(int mt, int nt) {
  const int slab = (mt + nt) * 2048, regs = mt * nt * 4 + (mt + nt) * 10 + 24;
  int best = 4, most = 0;
  for (int w = regs <= 256 ? 8 : 4; w >= 4; --w) {
    int d = 160 * 1024 / (w * slab);
    if (d > 8) d = 8;
    if (w * d > most) { most = w * d; best = w; }
  }
  return best;
}
template <int MT, int NT, bool PAIR>
struct StreamShape {
  static constexpr int L = (MT + NT) * 2, SLAB = L * 1024;     // loads of 1 KB and bytes of a slab
  static constexpr int WV = stream_waves(MT, NT);
  static constexpr int FIT = 160 * 1024 / (WV * SLAB), D = FIT > 8 ? 8 : FIT;
  static constexpr int NC = PAIR ? NT / 2 : NT;                // 16-column tiles of one product
  static constexpr int passes() { int p = 1; while (MT % p || WV * (MT / p) * NT > 160) ++p; return p; }
  static constexpr int IP = MT / passes();                     // 16-row tiles whose sums meet in LDS at a time
  static constexpr int RING = WV * D * SLAB, RED = WV * IP * NT * 1024, LDS = RING > RED ? RING : RED;
  static_assert(D >= 1 && (D - 1) * L < 64 && (!PAIR || NT % 2 == 0), "ring");
};
template <int MT, int NT, bool PAIR>
__global__ __launch_bounds__((StreamShape<MT, NT, PAIR>::WV * 64)) void stream_i8_kernel(const GemmI8 P) {
  using S = StreamShape<MT, NT, PAIR>;
  constexpr int L = S::L, D = S::D, WV = S::WV, NC = S::NC;
  extern __shared__ __attribute__((aligned(128))) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, kq = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // XCD x (workgroup ids are dealt round-robin) takes a contiguous range of the tiles: the row tiles of one column tile
  // together, or the other way round, whichever operand is larger is then read by one XCD alone
  const int x = blockIdx.x & 7, T = gridDim.x;
  const int tile = x * (T >> 3) + (x < (T & 7) ? x : (T & 7)) + (blockIdx.x >> 3);
  const bool by_m = P.M > (PAIR ? 2 * P.N : P.N);
  const int tm = by_m ? tile / P.tiles_n : tile % P.tiles_m, tn = by_m ? tile % P.tiles_n : tile / P.tiles_m;
  const int m0 = tm * (MT * 16), n0 = tn * NC * 16;
  unsigned char* const ring = smem + wave * (D * S::SLAB);
  // byte offsets of my lane's 16 codes: load i fills slab rows 8 i .. 8 i + 7, rows of A first
  uint32_t off[L];
#pragma unroll
  for (int i = 0; i < L; ++i) {
    const int r = i * 8 + (lane >> 3), c = ((lane & 7) ^ swz_key(r)) * 16;
    if (i < 2 * MT) {
      const int m = m0 + r < P.M ? r : P.M - 1 - m0;     // rows past the end repeat the last one and are not stored
      off[i] = (uint32_t)m * (uint32_t)P.lda + c;
    } else {
      const int j = (r - 16 * MT) >> 4, n = n0 + (j % NC) * 16 + (r & 15);
      off[i] = (uint32_t)((n < P.N ? n : P.N - 1) - n0) * (uint32_t)P.ldw + c;
    }
  }
  const int8_t* const A = P.A + (size_t)m0 * P.lda;
  const int8_t* const W = P.W + (size_t)n0 * P.ldw;
  const int8_t* const W2 = PAIR ? P.W2 + (size_t)n0 * P.ldw : W;
  const int nk = P.K / 128, mine = (nk - wave + WV - 1) / WV;            // slabs wave, wave + WV, ...
  auto load = [&](int i, int s, int stage) {
    buffer_load_lds16(i < 2 * MT ? A : (i - 2 * MT) / 2 < NC ? W : W2, (lptr_t)(ring + stage * S::SLAB + i * 1024), off[i], (wave + WV * s) * 128);
  };
  i32x4 acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
  const int at = l16 * 128 + ((kq ^ swz_key(l16)) << 4);
  // slab s, which has landed in `stage`; next: the stage is filled again with slab s + D, whose loads go out ahead of the products
  auto multiply = [&](int s, int stage, auto next) {
    const unsigned char* const p[2] = {ring + stage * S::SLAB + at, ring + stage * S::SLAB + (at ^ 64)};     // (odd tiles flip bit 2 of the key)
    i32x4 fa[2][MT], fb[2][NT];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int j = 0; j < NT; ++j) fb[h][j] = *(const i32x4*)(p[h ^ ((MT + j) & 1)] + (MT + j) * 2048);
#pragma unroll
      for (int i = 0; i < MT; ++i) fa[h][i] = *(const i32x4*)(p[h ^ (i & 1)] + i * 2048);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // (in registers before the stage is loaded over)
    __builtin_amdgcn_sched_barrier(0);
    // the loads spread over the products: back to back a wave waits some 70 cycles for each to be taken
    constexpr int NM = 2 * MT * NT, PER = NM / L > 1 ? NM / L / 2 : 1;
#pragma unroll
    for (int q = 0; q < NM; ++q) {
      const int h = q / (MT * NT), i = q / NT % MT, j = q % NT;
      if (decltype(next)::value && q % PER == 0 && q / PER < L) load(q / PER, s + D, stage);
      acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[h][j], fa[h][i], acc[i][j], 0, 0, 0);
    }
    if constexpr (decltype(next)::value) {
#pragma unroll
      for (int i = (NM + PER - 1) / PER; i < L; ++i) load(i, s + D, stage);
#pragma unroll
      for (int i = 0; i < L && i * PER < NM; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, PER, 0);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  };
#pragma unroll
  for (int s = 0; s < D; ++s)
    if (s < mine)
#pragma unroll
      for (int i = 0; i < L; ++i) load(i, s, s);
  int s = 0, stage = 0;
  for (; s + D < mine; ++s) {
    wait_vm<(D - 1) * L, false>();                       // slab s
    multiply(s, stage, std::true_type{});
    stage = stage + 1 == D ? 0 : stage + 1;
  }
  for (; s < mine; ++s) {                                // the last D: fewer are in flight with every step
    switch (mine - 1 - s) {
      case 7: if constexpr (D > 7) wait_vm<(D > 7 ? 7 : 0) * L, false>(); break;
      case 6: if constexpr (D > 6) wait_vm<(D > 6 ? 6 : 0) * L, false>(); break;
      case 5: if constexpr (D > 5) wait_vm<(D > 5 ? 5 : 0) * L, false>(); break;
      case 4: if constexpr (D > 4) wait_vm<(D > 4 ? 4 : 0) * L, false>(); break;
      case 3: if constexpr (D > 3) wait_vm<(D > 3 ? 3 : 0) * L, false>(); break;
      case 2: if constexpr (D > 2) wait_vm<(D > 2 ? 2 : 0) * L, false>(); break;
      case 1: wait_vm<L, false>(); break;
      default: wait_vm<0, false>(); break;
    }
    multiply(s, stage, std::false_type{});
    stage = stage + 1 == D ? 0 : stage + 1;
  }
  // (16-byte place of a lane's sums inside their 16x16 tile: turned by the column group, so that reading along a row meets 16 banks of 16 bytes)
  i32x4* const red = (i32x4*)smem;
  auto place = [](int i, int j, int row, int q) { return (i * NT + j) * 64 + q * 16 + (row ^ ((j * 4 + q) & 15)); };
  constexpr int IP = S::IP;
  auto sum = [&](int q) {
    i32x4 t = red[q];
#pragma unroll
    for (int w = 1; w < WV; ++w) t += red[q + w * IP * NT * 64];
    return t;
  };
  const bool by_rows = n0 >= P.vt_from;                  // (transposed: neighbouring threads take neighbouring rows)
#pragma unroll
  for (int i0 = 0; i0 < MT; i0 += IP) {
    __syncthreads();                                     // (the rings, or the sums before, are done with)
#pragma unroll
    for (int i = 0; i < IP; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) red[wave * (IP * NT * 64) + place(i, j, l16, kq)] = acc[i0 + i][j];
    // up to four of a thread's results at a time: what the first ones need comes in while the sums are gathered
    constexpr int ALL = IP * NC * 64, STEP = WV * 64, U = MT * NT >= 48 || ALL < 4 * STEP ? 2 : 4;
    Ahead ahead[U];
    int row[U], g[U];
    bool in[U];
    auto fetch = [&](int q0) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int q = q0 + u * STEP;
        row[u] = by_rows ? q % (IP * 16) : q / (NC * 4); g[u] = by_rows ? q / (IP * 16) : q % (NC * 4);
        in[u] = q < ALL && m0 + i0 * 16 + row[u] < P.M && n0 + g[u] * 4 < P.N;
        if (in[u]) ahead[u] = fetch4<PAIR>(P, m0 + i0 * 16 + row[u], n0 + g[u] * 4);
      }
    };
    fetch(tid);
    __syncthreads();
    for (int q0 = tid;;) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (!in[u]) continue;
        const int i = row[u] >> 4, j = g[u] >> 2, m = m0 + i0 * 16 + row[u], n = n0 + g[u] * 4;
        const i32x4 t = sum(place(i, j, row[u] & 15, g[u] & 3));
        i32x4 up;
        if constexpr (PAIR) up = sum(place(i, j + NC, row[u] & 15, g[u] & 3));
        if (any_lane(ahead[u].sa > LARGE)) ease4<PAIR>(ahead[u]);
        if constexpr (PAIR) put_pair4(P, m, n, t, up, ahead[u]);
        else put_row4(P, m, n, t, ahead[u]);
      }
      q0 += U * STEP;
      if (q0 >= ALL) break;
      fetch(q0);
    }
  }
}

// ---- launches ------------------------------------------------------------------------------------------------------------
namespace {

template <int BM, int BN, int WM, int WN, int NS>
void launch8(hipStream_t s, GemmI8& p) {
  p.tiles_m = (p.M + BM - 1) / BM;
  p.tiles_n = ((p.W2 ? 2 * p.N : p.N) + BN - 1) / BN;
  constexpr int lds = NS * (BM + BN) * 128 + 8 * 2048;
  static_assert(lds <= 160 * 1024, "LDS of a CU");
  auto kern = gemm8_i8_kernel<BM, BN, WM, WN, NS>;
  static std::atomic<unsigned> seen{0};
  if (first_use_on_device(seen)) (void)hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  const int units = p.tiles_m * p.tiles_n * p.splits;
  hipLaunchKernelGGL(kern, dim3(units < 256 ? units : 256), dim3(512), lds, s, p);
  if (p.splits > 1) {
    constexpr int per = 8 * (BM / WM / 16) * 4 * 64;
    hipLaunchKernelGGL((reduce_i8_kernel<BM, BN, WM, WN>), dim3(p.tiles_m * p.tiles_n * ((p.W2 ? per / 2 : per) / 256)), dim3(256), 0, s, p);
  }
}

template <int MT, int NT, bool PAIR>
void launch_stream_t(hipStream_t s, GemmI8& p) {
  using S = StreamShape<MT, NT, PAIR>;
  auto kern = stream_i8_kernel<MT, NT, PAIR>;
  static std::atomic<unsigned> seen{0};
  if (first_use_on_device(seen)) (void)hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, S::LDS);
  p.tiles_m = (p.M + MT * 16 - 1) / (MT * 16);
  p.tiles_n = (p.N + S::NC * 16 - 1) / (S::NC * 16);
  hipLaunchKernelGGL(kern, dim3(p.tiles_m * p.tiles_n), dim3(S::WV * 64), S::LDS, s, p);
}
template <int MT>
bool launch_stream_m(hipStream_t s, GemmI8& p, int nt) {
  if (p.W2) {
    switch (nt) {
      case 2: launch_stream_t<MT, 2, true>(s, p); return true;
      case 4: launch_stream_t<MT, 4, true>(s, p); return true;
      case 6: if constexpr (MT <= 5) { launch_stream_t<MT, 6, true>(s, p); return true; }
    }
    return false;
  }
  switch (nt) {
    case 1: launch_stream_t<MT, 1, false>(s, p); return true;
    case 2: launch_stream_t<MT, 2, false>(s, p); return true;
    case 3: launch_stream_t<MT, 3, false>(s, p); return true;
    case 4: launch_stream_t<MT, 4, false>(s, p); return true;
    case 6: if constexpr (MT == 4 || MT == 5) { launch_stream_t<MT, 6, false>(s, p); return true; }
  }
  return false;
}

// ---- the choice of tile ----
// The variant with the least estimated time, in microseconds: a start, the rounds of 256 workgroups, in each the slabs of one tile and a
// fixed part (first loads, sums of the waves, epilogue).  A slab of a stream tile takes 2 KB a row tile of what a CU pulls and a share of
// its products; a slab of an 8-wave tile takes longer the more CUs run one (the clock falls with the matrix load: 256x256 0.7 us for
// one, 1.2 with all of them busy, 1.3 round after round).  No estimate is below its bytes at 4.8 TB/s, with which the rest was fitted: weights from HBM
// come no faster, those in the memory-side cache up to a tenth (1 x 12288 x 4096), which only levels tiles that are all as fast as their bytes.
// The constants were fitted to 312 products of 1 to 8000 rows, 300 to 12288 columns and K from 512 to 10240 with every variant timed: the
// one chosen took 1.005 times the best one's time in the mean, 1.09 at most; over 140 other shapes 1.013 and 1.13 (the most where a last
// round of few tiles has a launch of its own).  Both sides near the borders: 128 rows, N = 4096, K = 4096 stream
// 7.6, 128x128 14; 200 rows, N = 12288 128x128 20, stream 23; 333 rows, N = 4096, K = 10240 stream 22.2, 128x128 34; 500 rows, N = 12288
// 128x256 27.8, 256x256 38.2; 1000 rows 52.7 and 44.2; 1000 rows, N = 4096 128x128 20.6, 128x256 25.4.  Two shares of K: 500 rows, N = 4096,
// K = 10240 to bf16 31.9 (26.4 and the reduction's 5.5), unsplit 36.6, stream 39.8; 248 rows, N = 6176, K = 9600 anything unsplit takes 27 % longer.
//   Columns that fill whole rounds of 256 8-wave tiles go ahead of the rest, which then takes the tile that suits it, where that saves 5 %:
// 528 tiles are two rounds and 16 tiles more.  2744 x 12288 x 4096 138 -> 125 us, a gated pair of 1000 x 10240 x 4096 92 -> 79; without the
// 5 % 2200 x 4096 x 10240 89 -> 94.  160 drawn shapes where it is chosen: 0.76 to 1.10 of the best 8-wave tile in one launch, 0.944 in the
// mean; 1 us for the second launch in the estimate would win 0.1 %, more of it or a larger margin lose.
struct Choice { int variant, splits; float us; };
struct Plan { Choice main, rest; int first; };      // first: columns of the main launch where the rest has one of its own, else 0

struct Tile { int bm, bn; float one, all, on, fixed; };            // a slab of the only tile, of 256 tiles, of round after round
constexpr Tile TILES[] = {{128, 128, 0.305f, 0.458f, 0.477f, 3.3f}, {128, 256, 0.43f, 0.70f, 0.75f, 5.7f},
                          {256, 128, 0.43f, 0.70f, 0.75f, 5.7f}, {256, 256, 0.70f, 1.19f, 1.29f, 9.6f}};

// cols: columns of the product, of a pair those of both
Choice choose(int M, long long cols, int K, bool pair, size_t scratch) {
  const int nk = K / 128;
  const float least = 0.4f + ((float)M * K + (float)cols * K + (pair ? 1.f : 2.f) * M * cols) / 4.8e6f;
  Choice best = {0, 1, 0.f};
  auto offer = [&](int variant, int splits, float us) {
    if (us < least) us = least + us * 1e-3f;
    if (!best.variant || us < best.us) best = Choice{variant, splits, us};
  };
  // (most rows first: at the same estimate two row tiles of one workgroup read a weight once, two workgroups twice; cold weights,
  // 32 rows, N = 4096, K = 10240: 13.7 us with 32 x 16 tiles, 14.7 with 16 x 32)
  for (int mt = 6; mt >= 1; --mt)
    for (int nt : {1, 2, 3, 4, 6}) {
      if ((pair ? nt % 2 != 0 : nt == 6 && mt < 4) || (nt == 6 && mt == 6)) continue;      // (not built)
      const long long wgs = (M + 16LL * mt - 1) / (16 * mt) * ((cols + 16 * nt - 1) / (16 * nt)), rounds = (wgs + 255) / 256;
      if (wgs > (1 << 22)) continue;                                                        // (512 threads each: a launch has less than 2^32)
      offer(100 * mt + nt, 1, 0.6f + (float)rounds * (nk * (0.0141f * (mt + nt) + 0.005f * mt * nt) + (rounds > 1 ? 1.95f : 2.9f) + 0.054f * mt * nt));
    }
  auto slab = [](const Tile& t, long long n) { return t.one + (t.all - t.one) * (float)n / 256.f; };
  for (const Tile& t : TILES) {
    const long long n = (M + t.bm - 1LL) / t.bm * ((cols + t.bn - 1) / t.bn), full = n > 256 ? n / 256 : 0, rest = n - full * 256;
    offer(t.bm * 1000 + t.bn, 1, 2.6f + (float)full * (nk * t.on + t.fixed) + (rest ? nk * slab(t, rest) + t.fixed : 0.f));
  }
  // Shares of K of 128x128 tiles, where these leave CUs empty: their sums go through memory to a second launch.
  const long long n = (M + 127LL) / 128 * ((cols + 127) / 128);
  for (int s = 2; s <= 4 && n * s <= 256 && nk >= 8 * s; ++s)
    if ((size_t)n * s * (128 * 128 * 4) <= scratch)
      offer(128128, s, 5.3f + (float)((nk + s - 1) / s) * slab(TILES[0], n * s) + 2.3f + (float)n * s * 0.018f);
  return best;
}

Plan make_plan(int M, int N, int K, bool pair, size_t scratch) {
  const long long cols = pair ? 2LL * N : N;
  Plan p = {choose(M, cols, K, pair, scratch), {0, 1, 0.f}, 0};
  float best = p.main.us * 0.95f;
  for (const Tile& t : TILES) {
    const long long tm = (M + t.bm - 1LL) / t.bm, n = tm * ((cols + t.bn - 1) / t.bn), full = n / 256;
    if (full < 1 || n % 256 == 0) continue;
    const long long first = full * 256 / tm * t.bn / 256 * 256;      // (256: transposed columns of the rest start at one of its tiles)
    if (first <= 0 || first >= cols) continue;
    const Choice rest = choose(M, cols - first, K, pair, scratch);
    const float us = 2.6f + (float)full * (K / 128 * (full > 1 ? t.on : t.all) + t.fixed) + rest.us;
    if (us < best) { best = us; p.main = Choice{t.bm * 1000 + t.bn, 1, us}; p.rest = rest; p.first = (int)(pair ? first / 2 : first); }
  }
  return p;
}

}  // namespace

// variant 100 MT + NT: a stream tile; BM*1000 + BN: an 8-wave tile, 128x128 ones with p.splits shares of K
bool launch_gemm_i8_variant(hipStream_t s, GemmI8& p, int variant) {
  if (variant != 128128) p.splits = 1;
  switch (variant) {
    case 256256: launch8<256, 256, 2, 4, 2>(s, p); return true;
    case 256128: launch8<256, 128, 4, 2, 3>(s, p); return true;
    case 128256: launch8<128, 256, 2, 4, 3>(s, p); return true;
    case 128128: launch8<128, 128, 4, 2, 4>(s, p); return true;
  }
  switch (variant / 100) {
    case 1: return launch_stream_m<1>(s, p, variant % 100);
    case 2: return launch_stream_m<2>(s, p, variant % 100);
    case 3: return launch_stream_m<3>(s, p, variant % 100);
    case 4: return launch_stream_m<4>(s, p, variant % 100);
    case 5: return launch_stream_m<5>(s, p, variant % 100);
    case 6: return launch_stream_m<6>(s, p, variant % 100);
  }
  return false;
}

int gemm_i8_plan(int M, int N, int K, bool pair, size_t scratch, int (&out)[3]) {
  const Plan p = make_plan(M, N, K, pair, scratch);
  out[0] = p.first ? p.rest.splits : p.main.splits; out[1] = p.first; out[2] = p.rest.variant;     // (a first launch has whole tiles)
  return p.main.variant;
}
size_t gemm_i8_work_bytes(int M, int N, int K, bool pair) {
  const Plan p = make_plan(M, N, K, pair, ~(size_t)0);
  const Choice& c = p.first ? p.rest : p.main;
  const long long n = N - p.first;
  return c.splits == 1 ? 0 : (size_t)((M + 127) / 128) * (((pair ? 2 * n : n) + 127) / 128) * c.splits * (128 * 128 * 4);
}

bool launch_gemm_i8(hipStream_t s, GemmI8& p) {
  const Plan plan = make_plan(p.M, p.N, p.K, p.W2 != nullptr, p.partial ? p.partial_bytes : 0);
  const int n1 = plan.first;
  if (!n1) {
    p.splits = plan.main.splits;
    return launch_gemm_i8_variant(s, p, plan.main.variant);
  }
  GemmI8 a = p, b = p;                                   // columns 0 .. n1 - 1, and the rest
  a.N = n1; a.splits = 1;
  if (a.vt_from > n1) a.vt_from = n1;
  b.N = p.N - n1; b.splits = plan.rest.splits;
  b.W += (size_t)n1 * p.ldw; b.sw += n1;
  if (b.W2) { b.W2 += (size_t)n1 * p.ldw; b.sw2 += n1; }
  if (b.bias) b.bias += n1;
  if (b.gate) b.gate += n1;
  if (b.out) b.out = (char*)b.out + (size_t)n1 * (p.kind == OUT_F32 || p.kind == OUT_RESID_F32 ? 4 : 2);
  if (p.vt_from < n1) { b.vt += (size_t)(n1 - p.vt_from) * p.ldvt; b.vt_from = 0; }
  else b.vt_from = p.vt_from - n1;
  return launch_gemm_i8_variant(s, a, plan.main.variant) && launch_gemm_i8_variant(s, b, plan.rest.variant);
}

}  // namespace dit
