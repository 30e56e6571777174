// What the kernels of the matrix product (exfold_linear_forward) share: the order of the tiles, and
// the epilogue: bias, activation, gate, residual and the rounding to y's type, from float32 sums.
#pragma once

#include "common.hpp"
#include "kernels.hpp"

namespace exfold {

// Tile of logical id L: panels of kPanel m-tiles, m-tile fastest in a panel, then the n-tiles, then
// the panels, then the splits, so that an XCD's consecutive ids share rows and weights (8192 x
// 1024 x 4096 83.6 -> 78.4 us against all m-tiles first).
constexpr int kPanel = 8;
__device__ __forceinline__ void tile_of(int L, int mts, int nts, int &mt, int &nt, int &ks) {
  ks = L / (mts * nts);
  L -= ks * mts * nts;
  const int panel = L / (kPanel * nts), in = L - panel * kPanel * nts, pm = min(kPanel, mts - panel * kPanel);
  nt = in / pm;
  mt = panel * kPanel + in - nt * pm;
}

// FAST: the result is rounded to bf16, and the hardware's exponential and reciprocal are taken: a
// few float32 ulps, and |u| more of them in the lower tail of the sigmoid, 2^-20 of |z| at most.
template <bool FAST> __device__ __forceinline__ float sigmoid_times(float z, float u) {
  if constexpr (FAST)
    return z * __builtin_amdgcn_rcpf(1.0f + __expf(-u));
  else
    return z / (1.0f + expf(-u));
}
// z Phi(z) = max(z, 0) - |z| Phi(-|z|) within 17 + 1.1 z^2 half steps of float32 of its value (erfcf of a
// rounded z / sqrt(2) has the z^2 too): Phi(-m) = exp(-m^2 / 2) times half the scaled complementary
// error function of m / sqrt(2), which is smooth in t = 1 / (1 + m / (2 sqrt(2))): a polynomial of
// degree 9 without constant term, fitted to least relative error over m < 13.3 (9e-8 with its
// float32 coefficients).  Of 2e7 normal z, 2.0e-5 round to another bf16 than the exact value in a
// float32 model of it (a degree of 7: 9.4e-5).  8192 x 8192 outputs of 512-long rows: 126.0 us, 122.6 with degree 7; 777 x
// 1408 outputs of 64-long rows: 6.3 us, 8.7 with the library's function, 5.0 without an activation.
__device__ __forceinline__ float gelu_few_ulps(float z) {
  // beyond 16 Phi(-m) is 0 in float32, and an infinite m would make 0 * m of it
  const float v = __builtin_elementwise_minimum(z, 16.0f), m = fabsf(v);
  const float t = __builtin_amdgcn_rcpf(fmaf(0.35355339f, m, 1.0f));
  float p = fmaf(-0.0294245053f, t, 0.141748533f);
  p = fmaf(p, t, -0.242478341f);
  p = fmaf(p, t, 0.137742981f);
  p = fmaf(p, t, -0.0124178017f);
  p = fmaf(p, t, 0.100961797f);
  p = fmaf(p, t, 0.121649213f);
  p = fmaf(p, t, 0.141174138f);
  p = fmaf(p, t, 0.141043991f);
  const float q = p * t * __builtin_amdgcn_exp2f(-0.72134752f * v * v);
  return fmaf(-m, q, __builtin_elementwise_maximum(z, 0.0f));  // NaN stays NaN
}
template <int ACT, bool FAST> __device__ __forceinline__ float activate(float z) {
  if constexpr (ACT == EXFOLD_ACT_RELU) return __builtin_elementwise_maximum(z, 0.0f);  // NaN stays NaN
  if constexpr (ACT == EXFOLD_ACT_SILU) return sigmoid_times<FAST>(z, z);
  // z Phi(z), by the complementary function: 1 + erf would lose the lower tail
  if constexpr (ACT == EXFOLD_ACT_GELU) return FAST ? gelu_few_ulps(z) : 0.5f * z * erfcf(z * -0.70710678f);
  // 0.5 z (1 + tanh u) = z / (1 + exp(-2 u)), u = sqrt(2 / pi) (z + 0.044715 z^3)
  if constexpr (ACT == EXFOLD_ACT_GELU_TANH)
    return sigmoid_times<FAST>(z, z * fmaf(0.07135481f * z, z, 1.59576912f));
  return z;
}

// Runs f with the activation as a compile-time constant (one uniform branch a tile).
template <typename F> __device__ __forceinline__ void with_act(int act, F f) {
  switch (act) {
    case EXFOLD_ACT_RELU: f(std::integral_constant<int, EXFOLD_ACT_RELU>{}); break;
    case EXFOLD_ACT_SILU: f(std::integral_constant<int, EXFOLD_ACT_SILU>{}); break;
    case EXFOLD_ACT_GELU: f(std::integral_constant<int, EXFOLD_ACT_GELU>{}); break;
    case EXFOLD_ACT_GELU_TANH: f(std::integral_constant<int, EXFOLD_ACT_GELU_TANH>{}); break;
    default: f(std::integral_constant<int, EXFOLD_ACT_NONE>{}); break;
  }
}

// Vectors at element alignment (global memory takes them at any byte).
typedef float f32x4_u __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned int u32x2_u __attribute__((ext_vector_type(2), aligned(2)));

__device__ __forceinline__ f32x4 load_quad(const float *p) { return *reinterpret_cast<const f32x4_u *>(p); }
__device__ __forceinline__ f32x4 load_quad(const bf16_t *p) {
  const u32x2_u q = *reinterpret_cast<const u32x2_u *>(p);
  return f32x4{__uint_as_float(q[0] << 16), __uint_as_float(q[0] & 0xffff0000u), __uint_as_float(q[1] << 16),
               __uint_as_float(q[1] & 0xffff0000u)};
}
__device__ __forceinline__ void store_quad(float *p, const f32x4 &v) { *reinterpret_cast<f32x4_u *>(p) = v; }
__device__ __forceinline__ void store_quad(bf16_t *p, const f32x4 &v) {
  typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
  const bf16x4 b = {(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
  *reinterpret_cast<u32x2_u *>(p) = __builtin_bit_cast(u32x2_u, b);
}
// Entries n .. n + 3 of a row of N; 0 past its end.
template <typename T> __device__ __forceinline__ f32x4 load_quad(const T *row, int n, int N) {
  if (n + 4 <= N) return load_quad(row + n);
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int e = 0; e < 3; ++e)
    if (n + e < N) v[e] = load_f32(row + n + e);
  return v;
}

// Bias of columns n .. n + 3 (gated: bz of the gate, bu of the up columns).
template <bool GATED> __device__ __forceinline__ void bias_quad(const LinearArgs &a, int n, f32x4 &bz, f32x4 &bu) {
  bz = bu = f32x4{0.f, 0.f, 0.f, 0.f};
  if (a.bias && n < a.N) {
    bz = load_quad(a.bias, n, a.N);
    if (GATED) bu = load_quad(a.bias + a.N, n, a.N);
  }
}
// Outputs (m, n) .. (m, n + 3), n < N, from their sums z (gated: gate sums z, up sums u), the bias
// and the residual r.
template <int ACT, bool GATED, typename O>
__device__ __forceinline__ void finish_quad(const LinearArgs &a, long long m, int n, f32x4 z, const f32x4 &u,
                                            const f32x4 &bz, const f32x4 &bu, const f32x4 &r) {
  z += bz;
#pragma unroll
  for (int e = 0; e < 4; ++e) z[e] = activate<ACT, sizeof(O) == 2>(z[e]);
  if constexpr (GATED) z *= u + bu;
  z += r;
  O *y = static_cast<O *>(a.y) + m * a.ldy + n;
  if (n + 4 <= a.N) {
    store_quad(y, z);
  } else {
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (n + e < a.N) y[e] = store_cvt<O>(z[e]);
  }
}

// The tiles' sums go through LDS, and a loop of a few rows a thread finishes them in row-major
// order: whole lines of r and y instead of 16-byte pieces of 32 rows, and a loop's instructions
// instead of a whole tile's.  Against finishing each wave's registers where they are: 777 x 1411 x
// 1003 with residual 22.8 -> 20.9 us, 1237 x 2816 x 4096 gated 44.6 -> 42.8, float32 600 x 2048 x
// 768 29.3 -> 28.6.
//
// `rows` rows of `COLS` outputs (gated: COLS gate sums, then COLS up sums) at red, PITCH floats a
// row, COPIES of them `copy` floats apart to be added in order; outputs (row0, n0) on.  The
// residual of a thread's rows of one turn is loaded before their outputs are stored (y may be
// the residual, so the compiler keeps the order written here).
template <int COPIES> __device__ __forceinline__ f32x4 lds_sum(const float *red, int copy) {
  f32x4 v = *reinterpret_cast<const f32x4 *>(red);
#pragma unroll
  for (int w = 1; w < COPIES; ++w) v += *reinterpret_cast<const f32x4 *>(red + w * copy);
  return v;
}
template <bool GATED, typename O, int COLS, int PITCH, int COPIES, int THREADS>
__device__ __forceinline__ void finish_tile(const LinearArgs &a, const float *red, int copy, long long row0, int n0, int rows) {
  constexpr int QN = COLS / 4, RN = THREADS / QN, U = 4;
  const int q = threadIdx.x % QN * 4, n = n0 + q;
  if (n >= a.N) return;
  f32x4 bz, bu;
  bias_quad<GATED>(a, n, bz, bu);
  const O *res = static_cast<const O *>(a.res);
  with_act(a.act, [&](auto act) {
#pragma unroll 1
    for (int m0 = threadIdx.x / QN; m0 < rows; m0 += RN * U) {
      f32x4 r[U];
#pragma unroll
      for (int i = 0; i < U; ++i) {
        r[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        const int m = m0 + i * RN;
        if (res && m < rows) r[i] = load_quad(res + (row0 + m) * a.ldr, n, a.N);
      }
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int m = m0 + i * RN;
        if (m >= rows) break;
        const float *at = red + m * PITCH + q;
        finish_quad<decltype(act)::value, GATED, O>(a, row0 + m, n, lds_sum<COPIES>(at, copy),
                                                    GATED ? lds_sum<COPIES>(at + COLS, copy) : f32x4{0.f, 0.f, 0.f, 0.f},
                                                    bz, bu, r[i]);
      }
    }
  });
}
// The same sums as partial sums of split ks (a.part).
template <bool GATED, int COLS, int PITCH, int COPIES, int THREADS>
__device__ __forceinline__ void store_partial(const LinearArgs &a, int ks, const float *red, int copy, int row0, int n0,
                                              int rows) {
  constexpr int H = GATED ? 2 : 1, QN = COLS * H / 4;
  const int np = linear_part_cols(a.N);
  for (int i = threadIdx.x; i < rows * QN; i += THREADS) {
    const int m = i / QN, c = i % QN * 4, n = n0 + (GATED ? c & (COLS - 1) : c);
    if (n < a.N)
      *reinterpret_cast<f32x4 *>(a.part + ((long long)ks * a.M + row0 + m) * np * H + (GATED && c >= COLS ? np : 0) + n) =
          lds_sum<COPIES>(red + m * PITCH + c, copy);
  }
}

// One output (m, n) from its sum z (gated: gate sum z, up sum u).
template <bool GATED, typename O>
__device__ __forceinline__ void finish1(const LinearArgs &a, long long m, int n, float z, float u) {
  if (a.bias) {
    z += a.bias[n];
    if (GATED) u += a.bias[a.N + n];
  }
  with_act(a.act, [&](auto act) { z = activate<decltype(act)::value, sizeof(O) == 2>(z); });
  if (GATED) z *= u;
  if (a.res) z += load_f32(static_cast<const O *>(a.res) + m * a.ldr + n);
  static_cast<O *>(a.y)[m * a.ldy + n] = store_cvt<O>(z);
}

}  // namespace exfold
