// Epilogue of the matrix product (exfold_linear_forward): bias, activation, gate, residual
// and the rounding to y's type, from float32 sums.
#pragma once

#include "common.hpp"
#include "kernels.hpp"

namespace exfold {

// FAST: the result is rounded to bf16, where the hardware's exponential and reciprocal
// (a few float32 ulps) change nothing that the rounding keeps.
template <bool FAST> __device__ __forceinline__ float sigmoid_times(float z, float u) {
  if constexpr (FAST)
    return z * __builtin_amdgcn_rcpf(1.0f + __expf(-u));
  else
    return z / (1.0f + expf(-u));
}
template <int ACT, bool FAST> __device__ __forceinline__ float activate(float z) {
  if constexpr (ACT == EXFOLD_ACT_RELU) return z > 0.f ? z : 0.f;
  if constexpr (ACT == EXFOLD_ACT_SILU) return sigmoid_times<FAST>(z, z);
  if constexpr (ACT == EXFOLD_ACT_GELU) return 0.5f * z * (1.0f + erff(z * 0.70710678f));
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

// Outputs (m, n) .. (m, n + 3) from their sums z (gated: gate sums z, up sums u); columns
// from a.N on are not touched.  quad: r and y move four values at a time.
template <int ACT, bool GATED, typename O>
__device__ __forceinline__ void finish4(const LinearArgs &a, bool quad, long long m, int n, const float (&z)[4],
                                        const float (&u)[4]) {
  constexpr bool FAST = sizeof(O) == 2;
  O *y = static_cast<O *>(a.y) + m * a.ldy + n;
  const O *r = a.res ? static_cast<const O *>(a.res) + m * a.ldr + n : nullptr;
  const bool whole = quad && n + 4 <= a.N;
  float rv[4] = {0.f, 0.f, 0.f, 0.f}, o[4];
  if (r) {
    if (whole) {
      if constexpr (sizeof(O) == 2) {
        const uint2 q = *reinterpret_cast<const uint2 *>(r);
        rv[0] = __uint_as_float(q.x << 16);
        rv[1] = __uint_as_float(q.x & 0xffff0000u);
        rv[2] = __uint_as_float(q.y << 16);
        rv[3] = __uint_as_float(q.y & 0xffff0000u);
      } else {
        const f32x4 q = *reinterpret_cast<const f32x4 *>(r);
#pragma unroll
        for (int e = 0; e < 4; ++e) rv[e] = q[e];
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (n + e < a.N) rv[e] = load_f32(r + e);
    }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int c = min(n + e, a.N - 1);
    float g = z[e], v = u[e];
    if (a.bias) {
      g += a.bias[c];
      if (GATED) v += a.bias[a.N + c];
    }
    g = activate<ACT, FAST>(g);
    if (GATED) g *= v;
    o[e] = g + rv[e];
  }
  if (whole) {
    if constexpr (sizeof(O) == 2) {
      typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
      *reinterpret_cast<bf16x4 *>(y) = bf16x4{(__bf16)o[0], (__bf16)o[1], (__bf16)o[2], (__bf16)o[3]};
    } else {
      *reinterpret_cast<f32x4 *>(y) = f32x4{o[0], o[1], o[2], o[3]};
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (n + e < a.N) y[e] = store_cvt<O>(o[e]);
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

// Whether rows of r and y can be moved four values at a time.
template <typename O> __device__ __forceinline__ bool quads(const LinearArgs &a) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(a.y) | reinterpret_cast<uintptr_t>(a.res) |
                       (uintptr_t)(a.ldy * sizeof(O)) | (uintptr_t)(a.res ? a.ldr * sizeof(O) : 0);
  return at % (4 * sizeof(O)) == 0;
}

}  // namespace exfold
