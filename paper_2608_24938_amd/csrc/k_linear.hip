// Matrix product with bias, activation and residual in its epilogue (exfold_linear_forward):
//   y = act(x W^T + b) + r,   gated: y = act(x W_g^T + b_g) * (x W_u^T + b_u) + r
// float32 sums, one rounding to y's type.
#include "common.hpp"
#include "kernels.hpp"

namespace exfold {

// ---------------------------------------------------------------------------
// Epilogue.
// ---------------------------------------------------------------------------

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

// Whether rows of r and y can be moved four values at a time.
template <typename O> __device__ __forceinline__ bool quads(const LinearArgs &a) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(a.y) | reinterpret_cast<uintptr_t>(a.res) |
                       (uintptr_t)(a.ldy * sizeof(O)) | (uintptr_t)(a.res ? a.ldr * sizeof(O) : 0);
  return at % (4 * sizeof(O)) == 0;
}

// ---------------------------------------------------------------------------
// Tiles of BM rows x BN weight rows (gated: BN / 2 gate rows and the BN / 2 up rows of the
// same columns), four waves of 32x32 MFMA tiles.  A stage is 128 bytes of the reduction (64
// bf16 or 32 float32 columns) of every row, staged through registers into one of two LDS
// buffers, its 16-byte pieces swizzled so that a fragment read spreads over the banks; the
// next stage's loads fly during the MFMAs.  A lane's piece of a row feeds one 32x32x16 bf16
// MFMA or four 32x32x2 float32 ones (any assignment of columns to steps is a valid order).
// VEC: rows start on 16 bytes and K is a whole number of pieces; else element loads, 64 (32)
// consecutive ones a wave.  Rows past the ends re-read the last one and are not stored;
// columns past K are zero.
// ---------------------------------------------------------------------------
template <typename E> __device__ __forceinline__ void mma32(const u32x4 &a, const u32x4 &b, f32x16 &c) {
  if constexpr (sizeof(E) == 2) {
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[e]), __uint_as_float(b[e]), c, 0, 0, 0);
  }
}

// LDS slot (16-byte units) of piece q of tile row r (8 pieces a row).
__device__ __forceinline__ int piece_at(int r, int q) { return r * 8 + (q ^ ((r ^ (r >> 1)) & 7)); }

template <typename E, int BM, int BN, bool GATED, bool VEC>
__global__ __launch_bounds__(256, 1) void linear_tile(const LinearArgs a, const LinearPlan p) {
  constexpr int KS = 128 / sizeof(E), EP = 16 / sizeof(E);
  constexpr int TM = BM / 64, TN = BN / 64;
  constexpr int PA = BM * 8 / 256, PB = BN * 8 / 256;                 // pieces a thread
  constexpr int SA = VEC ? 1 : BM * KS / 256, SB = VEC ? 1 : BN * KS / 256;  // elements a thread
  static_assert(!GATED || TN % 2 == 0, "a wave holds the gate and the up columns");
  __shared__ __attribute__((aligned(16))) u32x4 smem[2][(BM + BN) * 8];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wm = wave >> 1, wn = wave & 1;
  const int mts = (a.M + BM - 1) / BM, cols = GATED ? BN / 2 : BN, nts = (a.N + cols - 1) / cols;
  const int L = xcd_remap(blockIdx.x, mts * nts * p.ksplit);
  const int mt = L % mts, nt = L / mts % nts, ks = L / mts / nts;
  const int k0 = ks * p.kc, k1 = min(a.K, k0 + p.kc);
  const E *x = static_cast<const E *>(a.x), *w = static_cast<const E *>(a.w);
  // weight row of tile row r
  auto wrow = [&](int r) {
    if (!GATED) return min(nt * BN + r, a.N - 1);
    const int c = min(nt * (BN / 2) + (r & (BN / 2 - 1)), a.N - 1);
    return r < BN / 2 ? c : a.N + c;
  };
  auto xrow = [&](int r) { return min(mt * BM + r, a.M - 1); };

  const E *sa[VEC ? PA : 1], *sb[VEC ? PB : 1];
  if constexpr (VEC) {
#pragma unroll
    for (int i = 0; i < PA; ++i) sa[i] = x + xrow(i * 32 + (tid >> 3)) * a.ldx + (tid & 7) * EP;
#pragma unroll
    for (int i = 0; i < PB; ++i) sb[i] = w + wrow(i * 32 + (tid >> 3)) * a.ldw + (tid & 7) * EP;
  }
  u32x4 ra[VEC ? PA : 1], rb[VEC ? PB : 1];
  E ea[SA], eb[SB];
  auto load = [&](int k) __attribute__((always_inline)) {
    if constexpr (VEC) {
      const bool in = k + (tid & 7) * EP < k1;
#pragma unroll
      for (int i = 0; i < PA; ++i) ra[i] = in ? *reinterpret_cast<const u32x4 *>(sa[i] + k) : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
      for (int i = 0; i < PB; ++i) rb[i] = in ? *reinterpret_cast<const u32x4 *>(sb[i] + k) : u32x4{0u, 0u, 0u, 0u};
    } else {
      const int c = tid % KS, r0 = tid / KS;
      const bool in = k + c < k1;
#pragma unroll
      for (int i = 0; i < SA; ++i) ea[i] = in ? x[xrow(r0 + i * (256 / KS)) * a.ldx + k + c] : E(0);
#pragma unroll
      for (int i = 0; i < SB; ++i) eb[i] = in ? w[wrow(r0 + i * (256 / KS)) * a.ldw + k + c] : E(0);
    }
  };
  auto stage = [&](int buf) __attribute__((always_inline)) {
    u32x4 *As = smem[buf], *Bs = As + BM * 8;
    if constexpr (VEC) {
#pragma unroll
      for (int i = 0; i < PA; ++i) As[piece_at(i * 32 + (tid >> 3), tid & 7)] = ra[i];
#pragma unroll
      for (int i = 0; i < PB; ++i) Bs[piece_at(i * 32 + (tid >> 3), tid & 7)] = rb[i];
    } else {
      const int c = tid % KS, r0 = tid / KS;
#pragma unroll
      for (int i = 0; i < SA; ++i)
        reinterpret_cast<E *>(&As[piece_at(r0 + i * (256 / KS), c / EP)])[c % EP] = ea[i];
#pragma unroll
      for (int i = 0; i < SB; ++i)
        reinterpret_cast<E *>(&Bs[piece_at(r0 + i * (256 / KS), c / EP)])[c % EP] = eb[i];
    }
  };
  f32x16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
  // tile row of a wave's column block j: blocks wn, wn + 2, ... (gated: gate and up blocks in step)
  auto brow = [&](int j) { return (j * 2 + wn) * 32; };

  int buf = 0;
  load(k0);
  stage(0);
  __syncthreads();
  for (int k = k0; k < k1; k += KS) {
    const bool more = k + KS < k1;
    if (more) load(k + KS);
    const u32x4 *As = smem[buf], *Bs = As + BM * 8;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      u32x4 fa[TM], fb[TN];
#pragma unroll
      for (int i = 0; i < TM; ++i) fa[i] = As[piece_at((i * 2 + wm) * 32 + (lane & 31), 2 * s + (lane >> 5))];
#pragma unroll
      for (int j = 0; j < TN; ++j) fb[j] = Bs[piece_at(brow(j) + (lane & 31), 2 * s + (lane >> 5))];
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) mma32<E>(fb[j], fa[i], acc[i][j]);
    }
    if (more) stage(buf ^ 1);
    __syncthreads();
    buf ^= 1;
  }

  // Register r of tile (i, j): row (i 2 + wm) 32 + lane % 32, column brow(j) + 8 (r / 4) +
  // 4 (lane / 32) + r % 4 (the weights are the MFMA's first operand): runs of four columns.
  const int m0 = mt * BM + wm * 32 + (lane & 31);
  if (p.ksplit > 1) {
    const long long ld = linear_part_ld(a.N, GATED);
    const int nw = GATED ? 2 * a.N : a.N;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int m = m0 + i * 64;
      if (m >= a.M) continue;
      float *row = a.part + ((long long)ks * a.M + m) * ld;
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int c = brow(j) + 8 * g + 4 * (lane >> 5);
          const int in_half = GATED ? nt * (BN / 2) + (c & (BN / 2 - 1)) : nt * BN + c;
          const int base = GATED && c >= BN / 2 ? a.N : 0;
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (in_half + e < a.N) row[base + in_half + e] = acc[i][j][4 * g + e];
        }
    }
    (void)nw;
    return;
  }
  auto finish = [&](auto out) {
    using O = decltype(out);
    const bool quad = quads<O>(a);
    with_act(a.act, [&](auto act) {
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        const int m = m0 + i * 64;
        if (m >= a.M) continue;
#pragma unroll
        for (int j = 0; j < (GATED ? TN / 2 : TN); ++j)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const int n = nt * cols + brow(j) + 8 * g + 4 * (lane >> 5);
            if (n >= a.N) continue;
            float z[4], u[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              z[e] = acc[i][j][4 * g + e];
              if constexpr (GATED) u[e] = acc[i][j + TN / 2][4 * g + e];
            }
            finish4<decltype(act)::value, GATED, O>(a, quad, m, n, z, u);
          }
      }
    });
  };
  if (sizeof(E) == 4 || a.out_dtype == EXFOLD_F32)
    finish(float{});
  else if constexpr (sizeof(E) == 2)
    finish(bf16_t{});
}

// Joins the split partial sums in order, four columns a thread, and finishes them.
template <bool GATED, typename O>
__global__ __launch_bounds__(256) void linear_join(const LinearArgs a, int ksplit) {
  const long long ld = linear_part_ld(a.N, GATED), split = (long long)a.M * ld;
  const int quads_n = (a.N + 3) / 4;
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  if (i >= (long long)a.M * quads_n) return;
  const long long m = i / quads_n;
  const int n = (int)(i % quads_n) * 4;
  const float *row = a.part + m * ld;
  float z[4] = {0.f, 0.f, 0.f, 0.f}, u[4] = {0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < ksplit; ++s)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (n + e < a.N) {
        z[e] += row[s * split + n + e];
        if (GATED) u[e] += row[s * split + a.N + n + e];
      }
  const bool quad = quads<O>(a);
  with_act(a.act, [&](auto act) { finish4<decltype(act)::value, GATED, O>(a, quad, m, n, z, u); });
}

// ---------------------------------------------------------------------------
// Planning and launch.
// ---------------------------------------------------------------------------
LinearPlan plan_linear(int dtype, bool gated, bool vec, int M, int N, int K, int cu_count) {
  LinearPlan p{};
  p.kind = kLinTile;
  p.bm = 64;
  p.bn = 128;
  const int cols = gated ? p.bn / 2 : p.bn, stage = dtype == EXFOLD_BF16 ? 64 : 32;
  const long long tiles = (long long)((M + p.bm - 1) / p.bm) * ((N + cols - 1) / cols);
  const int stages = (K + stage - 1) / stage;
  int split = 1;
  while (tiles * split < cu_count && split < 16 && stages / (2 * split) >= 4) split *= 2;
  const int per = (stages + split - 1) / split;
  p.kc = per * stage;
  p.ksplit = (stages + per - 1) / per;
  p.grid = (int)(tiles * p.ksplit);
  return p;
}

template <typename E, bool GATED, bool VEC>
static void launch_tile(const LinearArgs &a, const LinearPlan &p, hipStream_t s) {
  linear_tile<E, 64, 128, GATED, VEC><<<p.grid, 256, 0, s>>>(a, p);
}

hipError_t launch_linear(const LinearArgs &a, const LinearPlan &p, bool vec, hipStream_t s) {
  if (a.M <= 0) return hipSuccess;
  auto tile = [&](auto e, auto gated, auto v) { launch_tile<decltype(e), decltype(gated)::value, decltype(v)::value>(a, p, s); };
  auto by_vec = [&](auto e, auto gated) { vec ? tile(e, gated, std::true_type{}) : tile(e, gated, std::false_type{}); };
  auto by_gate = [&](auto e) { a.gated ? by_vec(e, std::true_type{}) : by_vec(e, std::false_type{}); };
  if (a.dtype == EXFOLD_BF16) by_gate(bf16_t{}); else by_gate(float{});
  if (p.ksplit > 1) {
    const long long n = (long long)a.M * ((a.N + 3) / 4);
    const int grid = (int)((n + 255) / 256);
    auto join = [&](auto gated, auto o) { linear_join<decltype(gated)::value, decltype(o)><<<grid, 256, 0, s>>>(a, p.ksplit); };
    if (a.out_dtype == EXFOLD_BF16)
      a.gated ? join(std::true_type{}, bf16_t{}) : join(std::false_type{}, bf16_t{});
    else
      a.gated ? join(std::true_type{}, float{}) : join(std::false_type{}, float{});
  }
  return hipGetLastError();
}

}  // namespace exfold
