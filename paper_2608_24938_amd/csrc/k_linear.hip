// Matrix product with bias, activation and residual in its epilogue (exfold_linear_forward):
//   y = act(x W^T + b) + r,   gated: y = act(x W_g^T + b_g) * (x W_u^T + b_u) + r
// float32 sums, one rounding to y's type.
#include "common.hpp"
#include "kernels.hpp"
#include "linear_epilogue.hpp"

namespace exfold {

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

// ---------------------------------------------------------------------------
// Few rows (serving a token or four): the weights are read once and nothing is staged.  A
// workgroup takes RW weight rows (gated: RW / 2 columns' gate and up rows) over the whole
// reduction, its 256 threads on consecutive 16-byte pieces of each (element loads where the
// rows allow no pieces), two sweeps of loads in flight, products in float32 on the vector
// units; the threads' sums are added by DPP within rows of 16 lanes and then in order through
// LDS.
// ---------------------------------------------------------------------------
// Elements of a 16-byte piece as float32.
template <typename E> __device__ __forceinline__ void unpack_piece(const u32x4 &v, float (&f)[16 / sizeof(E)]) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if constexpr (sizeof(E) == 2) {
      f[2 * q] = __uint_as_float(v[q] << 16);
      f[2 * q + 1] = __uint_as_float(v[q] & 0xffff0000u);
    } else {
      f[q] = __uint_as_float(v[q]);
    }
  }
}

// Sum over the 16 lanes of a DPP row; every lane of the row gets it.
__device__ __forceinline__ float row_sum(float v) {
  v += __uint_as_float(dpp_u32<0xB1>(__float_as_uint(v), 0u));
  v += __uint_as_float(dpp_u32<0x4E>(__float_as_uint(v), 0u));
  v += __uint_as_float(dpp_u32<0x141>(__float_as_uint(v), 0u));
  v += __uint_as_float(dpp_u32<0x140>(__float_as_uint(v), 0u));
  return v;
}

template <typename E, int MT, int RW, bool GATED, bool VEC>
__global__ __launch_bounds__(256) void linear_few(const LinearArgs a) {
  constexpr int EP = 16 / sizeof(E), U = 2, COLS = GATED ? RW / 2 : RW;
  __shared__ float part[16][RW * MT];
  const int tid = threadIdx.x, n0 = blockIdx.x * COLS;
  const E *x = static_cast<const E *>(a.x), *w = static_cast<const E *>(a.w);
  const E *xr[MT], *wr[RW];
#pragma unroll
  for (int m = 0; m < MT; ++m) xr[m] = x + (long long)min(m, a.M - 1) * a.ldx;
#pragma unroll
  for (int r = 0; r < RW; ++r) {
    const int n = min(n0 + (GATED ? r % COLS : r), a.N - 1);
    wr[r] = w + (long long)(GATED && r >= COLS ? a.N + n : n) * a.ldw;
  }
  float acc[RW][MT];
#pragma unroll
  for (int r = 0; r < RW; ++r)
#pragma unroll
    for (int m = 0; m < MT; ++m) acc[r][m] = 0.f;
  if constexpr (VEC) {
    for (int k = tid * EP; k < a.K; k += 256 * EP * U) {
      u32x4 wv[U][RW], xv[U][MT];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int ku = k + u * 256 * EP;
        const bool in = ku < a.K;
#pragma unroll
        for (int r = 0; r < RW; ++r) wv[u][r] = in ? *reinterpret_cast<const u32x4 *>(wr[r] + ku) : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
        for (int m = 0; m < MT; ++m) xv[u][m] = in ? *reinterpret_cast<const u32x4 *>(xr[m] + ku) : u32x4{0u, 0u, 0u, 0u};
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float xf[MT][EP];
#pragma unroll
        for (int m = 0; m < MT; ++m) unpack_piece<E>(xv[u][m], xf[m]);
#pragma unroll
        for (int r = 0; r < RW; ++r) {
          float wf[EP];
          unpack_piece<E>(wv[u][r], wf);
#pragma unroll
          for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int e = 0; e < EP; ++e) acc[r][m] = fmaf(wf[e], xf[m][e], acc[r][m]);
        }
      }
    }
  } else {
    constexpr int UE = 4;
    for (int k = tid; k < a.K; k += 256 * UE) {
      E wv[UE][RW], xv[UE][MT];
#pragma unroll
      for (int u = 0; u < UE; ++u) {
        const int ku = k + u * 256;
        const bool in = ku < a.K;
#pragma unroll
        for (int r = 0; r < RW; ++r) wv[u][r] = in ? wr[r][ku] : E(0);
#pragma unroll
        for (int m = 0; m < MT; ++m) xv[u][m] = in ? xr[m][ku] : E(0);
      }
#pragma unroll
      for (int u = 0; u < UE; ++u)
#pragma unroll
        for (int r = 0; r < RW; ++r)
#pragma unroll
          for (int m = 0; m < MT; ++m) acc[r][m] = fmaf(load_f32(&wv[u][r]), load_f32(&xv[u][m]), acc[r][m]);
    }
  }
#pragma unroll
  for (int r = 0; r < RW; ++r)
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      const float v = row_sum(acc[r][m]);
      if ((tid & 15) == 0) part[tid >> 4][m * RW + r] = v;
    }
  __syncthreads();
  if (tid >= COLS * MT) return;
  const int m = tid / COLS, c = tid % COLS, n = n0 + c;
  if (m >= a.M || n >= a.N) return;
  float z = 0.f, g = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    z += part[i][m * RW + c];
    if (GATED) g += part[i][m * RW + COLS + c];
  }
  if (sizeof(E) == 4 || a.out_dtype == EXFOLD_F32)
    finish1<GATED, float>(a, m, n, z, g);
  else if constexpr (sizeof(E) == 2)
    finish1<GATED, bf16_t>(a, m, n, z, g);
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
constexpr int kFewRows = 4;

LinearPlan plan_linear(int dtype, bool gated, bool vec, int M, int N, int K, int cu_count) {
  LinearPlan p{};
  p.ksplit = 1;
  p.kc = K;
  const long long wrows = (long long)N * (gated ? 2 : 1);
  if (M <= kFewRows) {
    p.kind = kLinFew;
    p.bm = M <= 1 ? 1 : M <= 2 ? 2 : 4;
    p.bn = wrows >= 16LL * cu_count ? 8 : 2;
    const int cols = gated ? p.bn / 2 : p.bn;
    p.grid = (N + cols - 1) / cols;
    return p;
  }
  if (dtype == EXFOLD_BF16 && vec && K % 64 == 0 && K >= 128) {
    // 256 x 256 tiles, one a CU, where they fill the chip
    const long long tiles = (long long)((M + 255) / 256) * ((wrows + 255) / 256);
    if (4 * tiles >= 3 * cu_count) {
      p.kind = kLinWide;
      p.bm = p.bn = 256;
      p.grid = (int)tiles;
      return p;
    }
  }
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
static void launch_few(const LinearArgs &a, const LinearPlan &p, hipStream_t s) {
  auto go = [&](auto mt) {
    constexpr int MT = decltype(mt)::value;
    if (p.bn == 8) linear_few<E, MT, 8, GATED, VEC><<<p.grid, 256, 0, s>>>(a);
    else linear_few<E, MT, 2, GATED, VEC><<<p.grid, 256, 0, s>>>(a);
  };
  if (p.bm == 1) go(std::integral_constant<int, 1>{});
  else if (p.bm == 2) go(std::integral_constant<int, 2>{});
  else go(std::integral_constant<int, 4>{});
}

template <typename E, bool GATED, bool VEC>
static void launch_typed(const LinearArgs &a, const LinearPlan &p, hipStream_t s) {
  if (p.kind == kLinFew) launch_few<E, GATED, VEC>(a, p, s);
  else linear_tile<E, 64, 128, GATED, VEC><<<p.grid, 256, 0, s>>>(a, p);
}

hipError_t launch_linear(const LinearArgs &a, const LinearPlan &p, bool vec, hipStream_t s) {
  if (a.M <= 0) return hipSuccess;
  if (p.kind == kLinWide) return launch_linear_wide(a, p, s);
  auto typed = [&](auto e, auto gated) {
    using E = decltype(e);
    constexpr bool G = decltype(gated)::value;
    vec ? launch_typed<E, G, true>(a, p, s) : launch_typed<E, G, false>(a, p, s);
  };
  auto by_gate = [&](auto e) { a.gated ? typed(e, std::true_type{}) : typed(e, std::false_type{}); };
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
