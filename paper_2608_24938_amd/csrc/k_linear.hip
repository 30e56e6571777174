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
// bf16 or 32 float32 columns) of every row in LDS, its 16-byte pieces swizzled so that a
// fragment read spreads over the banks.  A lane's piece of a row feeds one 32x32x16 bf16 MFMA
// or four 32x32x2 float32 ones (any assignment of columns to steps is a valid order).  Rows
// past the ends re-read the last one and are not stored; columns past K are zero.
// ---------------------------------------------------------------------------
template <typename E> constexpr int mma_steps() { return sizeof(E) == 2 ? 1 : 4; }
template <typename E> __device__ __forceinline__ void mma32(const u32x4 &a, const u32x4 &b, int e, f32x16 &c) {
  if constexpr (sizeof(E) == 2)
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[e]), __uint_as_float(b[e]), c, 0, 0, 0);
}

// LDS slot (16-byte units) of piece q of tile row r (8 pieces a row).
__device__ __forceinline__ int piece_at(int r, int q) { return r * 8 + (q ^ ((r ^ (r >> 1)) & 7)); }

// A wave's TM x TN tiles of sums into LDS, row-major: register r of tile (i, j) is row arow(i) +
// lane % 32, column brow(j) + 8 (r / 4) + 4 (lane / 32) + r % 4 (the weights are the MFMA's first
// operand): runs of four columns.
template <int PITCH, int TM, int TN, typename RowA, typename RowB>
__device__ __forceinline__ void sums_to_lds(float *red, const f32x16 (&acc)[TM][TN], int lane, const RowA &arow,
                                            const RowB &brow) {
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<f32x4 *>(red + (arow(i) + (lane & 31)) * PITCH + brow(j) + 8 * g + 4 * (lane >> 5)) =
            f32x4{acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
}
// Outputs or partial sums of a tile from its sums in LDS (all threads, after a barrier).
template <typename E, int BM, int COLS, int PITCH, int COPIES, bool GATED>
__device__ __forceinline__ void tile_out(const LinearArgs &a, const LinearPlan &p, const float *red, int mt, int nt, int ks) {
  const int rows = min(BM, a.M - mt * BM);
  if (p.ksplit > 1)
    store_partial<GATED, COLS, PITCH, COPIES, 256>(a, ks, red, BM * PITCH, mt * BM, nt * COLS, rows);
  else if (sizeof(E) == 4 || a.out_dtype == EXFOLD_F32)
    finish_tile<GATED, float, COLS, PITCH, COPIES, 256>(a, red, BM * PITCH, mt * BM, nt * COLS, rows);
  else if constexpr (sizeof(E) == 2)
    finish_tile<GATED, bf16_t, COLS, PITCH, COPIES, 256>(a, red, BM * PITCH, mt * BM, nt * COLS, rows);
}

// A 16-byte piece of a row at any element alignment, `left` elements of which exist (the rest 0).
template <typename E> __device__ __forceinline__ u32x4 load_piece(const E *p, int left) {
  constexpr int EP = 16 / sizeof(E);
  u32x4 v = {0u, 0u, 0u, 0u};
  if (left >= EP) {
    __builtin_memcpy(&v, p, 16);
  } else {
#pragma unroll
    for (int e = 0; e < EP - 1; ++e)
      if (e < left) {
        if constexpr (sizeof(E) == 2) v[e / 2] |= (uint32_t)p[e] << (16 * (e & 1));
        else v[e] = __float_as_uint(p[e]);
      }
  }
  return v;
}

// Rows at any alignment: the stages pass through registers into one of two LDS buffers, loaded in
// 16-byte pieces that may lie across 16-byte borders (elements at a row's end), two stages ahead.
template <typename E, int BM, int BN, bool GATED>
__global__ __launch_bounds__(256, 2) void linear_tile(const LinearArgs a, const LinearPlan p) {
  constexpr int EP = 16 / sizeof(E), KS = 8 * EP;
  constexpr int TM = BM / 64, TN = BN / 64, COLS = GATED ? BN / 2 : BN;
  constexpr int PA = BM * 8 / 256, PB = BN * 8 / 256;  // pieces a thread
  static_assert(!GATED || TN % 2 == 0, "a wave holds the gate and the up columns");
  constexpr int PITCH = BN + 4;  // floats of a row of sums
  static_assert(BM * PITCH * 4 <= 2 * (BM + BN) * 128, "the sums fit the stages");
  __shared__ __attribute__((aligned(16))) u32x4 smem[2][(BM + BN) * 8];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wm = wave >> 1, wn = wave & 1;
  const int mts = (a.M + BM - 1) / BM, nts = (a.N + COLS - 1) / COLS;
  int mt, nt, ks;
  tile_of(xcd_remap(blockIdx.x, mts * nts * p.ksplit), mts, nts, mt, nt, ks);
  const int k0 = ks * p.kc, k1 = min(a.K, k0 + p.kc), kq = (tid & 7) * EP;
  const E *sa[PA], *sb[PB];
#pragma unroll
  for (int i = 0; i < PA; ++i)
    sa[i] = static_cast<const E *>(a.x) + min(mt * BM + i * 32 + (tid >> 3), a.M - 1) * a.ldx + kq;
#pragma unroll
  for (int i = 0; i < PB; ++i) {
    const int r = i * 32 + (tid >> 3), c = min(nt * COLS + (GATED ? r & (COLS - 1) : r), a.N - 1);
    sb[i] = static_cast<const E *>(a.w) + (GATED && r >= COLS ? a.N + c : c) * a.ldw + kq;
  }
  // two register sets: the loads of a stage fly during the MFMAs of the two before it
  u32x4 ra0[PA], rb0[PB], ra1[PA], rb1[PB];
  auto load = [&](int k, u32x4 (&ra)[PA], u32x4 (&rb)[PB]) __attribute__((always_inline)) {
    const int left = k1 - k - kq;
    if (k + KS <= k1) {
#pragma unroll
      for (int i = 0; i < PA; ++i) __builtin_memcpy(&ra[i], sa[i] + k, 16);
#pragma unroll
      for (int i = 0; i < PB; ++i) __builtin_memcpy(&rb[i], sb[i] + k, 16);
    } else {
#pragma unroll
      for (int i = 0; i < PA; ++i) ra[i] = load_piece(sa[i] + k, left);
#pragma unroll
      for (int i = 0; i < PB; ++i) rb[i] = load_piece(sb[i] + k, left);
    }
  };
  auto stage = [&](int buf, const u32x4 (&ra)[PA], const u32x4 (&rb)[PB]) __attribute__((always_inline)) {
    u32x4 *As = smem[buf], *Bs = As + BM * 8;
#pragma unroll
    for (int i = 0; i < PA; ++i) As[piece_at(i * 32 + (tid >> 3), tid & 7)] = ra[i];
#pragma unroll
    for (int i = 0; i < PB; ++i) Bs[piece_at(i * 32 + (tid >> 3), tid & 7)] = rb[i];
  };
  f32x16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
  // tile row of a wave's column block j: blocks wn, wn + 2, ... (gated: gate and up blocks in step)
  auto arow = [&](int i) { return (i * 2 + wm) * 32; };
  auto brow = [&](int j) { return (j * 2 + wn) * 32; };
  auto multiply = [&](int buf) __attribute__((always_inline)) {
    const u32x4 *As = smem[buf], *Bs = As + BM * 8;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      u32x4 fa[TM], fb[TN];
#pragma unroll
      for (int i = 0; i < TM; ++i) fa[i] = As[piece_at(arow(i) + (lane & 31), 2 * s + (lane >> 5))];
#pragma unroll
      for (int j = 0; j < TN; ++j) fb[j] = Bs[piece_at(brow(j) + (lane & 31), 2 * s + (lane >> 5))];
#pragma unroll
      for (int e = 0; e < mma_steps<E>(); ++e)
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int j = 0; j < TN; ++j) mma32<E>(fb[j], fa[i], e, acc[i][j]);
    }
  };
  load(k0, ra0, rb0);
  load(k0 + KS, ra1, rb1);
  stage(0, ra0, rb0);
  __syncthreads();
  for (int k = k0; k < k1; k += 2 * KS) {
    load(k + 2 * KS, ra0, rb0);
    multiply(0);
    stage(1, ra1, rb1);
    __syncthreads();
    if (k + KS >= k1) break;
    load(k + 3 * KS, ra1, rb1);
    multiply(1);
    stage(0, ra0, rb0);
    __syncthreads();
  }
  // the last stage's barrier is behind every wave's reads
  __syncthreads();
  float *red = reinterpret_cast<float *>(&smem[0][0]);
  sums_to_lds<PITCH>(red, acc, lane, arow, brow);
  __syncthreads();
  tile_out<E, BM, COLS, PITCH, 1, GATED>(a, p, red, mt, nt, ks);
}

// ---------------------------------------------------------------------------
// Ring tiles (rows in 16-byte pieces, more than four of them): BM rows x BN weight rows as
// above, but the stages go from global memory straight into an LDS ring of S buffers, S - 1
// stages ahead, with one barrier a stage: a wave waits until its own loads of the stage have
// landed and its LDS reads of the last one have ended, meets the others, refills the buffer
// they all have left, and multiplies.  Stages past the end of the range, and pieces past K,
// read zeros from a constant, so that every wave has the same number of loads in flight at
// every wait.
// KW: the four waves take one 16-byte step of a stage each on the whole tile instead of a
// quarter of the tile (few rows: the tile is small and the weights stream), and their sums are
// added in wave order through LDS.
// ONCE: one tile of rows, so no other workgroup reads these weights: non-temporal loads (16
// rows on 28672 x 4096 weights 48.1 -> 42.6 us; 8 on 4096 x 4096, which fit the last-level
// cache, 11.8 -> 11.5).
// ---------------------------------------------------------------------------
__device__ const u32x4 kZeroPiece[8] = {};

// One 16-byte piece a lane from global g into the 1 KiB LDS block at byte address lds
// (wave-uniform): lane l lands at lds + 16 l.  M0 holds the block address; nothing else in
// these kernels uses M0 (no indirect register moves).
template <bool ONCE> __device__ __forceinline__ void ring_load(const char *g, uint32_t lds) {
  if constexpr (ONCE)
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off nt" : : "v"(g), "s"(lds) : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(g), "s"(lds) : "memory", "m0");
}

template <typename E, int BM, int BN, int S, bool KW, bool GATED, bool ONCE>
__global__ __launch_bounds__(256, BM == 128 && S > 2 ? 1 : 2) void linear_ring(const LinearArgs a, const LinearPlan p) {
  constexpr int EP = 16 / sizeof(E), KS = 8 * EP, ROWS = BM + BN, NB = ROWS / 32;
  constexpr int TM = KW ? BM / 32 : BM / 64, TN = KW ? BN / 32 : BN / 64;
  constexpr int COLS = GATED ? BN / 2 : BN;
  static_assert(!GATED || TN % 2 == 0, "a wave holds the gate and the up columns");
  constexpr int PITCH = BN + 4;  // floats of a row of the waves' sums
  constexpr int RING = S * ROWS * 8, RED = (KW ? 4 : 1) * BM * PITCH / 4;
  __shared__ __attribute__((aligned(1024))) u32x4 smem[RING > RED ? RING : RED];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = KW ? 0 : wave >> 1, wn = KW ? 0 : wave & 1;
  const int mts = (a.M + BM - 1) / BM, nts = (a.N + COLS - 1) / COLS;
  int mt, nt, ks;
  tile_of(xcd_remap(blockIdx.x, mts * nts * p.ksplit), mts, nts, mt, nt, ks);
  const int k0 = ks * p.kc, k1 = min(a.K, k0 + p.kc), stages = (k1 - k0 + KS - 1) / KS;

  // 1 KiB block i of this wave: rows 8 (4 i + wave) .. + 7 of the stage, x rows first
  const char *src[NB];
  int kq[NB];  // this lane's piece of the row, in elements
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    const int r = 8 * (4 * i + wave) + (lane >> 3), q = (lane & 7) ^ ((r ^ (r >> 1)) & 7);
    const E *row;
    if (i < BM / 32) {
      row = static_cast<const E *>(a.x) + min(mt * BM + r, a.M - 1) * a.ldx;
    } else {
      const int b = r - BM, c = min(nt * COLS + (GATED ? b & (COLS - 1) : b), a.N - 1);
      row = static_cast<const E *>(a.w) + (GATED && b >= COLS ? a.N + c : c) * a.ldw;
    }
    kq[i] = k0 + q * EP;
    src[i] = reinterpret_cast<const char *>(row + kq[i]);
  }
  const uint32_t lds0 = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void *)smem + wave * 1024;
  auto issue = [&](int st, int slot) __attribute__((always_inline)) {
    const uint32_t to = lds0 + slot * (ROWS * 128);
    if (st < stages - 1) {
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        if (i < BM / 32) ring_load<false>(src[i] + (long long)st * 128, to + i * 4096);
        else ring_load<ONCE>(src[i] + (long long)st * 128, to + i * 4096);
      }
    } else {
#pragma unroll
      for (int i = 0; i < NB; ++i)
        ring_load<false>(kq[i] + st * KS < k1 ? src[i] + (long long)st * 128 : reinterpret_cast<const char *>(kZeroPiece), to + i * 4096);
    }
  };
  f32x16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
  auto arow = [&](int i) { return KW ? i * 32 : (i * 2 + wm) * 32; };
  auto brow = [&](int j) { return KW ? j * 32 : (j * 2 + wn) * 32; };

  constexpr int STEPS = KW ? 1 : 4;
  u32x4 fa[TM], fb[TN], na[TM], nb[TN];  // fragments of a step and of the next
  // byte offsets in a buffer of this lane's piece of step s in the wave's first row blocks; the
  // others are whole blocks further (the swizzle repeats every 16 rows)
  uint32_t at_a[STEPS], at_b[STEPS];
#pragma unroll
  for (int s = 0; s < STEPS; ++s) {
    const int q = 2 * (KW ? wave : s) + (lane >> 5);
    at_a[s] = piece_at(arow(0) + (lane & 31), q) * 16;
    at_b[s] = (BM * 8 + piece_at(brow(0) + (lane & 31), q)) * 16;
  }
  constexpr int STEP_ROWS = KW ? 32 : 64;
  auto read = [&](int slot, int s, u32x4 (&ra)[TM], u32x4 (&rb)[TN]) __attribute__((always_inline)) {
    const char *base = reinterpret_cast<const char *>(smem) + slot * (ROWS * 128);
#pragma unroll
    for (int j = 0; j < TN; ++j) rb[j] = *reinterpret_cast<const u32x4 *>(base + at_b[s] + j * STEP_ROWS * 128);
#pragma unroll
    for (int i = 0; i < TM; ++i) ra[i] = *reinterpret_cast<const u32x4 *>(base + at_a[s] + i * STEP_ROWS * 128);
    __builtin_amdgcn_sched_barrier(0);  // read now: the products of the step before cover the latency
  };
  auto multiply = [&](const u32x4 (&ra)[TM], const u32x4 (&rb)[TN]) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < mma_steps<E>(); ++e)
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) mma32<E>(rb[j], ra[i], e, acc[i][j]);
    __builtin_amdgcn_sched_barrier(0);
  };
#pragma unroll
  for (int st = 0; st < S; ++st) issue(st, st);
  asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" : : "n"((S - 1) * NB) : "memory");
  read(0, 0, fa, fb);
  int slot = 0;
  for (int st = 0; st < stages; ++st) {
#pragma unroll
    for (int s = 0; s < STEPS - 1; s += 2) {
      read(slot, s + 1, na, nb);
      multiply(fa, fb);
      if (s + 2 < STEPS) {
        read(slot, s + 2, fa, fb);
        multiply(na, nb);
      }
    }
    // the next stage has landed and this one is read: its buffer is filled again
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"((S - 2) * NB) : "memory");
    issue(st + S, slot);
    slot = slot == S - 1 ? 0 : slot + 1;
    if constexpr (STEPS > 1) {
      read(slot, 0, fa, fb);
      multiply(na, nb);
    } else {
      read(slot, 0, na, nb);
      multiply(fa, fb);
#pragma unroll
      for (int i = 0; i < TM; ++i) fa[i] = na[i];
#pragma unroll
      for (int j = 0; j < TN; ++j) fb[j] = nb[j];
    }
  }
  // no load into the ring is left, and every wave has read it
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" : : : "memory");

  float *red = reinterpret_cast<float *>(smem);
  sums_to_lds<PITCH>(red + (KW ? wave * BM * PITCH : 0), acc, lane, arow, brow);
  __syncthreads();
  tile_out<E, BM, COLS, PITCH, KW ? 4 : 1, GATED>(a, p, red, mt, nt, ks);
}

// ---------------------------------------------------------------------------
// Few rows (serving a token or four; a few times four where the weights are small): nothing is
// staged.  A workgroup takes MT rows and RW weight rows (gated: RW / 2 columns' gate and up
// rows) over the whole reduction, its 256 threads on consecutive 16-byte pieces of each (VEC:
// the rows start on 16 bytes and hold whole pieces), two sweeps of loads in flight, products
// in float32 on the vector units; the threads' sums are added by DPP within rows of 16 lanes
// and then in order through LDS.  One token, 2 x 1408 weight rows of 4096: 5.6 us, 4.1 TB/s.
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
  const int tid = threadIdx.x, n0 = blockIdx.x * COLS, m0 = blockIdx.y * MT;
  const E *x = static_cast<const E *>(a.x), *w = static_cast<const E *>(a.w);
  const E *xr[MT], *wr[RW];
#pragma unroll
  for (int m = 0; m < MT; ++m) xr[m] = x + (long long)min(m0 + m, a.M - 1) * a.ldx;
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
  auto piece = [&](const E *row, int k) {
    if constexpr (VEC)
      return k < a.K ? *reinterpret_cast<const u32x4 *>(row + k) : u32x4{0u, 0u, 0u, 0u};
    else
      return load_piece(row + k, a.K - k);
  };
  for (int k = tid * EP; k < a.K; k += 256 * EP * U) {
    u32x4 wv[U][RW], xv[U][MT];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int ku = k + u * 256 * EP;
#pragma unroll
      for (int r = 0; r < RW; ++r) wv[u][r] = piece(wr[r], ku);
#pragma unroll
      for (int m = 0; m < MT; ++m) xv[u][m] = piece(xr[m], ku);
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
  if (m0 + m >= a.M || n >= a.N) return;
  float z = 0.f, g = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    z += part[i][m * RW + c];
    if (GATED) g += part[i][m * RW + COLS + c];
  }
  if (sizeof(E) == 4 || a.out_dtype == EXFOLD_F32)
    finish1<GATED, float>(a, m0 + m, n, z, g);
  else if constexpr (sizeof(E) == 2)
    finish1<GATED, bf16_t>(a, m0 + m, n, z, g);
}

// Joins the split partial sums in order, four columns a thread, and finishes them.
template <bool GATED, typename O>
__global__ __launch_bounds__(256) void linear_join(const LinearArgs a, int ksplit) {
  const int np = linear_part_cols(a.N), quads_n = np / 4;
  const long long ld = (long long)np * (GATED ? 2 : 1), split = a.M * ld;
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  if (i >= (long long)a.M * quads_n) return;
  const long long m = i / quads_n;
  const int n = (int)(i % quads_n) * 4;
  const float *row = a.part + m * ld + n;
  f32x4 zs = {0.f, 0.f, 0.f, 0.f}, us = zs;
#pragma unroll 8
  for (int s = 0; s < ksplit; ++s) {
    zs += *reinterpret_cast<const f32x4 *>(row + s * split);
    if (GATED) us += *reinterpret_cast<const f32x4 *>(row + s * split + np);
  }
  f32x4 bz, bu, r = {0.f, 0.f, 0.f, 0.f};
  bias_quad<GATED>(a, n, bz, bu);
  if (a.res) r = load_quad(static_cast<const O *>(a.res) + m * a.ldr, n, a.N);
  with_act(a.act, [&](auto act) { finish_quad<decltype(act)::value, GATED, O>(a, m, n, zs, us, bz, bu, r); });
}

// ---------------------------------------------------------------------------
// Planning and launch.
// ---------------------------------------------------------------------------
constexpr int kFewRows = 4, kFewMost = 64;  // rows: always, at most (of more than 8 weight rows), on the vector units

// Tiles, what a stage of one takes a CU that holds one workgroup of them or several in turn,
// and what a tile takes besides (first loads, epilogue); measured, microseconds.  bf16: the
// bytes of the stage at about 65 GB/s a CU, wide tiles by their MFMAs; float32: the MFMAs.  The
// register-staged tiles wait for their loads, and two workgroups a CU overlap.
struct TileCost {
  int kind, bm, bn;
  float bf16, f32, once;
};
constexpr TileCost kTiles[] = {{kLinRing, 32, 64, 0.19f, 0.35f, 1.6f},  {kLinRing, 64, 64, 0.24f, 0.66f, 2.3f},
                               {kLinRing, 64, 128, 0.36f, 1.16f, 3.2f}, {kLinRing, 128, 128, 0.52f, 2.33f, 7.f},
                               {kLinWide, 256, 256, 1.5f, 0.f, 10.f},   {kLinTile, 64, 128, 1.1f, 1.6f, 3.2f}};

// Rows [0, rows_x) of x and [0, rows_w) of w, copied to rows of kp elements (whole pieces, zeros
// behind K) at 16-byte alignment, a piece a thread at a time.
template <typename E>
__global__ __launch_bounds__(256) void linear_copy(const LinearArgs a, const E *x, const E *w, E *to_x, E *to_w,
                                                  long long rows_x, long long rows_w, int kp) {
  constexpr int EP = 16 / sizeof(E);
  const int pieces = kp / EP;
  const long long n = (rows_x + rows_w) * pieces;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) {
    const long long r = i / pieces;
    const int k = (int)(i % pieces) * EP;
    const bool of_x = r < rows_x;
    const E *src = of_x ? x + r * a.ldx : w + (r - rows_x) * a.ldw;
    E *dst = of_x ? to_x + r * kp : to_w + (r - rows_x) * kp;
    *reinterpret_cast<u32x4 *>(dst + k) = load_piece(src + k, a.K - k);
  }
}

// The tile and split of the least estimated time: rounds of tiles over the CUs, or the
// weights' and rows' bytes from memory (about 4.8 TB/s) where those take longer, and for a
// split its partial sums, written and read, and the launch that joins them.  The estimate
// picks among kernels that all are right (600 x 2048 x 768 float32: taken 32 x 64 tiles, 29 us, 64 x
// 128 33 and 128 x 128 34; 64 x 4096 x 4096 bf16: taken a split in four, 13.4 us, none 15.3).  It
// charges a whole round for every cu_count ring tiles, though two of 64 x 64 share a CU, and so
// passes over them where they are a few more than the CUs (777 x 1408 x 1024 bf16: taken 64 x 128,
// 13.4 us, 64 x 64 12.4, 32 x 64 15.5, 128 x 128 19.7).
static double plan_tiles(bool bf16, bool gated, bool vec, int M, int N, int K, int cu_count, LinearPlan &p) {
  p = LinearPlan{};
  p.vec = vec;
  p.K = K;
  const long long wrows = (long long)N * (gated ? 2 : 1);
  const int stage = bf16 ? 64 : 32, stages = (K + stage - 1) / stage;
  const double memory = ((double)wrows * K + (double)M * K) * (bf16 ? 2 : 4) / 4.8e6;  // us
  double best = 0.0;
  for (const TileCost &t : kTiles) {
    if ((t.kind == kLinTile) == vec) continue;
    if (t.kind == kLinWide && (!bf16 || K % 64 != 0 || K < 128)) continue;
    const int cols = gated ? t.bn / 2 : t.bn;
    const long long tiles = (long long)((M + t.bm - 1) / t.bm) * ((N + cols - 1) / cols);
    for (int fill = 0; fill <= 2; ++fill) {  // not split, or one or two workgroups a CU
      long long split = 1;
      if (fill > 0) {
        split = fill * (long long)cu_count / tiles;
        if (split > stages / 6) split = stages / 6;
        if (split > 32) split = 32;
        if (split < 2 || t.kind == kLinWide) continue;
      }
      const int per = (int)((stages + split - 1) / split), ksplit = (stages + per - 1) / per;
      const long long wgs = tiles * ksplit, round = t.kind == kLinTile ? 2 * cu_count : cu_count;
      double us = (double)((wgs + round - 1) / round) * (per * (bf16 ? t.bf16 : t.f32) + t.once);
      // few streams are slower, and tiles of rows drift apart, so their weights come again
      const int again = (M + t.bm - 1) / t.bm - 1;
      const double slow = memory * ((2 * wgs < 3 * cu_count ? 1.15 : 1.0) + 0.2 * (again < 3 ? again : 3));
      if (us < slow && memory > 10.0) us = slow + 0.05 * us;
      if (ksplit > 1) us += 4.0 + ksplit * (double)M * wrows * 8 / 4e6;
      if (best > 0.0 && us >= best) continue;
      best = us;
      p.kind = t.kind;
      p.bm = t.bm;
      p.bn = t.bn;
      p.ksplit = ksplit;
      p.kc = ksplit > 1 ? per * stage : K;
      p.grid = (int)(tiles * ksplit);
      p.shared_cu = p.grid > cu_count;
    }
  }
  return best;
}

LinearPlan plan_linear(int dtype, bool gated, bool vec_x, bool vec_w, int M, int N, int K, int cu_count) {
  LinearPlan p{};
  const bool bf16 = dtype == EXFOLD_BF16, whole = K % (bf16 ? 8 : 4) == 0;
  const long long wrows = (long long)N * (gated ? 2 : 1);
  // Rows in groups of four on the vector units: the weights pass once a group and the rows once
  // a block of weight rows, mostly from the caches, at half the rate where pieces lie across
  // 16-byte borders; a round of workgroups takes its loads' latency whatever they read (8 x 343 x
  // 498 float32 at odd strides 3.7 us, 10.4 copied to tiles; 16 x 128 x 2048 bf16 3.3 and 6.9; 10
  // x 2 x 4464 x 120 float32, 3348 workgroups, 15.0).
  const int few_rows = M <= 1 ? 1 : M <= 2 ? 2 : 4, few_cols = (wrows >= 16LL * cu_count ? 8 : 2) / (gated ? 2 : 1);
  const int groups = (M + few_rows - 1) / few_rows, blocks = (N + few_cols - 1) / few_cols, esz = bf16 ? 2 : 4;
  const bool few_fits = M <= kFewMost || (wrows <= 8 && M <= (1 << 16));
  const double few = ((double)groups * wrows * K / 5e6 + (double)blocks * M * K / 10e6) * esz * (vec_w && whole ? 1 : 2) +
                     (double)groups * wrows * K * 4 / 30e6 +
                     2.5 * (double)(((long long)groups * blocks - 1) / ((few_cols > 2 ? 3 : 6) * (long long)cu_count) + 1);  // us
  auto take_few = [&] {
    p = LinearPlan{};
    p.kind = kLinFew;
    p.vec = vec_x && vec_w && whole;
    p.K = p.kc = K;
    p.ksplit = 1;
    p.bm = few_rows;
    p.bn = few_cols * (gated ? 2 : 1);
    p.grid = blocks * groups;
    return p;
  };
  if (M <= kFewRows) return take_few();
  if (vec_x && vec_w && whole) {
    const double tiles = plan_tiles(bf16, gated, true, M, N, K, cu_count, p);
    return few_fits && few < tiles ? take_few() : p;
  }
  // as the rows lie, or copied first: one launch more, the copies written and read.  Where K is no
  // whole number of pieces both operands are copied, with zeros up to a whole stage; else only
  // rows that start elsewhere are, and the length stays K for both.
  const double direct = plan_tiles(bf16, gated, false, M, N, K, cu_count, p);
  const int stage = bf16 ? 64 : 32, kp = whole ? K : (K + stage - 1) / stage * stage;
  const bool px = !vec_x || !whole, pw = !vec_w || !whole;
  LinearPlan q;
  const double copied = plan_tiles(bf16, gated, true, M, N, kp, cu_count, q) + 3.0 +
                        ((px ? M : 0) + (pw ? (double)wrows : 0.0)) * kp * (bf16 ? 2 : 4) * 2 / 4e6;
  if (few_fits && few < direct && few < copied) return take_few();
  if (copied < direct) {
    p = q;
    p.copy_x = px;
    p.copy_w = pw;
  }
  return p;
}

template <typename E, bool GATED, bool VEC>
static void launch_few(const LinearArgs &a, const LinearPlan &p, hipStream_t s) {
  auto go = [&](auto mt) {
    constexpr int MT = decltype(mt)::value;
    const int y = (a.M + MT - 1) / MT;
    const dim3 grid(p.grid / y, y);
    if (p.bn == 8) linear_few<E, MT, 8, GATED, VEC><<<grid, 256, 0, s>>>(a);
    else linear_few<E, MT, 2, GATED, VEC><<<grid, 256, 0, s>>>(a);
  };
  if (p.bm == 1) go(std::integral_constant<int, 1>{});
  else if (p.bm == 2) go(std::integral_constant<int, 2>{});
  else go(std::integral_constant<int, 4>{});
}

template <typename E, bool GATED, bool VEC>
static void launch_typed(const LinearArgs &a, const LinearPlan &p, hipStream_t s) {
  if (p.kind == kLinFew) {
    launch_few<E, GATED, VEC>(a, p, s);
  } else if constexpr (VEC) {
    // Buffers: as many stages as two workgroups a CU leave room for where the loads are waited
    // for, few where several workgroups a CU cover each other: float32 on 32 x 64 tiles (600 x
    // 2048 x 768: three 29.0 us, six 32.2), 128 x 128 tiles that are more than the CUs (2048 x 4096
    // x 4096: two 76.2 us, four 87.6; 128 x 28672 x 4096, 224 tiles: 74.6, 63.6; float32 ones are
    // always more, the plan estimates fewer behind twice as many of 64 x 128), and reductions of
    // two stages on 64 x 128 tiles (5498 x 7744 x 64: two 74.5 us, three 101.6).
    constexpr int S32 = sizeof(E) == 4 ? 3 : 6;
    const bool once = a.M <= p.bm;
    if (p.bm == 32 && once) linear_ring<E, 32, 64, S32, true, GATED, true><<<p.grid, 256, 0, s>>>(a, p);
    else if (p.bm == 32) linear_ring<E, 32, 64, S32, true, GATED, false><<<p.grid, 256, 0, s>>>(a, p);
    else if (p.bn == 64 && once) linear_ring<E, 64, 64, 4, true, GATED, true><<<p.grid, 256, 0, s>>>(a, p);
    else if (p.bn == 64) linear_ring<E, 64, 64, 4, true, GATED, false><<<p.grid, 256, 0, s>>>(a, p);
    else if (p.bm == 64 && p.kc <= 2 * 128 / (int)sizeof(E)) linear_ring<E, 64, 128, 2, false, GATED, false><<<p.grid, 256, 0, s>>>(a, p);
    else if (p.bm == 64) linear_ring<E, 64, 128, 3, false, GATED, false><<<p.grid, 256, 0, s>>>(a, p);
    else if (sizeof(E) == 4 || p.shared_cu) linear_ring<E, 128, 128, 2, false, GATED, false><<<p.grid, 256, 0, s>>>(a, p);
    else if constexpr (sizeof(E) == 2) linear_ring<E, 128, 128, 4, false, GATED, false><<<p.grid, 256, 0, s>>>(a, p);
  } else {
    linear_tile<E, 64, 128, GATED><<<p.grid, 256, 0, s>>>(a, p);
  }
}

template <typename E>
static void launch_copy(LinearArgs &a, const LinearPlan &p, hipStream_t s) {
  const long long rows_x = p.copy_x ? a.M : 0, rows_w = p.copy_w ? (long long)a.N * (a.gated ? 2 : 1) : 0;
  const long long n = (rows_x + rows_w) * (p.K / (16 / (int)sizeof(E)));
  E *to_x = static_cast<E *>(a.copied_x), *to_w = static_cast<E *>(a.copied_w);
  const long long blocks = (n + 255) / 256 < 16384 ? (n + 255) / 256 : 16384;
  linear_copy<E><<<(unsigned)blocks, 256, 0, s>>>(a, static_cast<const E *>(a.x), static_cast<const E *>(a.w), to_x,
                                                         to_w, rows_x, rows_w, p.K);
  if (p.copy_x) {
    a.x = to_x;
    a.ldx = p.K;
  }
  if (p.copy_w) {
    a.w = to_w;
    a.ldw = p.K;
  }
}

hipError_t launch_linear(const LinearArgs &args, const LinearPlan &p, hipStream_t s) {
  if (args.M <= 0) return hipSuccess;
  LinearArgs a = args;
  if (p.copy_x || p.copy_w) {
    if (a.dtype == EXFOLD_BF16) launch_copy<bf16_t>(a, p, s);
    else launch_copy<float>(a, p, s);
    a.K = p.K;
  }
  if (p.kind == kLinWide) return launch_linear_wide(a, p, s);
  auto typed = [&](auto e, auto gated) {
    using E = decltype(e);
    constexpr bool G = decltype(gated)::value;
    p.vec ? launch_typed<E, G, true>(a, p, s) : launch_typed<E, G, false>(a, p, s);
  };
  auto by_gate = [&](auto e) { a.gated ? typed(e, std::true_type{}) : typed(e, std::false_type{}); };
  if (a.dtype == EXFOLD_BF16) by_gate(bf16_t{}); else by_gate(float{});
  if (p.ksplit > 1) {
    const long long n = (long long)a.M * (linear_part_cols(a.N) / 4);
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
