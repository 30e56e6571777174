// Routing of tokens to experts from router logits: softmax or sigmoid scores over all
// experts, a bias that steers the selection only, group-limited selection, renormalised
// and scaled weights (exfold_route_experts; the rules stand in the header).
#include "common.hpp"
#include "kernels.hpp"

namespace exfold {

// Sixteen lanes a token, four tokens a wave: lane q of the sixteen (one DPP row, so every
// exchange between them stays in registers) holds experts R q .. R q + R - 1.
template <int CTRL> __device__ __forceinline__ double dpp_f64(double v) {
  const uint64_t b = (uint64_t)__double_as_longlong(v);
  return __longlong_as_double((long long)dpp_u64<CTRL>(b, b));
}
__device__ __forceinline__ double row_sum_f64(double v) {
  v += dpp_f64<0xB1>(v);
  v += dpp_f64<0x4E>(v);
  v += dpp_f64<0x141>(v);
  return v + dpp_f64<0x140>(v);
}
__device__ __forceinline__ double row_max_f64(double v) {
  v = fmax(v, dpp_f64<0xB1>(v));
  v = fmax(v, dpp_f64<0x4E>(v));
  v = fmax(v, dpp_f64<0x141>(v));
  return fmax(v, dpp_f64<0x140>(v));
}
__device__ __forceinline__ uint32_t row_max_u32(uint32_t v) {
  v = max(v, dpp_u32<0xB1>(v, v));
  v = max(v, dpp_u32<0x4E>(v, v));
  v = max(v, dpp_u32<0x141>(v, v));
  return max(v, dpp_u32<0x140>(v, v));
}
__device__ __forceinline__ uint32_t row_min_u32(uint32_t v) { return ~row_max_u32(~v); }

// The float whose order key is k.
__device__ __forceinline__ float key_float(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? k ^ 0x80000000u : ~k); }

// A logit as the definition takes it: NaN masked like -inf, +inf the largest float32.
__device__ __forceinline__ float clean_logit(float f) {
  return f > -__builtin_huge_valf() ? fminf(f, 3.402823466e+38f) : -__builtin_huge_valf();
}

constexpr int kRouteTokens = 16;  // tokens of a workgroup

// float64 values in LDS of a token of N experts in G groups (odd: the tokens of a wave start on other banks).
__host__ __device__ constexpr int route_lds_doubles(int N, int G) { return (N + G + 2) | 1; }

// The largest (value, then smallest id) is taken K times.  Without a bias the values are the
// logits and their 32-bit order keys decide.  With one they are float64 scores + bias: their
// roundings to float32 keep the order, so the same 32-bit rounds run on those, and float64
// decides only where two of a round's best round alike.  Scores of all experts are computed
// where something needs them (SC: a bias, or groups by their two largest; a softmax that is
// not renormalised needs its sum), else those of the K routes only.
template <typename E, int R, bool BIAS, bool SC>
__global__ __launch_bounds__(256) void route_experts_kernel(const RouteExpertsArgs a) {
  static_assert(SC || !BIAS, "a bias needs the scores");
  extern __shared__ double lds[];  // groups only: route_lds_doubles a token
  const int tid = threadIdx.x, q = tid & 15, slot = tid >> 4;
  const long long t = (long long)blockIdx.x * kRouteTokens + slot;
  const bool on = t < a.T;
  const int N = a.N, K = a.K, e0 = q * R;
  const E *row = static_cast<const E *>(a.logits) + (on ? t : a.T - 1) * a.ld;
  const double inf = __builtin_huge_val();

  float l[R];
  if (a.vec) {
    constexpr int EP = 16 / sizeof(E);
#pragma unroll
    for (int c = 0; c < (R + EP - 1) / EP; ++c) {
      u32x4 v = u32x4{0u, 0u, 0u, 0u};
      if constexpr (R >= EP) v = *reinterpret_cast<const u32x4 *>(row + e0 + c * EP);
#pragma unroll
      for (int i = 0; i < EP; ++i)
        if (c * EP + i < R) {
          if constexpr (sizeof(E) == 2)
            l[c * EP + i] = __uint_as_float((i & 1) ? v[i / 2] & 0xffff0000u : v[i / 2] << 16);
          else
            l[c * EP + i] = __uint_as_float(v[i]);
        }
    }
  } else {
#pragma unroll
    for (int j = 0; j < R; ++j) l[j] = e0 + j < N ? load_f32(row + e0 + j) : -__builtin_huge_valf();
  }
#pragma unroll
  for (int j = 0; j < R; ++j) l[j] = clean_logit(l[j]);

  // softmax: exp(l - top), top finite where any logit is
  float topf = l[0];
#pragma unroll
  for (int j = 1; j < R; ++j) topf = fmaxf(topf, l[j]);
  topf = key_float(row_max_u32(float_key(topf)));
  const double top = topf > -__builtin_huge_valf() ? (double)topf : 0.0;
  const bool soft = a.score == EXFOLD_SCORE_SOFTMAX;
  auto raw = [&](float x) { return soft ? exp((double)x - top) : 1.0 / (1.0 + exp(-(double)x)); };  // 0 where masked

  double p[SC ? R : 1], sum = 1.0;
  if constexpr (SC) {
#pragma unroll
    for (int j = 0; j < R; ++j) p[j] = raw(l[j]);
  }
  if (soft && (SC || !a.renorm)) {
    double part = 0.0;
#pragma unroll
    for (int j = 0; j < R; ++j) {
      if constexpr (SC) part += p[j];
      else part += raw(l[j]);
    }
    sum = row_sum_f64(part);
    if (!(sum > 0.0)) sum = 1.0;  // every expert masked
  }
  uint32_t key[R];
#pragma unroll
  for (int j = 0; j < R; ++j) {
    if constexpr (SC) {
      double s = soft ? p[j] / sum : p[j];
      if constexpr (BIAS) s += (double)a.bias[min(e0 + j, N - 1)];
      p[j] = (l[j] > -__builtin_huge_valf() && s > -inf) ? s : -inf;  // the value of the expert; NaN masks
    }
    key[j] = e0 + j < N ? float_key(BIAS ? (float)p[SC ? j : 0] : l[j]) : 0u;
  }

  if (a.n_groups > 1) {
    const int G = a.n_groups, size = N / G;
    const bool top2 = SC && a.group_value == EXFOLD_GROUP_TOP2;
    double *sv = lds + slot * route_lds_doubles(N, G), *gv = sv + N + 1;  // values of the experts, of the groups
#pragma unroll
    for (int j = 0; j < R; ++j)
      if (e0 + j < N) sv[e0 + j] = (BIAS || top2) ? p[SC ? j : 0] : (double)l[j];
    wave_lds_order();
    for (int g = q; g < G; g += 16) {
      double m1 = -inf, m2 = -inf;
      for (int i = 0, at = q % size; i < size; ++i, at = at + 1 == size ? 0 : at + 1) {  // staggered over the banks
        const double s = sv[g * size + at];
        m2 = fmax(m2, fmin(m1, s));
        m1 = fmax(m1, s);
      }
      gv[g] = (top2 && m2 > -inf) ? m1 + m2 : m1;
    }
    wave_lds_order();
    for (int g = q; g < G; g += 16) {
      const double mine = gv[g];
      int rank = 0;
      for (int o = 0; o < G; ++o) {
        const double other = gv[o];
        rank += other > mine || (other == mine && o < g);
      }
      sv[g] = rank < a.keep_groups ? 1.0 : 0.0;  // the experts' values have been read
    }
    wave_lds_order();
    int g = e0 / size, r = e0 % size;
#pragma unroll
    for (int j = 0; j < R; ++j) {
      if (e0 + j < N && sv[g] == 0.0) key[j] = 0u;
      if (++r == size) {
        r = 0;
        ++g;
      }
    }
  }

  // Lane k of the row gets route k.  A key of 0 is taken or not a candidate; a masked one is above.
  int my_id = 0;
  uint32_t my_key = 0u;
  for (int k = 0; k < K; ++k) {
    uint32_t m = key[0];
#pragma unroll
    for (int j = 1; j < R; ++j) m = max(m, key[j]);
    m = row_max_u32(m);
    uint32_t id = 0xffffu, n = 0u;
#pragma unroll
    for (int j = R - 1; j >= 0; --j)
      if (key[j] == m) {
        id = e0 + j;
        ++n;
      }
    if constexpr (BIAS) {
      const uint64_t has = __ballot(n > 0u);
      const uint32_t lanes = (uint32_t)(has >> (threadIdx.x & 48)) & 0xffffu;
      if (__any(n > 1u || (lanes & (lanes - 1u)) != 0u)) {  // some row's best round alike
        double best = -inf;
#pragma unroll
        for (int j = 0; j < R; ++j)
          if (key[j] == m) best = fmax(best, p[j]);
        best = row_max_f64(best);
        id = 0xffffu;
#pragma unroll
        for (int j = R - 1; j >= 0; --j)
          if (key[j] == m && p[j] == best) id = e0 + j;
      }
    }
    id = row_min_u32(id);
#pragma unroll
    for (int j = 0; j < R; ++j)
      if (id == (uint32_t)(e0 + j)) key[j] = 0u;
    if (q == k) {
      my_id = (int)id;
      my_key = m;
    }
  }

  my_id = clamp_id(my_id, N);
  double w = 0.0;
  if (q < K) {
    float lk = key_float(my_key);
    bool live = true;
    if constexpr (BIAS) {
      lk = clean_logit(load_f32(row + my_id));
      live = a.bias[my_id] > -__builtin_huge_valf();
    }
    if (live && lk > -__builtin_huge_valf()) w = raw(lk) / sum;
  }
  if (a.renorm) {
    const double total = row_sum_f64(w);
    w = total > 0.0 ? w / total : 0.0;
  }
  if (on && q < K) {
    a.ids[t * K + q] = my_id;
    a.w[t * K + q] = (float)(w * (double)a.scale);
  }
}

template <typename E, int R>
static void launch_rows(const RouteExpertsArgs &a, hipStream_t s) {
  const int grid = (a.T + kRouteTokens - 1) / kRouteTokens;
  // at most 16 * 515 * 8 bytes = 64.4 KiB
  const size_t lds = a.n_groups > 1 ? sizeof(double) * kRouteTokens * route_lds_doubles(a.N, a.n_groups) : 0;
  if (a.bias) route_experts_kernel<E, R, true, true><<<grid, 256, lds, s>>>(a);
  else if (a.n_groups > 1 && a.group_value == EXFOLD_GROUP_TOP2) route_experts_kernel<E, R, false, true><<<grid, 256, lds, s>>>(a);
  else route_experts_kernel<E, R, false, false><<<grid, 256, lds, s>>>(a);
}

hipError_t launch_route_experts(const RouteExpertsArgs &args, hipStream_t s) {
  if (args.T <= 0) return hipSuccess;
  RouteExpertsArgs a = args;
  auto by_size = [&](auto e) {
    using E = decltype(e);
    const int R = a.N <= 32 ? 2 : a.N <= 64 ? 4 : a.N <= 128 ? 8 : 16;
    // 16-byte loads where each lane's experts are whole pieces
    a.vec = a.N == 16 * R && R * sizeof(E) % 16 == 0 && reinterpret_cast<uintptr_t>(a.logits) % 16 == 0 &&
            a.ld * (long long)sizeof(E) % 16 == 0;
    if (R == 2) launch_rows<E, 2>(a, s);
    else if (R == 4) launch_rows<E, 4>(a, s);
    else if (R == 8) launch_rows<E, 8>(a, s);
    else launch_rows<E, 16>(a, s);
  };
  if (a.dtype == EXFOLD_BF16) by_size(bf16_t{});
  else by_size(float{});
  return hipGetLastError();
}

}  // namespace exfold
