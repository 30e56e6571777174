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

// The value of a group from its two largest members, and the comparison of a round: u32 order
// keys or float64.
template <typename V> __device__ __forceinline__ V row_max(V v);
template <> __device__ __forceinline__ uint32_t row_max<uint32_t>(uint32_t v) { return row_max_u32(v); }
template <> __device__ __forceinline__ double row_max<double>(double v) { return row_max_f64(v); }
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return max(a, b); }
__device__ __forceinline__ double larger(double a, double b) { return fmax(a, b); }
__device__ __forceinline__ uint32_t smaller(uint32_t a, uint32_t b) { return min(a, b); }
__device__ __forceinline__ double smaller(double a, double b) { return fmin(a, b); }
template <int CTRL> __device__ __forceinline__ uint32_t dpp_any(uint32_t v) { return dpp_u32<CTRL>(v, v); }
template <int CTRL> __device__ __forceinline__ double dpp_any(double v) { return dpp_f64<CTRL>(v); }

// Candidates of the kept groups: bit j of the result for expert R q + j (all of value[], N of
// them).  lowest: below every value of an expert that is not masked, at most that of one that is.
// Groups of whole lanes, 2^i of them, stay in registers; others go through LDS.
template <int R, bool TOP2, typename V>
__device__ __forceinline__ uint32_t kept_candidates(const RouteExpertsArgs &a, const V (&value)[R], V lowest, int q, V *lds) {
  const int N = a.N, G = a.n_groups, size = N / G, e0 = q * R;
  const int lanes = size / R;
  uint32_t cand = 0u;
  auto merge = [&](V &m1, V &m2, V o1, V o2) {
    m2 = larger(smaller(m1, o1), larger(m2, o2));
    m1 = larger(m1, o1);
  };
  auto join = [&](V m1, V m2) -> V {  // masked members add nothing
    if constexpr (TOP2) return m2 > lowest ? m1 + m2 : m1;
    else return m1;
  };
  if (N == 16 * R && size % R == 0 && (lanes & (lanes - 1)) == 0) {
    V m1 = value[0], m2 = lowest;
#pragma unroll
    for (int j = 1; j < R; ++j) merge(m1, m2, value[j], lowest);
    if (lanes > 1) merge(m1, m2, dpp_any<0xB1>(m1), dpp_any<0xB1>(m2));
    if (lanes > 2) merge(m1, m2, dpp_any<0x4E>(m1), dpp_any<0x4E>(m2));
    if (lanes > 4) merge(m1, m2, dpp_any<0x141>(m1), dpp_any<0x141>(m2));  // at most 8: two groups or more
    const V mine = join(m1, m2);
    const uint32_t g = (uint32_t)(q / lanes);
    // rounds: the largest value of the groups that are left, then the smallest group of it
    bool left = true, keep = false;
    for (int k = 0; k < a.keep_groups; ++k) {
      const V best = row_max(left ? mine : lowest);
      const uint32_t win = row_min_u32(left && mine == best ? g : 0xffffu);
      if (win == g) keep = true, left = false;
    }
    cand = keep ? (1u << R) - 1u : 0u;
  } else {
    V *sv = lds, *gv = lds + N + 1;  // values of the experts, of the groups
#pragma unroll
    for (int j = 0; j < R; ++j)
      if (e0 + j < N) sv[e0 + j] = value[j];
    wave_lds_order();
    for (int g = q; g < G; g += 16) {
      V m1 = lowest, m2 = lowest;
      for (int i = 0, at = q % size; i < size; ++i, at = at + 1 == size ? 0 : at + 1)  // staggered over the banks
        merge(m1, m2, sv[g * size + at], lowest);
      gv[g] = join(m1, m2);
    }
    wave_lds_order();
    for (int g = q; g < G; g += 16) {
      const V mine = gv[g];
      int rank = 0;
      for (int o = 0; o < G; ++o) {
        const V other = gv[o];
        rank += other > mine || (other == mine && o < g);
      }
      sv[g] = rank < a.keep_groups ? V(1) : V(0);  // the experts' values have been read
    }
    wave_lds_order();
    int g = e0 / size, r = e0 % size;
#pragma unroll
    for (int j = 0; j < R; ++j) {
      if (e0 + j < N && sv[g] != V(0)) cand |= 1u << j;
      if (++r == size) {
        r = 0;
        ++g;
      }
    }
  }
  return cand;
}

// K rounds take the largest (value, then smallest id).  Without a bias the values are the
// logits, compared by their 32-bit order keys; a round runs on keys whose low byte holds the
// expert (255 - id, so the smaller id is the larger key): one maximum gives value and expert.
// That is exact unless two values share the upper 24 bits of their keys; two such are next to
// each other in the order of the rounds, so comparing each winner with the one before (and the
// K-th with the next) finds them, and the wave is routed again on whole keys, whose rounds
// search the expert of the maximum.  bf16 logits have nothing in the low bytes and never need
// it.  With a bias the values are float64 scores + bias; their roundings to float32 keep the
// order, so the whole-key rounds run on those, and float64 decides where a round's best round
// alike (24 bits are shared more often there: 8192 tokens of 128 experts 10.4 us, 11.9 with
// the first kind of rounds).
// Scores of all experts are computed where something needs them (SC: a bias, or groups by
// their two largest; a softmax that is not renormalised needs its sum), else those of the K
// routes only.
// Bound by its instructions: 65536 tokens of 256 experts, bf16, in 8 groups 26.8 us (58 us with
// whole-key rounds and groups through LDS; the bytes take 7), 8192 of 128 with a bias 9.3 us.
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
  const float inff = __builtin_huge_valf();

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
    for (int j = 0; j < R; ++j) l[j] = e0 + j < N ? load_f32(row + e0 + j) : -inff;
  }
#pragma unroll
  for (int j = 0; j < R; ++j) l[j] = clean_logit(l[j]);

  // softmax: exp(l - top), top finite where any logit is
  float topf = l[0];
#pragma unroll
  for (int j = 1; j < R; ++j) topf = fmaxf(topf, l[j]);
  topf = key_float(row_max_u32(float_key(topf)));
  const double top = topf > -inff ? (double)topf : 0.0;
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
  if constexpr (SC) {
#pragma unroll
    for (int j = 0; j < R; ++j) {
      double s = soft ? p[j] / sum : p[j];
      if constexpr (BIAS) s += (double)a.bias[min(e0 + j, N - 1)];
      p[j] = (l[j] > -inff && s > -inf) ? s : -inf;  // the value of the expert; NaN masks
    }
  }
  auto key_of = [&](int j) { return float_key(BIAS ? (float)p[SC ? j : 0] : l[j]); };

  // candidates: the experts, of the kept groups
  uint32_t cand = e0 >= N ? 0u : N - e0 >= R ? (1u << R) - 1u : (1u << (N - e0)) - 1u;
  if (a.n_groups > a.keep_groups) {
    double *mine = lds + slot * route_lds_doubles(N, a.n_groups);
    if (SC && a.group_value == EXFOLD_GROUP_TOP2) {
      if constexpr (SC) cand = kept_candidates<R, true>(a, p, -inf, q, mine);
    } else if constexpr (BIAS) {
      cand = kept_candidates<R, false>(a, p, -inf, q, mine);
    } else {
      uint32_t key[R];
#pragma unroll
      for (int j = 0; j < R; ++j) key[j] = key_of(j);
      cand = kept_candidates<R, false>(a, key, 0u, q, reinterpret_cast<uint32_t *>(mine));
    }
  }

  // Lane k of the row gets route k.  A key of 0 is taken or no candidate; a masked one is above.
  uint32_t key[R];
  int my_id = 0;
  bool whole = BIAS;
  if constexpr (!BIAS) {
    constexpr bool EXACT = sizeof(E) == 2;  // nothing in the keys' low bytes
    uint32_t mine = 0u, last = 0u;
    bool close = false;
#pragma unroll
    for (int j = 0; j < R; ++j) key[j] = (cand >> j & 1u) ? (key_of(j) & ~255u) | (uint32_t)(255 - e0 - j) : 0u;
    for (int k = 0; k < K + (EXACT ? 0 : 1); ++k) {
      uint32_t m = key[0];
#pragma unroll
      for (int j = 1; j < R; ++j) m = max(m, key[j]);
      m = row_max_u32(m);
#pragma unroll
      for (int j = 0; j < R; ++j) key[j] = key[j] == m ? 0u : key[j];
      if (q == k) mine = m;
      close = close || ((m ^ last) < 256u && m >= 0x00800000u);  // masked ones are all alike
      last = m;
    }
    my_id = 255 - (int)(mine & 255u);
    whole = !EXACT && __any(close);
  }
  if (whole) {
#pragma unroll
    for (int j = 0; j < R; ++j) key[j] = (cand >> j & 1u) ? key_of(j) : 0u;
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
        const uint32_t lanes = (uint32_t)(__ballot(n > 0u) >> (threadIdx.x & 48)) & 0xffffu;
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
      if (q == k) my_id = (int)id;
    }
  }

  my_id = clamp_id(my_id, N);
  double w = 0.0;
  if (q < K) {
    const float lk = clean_logit(load_f32(row + my_id));
    const bool live = lk > -inff && (!BIAS || a.bias[my_id] > -inff);
    if (live) w = raw(lk) / sum;
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
  const size_t lds = a.n_groups > a.keep_groups ? sizeof(double) * kRouteTokens * route_lds_doubles(a.N, a.n_groups) : 0;
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
