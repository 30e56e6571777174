// Routing of tokens to experts from router logits: softmax or sigmoid scores over all
// experts, a bias that steers the selection only, group-limited selection, renormalised
// and scaled weights (exfold_route_experts; the rules stand in the header).
#include "common.hpp"
#include "kernels.hpp"

namespace exfold {

// One wave a token, experts lane + 64 j, everything in float64.
template <typename E>
__global__ __launch_bounds__(64) void route_experts_kernel(const RouteExpertsArgs a) {
  __shared__ double sv[kMaxExperts];
  __shared__ double gv[kMaxExperts];
  const int lane = threadIdx.x;
  const long long t = blockIdx.x;
  const int N = a.N, K = a.K, G = a.n_groups, size = N / G;
  const E *row = static_cast<const E *>(a.logits) + t * a.ld;
  const double inf = __builtin_huge_val();
  constexpr int R = kMaxExperts / 64;
  double l[R], p[R], v[R];
  bool live[R];
  double top = -inf;
#pragma unroll
  for (int j = 0; j < R; ++j) {
    const int e = lane + 64 * j;
    const float f = e < N ? load_f32(row + e) : -__builtin_huge_valf();
    live[j] = f > -__builtin_huge_valf();  // false for NaN
    l[j] = live[j] ? (double)fminf(f, 3.402823466e+38f) : -inf;
    top = fmax(top, l[j]);
  }
  for (int m = 1; m < 64; m <<= 1) top = fmax(top, __shfl_xor(top, m));
  if (a.score == EXFOLD_SCORE_SOFTMAX) {
    double sum = 0.0;
#pragma unroll
    for (int j = 0; j < R; ++j) {
      p[j] = live[j] ? exp(l[j] - top) : 0.0;
      sum += p[j];
    }
    for (int m = 1; m < 64; m <<= 1) sum += __shfl_xor(sum, m);
#pragma unroll
    for (int j = 0; j < R; ++j) p[j] = live[j] ? p[j] / sum : 0.0;
  } else {
#pragma unroll
    for (int j = 0; j < R; ++j) p[j] = live[j] ? 1.0 / (1.0 + exp(-l[j])) : 0.0;
  }
#pragma unroll
  for (int j = 0; j < R; ++j) {
    const int e = lane + 64 * j;
    const double b = (a.bias && e < N) ? (double)a.bias[e] : 0.0;
    const double s = p[j] + b;
    if (!(s > -inf)) live[j] = false;  // a bias of -inf or NaN masks too
    v[j] = !live[j] ? -inf : a.bias ? s : l[j];
    if (e < N) sv[e] = !live[j] ? -inf : (a.group_value == EXFOLD_GROUP_TOP2) ? s : v[j];
  }
  __syncthreads();
  bool out[R];
#pragma unroll
  for (int j = 0; j < R; ++j) out[j] = lane + 64 * j >= N;
  if (G > 1) {
    for (int g = lane; g < G; g += 64) {
      double m1 = -inf, m2 = -inf;
      for (int i = 0; i < size; ++i) {
        const double s = sv[g * size + i];
        m2 = fmax(m2, fmin(m1, s));
        m1 = fmax(m1, s);
      }
      gv[g] = (a.group_value == EXFOLD_GROUP_TOP2 && m2 > -inf) ? m1 + m2 : m1;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const int g = min((lane + 64 * j) / size, G - 1);
      int rank = 0;
      for (int o = 0; o < G; ++o) rank += gv[o] > gv[g] || (gv[o] == gv[g] && o < g);
      out[j] = out[j] || rank >= a.keep_groups;
    }
  }
  // K rounds: the largest (v, smaller id first) of the candidates that are left
  double mine = 0.0, total = 0.0;
  int my_id = 0;
  for (int k = 0; k < K; ++k) {
    double best = -inf, bp = 0.0;
    int id = kMaxExperts;
#pragma unroll
    for (int j = 0; j < R; ++j)
      if (!out[j] && (id == kMaxExperts || v[j] > best)) {
        best = v[j];
        bp = live[j] ? p[j] : 0.0;
        id = lane + 64 * j;
      }
    for (int m = 1; m < 64; m <<= 1) {
      const double ov = __shfl_xor(best, m), op = __shfl_xor(bp, m);
      const int oi = __shfl_xor(id, m);
      if (oi != kMaxExperts && (id == kMaxExperts || ov > best || (ov == best && oi < id))) {
        best = ov;
        bp = op;
        id = oi;
      }
    }
#pragma unroll
    for (int j = 0; j < R; ++j)
      if (lane + 64 * j == id) out[j] = true;
    if (lane == k) {
      mine = bp;
      my_id = id;
    }
    total += bp;
  }
  if (lane < K) {
    if (a.renorm) mine = total > 0.0 ? mine / total : 0.0;
    a.ids[t * K + lane] = clamp_id(my_id, N);
    a.w[t * K + lane] = (float)(mine * (double)a.scale);
  }
}

hipError_t launch_route_experts(const RouteExpertsArgs &a, hipStream_t s) {
  if (a.T <= 0) return hipSuccess;
  if (a.dtype == EXFOLD_BF16)
    route_experts_kernel<bf16_t><<<a.T, 64, 0, s>>>(a);
  else
    route_experts_kernel<float><<<a.T, 64, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace exfold
