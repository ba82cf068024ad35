// Token-choice routing by scores: softmax or sigmoid scores, a selection bias, expert groups, renormalised and scaled
// gate weights, and the backward pass.
//
//   s = softmax(z) or sigmoid(z),  v = s + bias;  the top_groups groups with the largest sum of their group_best largest v stay;
//   of their experts the k with the largest v;  w = s / sum of the chosen s (or s) * scale
//
// Which of two experts is ahead is decided on v in 64 bits: of 64 Ki tokens over 256 experts some two have neighbours
// closer than a 32-bit rounding at the border of the selection, and an index cannot be a little wrong.
#include "common.h"
#include "profile.h"

namespace dynmo {

constexpr int kMaxRouteExperts = 256;

// An expert whose logit is NaN or -inf, or whose order value is, is never chosen; +inf counts as the largest finite number,
// so that a softmax over it has a value.
__device__ __forceinline__ float clean_logit(float z) { return z != z ? -INFINITY : fminf(z, 3.402823466e38f); }

// Between a wavefront's LDS writes and the reads of them by its other lanes: its LDS accesses complete in order, the compiler has to keep it.
__device__ __forceinline__ void wave_lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

struct Best {
  double v;
  int idx;
};
__device__ __forceinline__ Best better(const Best& a, const Best& b) { return a.v > b.v || (a.v == b.v && a.idx < b.idx) ? a : b; }

// A token owns LPT adjacent lanes of a wavefront; lane j of them holds the experts j, j + LPT, ... (VPL of them).
template <int LPT, int VPL>
__global__ __launch_bounds__(256) void route_scored_kernel(const float* __restrict__ logits, const float* __restrict__ bias,
                                                           int32_t* __restrict__ expert_idx, float* __restrict__ gate_w, int T, int E,
                                                           int k, const dynmo_route_rule rule) {
  constexpr int kTokens = 64 / LPT;
  __shared__ double order[4][kTokens][LPT * VPL], scores[4][kTokens][LPT * VPL], group[4][kTokens][LPT * VPL];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, j = lane % LPT, tok = lane / LPT;
  const long t = ((long)blockIdx.x * 4 + wave) * kTokens + tok;
  float z[VPL], top = -INFINITY;
  double s[VPL];
#pragma unroll
  for (int q = 0; q < VPL; ++q) {
    const int e = q * LPT + j;
    z[q] = t < T && e < E ? clean_logit(logits[t * E + e]) : -INFINITY;
    top = fmaxf(top, z[q]);
  }
  if (rule.score == DYNMO_SCORE_SOFTMAX) {
#pragma unroll
    for (int m = 1; m < LPT; m <<= 1) top = fmaxf(top, __shfl_xor(top, m, 64));
    double sum = 0.0;
#pragma unroll
    for (int q = 0; q < VPL; ++q) sum += s[q] = z[q] == -INFINITY ? 0.0 : exp((double)z[q] - (double)top);
#pragma unroll
    for (int m = 1; m < LPT; m <<= 1) sum += __shfl_xor(sum, m, 64);
#pragma unroll
    for (int q = 0; q < VPL; ++q) s[q] /= sum > 0.0 ? sum : 1.0;
  } else {
#pragma unroll
    for (int q = 0; q < VPL; ++q) s[q] = 1.0 / (1.0 + exp(-(double)z[q]));
  }
  double v[VPL];
#pragma unroll
  for (int q = 0; q < VPL; ++q) {
    const int e = q * LPT + j;
    v[q] = s[q] + (bias && e < E ? (double)bias[e] : 0.0);
    if (!(v[q] > -INFINITY) || z[q] == -INFINITY) v[q] = -INFINITY;
    order[wave][tok][e] = v[q];
    scores[wave][tok][e] = s[q];
  }
  wave_lds_order();
  if (rule.groups > 1) {
    const int size = E / rule.groups;
    double sum[VPL];
#pragma unroll
    for (int q = 0; q < VPL; ++q) {
      const int g = q * LPT + j;
      double first = -INFINITY, second = -INFINITY;
      for (int i = 0; g < rule.groups && i < size; ++i) {
        const double x = order[wave][tok][g * size + i];
        second = x > first ? first : x > second ? x : second;
        first = x > first ? x : first;
      }
      sum[q] = rule.group_best == 2 && second > -INFINITY ? first + second : first;
      group[wave][tok][g] = sum[q];
    }
    wave_lds_order();
    bool stays[VPL];
#pragma unroll
    for (int q = 0; q < VPL; ++q) {
      const int g = q * LPT + j;
      int ahead = 0;
      for (int o = 0; o < rule.groups; ++o) {
        const double x = group[wave][tok][o];
        ahead += x > sum[q] || (x == sum[q] && o < g);
      }
      stays[q] = ahead < rule.top_groups;
    }
    wave_lds_order();
#pragma unroll
    for (int q = 0; q < VPL; ++q) group[wave][tok][q * LPT + j] = stays[q] ? 1.0 : 0.0;
    wave_lds_order();
#pragma unroll
    for (int q = 0; q < VPL; ++q) {
      const int e = q * LPT + j;
      if (e < E && group[wave][tok][e / size] == 0.0) v[q] = -INFINITY;
    }
  }
  int idx[VPL];
  double w[VPL], total = 0.0;
#pragma unroll
  for (int q = 0; q < VPL; ++q) idx[q] = -1, w[q] = 0.0;
  for (int slot = 0; slot < k; ++slot) {
    Best best = {v[0], j};
#pragma unroll
    for (int q = 1; q < VPL; ++q) best = better(best, Best{v[q], q * LPT + j});
#pragma unroll
    for (int m = 1; m < LPT; m <<= 1) best = better(best, Best{__shfl_xor(best.v, m, 64), __shfl_xor(best.idx, m, 64)});
    if (best.v == -INFINITY) best.idx = -1;
    const double score = best.idx < 0 ? 0.0 : scores[wave][tok][best.idx];
    total += score;
#pragma unroll
    for (int q = 0; q < VPL; ++q) {
      if (q * LPT + j == slot) {
        idx[q] = best.idx;
        w[q] = score;
      }
      if (q * LPT + j == best.idx) v[q] = -INFINITY;  // taken
    }
  }
  const double by = rule.renormalize ? (total > 0.0 ? (double)rule.scale / total : 0.0) : (double)rule.scale;
#pragma unroll
  for (int q = 0; q < VPL; ++q) {
    const int slot = q * LPT + j;
    if (t < T && slot < k) {
      expert_idx[t * k + slot] = idx[q];
      gate_w[t * k + slot] = (float)(w[q] * by);
    }
  }
}

// ds_j = (g_j - sum_i g_i s_i / S) / S with S the sum of the chosen scores (or g_j), g = dgate * scale; then through the scores:
// sigmoid ds s (1 - s) at the chosen experts, softmax p_e ([e chosen] ds_e - sum_j ds_j p_j) everywhere.
template <int LPT, int VPL>
__global__ __launch_bounds__(256) void route_scored_bwd_kernel(const float* __restrict__ dgate, const float* __restrict__ logits,
                                                               const int32_t* __restrict__ expert_idx, float* __restrict__ dlogits,
                                                               int T, int E, int k, const dynmo_route_rule rule) {
  constexpr int kTokens = 64 / LPT;
  __shared__ float scores[4][kTokens][LPT * VPL], grads[4][kTokens][LPT * VPL];
  __shared__ int chosen[4][kTokens][LPT * VPL];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, j = lane % LPT, tok = lane / LPT;
  const long t = ((long)blockIdx.x * 4 + wave) * kTokens + tok;
  float z[VPL], s[VPL], top = -INFINITY;
#pragma unroll
  for (int q = 0; q < VPL; ++q) {
    const int e = q * LPT + j;
    z[q] = t < T && e < E ? clean_logit(logits[t * E + e]) : -INFINITY;
    top = fmaxf(top, z[q]);
  }
  if (rule.score == DYNMO_SCORE_SOFTMAX) {
#pragma unroll
    for (int m = 1; m < LPT; m <<= 1) top = fmaxf(top, __shfl_xor(top, m, 64));
    float sum = 0.f;
#pragma unroll
    for (int q = 0; q < VPL; ++q) sum += s[q] = z[q] == -INFINITY ? 0.f : __expf(z[q] - top);
#pragma unroll
    for (int m = 1; m < LPT; m <<= 1) sum += __shfl_xor(sum, m, 64);
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
#pragma unroll
    for (int q = 0; q < VPL; ++q) s[q] *= inv;
  } else {
#pragma unroll
    for (int q = 0; q < VPL; ++q) s[q] = sigmoidf_(z[q]);
  }
#pragma unroll
  for (int q = 0; q < VPL; ++q) scores[wave][tok][q * LPT + j] = s[q];
  wave_lds_order();
  float g[VPL], w[VPL], total = 0.f, inner = 0.f;
  int idx[VPL];
#pragma unroll
  for (int q = 0; q < VPL; ++q) {
    const int slot = q * LPT + j;
    const bool used = t < T && slot < k;
    idx[q] = used ? expert_idx[t * k + slot] : -1;
    if (idx[q] < 0 || idx[q] >= E) idx[q] = -1;
    g[q] = idx[q] >= 0 ? dgate[t * k + slot] * rule.scale : 0.f;
    w[q] = idx[q] >= 0 ? scores[wave][tok][idx[q]] : 0.f;
    total += w[q];
    inner += g[q] * w[q];
  }
#pragma unroll
  for (int m = 1; m < LPT; m <<= 1) {
    total += __shfl_xor(total, m, 64);
    inner += __shfl_xor(inner, m, 64);
  }
  if (rule.renormalize) {
    const float inv = total > 0.f ? 1.f / total : 0.f;
#pragma unroll
    for (int q = 0; q < VPL; ++q) g[q] = idx[q] >= 0 ? (g[q] - inner * inv) * inv : 0.f;
    inner = 0.f;  // sum_j ds_j s_j
  }
#pragma unroll
  for (int q = 0; q < VPL; ++q) {
    chosen[wave][tok][q * LPT + j] = idx[q];
    grads[wave][tok][q * LPT + j] = g[q];
  }
  wave_lds_order();
  float ds[VPL];
#pragma unroll
  for (int q = 0; q < VPL; ++q) ds[q] = 0.f;
  for (int slot = 0; slot < k; ++slot) {
    const int e = chosen[wave][tok][slot];
    const float d = grads[wave][tok][slot];
#pragma unroll
    for (int q = 0; q < VPL; ++q)
      if (e == q * LPT + j) ds[q] += d;
  }
#pragma unroll
  for (int q = 0; q < VPL; ++q) {
    const int e = q * LPT + j;
    if (t < T && e < E)
      dlogits[t * E + e] = rule.score == DYNMO_SCORE_SOFTMAX ? s[q] * (ds[q] - inner) : ds[q] == 0.f ? 0.f : ds[q] * s[q] * sigmoidf_(-z[q]);
  }
}

static int32_t check_route(const dynmo_desc* d, const dynmo_route_rule* r) {
  const int32_t rc = check_desc(d, kMaxRouteExperts);
  if (rc) return rc;
  if (!r || (r->score != DYNMO_SCORE_SOFTMAX && r->score != DYNMO_SCORE_SIGMOID)) return DYNMO_EINVAL;
  if (r->groups < 1 || d->E % r->groups || r->top_groups < 1 || r->top_groups > r->groups) return DYNMO_EINVAL;
  if (r->group_best < 1 || r->group_best > 2 || (r->renormalize != 0 && r->renormalize != 1)) return DYNMO_EINVAL;
  if (!(r->scale - r->scale == 0.f)) return DYNMO_EINVAL;                  // NaN or infinite
  if (d->k > r->top_groups * (d->E / r->groups)) return DYNMO_EINVAL;  // more slots than experts that can be chosen
  return DYNMO_OK;
}

// f(lanes per token, experts per lane) for this number of experts
template <typename F>
static int32_t by_experts(int E, F&& f) {
  using std::integral_constant;
  const integral_constant<int, 1> one;
  if (E <= 1) return f(one, one);
  if (E <= 2) return f(integral_constant<int, 2>{}, one);
  if (E <= 4) return f(integral_constant<int, 4>{}, one);
  if (E <= 8) return f(integral_constant<int, 8>{}, one);
  if (E <= 16) return f(integral_constant<int, 16>{}, one);
  if (E <= 32) return f(integral_constant<int, 32>{}, one);
  if (E <= 64) return f(integral_constant<int, 64>{}, one);
  if (E <= 128) return f(integral_constant<int, 64>{}, integral_constant<int, 2>{});
  return f(integral_constant<int, 64>{}, integral_constant<int, 4>{});
}

static dim3 blocks_of(int T, int tokens_per_wave) { return dim3((unsigned)((T + 4L * tokens_per_wave - 1) / (4L * tokens_per_wave))); }

}  // namespace dynmo

using namespace dynmo;

extern "C" int32_t dynmo_route_scored(const dynmo_desc* d, const dynmo_route_rule* rule, const float* logits, const float* bias,
                                      int32_t* expert_idx, float* gate_w, void* stream) {
  const int32_t rc = check_route(d, rule);
  if (rc) return rc;
  if (!logits || !expert_idx || !gate_w) return DYNMO_EINVAL;
  if (d->T == 0) return DYNMO_OK;
  return by_experts(d->E, [&](auto lpt, auto vpl) -> int32_t {
    constexpr int LPT = decltype(lpt)::value, VPL = decltype(vpl)::value;
    hipStream_t st = (hipStream_t)stream;
    DYNMO_TIMED_LAUNCH(K_ROUTE_TOPK, st, route_scored_kernel<LPT, VPL><<<blocks_of(d->T, 64 / LPT), dim3(256), 0, st>>>(
                                             logits, bias, expert_idx, gate_w, d->T, d->E, d->k, *rule));
    return DYNMO_OK;
  });
}

extern "C" int32_t dynmo_route_scored_bwd(const dynmo_desc* d, const dynmo_route_rule* rule, const float* dgate, const float* logits,
                                          const int32_t* expert_idx, float* dlogits, void* stream) {
  const int32_t rc = check_route(d, rule);
  if (rc) return rc;
  if (!dgate || !logits || !expert_idx || !dlogits) return DYNMO_EINVAL;
  if (d->T == 0) return DYNMO_OK;
  return by_experts(d->E, [&](auto lpt, auto vpl) -> int32_t {
    constexpr int LPT = decltype(lpt)::value, VPL = decltype(vpl)::value;
    hipStream_t st = (hipStream_t)stream;
    DYNMO_TIMED_LAUNCH(K_ROUTE_TOPK_BWD, st, route_scored_bwd_kernel<LPT, VPL><<<blocks_of(d->T, 64 / LPT), dim3(256), 0, st>>>(
                                                 dgate, logits, expert_idx, dlogits, d->T, d->E, d->k, *rule));
    return DYNMO_OK;
  });
}
