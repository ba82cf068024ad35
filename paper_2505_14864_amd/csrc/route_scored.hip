// Token-choice routing by scores: softmax or sigmoid scores, a selection bias, expert groups, renormalised and scaled
// gate weights, and the backward pass.
//
//   s = softmax(z) or sigmoid(z),  v = s + bias;  the top_groups groups with the largest sum of their group_best largest v stay;
//   of their experts the k with the largest v;  w = s / sum of the chosen s (or s) * scale
//
// Which of two experts is ahead is decided on v in 64 bits: of 64 Ki tokens over 256 experts some have neighbours
// closer than a 32-bit rounding at the border of the selection, and an index cannot be a little wrong.  Done for all of it, 64 bits took
// ten times the time of the rest, so the selection is made in 32 bits first, with a bound on what their roundings can move; a
// token with two values in question closer than that (a few in a thousand, and all that have equal ones) is routed again in 64.
//
// Bound: the vector instructions of the k rounds, with few tokens the launch and their latency.  A lane holds four neighbouring experts, a token
// as many lanes as it needs, 4, 16 or 64, so that up to 16 tokens share a wavefront; a maximum over a token's lanes takes two, four or
// eight vector instructions for all of them at once, and the winner's own lane stores its index and weight: nothing else crosses lanes.
//
// Measured: 65536 tokens x 64 experts, k = 8, with a bias 20 us, without one 15 (all of it in 64 bits, a token per wavefront: 101 with it),
// 4096 x 256 in eight groups 8 to 12, by whether a token is in doubt (18), 3001 x 60 in five groups 4.6 (9), one token 2.1, 65536 x 256 in groups 92; backward
// 65536 x 256 21 us: 67 MB of gradients written and 38 MB read (counted), the cache lines that the chosen logits lie in; with weights as the softmax gives
// them, and so all logits read, 27 us.
#include "common.h"
#include "profile.h"

namespace dynmo {

constexpr int kMaxRouteExperts = 256;

// An expert whose logit is NaN or -inf, or whose order value is, is never chosen; +inf counts as the largest finite number,
// so that a softmax over it has a value.
__device__ __forceinline__ float clean_logit(float z) { return z != z ? -INFINITY : fminf(z, 3.402823466e38f); }

// The value that the lane has whose place among LPT neighbours is mirrored in one more bit: after log2(LPT) steps of op(v, neighbour)
// every lane has the result over all of them.
template <int CTRL>
__device__ __forceinline__ float moved(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
template <int LPT, typename Op>
__device__ __forceinline__ float over_lanes(float v, Op op) {
  static_assert(LPT == 4 || LPT == 16 || LPT == 64, "");
  v = op(v, moved<0xB1>(v));  // lane ^ 1
  v = op(v, moved<0x4E>(v));  // lane ^ 2
  if constexpr (LPT >= 16) {
    v = op(v, moved<0x141>(v));  // 7 - lane of eight
    v = op(v, moved<0x140>(v));  // 15 - lane of sixteen
  }
  if constexpr (LPT == 64) {  // a swap of two copies leaves the two halves of each pair of rows, and of the wavefront, everywhere
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
  return v;
}
// integers in the order of the floating values (no NaN), and back
__device__ __forceinline__ int order_key(float v) {
  const int b = __float_as_int(v);
  return b ^ ((b >> 31) & 0x7fffffff);
}
__device__ __forceinline__ float order_value(int k) { return __int_as_float(k ^ ((k >> 31) & 0x7fffffff)); }

template <int LPT>
__device__ __forceinline__ int max_over(int v) {
  v = max(v, __builtin_amdgcn_update_dpp(INT32_MIN, v, 0xB1, 0xf, 0xf, false));
  v = max(v, __builtin_amdgcn_update_dpp(INT32_MIN, v, 0x4E, 0xf, 0xf, false));
  if constexpr (LPT >= 16) {
    v = max(v, __builtin_amdgcn_update_dpp(INT32_MIN, v, 0x141, 0xf, 0xf, false));
    v = max(v, __builtin_amdgcn_update_dpp(INT32_MIN, v, 0x140, 0xf, 0xf, false));
  }
  if constexpr (LPT == 64) {
    auto r = __builtin_amdgcn_permlane16_swap((uint32_t)v, (uint32_t)v, false, false);
    v = max((int)r[0], (int)r[1]);
    r = __builtin_amdgcn_permlane32_swap((uint32_t)v, (uint32_t)v, false, false);
    v = max((int)r[0], (int)r[1]);
  }
  return v;
}
template <int LPT>
__device__ __forceinline__ float max_over(float v) {
  return over_lanes<LPT>(v, [](float a, float b) { return fmaxf(a, b); });
}
template <int LPT>
__device__ __forceinline__ float sum_over(float v) {
  return over_lanes<LPT>(v, [](float a, float b) { return a + b; });
}

// The first in the order of two experts, and of all the token's
struct Ranked {
  double v;
  int e;
};
__device__ __forceinline__ Ranked ahead_of(Ranked a, Ranked b) { return b.v > a.v || (b.v == a.v && b.e < a.e) ? b : a; }
template <int CTRL>
__device__ __forceinline__ Ranked moved(Ranked r) {
  const long long w = __double_as_longlong(r.v);
  const int lo = __builtin_amdgcn_update_dpp(0, (int)w, CTRL, 0xf, 0xf, true), hi = __builtin_amdgcn_update_dpp(0, (int)(w >> 32), CTRL, 0xf, 0xf, true);
  return {__longlong_as_double((long long)hi << 32 | (uint32_t)lo), __builtin_amdgcn_update_dpp(0, r.e, CTRL, 0xf, 0xf, true)};
}
template <int LPT>
__device__ __forceinline__ Ranked first_over(Ranked r) {
  r = ahead_of(r, moved<0xB1>(r));
  r = ahead_of(r, moved<0x4E>(r));
  if constexpr (LPT >= 16) {
    r = ahead_of(r, moved<0x141>(r));
    r = ahead_of(r, moved<0x140>(r));
  }
  if constexpr (LPT == 64) {
    auto both = [&](auto swap) {
      const long long w = __double_as_longlong(r.v);
      const auto lo = swap((uint32_t)w), hi = swap((uint32_t)(w >> 32)), e = swap((uint32_t)r.e);
      r = ahead_of({__longlong_as_double((long long)hi[0] << 32 | lo[0]), (int)e[0]}, {__longlong_as_double((long long)hi[1] << 32 | lo[1]), (int)e[1]});
    };
    both([](uint32_t x) { return __builtin_amdgcn_permlane16_swap(x, x, false, false); });
    both([](uint32_t x) { return __builtin_amdgcn_permlane32_swap(x, x, false, false); });
  }
  return r;
}

// A token owns LPT adjacent lanes; lane j of them holds VPL experts, four neighbours each time.
template <int LPT>
__device__ __forceinline__ int expert_of(int q, int j) {
  return q / 4 * (4 * LPT) + j * 4 + q % 4;
}
// VEC: E is a multiple of four and the logits are 16-byte aligned
template <int LPT, int VPL, bool VEC>
__device__ __forceinline__ void load_logits(const float* __restrict__ row, int j, int E, bool live, float* z) {
#pragma unroll
  for (int q = 0; q < VPL; q += 4) {
    const int e = expert_of<LPT>(q, j);
    float v[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    if constexpr (VEC) {
      if (live && e < E) unpack16<float>(*(const u32x4*)(row + e), v);
    } else {
#pragma unroll
      for (int c = 0; c < 4; ++c)
        if (live && e + c < E) v[c] = row[e + c];
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) z[q + c] = clean_logit(v[c]);
  }
}

// Scores in 32 bits; *top: the largest logit, -inf where there is none (softmax only)
template <int LPT, int VPL>
__device__ __forceinline__ void scores32(int score, const float* z, float* s, float* top, float* inv) {
  if (score == DYNMO_SCORE_SOFTMAX) {
    float mx = z[0];
#pragma unroll
    for (int q = 1; q < VPL; ++q) mx = fmaxf(mx, z[q]);
    mx = max_over<LPT>(mx);
    float sum = 0.f;
#pragma unroll
    for (int q = 0; q < VPL; ++q) sum += s[q] = z[q] == -INFINITY ? 0.f : __expf(z[q] - mx);
    sum = sum_over<LPT>(sum);
    *inv = sum > 0.f ? 1.f / sum : 0.f;
    *top = mx;
#pragma unroll
    for (int q = 0; q < VPL; ++q) s[q] *= *inv;
  } else {
#pragma unroll
    for (int q = 0; q < VPL; ++q) s[q] = sigmoidf_(z[q]);
  }
}

// The experts of the groups that do not stay lose their order value.  `order`: an LDS row of 4 LPT values for this token.
// *least, *most (32 bits only): the group scores of the last group that stays and of the first that does not.
template <int LPT, typename Real>
__device__ __forceinline__ void drop_groups(const dynmo_route_rule& rule, int E, int j, Real* order, Real* v, float* least, float* most) {
  const Real none = -INFINITY;
  const int size = E / rule.groups, lane = threadIdx.x & 63;
  auto add = [&](Real x, Real* first, Real* second) {
    *second = x > *first ? *first : x > *second ? x : *second;
    *first = x > *first ? x : *first;
  };
  auto score = [&](Real first, Real second) { return rule.group_best == 2 && second > none ? first + second : first; };
  Real low = INFINITY, high = none;
  auto count = [&](Real own, int g) {  // whether group g stays
    int before = 0;
#pragma unroll 4
    for (int o = 0; o < rule.groups; ++o) {
      const Real x = order[o];
      before += x > own || (x == own && o < g);
    }
    const bool stays = before < rule.top_groups;
    if (stays) low = own < low ? own : low;
    else high = own > high ? own : high;
    return stays;
  };
  if (size % 4 == 0) {  // a lane's experts are of one group, and no group has more than one lane to look after it
    Real first = none, second = none;
#pragma unroll
    for (int q = 0; q < 4; ++q) add(v[q], &first, &second);
    order[2 * j] = first;
    order[2 * j + 1] = second;
    wave_lds_order();
    first = second = none;
    if (j < rule.groups) {
#pragma unroll 4
      for (int i = 0; i < size / 4; ++i) {
        add(order[2 * (j * (size / 4) + i)], &first, &second);
        add(order[2 * (j * (size / 4) + i) + 1], &first, &second);
      }
    }
    wave_lds_order();
    const Real own = score(first, second);
    order[j] = own;
    wave_lds_order();
    const bool stays = j < rule.groups && count(own, j);
    const unsigned long long kept = __ballot(stays) >> (lane - j);
    if (4 * j < E && !(kept >> (4 * j / size) & 1)) {
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = none;
    }
  } else {
#pragma unroll
    for (int q = 0; q < 4; ++q) order[4 * j + q] = v[q];
    wave_lds_order();
    Real own[4];  // the scores of groups j, j + LPT, ..
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int g = q * LPT + j;
      Real first = none, second = none;
      if (g < rule.groups) {
#pragma unroll 4
        for (int i = 0; i < size; ++i) add(order[g * size + i], &first, &second);
      }
      own[q] = score(first, second);
    }
    wave_lds_order();
#pragma unroll
    for (int q = 0; q < 4; ++q) order[q * LPT + j] = own[q];
    wave_lds_order();
    bool stays[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) stays[q] = q * LPT + j < rule.groups && count(own[q], q * LPT + j);
    wave_lds_order();
#pragma unroll
    for (int q = 0; q < 4; ++q) order[q * LPT + j] = stays[q] ? 1 : 0;
    wave_lds_order();
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (4 * j + q < E && order[(4 * j + q) / size] == 0) v[q] = none;
  }
  wave_lds_order();
  if constexpr (sizeof(Real) == 4) {
    *least = -max_over<LPT>(-low);
    *most = max_over<LPT>(high);
  }
}

template <int LPT, bool VEC>
__global__ __launch_bounds__(256) void route_scored_kernel(const float* __restrict__ logits, const float* __restrict__ bias,
                                                           int32_t* __restrict__ expert_idx, float* __restrict__ gate_w, int T, int E,
                                                           int k, const dynmo_route_rule rule) {
  constexpr int kTokens = 64 / LPT, VPL = 4;
  __shared__ double order[4][kTokens][LPT * VPL];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, j = lane % LPT, tok = lane / LPT;
  const long t = ((long)blockIdx.x * 4 + wave) * kTokens + tok;
  const bool live = t < T, softmax = rule.score == DYNMO_SCORE_SOFTMAX;
  float z[VPL], s[VPL], v[VPL], top = 0.f, inv = 1.f;
  load_logits<LPT, VPL, VEC>(logits + t * E, j, E, live, z);
  scores32<LPT, VPL>(rule.score, z, s, &top, &inv);
  // Scores are monotonous in the logits: without a bias, and without sums of scores, the logits themselves are the order.
  const bool by_logit = bias == nullptr && (rule.groups == 1 || rule.group_best == 1);
  float size = 0.f;  // of the largest finite order value
#pragma unroll
  for (int q = 0; q < VPL; ++q) {
    const int e = expert_of<LPT>(q, j);
    v[q] = by_logit ? z[q] : s[q] + (bias && e < E ? bias[e] : 0.f);
    if (!(v[q] > -INFINITY) || z[q] == -INFINITY) v[q] = -INFINITY;
    if (fabsf(v[q]) < INFINITY) size = fmaxf(size, fabsf(v[q]));
  }
  // How far apart two order values have to be for their order to be that of the 64-bit ones, with twice to three times the bound of their
  // errors.  In units of 2^-24: an exponential is off by 2 and 1.5 |x| relative (the hardware's ulp, the product with log2 e).  The logistic function
  // of it by 0.25 x 2 + 0.22 x 1.5 for the exponential, whose slope weakens with x, and one each for its sum and its quotient: 2.8, twice for
  // two values.  A softmax score, of the largest one: 0.37 x 2.5 + 2 for the exponential of a rounded difference, one for the product, and up to 14 for
  // the common factor: 22 for two.  The sum with the bias: one of its own size, each.  By logits: the 64-bit scores have
  // to differ, too: e^z by 2^-40 relative, and the logistic function, whose slope up to z = 16 is at least 2^-24, by 2^-47; where it is flatter
  // than that, and where both exponentials may vanish, the token is left to the 64 bits.
  const float upper = by_logit && !softmax ? 16.f : INFINITY, lower = by_logit ? (softmax ? top : 0.f) - 600.f : -INFINITY;
  auto apart = [&](float larger) {
    if (by_logit) return softmax ? 0x1p-40f * (1.f + larger) : 0x1p-23f;
    return (softmax ? 0x1p-18f * inv : 0x1p-20f) + 0x1p-22f * larger;
  };
  bool doubtful = false, doubtful_groups = false;
  if (rule.groups > 1) {
    size = max_over<LPT>(size);
    float least, most;
    drop_groups<LPT, float>(rule, E, j, (float*)order[wave][tok], v, &least, &most);
    // sums of two, in which large values may have cancelled each other, or left the range
    const float larger = by_logit ? fmaxf(fabsf(least), fabsf(most)) : size;
    doubtful_groups = (most > -INFINITY && !(least - most > 2.f * apart(larger) && least <= upper && least >= lower)) || (!by_logit && !(size < 1e30f));
  }
  // The rounds compare integers in the same order, whose maximum over neighbouring lanes is one instruction.
  int slot[VPL], key[VPL];
  bool can[VPL];
#pragma unroll
  for (int q = 0; q < VPL; ++q) {
    slot[q] = -1;
    can[q] = v[q] > -INFINITY;
    key[q] = order_key(v[q] + 0.f);  // -0 counts as 0
  }
  const int none = order_key(-INFINITY);
  float last = NAN, before = NAN, largest = -INFINITY, gap = INFINITY;
  int filled = 0;
  auto round = [&](int n) {
    int best = key[0];
#pragma unroll
    for (int q = 1; q < VPL; ++q) best = max(best, key[q]);
    best = max_over<LPT>(best);
    const float value = order_value(best);
    const bool any = best > none;
    gap = fminf(gap, any ? last - value : INFINITY);  // equal infinities leave no gap, but are taken together
    before = any ? last : before;
    last = any ? value : last;
    if (n == 0) largest = value;
    return any ? best : INT32_MIN;  // no value has that key
  };
  for (int n = 0; n < k; ++n) {
    const int best = round(n);
    filled = best != INT32_MIN ? n + 1 : filled;
#pragma unroll
    for (int q = 0; q < VPL; ++q) {
      const bool taken = key[q] == best;
      slot[q] = taken ? n : slot[q];
      key[q] = taken ? none : key[q];
    }
  }
  round(k);  // the first that is not chosen
  doubtful |= filled > 0 && (!(gap > apart(fmaxf(fabsf(largest), fabsf(last)))) || largest > upper || before < lower);
  float total = 0.f, taken = 0.f;
#pragma unroll
  for (int q = 0; q < VPL; ++q) {
    total += slot[q] >= 0 ? s[q] : 0.f;
    taken += slot[q] >= 0 ? 1.f : 0.f;
  }
  total = sum_over<LPT>(total);
  taken = sum_over<LPT>(taken);
  const float by = rule.renormalize ? (total > 0.f ? rule.scale / total : 0.f) : rule.scale;
#pragma unroll
  for (int q = 0; q < VPL; ++q) s[q] *= by;
  doubtful |= taken != (float)filled;                                          // equal values were taken together
  doubtful |= rule.renormalize && filled > 0 && !(total > 0x1p-10f);  // small scores, whose exponentials are less exact
  doubtful_groups &= live;
  doubtful = (doubtful || doubtful_groups) && live;
  if (__ballot(doubtful)) {  // all lanes of the wavefront go along
    double s64[VPL], v64[VPL], sum64 = 0.0;
#pragma unroll
    for (int q = 0; q < VPL; ++q) {
      s64[q] = softmax ? (z[q] == -INFINITY ? 0.0 : exp((double)z[q] - (double)top)) : 1.0 / (1.0 + exp(-(double)z[q]));
      sum64 += s64[q];
    }
    if (softmax) {
#pragma unroll
      for (int m = 1; m < LPT; m <<= 1) sum64 += __shfl_xor(sum64, m, 64);
    }
#pragma unroll
    for (int q = 0; q < VPL; ++q) {
      const int e = expert_of<LPT>(q, j);
      if (softmax) s64[q] /= sum64 > 0.0 ? sum64 : 1.0;
      v64[q] = s64[q] + (bias && e < E ? (double)bias[e] : 0.0);
      if (!(v64[q] > -INFINITY) || z[q] == -INFINITY) v64[q] = -INFINITY;
    }
    if (__ballot(doubtful_groups)) {
      drop_groups<LPT, double>(rule, E, j, order[wave][tok], v64, nullptr, nullptr);
    } else {
#pragma unroll
      for (int q = 0; q < VPL; ++q) v64[q] = can[q] ? v64[q] : -INFINITY;
    }
    int slot64[VPL], filled64 = 0;
#pragma unroll
    for (int q = 0; q < VPL; ++q) slot64[q] = -1;
    for (int n = 0; n < k; ++n) {
      Ranked best = {v64[0], expert_of<LPT>(0, j)};
#pragma unroll
      for (int q = 1; q < VPL; ++q) best = ahead_of(best, {v64[q], expert_of<LPT>(q, j)});
      best = first_over<LPT>(best);
      if (best.v > -INFINITY) filled64 = n + 1;  // lanes of other tokens take part in what follows
#pragma unroll
      for (int q = 0; q < VPL; ++q) {
        const bool mine = expert_of<LPT>(q, j) == best.e && best.v > -INFINITY;
        slot64[q] = mine ? n : slot64[q];
        v64[q] = mine ? -INFINITY : v64[q];
      }
    }
    auto chosen_sum = [&]() {
      double sum = 0.0;
#pragma unroll
      for (int q = 0; q < VPL; ++q) sum += slot64[q] >= 0 ? s64[q] : 0.0;
#pragma unroll
      for (int n = 1; n < LPT; n <<= 1) sum += __shfl_xor(sum, n, 64);
      return sum;
    };
    double total64 = rule.renormalize ? chosen_sum() : 1.0;
    if (__ballot(total64 < 1e-290)) {  // scores that vanish: relative to the largest chosen one (of a sigmoid, to e^z of it where that is below one)
      float m = -INFINITY;
#pragma unroll
      for (int q = 0; q < VPL; ++q) m = slot64[q] >= 0 ? fmaxf(m, z[q]) : m;
      m = max_over<LPT>(m);
      if (!softmax) m = fminf(m, 0.f);
#pragma unroll
      for (int q = 0; q < VPL; ++q) {
        const double up = softmax || z[q] <= 0.f ? exp((double)z[q] - (double)m) : 1.0;
        s64[q] = slot64[q] >= 0 ? (softmax ? up : up / (1.0 + exp(-fabs((double)z[q])))) : 0.0;
      }
      total64 = chosen_sum();
    }
    if (sum_over<LPT>(doubtful ? 1.f : 0.f) > 0.f) {
      filled = filled64;
#pragma unroll
      for (int q = 0; q < VPL; ++q) {
        slot[q] = slot64[q];
        s[q] = (float)(s64[q] / total64 * rule.scale);  // of tokens with a chosen expert; others have nothing to store
      }
    }
  }
  if (!live) return;
#pragma unroll
  for (int q = 0; q < VPL; ++q)
    if (slot[q] >= 0) {
      expert_idx[t * k + slot[q]] = expert_of<LPT>(q, j);
      gate_w[t * k + slot[q]] = s[q];
    }
  for (int n = filled + j; n < k; n += LPT) {  // no expert is left for these
    expert_idx[t * k + n] = -1;
    gate_w[t * k + n] = 0.f;
  }
}

// With g = dgate * scale, s the chosen scores and w = s / sum s:
//   renormalised         dlogit_j = w_j (g_j - sum_i g_i w_i), for the sigmoid times 1 - s_j: at the chosen experts, zero elsewhere
//   sigmoid as it is     dlogit_j = g_j s_j (1 - s_j)
//   softmax as it is     dlogit_e = p_e ([e chosen] g_e - sum_i g_i p_i)
// Only the last one needs more than the chosen logits.  The w are taken relative to the largest chosen score (of a sigmoid, to e^z of it where that is
// below one): the chosen ones may lie far below the rest, kept up by the bias.
// Bound by memory, with few tokens by the launch and the latency of two dependent reads.  The slots' gradients meet their experts in an LDS row per
// token, slot after slot, so that an expert in several slots gets their sum in a fixed order.
template <int LPT, int VPL, bool VEC>
__global__ __launch_bounds__(256) void route_scored_bwd_kernel(const float* __restrict__ dgate, const float* __restrict__ logits,
                                                               const int32_t* __restrict__ expert_idx, float* __restrict__ dlogits,
                                                               int T, int E, int k, const dynmo_route_rule rule) {
  constexpr int kTokens = 64 / LPT;
  __shared__ __attribute__((aligned(16))) float grads[4][kTokens][LPT * VPL];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, j = lane % LPT, tok = lane / LPT;
  const long t = ((long)blockIdx.x * 4 + wave) * kTokens + tok;
  const bool live = t < T, softmax = rule.score == DYNMO_SCORE_SOFTMAX, all = softmax && !rule.renormalize;
  float* const row = grads[wave][tok];
  const float* const lg = logits + t * E;
  float z[VPL], s[VPL], top = 0.f, inv = 1.f;
  if (all) {
    load_logits<LPT, VPL, VEC>(lg, j, E, live, z);
    scores32<LPT, VPL>(rule.score, z, s, &top, &inv);
  }
#pragma unroll
  for (int q = 0; q < VPL; q += 4) *(u32x4*)(row + expert_of<LPT>(q, j)) = u32x4{0u, 0u, 0u, 0u};
  wave_lds_order();
  // slot `n` of the token: its expert (-1: none), that expert's logit and the gradient before its scaling
  auto slot = [&](int n, float* x, float* g) {
    *x = -INFINITY;
    *g = 0.f;
    if (!live || n >= k) return -1;
    const int e = expert_idx[t * k + n];
    if (e < 0 || e >= E) return -1;
    *x = clean_logit(lg[e]);
    *g = dgate[t * k + n];
    return e;
  };
  float x, g;
  int e = slot(j, &x, &g);  // with more slots than lanes they are looked up again
  // What all the gradients of renormalised weights have in common has no effect; that of some slot with an expert is taken off all of them, so
  // that one chosen expert, or equal gradients, give zero and not the rounding of a difference.
  float common = 0.f;
  if (rule.renormalize) {
    float some = g;
    top = x;
    for (int n = j + LPT; n < k; n += LPT) {
      slot(n, &x, &g);
      some = top > -INFINITY ? some : g;
      top = fmaxf(top, x);
    }
    const unsigned long long have = __ballot(top > -INFINITY) >> (lane - j) & ((1ull << LPT) - 1ull);
    some = __shfl(some, have ? lane - j + __builtin_ctzll(have) : lane, 64);
    common = have ? some : 0.f;
    top = max_over<LPT>(top);
    if (!softmax) top = fminf(top, 0.f);
  }
  auto scaled = [&](float v) { return (v - common) * rule.scale; };
  auto score = [&](float v) {  // in units of e^top (not all: 1)
    if (v == -INFINITY) return 0.f;
    if (softmax) return __expf(v - top) * inv;
    return v > 0.f ? sigmoidf_(v) : __expf(v - top) * sigmoidf_(-v);
  };
  float total = 0.f, inner = 0.f;
  for (int n = j; n < k; n += LPT) {
    if (k > LPT) slot(n, &x, &g);
    total += score(x);
    inner += x > -INFINITY ? scaled(g) * score(x) : 0.f;
  }
  total = sum_over<LPT>(total);
  inner = sum_over<LPT>(inner);
  const float by = !rule.renormalize ? 1.f : total > 0.f ? 1.f / total : 0.f;
  for (int base = 0; base < k; base += LPT) {
    if (k > LPT) e = slot(base + j, &x, &g);
    float d = scaled(g);  // all: what the expert's own score is multiplied with below
    if (!all) d = score(x) * by * (rule.renormalize ? d - inner * by : d) * (softmax ? 1.f : sigmoidf_(-x));
    if (x == -INFINITY) d = 0.f;
    for (int i = 0; i < LPT && base + i < k; ++i) {
      if (j == i && e >= 0) __hip_atomic_fetch_add(row + e, d, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WAVEFRONT);
      wave_lds_order();
    }
  }
  wave_lds_order();
  if (!live) return;
  float* const out = dlogits + t * E;
#pragma unroll
  for (int q = 0; q < VPL; q += 4) {
    const int at = expert_of<LPT>(q, j);
    float d[4];
    unpack16<float>(*(const u32x4*)(row + at), d);
    if (all) {
#pragma unroll
      for (int c = 0; c < 4; ++c) d[c] = s[q + c] * (d[c] - inner);
    }
    if constexpr (VEC) {
      if (at < E) *(u32x4*)(out + at) = pack16<float>(d);
    } else {
#pragma unroll
      for (int c = 0; c < 4; ++c)
        if (at + c < E) out[at + c] = d[c];
    }
  }
}

static int64_t blocks_of(int T, int tokens_per_wave) { return (T + 4L * tokens_per_wave - 1) / (4L * tokens_per_wave); }

static int32_t check_route(const dynmo_desc* d, const dynmo_route_rule* r) {
  const int32_t rc = check_desc(d, kMaxRouteExperts);
  if (rc) return rc;
  if (!r || (r->score != DYNMO_SCORE_SOFTMAX && r->score != DYNMO_SCORE_SIGMOID)) return DYNMO_EINVAL;
  if (r->groups < 1 || d->E % r->groups || r->top_groups < 1 || r->top_groups > r->groups) return DYNMO_EINVAL;
  if (d->T >= 1 << 26) return DYNMO_EUNSUPPORTED;
  if (d->E > 64 && blocks_of(d->T, 1) >= 1 << 24) return DYNMO_EUNSUPPORTED;  // forward, workgroups of four tokens: a launch has fewer than 2^32 threads
  if (r->group_best < 1 || r->group_best > 2 || (r->renormalize != 0 && r->renormalize != 1)) return DYNMO_EINVAL;
  if (!(r->scale - r->scale == 0.f)) return DYNMO_EINVAL;                  // NaN or infinite
  if (d->k > r->top_groups * (d->E / r->groups)) return DYNMO_EINVAL;  // more slots than experts that can be chosen
  return DYNMO_OK;
}

// f(lanes per token, experts per lane, whether rows can be read 16 bytes at a time).  The backward pass has nothing to search for and takes 16
// lanes per token for more than 64 experts, too.
template <bool BACKWARD, typename F>
static int32_t by_experts(int E, bool aligned, F&& f) {
  using std::integral_constant;
  auto with = [&](auto lpt, auto vpl) -> int32_t {
    return E % 4 == 0 && aligned ? f(lpt, vpl, std::true_type{}) : f(lpt, vpl, std::false_type{});
  };
  if (E <= 16) return with(integral_constant<int, 4>{}, integral_constant<int, 4>{});
  if (E <= 64) return with(integral_constant<int, 16>{}, integral_constant<int, 4>{});
  if constexpr (!BACKWARD) return with(integral_constant<int, 64>{}, integral_constant<int, 4>{});
  else if (E <= 128) return with(integral_constant<int, 16>{}, integral_constant<int, 8>{});
  else return with(integral_constant<int, 16>{}, integral_constant<int, 16>{});
}

}  // namespace dynmo

using namespace dynmo;

extern "C" int32_t dynmo_route_scored(const dynmo_desc* d, const dynmo_route_rule* rule, const float* logits, const float* bias,
                                      int32_t* expert_idx, float* gate_w, void* stream) {
  const int32_t rc = check_route(d, rule);
  if (rc) return rc;
  if (!logits || !expert_idx || !gate_w) return DYNMO_EINVAL;
  if (d->T == 0) return DYNMO_OK;
  return by_experts<false>(d->E, !misaligned16(logits), [&](auto lpt, auto, auto vec) -> int32_t {
    constexpr int LPT = decltype(lpt)::value;
    hipStream_t st = (hipStream_t)stream;
    DYNMO_TIMED_LAUNCH(K_ROUTE_TOPK, st, route_scored_kernel<LPT, decltype(vec)::value><<<dim3((unsigned)blocks_of(d->T, 64 / LPT)), dim3(256), 0, st>>>(
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
  return by_experts<true>(d->E, !misaligned16(logits, dlogits), [&](auto lpt, auto vpl, auto vec) -> int32_t {
    constexpr int LPT = decltype(lpt)::value, VPL = decltype(vpl)::value;
    hipStream_t st = (hipStream_t)stream;
    DYNMO_TIMED_LAUNCH(K_ROUTE_TOPK_BWD, st,
                       route_scored_bwd_kernel<LPT, VPL, decltype(vec)::value><<<dim3((unsigned)blocks_of(d->T, 64 / LPT)), dim3(256), 0, st>>>(
                           dgate, logits, expert_idx, dlogits, d->T, d->E, d->k, *rule));
    return DYNMO_OK;
  });
}
