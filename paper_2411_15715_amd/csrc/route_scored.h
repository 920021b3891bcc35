// Choice of experts by scores (hipcc only): softmax over all logits or sigmoid of each, a bias for the choice, groups, k of them.
//
//   s_e = e^(x_e - max) / sum e^(x - max)   or   1 / (1 + e^-x_e),      c_e = s_e + b_e
//   a group's worth: the sum of its group_best largest c;   the top_groups worthiest stay open
//   the k largest c of the open groups (ties: the lower expert),   w = scale s / sum of the k s   (or scale s)
// Scores, sums and comparisons are in 64 bits: two experts whose c differ by less than 2^-24 of it would come out in the order of their
// roundings, and the sum with a bias rounds scores that do differ together (of 8192 tokens on 256 experts dozens).
// A wave a token, bound by its some 1000 vector instructions: 8192 tokens, top-8 of 256 in 8 groups, 17.8 us; 1 token, top-8 of 64, with the tables 4.5.
#pragma once
#include "si_internal.h"
#include "route_device.h"
#include "wave_device.h"

namespace si {

struct ScoreLds {  // of a wave
  double s[MAX_EXPERTS];
  uint64_t c[MAX_EXPERTS];    // keys of s + b; then, of the groups, their worth
  uint32_t open[MAX_EXPERTS];
};

// order-preserving map to an unsigned integer and back; NaN: 0, below -infinity
__device__ __forceinline__ uint64_t score_key(double v) {
  const uint64_t u = (uint64_t)__double_as_longlong(v);
  return v != v ? 0 : u >> 63 ? ~u : u | 1ull << 63;
}
__device__ __forceinline__ double score_of(uint64_t key) {
  return __longlong_as_double((long long)(key == 0 ? ~0ull : key >> 63 ? key & ~(1ull << 63) : ~key));
}

// Which groups are open: lds.open[g].  lds.c holds the experts' keys.
__device__ __forceinline__ void open_groups(int E, const si_score_t& rule, int lane, ScoreLds& lds) {
  const int n = rule.n_groups, of_group = E / n;
  uint64_t worth[MAX_EXPERTS / 64];
  if (rule.group_best <= 2) {
    // P neighbouring lanes look at a group and keep its two largest keys.  (One lane a group, of 8 with 32 experts each, for 8192 tokens: the launch
    // 38.9 us, this way and with the rounds below 17.8.)
    int P = 1;
    while (2 * P * n <= 64 && 2 * P <= of_group) P *= 2;
#pragma unroll
    for (int i = 0; i < MAX_EXPERTS / 64; ++i) {
      const int g = (lane + 64 * i) / P;  // (i > 0: P is 1, or there is none)
      worth[i] = 0;
      if (64 * i >= n * P) continue;
      uint64_t a = 0, b = 0;
      if (g < n)
        for (int e = lane % P; e < of_group; e += P) {
          const uint64_t c = lds.c[g * of_group + e];
          b = max(b, min(a, c));
          a = max(a, c);
        }
      for (int d = 1; d < P; d *= 2) {
        const uint64_t a2 = __shfl_xor(a, d), b2 = __shfl_xor(b, d);
        b = max(max(b, b2), min(a, a2));
        a = max(a, a2);
      }
      worth[i] = rule.group_best == 1 ? a : score_key(score_of(a) + score_of(b));
    }
    wave_lds();
#pragma unroll
    for (int i = 0; i < MAX_EXPERTS / 64; ++i) {
      const int g = (lane + 64 * i) / P;
      if (g < n && lane % P == 0 && 64 * i < n * P) lds.c[g] = worth[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < MAX_EXPERTS / 64; ++i) {
      const int g = lane + 64 * i;
      worth[i] = 0;
      if (g >= n) continue;
      // the largest, then the largest after it in the order of (key, place), and so on
      const uint64_t* c = lds.c + g * of_group;
      double sum = 0.0;
      uint64_t last = ~0ull;
      int last_at = -1;
      for (int r = 0; r < rule.group_best; ++r) {
        uint64_t best = 0;
        int at = of_group;
        for (int e = 0; e < of_group; ++e) {
          const bool left = c[e] < last || (c[e] == last && e > last_at);
          if (left && (at == of_group || c[e] > best)) { best = c[e]; at = e; }
        }
        sum += score_of(best);
        last = best;
        last_at = at;
      }
      worth[i] = score_key(sum);
    }
    wave_lds();
#pragma unroll
    for (int i = 0; i < MAX_EXPERTS / 64; ++i)
      if (lane + 64 * i < n) lds.c[lane + 64 * i] = worth[i];
  }
  wave_lds();
  for (int g = lane; g < n; g += 64) {
    const uint64_t mine = lds.c[g];
    int before = 0;
    for (int h = 0; h < n; ++h) before += lds.c[h] > mine || (lds.c[h] == mine && h < g);
    lds.open[g] = before < rule.top_groups;
  }
  wave_lds();
}

// N experts a lane: lane + 64 i
template <int N, class F> __device__ __forceinline__ void scored_rounds(const float* __restrict__ l, int E, int k, const si_score_t& rule, int lane, ScoreLds& lds, F put) {
  float x[N];
  double s[N];
  uint64_t key[N];
  int ex[N];  // the expert of a key, or MAX_EXPERTS: none
#pragma unroll
  for (int i = 0; i < N; ++i) {
    ex[i] = lane + 64 * i < E ? lane + 64 * i : MAX_EXPERTS;
    x[i] = lane + 64 * i < E ? l[lane + 64 * i] : -INFINITY;
  }
  if (rule.score == SI_SCORE_SOFTMAX) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) m = max(m, x[i] == x[i] ? route_key(x[i]) : 0u);
    m = wave_max(m);
    const float top = m == 0 ? -INFINITY : __uint_as_float(m & 0x80000000u ? m & 0x7fffffffu : ~m);
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      // (what is as large as the largest has e^0, infinite or not; all of -infinity: nothing has a score)
      s[i] = x[i] == -INFINITY ? 0.0 : x[i] == top ? 1.0 : exp((double)x[i] - (double)top);
      sum += s[i];
    }
    sum = wave_total(sum);
    const double inv = sum == 0.0 ? 0.0 : 1.0 / sum;
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] *= inv;
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = 1.0 / (1.0 + exp(-(double)x[i]));
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    key[i] = 0;
    if (ex[i] == MAX_EXPERTS) continue;
    key[i] = score_key(s[i] + (rule.bias ? (double)rule.bias[lane + 64 * i] : 0.0));
    lds.s[lane + 64 * i] = s[i];
    if (rule.n_groups > 1) lds.c[lane + 64 * i] = key[i];
  }
  wave_lds();
  if (rule.n_groups > 1) {
    open_groups(E, rule, lane, lds);
    const int of_group = E / rule.n_groups, inv = (65535 + of_group) / of_group;  // (e inv >> 16 is e / of_group for all e < 256)
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (ex[i] < MAX_EXPERTS && !lds.open[ex[i] * inv >> 16]) { key[i] = 0; ex[i] = MAX_EXPERTS; }
  }
  // The keys of a lane in order, (larger key, then lower expert) first, so that a round looks at one of them
  auto before = [](uint64_t k0, int e0, uint64_t k1, int e1) { return k0 > k1 || (k0 == k1 && e0 < e1); };
  auto order = [&](int i, int j) {
    if (before(key[j], ex[j], key[i], ex[i])) {
      const uint64_t t = key[i]; key[i] = key[j]; key[j] = t;
      const int e = ex[i]; ex[i] = ex[j]; ex[j] = e;
    }
  };
  if constexpr (N == 2) order(0, 1);
  if constexpr (N == 4) { order(0, 1); order(2, 3); order(0, 2); order(1, 3); order(1, 2); }
  // k rounds: the largest key of the wave, by its upper half where only one lane has that, then the lowest expert that has it
  int sel[N];
#pragma unroll
  for (int i = 0; i < N; ++i) sel[i] = 0;
  for (int r = 0; r < k; ++r) {
    const uint32_t hi = (uint32_t)(key[0] >> 32), top = wave_max(hi);
    unsigned long long who = __ballot(hi == top);
    if (who & (who - 1)) {
      const uint32_t lo = (uint32_t)key[0], low = wave_max(hi == top ? lo : 0u);
      const bool equal = hi == top && lo == low;
      const uint32_t e = equal ? MAX_EXPERTS - (uint32_t)ex[0] : 0u, first = wave_max(e);  // (of no expert: 0)
      who = __ballot(equal && e == first);
    }
    const int w = __builtin_ctzll(who), e = __builtin_amdgcn_readlane(ex[0], w);
#pragma unroll
    for (int g = 0; g < N; ++g)
      if ((g == 0 || k > 64) && lane + 64 * g == r) sel[g] = e;
    if (lane == w) {
#pragma unroll
      for (int i = 0; i + 1 < N; ++i) { key[i] = key[i + 1]; ex[i] = ex[i + 1]; }
      key[N - 1] = 0;
      ex[N - 1] = MAX_EXPERTS;
    }
  }
  double v[N], sum = 0.0;
#pragma unroll
  for (int g = 0; g < N; ++g) {
    v[g] = lane + 64 * g < k ? lds.s[sel[g]] : 0.0;
    sum += v[g];
  }
  const double scale = rule.scale == 0.f ? 1.0 : (double)rule.scale;
  if (rule.renorm) {
    sum = wave_total(sum);
#pragma unroll
    for (int g = 0; g < N; ++g) v[g] = sum == 0.0 ? 0.0 : v[g] / sum;
  }
#pragma unroll
  for (int g = 0; g < N; ++g)
    if (lane + 64 * g < k) put(lane + 64 * g, sel[g], (float)(v[g] * scale));
}

template <class F> __device__ __forceinline__ void scored_token(const float* __restrict__ l, int E, int k, const si_score_t& rule, int lane, ScoreLds& lds, F put) {
  if (E <= 64) scored_rounds<1>(l, E, k, rule, lane, lds, put);
  else if (E <= 128) scored_rounds<2>(l, E, k, rule, lane, lds, put);
  else scored_rounds<4>(l, E, k, rule, lane, lds, put);
}

}  // namespace si
