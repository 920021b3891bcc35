// Choice of experts by scores (hipcc only): softmax over all logits or sigmoid of each, a bias for the choice, groups, k of them.
//
//   s_e = e^(x_e - max) / sum e^(x - max)   or   1 / (1 + e^-x_e),      c_e = s_e + b_e
//   a group's worth: the sum of its group_best largest c;   the top_groups worthiest stay open
//   the k largest c of the open groups (ties: the lower expert),   w = scale s / sum of the k s   (or scale s)
// Scores, sums and comparisons are in 64 bits: two experts whose c differ by less than 2^-24 of it would come out in the order of their
// roundings, and the sum with a bias rounds scores that do differ together (of 8192 tokens on 256 experts dozens).
#pragma once
#include "si_internal.h"
#include "route_device.h"

namespace si {

struct ScoreLds {  // of a wave
  double c[MAX_EXPERTS];      // then, of the groups, their worth
  uint32_t open[MAX_EXPERTS];
};

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int d = 32; d > 0; d /= 2) v += __shfl_xor(v, d);
  return v;
}

// order-preserving map to an unsigned integer; NaN: 0, below -infinity
__device__ __forceinline__ uint64_t score_key(double v) {
  const uint64_t u = (uint64_t)__double_as_longlong(v);
  return v != v ? 0 : u >> 63 ? ~u : u | 1ull << 63;
}

// LDS of a wave: its accesses are in order, only the compiler has to keep it
__device__ __forceinline__ void wave_lds() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
}

// N experts a lane: lane + 64 i
template <int N, class F> __device__ __forceinline__ void scored_rounds(const float* __restrict__ l, int E, int k, const si_score_t& rule, int lane, ScoreLds& lds, F put) {
  float x[N];
  double s[N];
  uint64_t key[N];
  bool in[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    in[i] = lane + 64 * i < E;
    x[i] = in[i] ? l[lane + 64 * i] : -INFINITY;
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
    sum = wave_sum(sum);
    const double inv = sum == 0.0 ? 0.0 : 1.0 / sum;
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] *= inv;
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = 1.0 / (1.0 + exp(-(double)x[i]));
  }
  if (rule.n_groups > 1) {
    const int of_group = E / rule.n_groups;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (in[i]) lds.c[lane + 64 * i] = s[i] + (rule.bias ? (double)rule.bias[lane + 64 * i] : 0.0);
    wave_lds();
    uint64_t worth[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int g = lane + 64 * i;
      worth[i] = 0;
      if (g >= rule.n_groups) continue;
      const double* c = lds.c + g * of_group;
      // the largest, then the largest after it in the order of (value, place), and so on
      double sum = 0.0;
      uint64_t last = ~0ull;
      int last_at = -1;
      for (int r = 0; r < rule.group_best; ++r) {
        uint64_t best = 0;
        int at = of_group;
        for (int e = 0; e < of_group; ++e) {
          const uint64_t ke = score_key(c[e]);
          const bool left = ke < last || (ke == last && e > last_at);
          if (left && (at == of_group || ke > best)) { best = ke; at = e; }
        }
        sum += c[at];
        last = best;
        last_at = at;
      }
      worth[i] = score_key(sum);
    }
    wave_lds();
    uint64_t* all = reinterpret_cast<uint64_t*>(lds.c);
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (lane + 64 * i < rule.n_groups) all[lane + 64 * i] = worth[i];
    wave_lds();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int g = lane + 64 * i;
      if (g >= rule.n_groups) continue;
      int before = 0;
      for (int h = 0; h < rule.n_groups; ++h) before += all[h] > worth[i] || (all[h] == worth[i] && h < g);
      lds.open[g] = before < rule.top_groups;
    }
    wave_lds();
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (in[i]) in[i] = lds.open[(lane + 64 * i) / of_group] != 0;
  }
  unsigned long long open[N];  // lanes whose i-th expert may be chosen yet
#pragma unroll
  for (int i = 0; i < N; ++i) {
    key[i] = in[i] ? score_key(s[i] + (rule.bias ? (double)rule.bias[lane + 64 * i] : 0.0)) : 0;
    open[i] = __ballot(in[i]);
  }
  // k rounds: the largest key of the wave, its upper half first, then the lowest expert that has it
  double sel_s[N];
  int sel_e[N];
#pragma unroll
  for (int i = 0; i < N; ++i) { sel_s[i] = 0.0; sel_e[i] = 0; }
  double sum = 0.0;
  for (int r = 0; r < k; ++r) {
    uint64_t m = key[0];
#pragma unroll
    for (int i = 1; i < N; ++i) m = max(m, key[i]);
    const uint32_t hi = wave_max((uint32_t)(m >> 32)), lo = wave_max((uint32_t)(m >> 32) == hi ? (uint32_t)m : 0u);
    m = (uint64_t)hi << 32 | lo;
    bool found = false;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const unsigned long long c = __ballot(key[i] == m) & open[i];
      if (!found && c) {
        const int w = __builtin_ctzll(c);
        const uint64_t bits = (uint64_t)__double_as_longlong(s[i]);
        const double v = __longlong_as_double((long long)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(bits >> 32), w) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)bits, w)));
        sum += v;
#pragma unroll
        for (int g = 0; g < N; ++g)
          if (lane + 64 * g == r) { sel_s[g] = v; sel_e[g] = w + 64 * i; }
        if (lane == w) key[i] = 0;
        open[i] &= ~(1ull << w);
        found = true;
      }
    }
  }
  const double scale = rule.scale == 0.f ? 1.0 : (double)rule.scale;
#pragma unroll
  for (int g = 0; g < N; ++g)
    if (lane + 64 * g < k) put(lane + 64 * g, sel_e[g], (float)(rule.renorm ? (sum == 0.0 ? 0.0 : sel_s[g] / sum * scale) : sel_s[g] * scale));
}

template <class F> __device__ __forceinline__ void scored_token(const float* __restrict__ l, int E, int k, const si_score_t& rule, int lane, ScoreLds& lds, F put) {
  if (E <= 64) scored_rounds<1>(l, E, k, rule, lane, lds, put);
  else scored_rounds<4>(l, E, k, rule, lane, lds, put);
}

}  // namespace si
