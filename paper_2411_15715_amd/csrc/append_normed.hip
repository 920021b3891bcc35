// New tokens into the paged cache with a norm of each head of q and k before its rotation, in the same pass:
//   n = w x / sqrt(mean(x^2) + eps) + b   (of x, or of x - mean(x)),   then R(p) n, rounded once
// L lanes have a head, 16 of its elements each (12 of 16 lanes with heads of 192, 6 of 8 with 96): the two vectors of 8 that turn into
// each other, so that statistics, weights and rotation meet in registers and nothing is read twice.  Sums are over the 16 elements of a lane, then
// over neighbouring lanes; the second moment of a norm about the mean is taken about the mean.  v goes its way as without the norm.
// Bound by memory, as the append without a norm: 4099 tokens of 64 + 8 heads of 128 (160 MB) into e4m3 38.3 us, 4.2 TB/s (without norm 38.2); in
// between, by the waves that fit: with 150 registers, the weights of q and k among them, 66 us, with 64 forced 46.  8 tokens: 4.7 us in the kernel.
#include "si_error.h"
#include "append_device.h"
#include "wave_device.h"

#include <algorithm>
#include <cmath>

namespace si {
namespace {

typedef u32x4 u32x4_a4 __attribute__((aligned(4)));

struct NormedArgs {
  Args g;
  si_head_norm_t n;
};

template <int CTRL> __device__ __forceinline__ float plus_dpp(float v) {
  return v + __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xf, 0xf, true));
}
// over L neighbouring lanes, the same in all of them
template <int L> __device__ __forceinline__ float sum_of(float v) {
  v = plus_dpp<0xb1>(v);                         // lanes 1 0 3 2
  v = plus_dpp<0x4e>(v);                         // lanes 2 3 0 1
  if constexpr (L >= 8) v = plus_dpp<0x141>(v);  // 8 lanes mirrored
  if constexpr (L >= 16) v = plus_dpp<0x140>(v); // 16 lanes mirrored
  return v;
}

__device__ __forceinline__ float weight_at(const void* w, int type, int at) {
  return type == SI_BF16 ? widen(static_cast<const uint16_t*>(w)[at]) : static_cast<const float*>(w)[at];
}
__device__ __forceinline__ void weights_at(const void* w, int type, int at, float (&f)[8]) {
  if (type == SI_BF16) {
    const u32x4 v = *reinterpret_cast<const u32x4_a2*>(static_cast<const uint16_t*>(w) + at);
    widen8(v, f);
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const u32x4 v = *reinterpret_cast<const u32x4_a4*>(static_cast<const float*>(w) + at + 4 * h);
#pragma unroll
      for (int i = 0; i < 4; ++i) f[4 * h + i] = __uint_as_float(v[i]);
    }
  }
}
// GENERAL: each head has weights of its own, or the halves of the rotated part do not begin at a vector of 8, so that the other element of a
// pair is in another lane.  Else the weights that all heads share lie in LDS, in fp32, and a lane has both elements of its pairs.
template <int TYPE, int L, bool GENERAL> __device__ void normed_part(const NormedArgs& na, int block) {
  __shared__ float2 s_turn[MAX_TOKENS][MAX_ANGLES];
  __shared__ Token s_token[MAX_TOKENS];
  __shared__ float s_x[GENERAL ? THREADS / L : 1][GENERAL ? 16 * L : 1];
  __shared__ __align__(16) float s_w[2][GENERAL ? 4 : 16 * L], s_b[2][GENERAL ? 4 : 16 * L];  // of q, of k
  constexpr int E = TYPE == SI_KV_E4M3 ? 16 : 8;
  const Args& g = na.g;
  const si_append_t& a = g.a;
  const si_head_norm_t& nm = na.n;
  const int d = g.c.head_dim, rot = a.rot_dim, half = rot / 2, tid = threadIdx.x, j = tid % L;
  const int t0 = block / g.qk_columns * g.per_block, n = min(g.per_block, a.n_tokens - t0), column = block % g.qk_columns;
  const int n_heads = a.q ? a.n_heads : 0, heads = n_heads + g.c.n_kv_heads;
  const int span = (heads + g.qk_columns - 1) / g.qk_columns, h0 = column * span, width = max(0, min(heads, h0 + span) - h0), all = width * n * L;
  const bool here = 16 * j < d, by_halves = !GENERAL && !a.rot_pairs;
  // first elements of this lane's two vectors
  const int d0 = by_halves && j < rot / 16 ? 8 * j : 16 * j, d1 = by_halves && j < rot / 16 ? 8 * j + half : 16 * j + 8;

  struct Unit {
    u32x4 x, y;
    int t, head;
  };
  auto fetch = [&](int f) {
    Unit k;
    k.t = 0;
    int u = f / L;
    while (u >= width) { u -= width; ++k.t; }
    k.head = u + h0;
    const bool is_q = k.head < n_heads;
    const uint16_t* p = static_cast<const uint16_t*>(is_q ? a.q : a.k) + (int64_t)(t0 + k.t) * (is_q ? a.q_stride : a.k_stride) + (is_q ? k.head : k.head - n_heads) * d;
    k.x = k.y = u32x4{0, 0, 0, 0};
    if (here) {
      k.x = __builtin_nontemporal_load(reinterpret_cast<const u32x4_a2*>(p + d0));
      k.y = __builtin_nontemporal_load(reinterpret_cast<const u32x4_a2*>(p + d1));
    }
    return k;
  };
  Unit next;
  if (tid < all) next = fetch(tid);
  if constexpr (!GENERAL)
    for (int i = tid; i < 2 * d; i += THREADS) {
      const int which = i >= d, at = i - which * d;
      const void *w = which ? nm.w_k : nm.w_q, *b = which ? nm.b_k : nm.b_q;
      s_w[which][at] = w ? weight_at(w, nm.w_type, at) : 1.f;
      s_b[which][at] = b ? weight_at(b, nm.w_type, at) : 0.f;
    }
  for (int i = tid; i < n * half; i += THREADS) s_turn[i / half][i % half] = turn(a.pos[t0 + i / half], a.inv_freq[i % half]);
  if (tid < n) {
    const int seq = a.seq[t0 + tid], pos = a.pos[t0 + tid];
    Token t{-1, 0};
    if (seq != -1) {
      int why = 0;
      const int page = kv_page_of(g.c, seq, pos, why);
      if (page >= 0) {
        const int in_page = pos % g.c.page_tokens;
        t.k = page * kv_page_elems(g.c) + kv_head_offset(g.c, g.layer, 0, 0) + (int64_t)(in_page / (4 * E)) * (4 * E * d);
        t.slot = kv_slot(E, in_page % (4 * E));
      } else if (column == 0) {
        atomicOr(g.c.status, why);
      }
    }
    s_token[tid] = t;
  }
  __syncthreads();
  const float per_d = 1.f / (float)d;
  for (int f = tid; f < all; f += THREADS) {
    const Unit k = next;
    if (f + THREADS < all) next = fetch(f + THREADS);
    const Token tok = s_token[k.t];
    const bool is_q = k.head < n_heads;
    const int head = is_q ? k.head : k.head - n_heads;
    float x[8], y[8];
    widen8(k.x, x);
    widen8(k.y, y);
    if (nm.kind == SI_NORM_MEAN) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += x[i] + y[i];
      const float mean = sum_of<L>(sum) * per_d;
#pragma unroll
      for (int i = 0; i < 8; ++i) { x[i] -= mean; y[i] -= mean; }
    }
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += x[i] * x[i] + y[i] * y[i];
    const float rs = rsqrtf(sum_of<L>(here ? sum : 0.f) * per_d + nm.eps);
    if (here) {
      if constexpr (GENERAL) {
        const void *w = is_q ? nm.w_q : nm.w_k, *b = is_q ? nm.b_q : nm.b_k;
        const int first = nm.per_head ? head * d : 0;
        auto take = [&](int at, float (&v)[8]) {
          float t[8];
          if (w) {
            weights_at(w, nm.w_type, first + at, t);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] *= t[i];
          }
          if (b) {
            weights_at(b, nm.w_type, first + at, t);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += t[i];
          }
        };
#pragma unroll
        for (int i = 0; i < 8; ++i) { x[i] *= rs; y[i] *= rs; }
        take(d0, x);
        take(d1, y);
      } else {
        const float *w = s_w[!is_q], *b = s_b[!is_q];
        const bool biased = (is_q ? nm.b_q : nm.b_k) != nullptr;
#pragma unroll
        for (int i = 0; i < 8; ++i) { x[i] = x[i] * rs * w[d0 + i]; y[i] = y[i] * rs * w[d1 + i]; }
        if (biased)
#pragma unroll
          for (int i = 0; i < 8; ++i) { x[i] += b[d0 + i]; y[i] += b[d1 + i]; }
      }
    }
    if constexpr (GENERAL) {
      float* row = s_x[tid / L];
#pragma unroll
      for (int i = 0; i < 8; ++i) { row[d0 + i] = x[i]; row[d1 + i] = y[i]; }
      wave_lds();
      for (int u = j; u < half; u += L) {
        const float2 cs = s_turn[k.t][u];
        const int i0 = a.rot_pairs ? 2 * u : u, i1 = a.rot_pairs ? 2 * u + 1 : u + half;
        const float p = row[i0], q = row[i1];
        row[i0] = p * cs.x - q * cs.y;
        row[i1] = q * cs.x + p * cs.y;
      }
      wave_lds();
#pragma unroll
      for (int i = 0; i < 8; ++i) { x[i] = row[d0 + i]; y[i] = row[d1 + i]; }
      wave_lds();
    } else if (by_halves) {
      if (j < rot / 16) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float2 cs = s_turn[k.t][8 * j + i];
          const float p = x[i], q = y[i];
          x[i] = p * cs.x - q * cs.y;
          y[i] = q * cs.x + p * cs.y;
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float& p = i < 4 ? x[(2 * i) % 8] : y[(2 * i) % 8];
        float& q = i < 4 ? x[(2 * i + 1) % 8] : y[(2 * i + 1) % 8];
        if (8 * j + i < half) {
          const float2 cs = s_turn[k.t][8 * j + i];
          const float p0 = p, q0 = q;
          p = p0 * cs.x - q0 * cs.y;
          q = q0 * cs.x + p0 * cs.y;
        }
      }
    }
    if (!here) continue;
    if (is_q) {
      uint16_t* dst = static_cast<uint16_t*>(a.q_out) + (int64_t)(t0 + k.t) * a.q_out_stride + head * d;
      const bool out = tok.k < 0;
      *reinterpret_cast<u32x4_a2*>(dst + d0) = out ? u32x4{0, 0, 0, 0} : pack8(x);
      *reinterpret_cast<u32x4_a2*>(dst + d1) = out ? u32x4{0, 0, 0, 0} : pack8(y);
    } else if (tok.k >= 0) {
      store_k<TYPE>(g, tok, head, d0, x);
      store_k<TYPE>(g, tok, head, d1, y);
    }
  }
}

template <int TYPE, int L, bool GENERAL> __global__ __launch_bounds__(THREADS) void k_append_normed(NormedArgs na) {
  const Args& g = na.g;
  if ((int)blockIdx.x < g.v_blocks) v_part<TYPE>(g, blockIdx.x);
  else {
    const int block = on_one_die(blockIdx.x - g.v_blocks, gridDim.x - g.v_blocks, g.run);
    normed_part<TYPE, L, GENERAL>(na, block);
  }
}

// How a call is cut into blocks; returns their number.
int64_t cut(Args& g, int lanes) {
  const si_cache_t& c = g.c;
  const si_append_t& a = g.a;
  const int units = ((a.q ? a.n_heads : 0) + c.n_kv_heads) * lanes;
  // A block has the heads of up to 4 tokens, whose angles and weights are formed once, as long as there are some 1000 blocks: 4099 tokens of 576 lanes in
  // blocks of 1, 2, 4 tokens 40.7, 40.2, 39.0 us (e4m3), by three blocks a token 54.8; 1931 of 256 lanes 14.2, 13.4, 15.6.  With few tokens a
  // lane has one head (what waits there is memory).
  const int want = THREADS * (a.n_tokens >= 256 ? 9 : 1);
  if (units >= want) g.qk_columns = (units + want - 1) / want;
  else if (a.n_tokens >= 256) g.per_block = std::clamp(a.n_tokens / 960, 1, std::min(MAX_TOKENS, want / units));
  const int E = kv_vec(c.type);
  g.v_columns = (c.n_kv_heads * c.head_dim + THREADS - 1) / THREADS;
  g.v_blocks = (a.n_tokens + E - 1) / E * g.v_columns;
  g.run = 32 / g.per_block * g.qk_columns;
  return (int64_t)((a.n_tokens + g.per_block - 1) / g.per_block) * g.qk_columns + g.v_blocks;
}

template <int TYPE, bool GENERAL> hipError_t launch(const NormedArgs& na, int lanes, int64_t blocks, hipStream_t stream) {
  const dim3 grid((unsigned)blocks);
  if (lanes == 4) hipLaunchKernelGGL((k_append_normed<TYPE, 4, GENERAL>), grid, dim3(THREADS), 0, stream, na);
  else if (lanes == 8) hipLaunchKernelGGL((k_append_normed<TYPE, 8, GENERAL>), grid, dim3(THREADS), 0, stream, na);
  else hipLaunchKernelGGL((k_append_normed<TYPE, 16, GENERAL>), grid, dim3(THREADS), 0, stream, na);
  return hipGetLastError();
}

bool misaligned(const void* p, int to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

}  // namespace
}  // namespace si

extern "C" int si_cache_append_normed(const si_cache_t* c, int32_t layer, const si_append_t* a, const si_head_norm_t* n, void* stream) {
  using namespace si;
  const char* who = "si_cache_append_normed";
  bool nothing;
  if (int rc = check_append(c, layer, a, who, &nothing)) return rc;
  if (!n) return set_error(SI_EINVAL, "%s: the norm's descriptor is NULL", who);
  if (n->kind != SI_NORM_NONE && n->kind != SI_NORM_RMS && n->kind != SI_NORM_MEAN) return set_error(SI_EINVAL, "%s: unknown norm %d", who, n->kind);
  if (n->w_type != SI_F32 && n->w_type != SI_BF16) return set_error(SI_EINVAL, "%s: unknown type %d of the weights", who, n->w_type);
  if (!(n->eps >= 0.f) || !std::isfinite(n->eps)) return set_error(SI_EINVAL, "%s: eps is negative or not finite", who);
  const int to = n->w_type == SI_F32 ? 4 : 2;
  if (misaligned(n->w_q, to) || misaligned(n->b_q, to) || misaligned(n->w_k, to) || misaligned(n->b_k, to))
    return set_error(SI_EINVAL, "%s: a weight or bias is not aligned to its type", who);
  if (nothing) return SI_OK;
  if (n->kind == SI_NORM_NONE) return si_cache_append(c, layer, a, stream);
  NormedArgs na{{*c, *a, layer, 1, 1, 0, 0, 1}, *n};
  const int lanes = c->head_dim <= 64 ? 4 : c->head_dim <= 128 ? 8 : 16;
  const int64_t blocks = cut(na.g, lanes);
  if (blocks >= (1 << 24))  // (a launch has fewer than 2^32 threads)
    return set_error(SI_EINVAL, "%s: too many tokens and heads in one call (%d, %d)", who, a->n_tokens, a->n_heads);
  const bool general = n->per_head || (!a->rot_pairs && a->rot_dim % 16 != 0);
  const auto f = c->type == SI_KV_BF16 ? (general ? launch<SI_KV_BF16, true> : launch<SI_KV_BF16, false>) : (general ? launch<SI_KV_E4M3, true> : launch<SI_KV_E4M3, false>);
  const hipError_t e = f(na, lanes, blocks, (hipStream_t)stream);
  if (e != hipSuccess) return set_error(SI_EHIP, "append launch failed: %s", hipGetErrorString(e));
  return SI_OK;
}
