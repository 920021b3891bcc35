// Attention of a few new tokens over the paged cache: the kernel (hipcc only; instantiated by attend_bf16.hip and attend_e4m3.hip).
//
// The rows of a block are the query heads that share a kv head, for all new tokens: up to 16 NT of them.  Per cache block of
// B tokens a wave forms S^T = K Q^T (matrix instructions with K as the left operand) and O^T += V^T P^T.  The cache holds K and V in the
// operand order of these instructions, so a wave loads both from memory into the registers that multiply, 16 bytes a lane and
// 1 KB in a run; and the tokens of a K block are placed so that the scores a lane receives are those of the
// tokens whose weights it has to hold for the second product: nothing passes through LDS or between lanes but the maximum of a row.
// Running maximum m and sum l (base 2) per row; the waves of a block and the blocks of a split sequence are joined by
//   m = max m_i,  l = sum l_i 2^(m_i - m),  o = sum o_i 2^(m_i - m)
// by the block that finishes last, in the order of the splits, so that the result does not depend on who that is.
#pragma once
#include <hip/hip_runtime.h>

#include "kv_layout.h"

namespace si {

constexpr int ATTEND_WAVES = 4;
constexpr int ATTEND_THREADS = 64 * ATTEND_WAVES;
constexpr int ATTEND_COUNTERS = 16384;  // units (sequence, kv head, row group) of a launch that may be split

struct AttendArgs {
  si_cache_t c;
  si_attend_t a;
  int layer;
  int rows;      // rows of a unit in all: n_new * heads per kv head
  int groups;    // row groups
  int splits;    // parts that a sequence of max_len is cut into
  int chunk;     // cache blocks of a part, at least
  float scale2;  // scale * log2(e)
  float* part;   // [unit][split][16 NT rows][D + 2]: o, then m, l of each row
  uint32_t* count;
};

hipError_t launch_attend_bf16(const AttendArgs& g, int nt, hipStream_t stream);
hipError_t launch_attend_e4m3(const AttendArgs& g, int nt, hipStream_t stream);

#if defined(__HIPCC__)
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_a2 __attribute__((aligned(2)));
typedef u32x2 u32x2_a2 __attribute__((aligned(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  const bf16x2 p = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, p);
}
__device__ __forceinline__ bf16x8 operand(const u32x4& v) { return __builtin_bit_cast(bf16x8, v); }
// eight e4m3 codes as bf16 (exact)
__device__ __forceinline__ bf16x8 operand8(uint32_t lo, uint32_t hi) {
  u32x4 r;
  r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false));
  r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true));
  r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false));
  r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true));
  return operand(r);
}

// over the lanes of a wave that hold the same row (16 apart)
__device__ __forceinline__ float max_of_row(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_of_row(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// 2^x for x <= 0 or -infinity
__device__ __forceinline__ float pow2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float finite_base(float m) { return m == -INFINITY ? 0.f : m; }

// Values that other blocks (on other dies, with caches of their own) read within the launch: device-scope accesses go to memory
__device__ __forceinline__ void put2(float* p, float a, float b) {
  const uint64_t v = (uint64_t)__float_as_uint(a) | (uint64_t)__float_as_uint(b) << 32;
  __hip_atomic_store(reinterpret_cast<uint64_t*>(p), v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 get2(const float* p) {
  const uint64_t v = __hip_atomic_load(reinterpret_cast<const uint64_t*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return make_float2(__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32)));
}

template <int TYPE, int D, int NT> struct Attend {
  static constexpr int E = TYPE == SI_KV_E4M3 ? 16 : 8, B = 4 * E, J = E / 4;  // J score tiles of 16 tokens
  static constexpr int NL = D / 16;                                           // loads of 16 bytes of K, and of V, a lane and block
  static constexpr int H = E / 8;                                             // operands of 8 elements in 16 bytes
  static constexpr int ROWS = 16 * NT, PAD = D + 4;                           // (rows of 16 banks more: the four groups of lanes write side by side)
  static constexpr int PART = ROWS * (D + 2);

  struct Lds {
    float o[ATTEND_WAVES][16][PAD];
    float m[ATTEND_WAVES][16], l[ATTEND_WAVES][16];
    uint32_t arrived;
  };

  // words of 16 bytes of V of this lane (E tokens from t0 on) that lie in [lo, hi)
  static __device__ __forceinline__ u32x4 token_mask(int t0, int lo, int hi) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[i] = 0;
#pragma unroll
      for (int e = 0; e < E / 4; ++e) {
        const int t = t0 + i * (E / 4) + e;
        if (t >= lo && t < hi) w[i] |= (E == 8 ? 0xffffu : 0xffu) << (e * (E == 8 ? 16 : 8));
      }
    }
    return w;
  }
  static __device__ __forceinline__ bool not_finite(const u32x4& v) {
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < E / 4; ++e) {
        if constexpr (E == 8) bad |= (v[i] >> (16 * e) & 0x7f80u) == 0x7f80u;
        else bad |= (v[i] >> (8 * e) & 0x7fu) == 0x7fu;
      }
    return bad;
  }

  static __device__ __forceinline__ void write_row(const AttendArgs& g, int seq_i, int kv, int row, int dim, const f32x4& o, float m, float l, float scale_v) {
    const int per = g.a.n_heads / g.c.n_kv_heads, j = row / per, head = kv * per + row % per;
    const int64_t r = (int64_t)seq_i * g.a.n_new + j;
    const float inv = l == 0.f ? 0.f : scale_v / l;
    *reinterpret_cast<u32x2_a2*>(static_cast<uint16_t*>(g.a.out) + r * g.a.out_stride + (int64_t)head * D + dim) =
        u32x2{bf16_pair(o[0] * inv, o[1] * inv), bf16_pair(o[2] * inv, o[3] * inv)};
    if (dim == 0 && g.a.lse) g.a.lse[r * g.a.n_heads + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
  }

  static __device__ void run(const AttendArgs& g, Lds& s) {
    const si_cache_t& c = g.c;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), grp = lane / 16, col = lane % 16;
    const int split = blockIdx.x, kv = blockIdx.y / g.groups, row0 = blockIdx.y % g.groups * ROWS, seq_i = blockIdx.z;
    const int per = g.a.n_heads / c.n_kv_heads, n_new = g.a.n_new;
    const int row_end = min(g.rows, row0 + ROWS);
    const bool reports = blockIdx.y == 0 && threadIdx.x == 0;

    // what the rows of this group see: [lo, hi), every one of them [lo_all, hi_all)
    const int seq = g.a.seqs ? g.a.seqs[seq_i] : seq_i;
    int len = 0;
    if (seq >= 0 && seq < c.n_seqs) {
      len = c.lens[seq];
      const int most = c.max_pages * c.page_tokens;
      if (len < 0 || len > most) {
        if (reports && split == 0) atomicOr(c.status, SI_CACHE_BAD_LEN);
        len = len < 0 ? 0 : most;
      }
    } else if (reports && split == 0) {
      atomicOr(c.status, SI_CACHE_BAD_SEQ);
    }
    const int window = g.a.window < len ? g.a.window : 0;
    const int first = len - n_new + 1;  // where the sight of token 0 ends
    const int hi = max(0, first + (row_end - 1) / per), hi_all = max(0, first + row0 / per);
    const int lo = window ? max(0, first + row0 / per - window) : 0, lo_all = window ? max(0, first + (row_end - 1) / per - window) : 0;
    const int fb = lo / B, nb = hi > lo ? (hi + B - 1) / B - fb : 0;
    const int chunk = max(g.chunk, (nb + g.splits - 1) / g.splits), active = max(1, (nb + chunk - 1) / chunk);
    if (split >= active) return;
    const int b0 = fb + split * chunk, b1 = min(b0 + chunk, fb + nb);

    const int32_t* table = c.table + (int64_t)max(seq, 0) * c.max_pages;  // (read where nb > 0 only)
    const int64_t page_bytes = kv_page_elems(c) * (TYPE == SI_KV_E4M3 ? 1 : 2), block_bytes = 64 * D;
    const char* k_base = static_cast<const char*>(c.pages) + kv_head_offset(c, g.layer, 0, kv) * (TYPE == SI_KV_E4M3 ? 1 : 2);
    const char* v_base = static_cast<const char*>(c.pages) + kv_head_offset(c, g.layer, 1, kv) * (TYPE == SI_KV_E4M3 ? 1 : 2);
    const int blocks_per_page = c.page_tokens / B;
    const int k_lane = grp * (B * 16) + col * 16, v_lane = grp * (D * 16) + col * 16;

    u32x4 q[NT][D / 32];
    int q_lo[NT], q_hi[NT], q_tok[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int row = row0 + 16 * t + col, j = row / per;
      const bool in = row < row_end;
      q_tok[t] = in ? j : -1;
      q_hi[t] = in ? max(0, first + j) : 0;
      q_lo[t] = in && window ? max(0, first + j - window) : 0;
      const uint16_t* p = static_cast<const uint16_t*>(g.a.q) + ((int64_t)seq_i * n_new + j) * g.a.q_stride + (int64_t)(kv * per + row % per) * D;
#pragma unroll
      for (int x = 0; x < D / 32; ++x) {
        // operand x of K covers, in this lane, elements 32 x + 8 grp of a head (bf16), or half x % 2 of the 16 from 64 (x / 2) + 16 grp on
        const int dim = E == 8 ? 32 * x + 8 * grp : 64 * (x / 2) + 16 * grp + 8 * (x % 2);
        q[t][x] = in ? u32x4(*reinterpret_cast<const u32x4_a2*>(p + dim)) : u32x4{0, 0, 0, 0};
      }
    }
    const float sc = g.scale2 * (TYPE == SI_KV_E4M3 && c.scale_k ? c.scale_k[kv] : 1.f);
    const float scale_v = TYPE == SI_KV_E4M3 && c.scale_v ? c.scale_v[kv] : 1.f;

    f32x4 o[NT][NL];
    float m[NT], l[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      m[t] = -INFINITY;
      l[t] = 0.f;
#pragma unroll
      for (int i = 0; i < NL; ++i) o[t][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // page numbers of the wave's next 64 blocks, one a lane
    int pages = 0;
    auto page_of = [&](int turn) {
      if (turn % 64 == 0) {
        const int b = b0 + wave + ATTEND_WAVES * (turn + lane);
        pages = b < b1 ? table[b / blocks_per_page] : 0;
      }
      const int p = __builtin_amdgcn_readlane(pages, turn % 64);
      return p >= 0 && p < c.n_pages ? p : -1;
    };
    u32x4 kf[NL], vf[NL];
    auto load_k = [&](int page, int b) {
      const char* p = k_base + max(page, 0) * page_bytes + (b % blocks_per_page) * block_bytes;
#pragma unroll
      for (int i = 0; i < NL; ++i) kf[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p + k_lane + (i / J) * (4 * B * 16) + (i % J) * 256));
    };
    auto load_v = [&](int page, int b) {
      const char* p = v_base + max(page, 0) * page_bytes + (b % blocks_per_page) * block_bytes;
#pragma unroll
      for (int i = 0; i < NL; ++i) vf[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p + v_lane + i * 256));
    };

    int turn = 0, b = b0 + wave, page = 0;
    if (b < b1) {
      page = page_of(0);
      load_k(page, b);
      load_v(page, b);
    }
    bool bad_page = false;
    for (; b < b1; b += ATTEND_WAVES) {
      // scores of the block: tile j, element i of this lane is token grp * E + 4 j + i
      f32x4 x[NT][J];
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int j = 0; j < J; ++j) x[t][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < NL; ++i)
#pragma unroll
        for (int h = 0; h < H; ++h) {
          const bf16x8 kk = E == 8 ? operand(kf[i]) : operand8(kf[i][2 * h], kf[i][2 * h + 1]);
#pragma unroll
          for (int t = 0; t < NT; ++t) x[t][i % J] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kk, operand(q[t][(i / J) * H + h]), x[t][i % J], 0, 0, 0);
        }
      const int b_next = b + ATTEND_WAVES;
      int page_next = 0;
      if (b_next < b1) {
        page_next = page_of(++turn);
        load_k(page_next, b_next);
      }
      const int t0 = b * B;
      const bool seen = page >= 0;
      bad_page |= !seen;
      const bool edge = !seen || t0 < lo_all || t0 + B > hi_all;  // (not all rows see all tokens)
      u32x4 p[NT][H];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float v = x[t][j][i] * sc;
            if (edge) {
              const int pos = t0 + grp * E + 4 * j + i;
              v = seen && pos >= q_lo[t] && pos < q_hi[t] ? v : -INFINITY;
            }
            x[t][j][i] = v;
            top = fmaxf(top, v);
          }
        const float m_new = fmaxf(m[t], max_of_row(top)), base = finite_base(m_new);
        if (__any(m_new > m[t])) {
          const float f = pow2(m[t] - base);
          l[t] *= f;
#pragma unroll
          for (int i = 0; i < NL; ++i) o[t][i] *= f;
          m[t] = m_new;
        }
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const int j = 2 * h + w / 2, i = 2 * (w % 2);
            const float a = pow2(x[t][j][i] - base), e = pow2(x[t][j][i + 1] - base);
            l[t] += a + e;
            p[t][h][w] = bf16_pair(a, e);
          }
      }
      bool apart = false;
      if (edge) {
        // what no row sees may be anything: weight 0 times infinity would be NaN
        const u32x4 keep = seen ? token_mask(t0 + grp * E, lo, hi) : u32x4{0, 0, 0, 0};
        bool bad = false;
#pragma unroll
        for (int i = 0; i < NL; ++i) {
          vf[i] &= keep;
          bad |= not_finite(vf[i]);
        }
        apart = n_new > 1 && __any(bad);
      }
      if (!apart) {
#pragma unroll
        for (int i = 0; i < NL; ++i)
#pragma unroll
          for (int h = 0; h < H; ++h) {
            const bf16x8 vv = E == 8 ? operand(vf[i]) : operand8(vf[i][2 * h], vf[i][2 * h + 1]);
#pragma unroll
            for (int t = 0; t < NT; ++t) o[t][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vv, operand(p[t][h]), o[t][i], 0, 0, 0);
          }
      } else {
        // a value that is not finite, seen by some of the tokens: one product for each of them
        for (int j = row0 / per; j <= (row_end - 1) / per; ++j) {
          const u32x4 keep = token_mask(t0 + grp * E, window ? max(0, first + j - window) : 0, max(0, first + j));
#pragma unroll
          for (int i = 0; i < NL; ++i) {
            const u32x4 v = vf[i] & keep;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
              f32x4 r = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
              for (int h = 0; h < H; ++h) r = __builtin_amdgcn_mfma_f32_16x16x32_bf16(E == 8 ? operand(v) : operand8(v[2 * h], v[2 * h + 1]), operand(p[t][h]), r, 0, 0, 0);
              if (q_tok[t] == j) o[t][i] += r;
            }
          }
        }
      }
      if (b_next < b1) load_v(page_next, b_next);
      page = page_next;
    }
    if (bad_page && lane == 0) atomicOr(c.status, SI_CACHE_BAD_PAGE);

    // the waves of the block, 16 rows at a time
    const int unit = seq_i * gridDim.y + blockIdx.y;
    float* part = g.part + ((int64_t)unit * g.splits + split) * PART;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      if (t > 0) __syncthreads();
      const float sum = sum_of_row(l[t]);
      if (grp == 0) { s.m[wave][col] = m[t]; s.l[wave][col] = sum; }
#pragma unroll
      for (int i = 0; i < NL; ++i) *reinterpret_cast<f32x4*>(&s.o[wave][col][16 * i + 4 * grp]) = o[t][i];
      __syncthreads();
      for (int i = threadIdx.x; i < 16 * D / 4; i += ATTEND_THREADS) {
        const int r = i / (D / 4), dim = i % (D / 4) * 4;
        if (row0 + 16 * t + r >= row_end) continue;
        float mm = -INFINITY;
#pragma unroll
        for (int w = 0; w < ATTEND_WAVES; ++w) mm = fmaxf(mm, s.m[w][r]);
        const float base = finite_base(mm);
        float ll = 0.f;
        f32x4 oo = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < ATTEND_WAVES; ++w) {
          const float f = pow2(s.m[w][r] - base);
          ll += s.l[w][r] * f;
          oo += *reinterpret_cast<const f32x4*>(&s.o[w][r][dim]) * f;
        }
        if (active == 1) {
          write_row(g, seq_i, kv, row0 + 16 * t + r, dim, oo, mm, ll, scale_v);
        } else {
          float* to = part + (16 * t + r) * (D + 2);
          put2(to + dim, oo[0], oo[1]);
          put2(to + dim + 2, oo[2], oo[3]);
          if (dim == 0) put2(to + D, mm, ll);
        }
      }
    }
    if (active == 1) return;

    // the splits of the unit: the last block to arrive joins them.  Its own stores have reached memory before it is counted
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) s.arrived = __hip_atomic_fetch_add(g.count + unit, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (s.arrived != (uint32_t)active - 1) return;
    asm volatile("" ::: "memory");
    if (threadIdx.x == 0) __hip_atomic_store(g.count + unit, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const float* parts = g.part + (int64_t)unit * g.splits * PART;
    for (int i = threadIdx.x; i < (row_end - row0) * (D / 4); i += ATTEND_THREADS) {
      const int r = i / (D / 4), dim = i % (D / 4) * 4;
      float mm = -INFINITY, ll = 0.f;
      f32x4 oo = {0.f, 0.f, 0.f, 0.f};
      constexpr int AHEAD = 8;
      for (int s0 = 0; s0 < active; s0 += AHEAD) {
        float2 ml[AHEAD], v[AHEAD][2];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
          const float* from = parts + (int64_t)min(s0 + k, active - 1) * PART + r * (D + 2);
          ml[k] = get2(from + D);
          v[k][0] = get2(from + dim);
          v[k][1] = get2(from + dim + 2);
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
          if (s0 + k >= active) break;
          const float m_new = fmaxf(mm, ml[k].x), base = finite_base(m_new), f = pow2(mm - base), h = pow2(ml[k].x - base);
          mm = m_new;
          ll = ll * f + ml[k].y * h;
          oo = oo * f + f32x4{v[k][0].x, v[k][0].y, v[k][1].x, v[k][1].y} * h;
        }
      }
      write_row(g, seq_i, kv, row0 + r, dim, oo, mm, ll, scale_v);
    }
  }
};

template <int TYPE, int D, int NT> __global__ __launch_bounds__(ATTEND_THREADS) void k_attend(AttendArgs g) {
  __shared__ typename Attend<TYPE, D, NT>::Lds s;
  Attend<TYPE, D, NT>::run(g, s);
}

template <int TYPE, int D, int NT> hipError_t launch(const AttendArgs& g, hipStream_t stream) {
  hipLaunchKernelGGL((k_attend<TYPE, D, NT>), dim3(g.splits, g.c.n_kv_heads * g.groups, g.a.n), dim3(ATTEND_THREADS), 0, stream, g);
  return hipGetLastError();
}
template <int TYPE, int D, int MOST> hipError_t launch_rows(const AttendArgs& g, int nt, hipStream_t stream) {
  if (nt == 1) return launch<TYPE, D, 1>(g, stream);
  if constexpr (MOST >= 4) {
    if (nt == 3) return launch<TYPE, D, 3>(g, stream);
    if (nt == 4) return launch<TYPE, D, 4>(g, stream);
  }
  return launch<TYPE, D, 2>(g, stream);
}

}  // namespace
#endif

}  // namespace si
