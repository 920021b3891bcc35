// Pieces that the kernels writing new tokens into the cache share (hipcc only): rounding to the cache's type, angles, places, and the whole way of v.
#pragma once
#include "si_internal.h"
#include "kv_layout.h"

namespace si {
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_a2 __attribute__((aligned(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int THREADS = 256;
constexpr int MAX_TOKENS = 4;    // tokens of a block of the q / k part
constexpr int MAX_ANGLES = 128;  // head_dim / 2

struct Args {
  si_cache_t c;
  si_append_t a;
  int layer;
  int per_block;    // tokens of a block of the q / k part
  int qk_columns;   // blocks of the q / k part along the units of a token
  int v_columns;    // blocks of the v part along its columns
  int v_blocks;     // and in all
  int run;          // blocks of the q / k part that follow each other on one die
};

__device__ __forceinline__ uint16_t bf16_bits(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  const bf16x2 p = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, p);
}
__device__ __forceinline__ float widen(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }

// x / scale, cut to the largest code (the comparisons leave NaN alone).  The quotient is the correctly rounded one: a product with the
// reciprocal differs from it at the borders between codes
__device__ __forceinline__ float code_value(float x, float scale) {
  x = x / scale;
  x = x < -448.f ? -448.f : x;
  return x > 448.f ? 448.f : x;
}
__device__ __forceinline__ uint32_t four_codes(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

__device__ __forceinline__ void widen8(const u32x4& v, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(v[i] << 16); f[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u); }
}
__device__ __forceinline__ u32x4 pack8(const float (&f)[8]) {
  return u32x4{bf16_pair(f[0], f[1]), bf16_pair(f[2], f[3]), bf16_pair(f[4], f[5]), bf16_pair(f[6], f[7])};
}

// cos and sin of pos * freq: the product and its whole turns in 64 bits (at position 10^6 an angle in 32 bits is off by 0.06)
__device__ __forceinline__ float2 turn(int pos, float freq) {
  const double t = (double)pos * (double)freq * 0.15915494309189533577;
  float s, c;
  sincospif((float)(2.0 * (t - rint(t))), &s, &c);
  return make_float2(c, s);
}

struct Token {
  int64_t k;  // first element of the token's K block at head 0, or -1: left out
  int slot;   // of the block
};

template <int TYPE> __device__ __forceinline__ void store_k(const Args& g, const Token& t, int head, int dim, const float (&f)[8]) {
  constexpr int E = TYPE == SI_KV_E4M3 ? 16 : 8;
  const int64_t at = t.k + head * kv_head_elems(g.c) + dim / E * (4 * E * E) + t.slot * E + dim % E;
  if constexpr (TYPE == SI_KV_BF16) {
    *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(g.c.pages) + at) = pack8(f);
  } else {
    const float s = g.c.scale_k ? g.c.scale_k[head] : 1.f;
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = code_value(f[i], s);
    *reinterpret_cast<u32x2*>(static_cast<uint8_t*>(g.c.pages) + at) = u32x2{four_codes(x[0], x[1], x[2], x[3]), four_codes(x[4], x[5], x[6], x[7])};
  }
}
template <int TYPE> __device__ __forceinline__ void store_k1(const Args& g, const Token& t, int head, int dim, float f) {
  constexpr int E = TYPE == SI_KV_E4M3 ? 16 : 8;
  const int64_t at = t.k + head * kv_head_elems(g.c) + dim / E * (4 * E * E) + t.slot * E + dim % E;
  if constexpr (TYPE == SI_KV_BF16) static_cast<uint16_t*>(g.c.pages)[at] = bf16_bits(f);
  else static_cast<uint8_t*>(g.c.pages)[at] = (uint8_t)four_codes(code_value(f, g.c.scale_k ? g.c.scale_k[head] : 1.f), 0.f, 0.f, 0.f);
}

// v of E tokens and THREADS columns (element of a head).  The layout holds E consecutive positions of an element in 16 bytes: where E
// tokens of the call fill such a chunk in order, the thread that meets the first of them stores it whole (the others are passed over,
// whichever block they belong to); else elements are stored one by one.
template <int TYPE> __device__ void v_part(const Args& g, int block) {
  constexpr int E = TYPE == SI_KV_E4M3 ? 16 : 8;
  __shared__ int64_t s_at[E];
  __shared__ int s_mode[E];  // 0: nothing to do, 1: this token alone, E: E tokens from this one on
  const si_append_t& a = g.a;
  const int d = g.c.head_dim, i0 = block / g.v_columns * E, tid = threadIdx.x;
  if (tid < E) {
    const int i = i0 + tid;
    int mode = 0;
    int64_t at = 0;
    const int seq = i < a.n_tokens ? a.seq[i] : -1;
    if (seq != -1) {
      const int pos = a.pos[i];
      int why = 0;  // (the q / k part reports it)
      const int page = kv_page_of(g.c, seq, pos, why);
      if (page >= 0) {
        const int in_page = pos % g.c.page_tokens, start = i - pos % E;
        at = page * kv_page_elems(g.c) + kv_head_offset(g.c, g.layer, 1, 0) + (int64_t)(in_page / (4 * E)) * (4 * E * d) +
             kv_v_offset(E, d, in_page % (4 * E), 0);
        bool whole = start >= 0 && start + E <= a.n_tokens;
        if (whole)
          for (int k = 0; k < E; ++k) whole = whole && a.seq[start + k] == seq && a.pos[start + k] == pos - pos % E + k;
        mode = !whole ? 1 : i == start ? E : 0;
      }
    }
    s_at[tid] = at;
    s_mode[tid] = mode;
  }
  __syncthreads();
  const int column = block % g.v_columns * THREADS + tid;
  if (column >= g.c.n_kv_heads * d) return;
  const int head = column / d, dim = column - head * d;
  const uint16_t* v = static_cast<const uint16_t*>(a.v) + column;
  const int64_t to = head * kv_head_elems(g.c) + (int64_t)dim * E;
  const float s = TYPE == SI_KV_E4M3 && g.c.scale_v ? g.c.scale_v[head] : 1.f;
  for (int k = 0; k < E; ++k) {
    const int mode = s_mode[k];
    if (mode == 0) continue;
    const uint16_t* p = v + (int64_t)(i0 + k) * a.v_stride;
    const int64_t at = s_at[k] + to;
    if (mode == 1) {
      if constexpr (TYPE == SI_KV_BF16) static_cast<uint16_t*>(g.c.pages)[at] = *p;
      else static_cast<uint8_t*>(g.c.pages)[at] = (uint8_t)four_codes(code_value(widen(*p), s), 0.f, 0.f, 0.f);
      continue;
    }
    uint16_t x[E];
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = p[e * a.v_stride];
    if constexpr (TYPE == SI_KV_BF16) {
      u32x4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = x[2 * e] | (uint32_t)x[2 * e + 1] << 16;
      *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(g.c.pages) + at) = w;
    } else {
      u32x4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        w[e] = four_codes(code_value(widen(x[4 * e]), s), code_value(widen(x[4 * e + 1]), s), code_value(widen(x[4 * e + 2]), s), code_value(widen(x[4 * e + 3]), s));
      *reinterpret_cast<u32x4*>(static_cast<uint8_t*>(g.c.pages) + at) = w;
    }
  }
}

// Blocks go to the 8 dies in turn.  A line of a K block holds 16 bytes of eight tokens: the runs of blocks that have 32 neighbouring tokens go to
// one die, whose cache puts the pieces together (else all dies write pieces of the same lines: 4099 tokens of 64 + 8 heads of 128, calls with other
// inputs between, bf16 42.8 us, this way 40.7; e4m3 40.7 both ways)
__device__ __forceinline__ int on_one_die(int b, int blocks, int run) {
  const int all = blocks / (8 * run) * (8 * run);
  if (b >= all) return b;  // (what is left over stays in order)
  const int die = b % 8, i = b / 8;
  return (i / run * 8 + die) * run + i % run;
}

}  // namespace
}  // namespace si
