// New tokens into the paged key-value cache: rotary positions for q and k, rounding to the cache's type, and the places of the layout.
// Bound by memory and by the pieces of 16 bytes that the layout takes a row of k apart into: 4099 tokens of 64 + 8 heads of 128 (160 MB) into e4m3
// 37.6 us, 4.3 TB/s, where a copy of as much takes 31; into bf16 36.2.  q is a plain pass beside it.  8 tokens: 4.2 us in the kernel, three trips
// to memory one after the other (sequence, page, store) and a cold instruction cache.
#include "si_internal.h"
#include "si_error.h"
#include "append_device.h"

#include <algorithm>

namespace si {
namespace {

// Units of a head: pairs and elements by themselves, and all of them
__host__ __device__ inline int singles(int rot) { return rot % 16 == 0 ? 0 : rot / 2 + (16 - rot % 16); }
__host__ __device__ inline int units_of_head(int rot, int d) { return rot % 16 == 0 ? d / 16 : singles(rot) + (d - rot / 16 * 16 - 16) / 16; }

// q and k of per_block tokens.  A thread takes 16 elements of a head: with rot_dim a multiple of 16 the two vectors that turn into each
// other (or 16 neighbours), so that every element is read once and q may be turned in place; else the elements up to the next multiple of 16
// as single pairs and single ones.
// What a thread needs first is on its way while the angles are formed, and what it needs next while it turns what it has.
template <int TYPE> __device__ void qk_part(const Args& g, int block) {
  __shared__ float2 s_turn[MAX_TOKENS][MAX_ANGLES];
  __shared__ Token s_token[MAX_TOKENS];
  constexpr int E = TYPE == SI_KV_E4M3 ? 16 : 8;
  const si_append_t& a = g.a;
  const int d = g.c.head_dim, half = a.rot_dim / 2, tid = threadIdx.x;
  const int t0 = block / g.qk_columns * g.per_block, n = min(g.per_block, a.n_tokens - t0), column = block % g.qk_columns;
  const int n_heads = a.q ? a.n_heads : 0, heads = n_heads + g.c.n_kv_heads;
  const int single = singles(a.rot_dim), per_head = units_of_head(a.rot_dim, d), first_wide = (a.rot_dim + 15) / 16;
  const uint32_t inv = (uint32_t)(0x100000000ull / per_head) + 1;  // u / per_head = umulhi(u, inv) while u * per_head < 2^32
  const int units = heads * per_head, span = (units + g.qk_columns - 1) / g.qk_columns;
  const int u0 = column * span, u1 = min(units, u0 + span), all = max(0, u1 - u0) * n;

  struct Unit {
    u32x4 x, y;
    int t, head, j;  // token of the block, head (k: after q's), unit of the head
  };
  auto source = [&](const Unit& k) {
    const bool is_q = k.head < n_heads;
    return static_cast<const uint16_t*>(is_q ? a.q : a.k) + (int64_t)(t0 + k.t) * (is_q ? a.q_stride : a.k_stride) + (is_q ? k.head : k.head - n_heads) * d;
  };
  // first elements of the two vectors of a unit
  auto dim0 = [&](int j) { return j < a.rot_dim / 16 && !a.rot_pairs ? 8 * j : 16 * j; };
  auto dim1 = [&](int j) { return j < a.rot_dim / 16 && !a.rot_pairs ? 8 * j + half : 16 * j + 8; };
  auto fetch = [&](int f) {
    Unit k;
    k.t = 0;
    int u = f;
    while (u >= u1 - u0) { u -= u1 - u0; ++k.t; }
    u += u0;
    k.head = (int)__umulhi((uint32_t)u, inv);
    k.j = u - k.head * per_head - single;  // negative: a pair or an element by itself
    if (k.j >= 0) {
      k.j += single > 0 ? first_wide : 0;
      const uint16_t* p = source(k);
      k.x = __builtin_nontemporal_load(reinterpret_cast<const u32x4_a2*>(p + dim0(k.j)));
      k.y = __builtin_nontemporal_load(reinterpret_cast<const u32x4_a2*>(p + dim1(k.j)));
    }
    return k;
  };
  Unit next;
  if (tid < all) next = fetch(tid);
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
  for (int f = tid; f < all; f += THREADS) {
    const Unit k = next;
    if (f + THREADS < all) next = fetch(f + THREADS);
    const Token tok = s_token[k.t];
    const bool is_q = k.head < n_heads;
    const int head = is_q ? k.head : k.head - n_heads, j = k.j;
    if (!is_q && tok.k < 0) continue;
    uint16_t* dst = static_cast<uint16_t*>(a.q_out) + (int64_t)(t0 + k.t) * a.q_out_stride + head * d;
    if (j >= 0) {
      float x[8], y[8];
      widen8(k.x, x);
      widen8(k.y, y);
      if (j < a.rot_dim / 16) {  // (never, where there are single pairs)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float2 cs = s_turn[k.t][8 * j + i];
          float& p = a.rot_pairs ? (i < 4 ? x[(2 * i) % 8] : y[(2 * i) % 8]) : x[i];
          float& q = a.rot_pairs ? (i < 4 ? x[(2 * i + 1) % 8] : y[(2 * i + 1) % 8]) : y[i];
          const float p0 = p, q0 = q;
          p = p0 * cs.x - q0 * cs.y;
          q = q0 * cs.x + p0 * cs.y;
        }
      }
      if (is_q) {
        const bool out = tok.k < 0;
        *reinterpret_cast<u32x4_a2*>(dst + dim0(j)) = out ? u32x4{0, 0, 0, 0} : pack8(x);
        *reinterpret_cast<u32x4_a2*>(dst + dim1(j)) = out ? u32x4{0, 0, 0, 0} : pack8(y);
      } else {
        store_k<TYPE>(g, tok, head, dim0(j), x);
        store_k<TYPE>(g, tok, head, dim1(j), y);
      }
    } else {
      const int u = j + single;
      const bool turned = u < half;
      const int d0 = turned ? (a.rot_pairs ? 2 * u : u) : u + half, d1 = a.rot_pairs ? d0 + 1 : d0 + half;
      const uint16_t* src = source(k);
      float x = widen(src[d0]), y = turned ? widen(src[d1]) : 0.f;
      if (turned) {
        const float2 cs = s_turn[k.t][u];
        const float x0 = x;
        x = x0 * cs.x - y * cs.y;
        y = y * cs.x + x0 * cs.y;
      }
      if (is_q) {
        dst[d0] = tok.k < 0 ? 0 : bf16_bits(x);
        if (turned) dst[d1] = tok.k < 0 ? 0 : bf16_bits(y);
      } else {
        store_k1<TYPE>(g, tok, head, d0, x);
        if (turned) store_k1<TYPE>(g, tok, head, d1, y);
      }
    }
  }
}

template <int TYPE> __global__ __launch_bounds__(THREADS) void k_append(Args g) {
  // (v first: its blocks have the longer way from load to store)
  if ((int)blockIdx.x < g.v_blocks) v_part<TYPE>(g, blockIdx.x);
  else qk_part<TYPE>(g, on_one_die(blockIdx.x - g.v_blocks, gridDim.x - g.v_blocks, g.run));
}

bool misaligned(const void* p, int to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

// How a call is cut into blocks; returns their number.
int64_t cut(Args& g) {
  const si_cache_t& c = g.c;
  const si_append_t& a = g.a;
  const int per_head = units_of_head(a.rot_dim, c.head_dim), units = ((a.q ? a.n_heads : 0) + c.n_kv_heads) * per_head;
  // A block has up to four units a thread, of one token or of up to 4 where these have few (4099 tokens of 576 units: 51 us with the angles formed
  // by two blocks of a token, 39 by one); with few tokens one unit a thread (what waits there is memory, not the threads)
  const int want = THREADS * (a.n_tokens >= 256 ? 4 : 1);
  if (units >= want) g.qk_columns = (units + want - 1) / want;
  else if (a.n_tokens >= 256) g.per_block = std::min(MAX_TOKENS, want / units);
  const int E = kv_vec(c.type);
  g.v_columns = (c.n_kv_heads * c.head_dim + THREADS - 1) / THREADS;
  g.v_blocks = (a.n_tokens + E - 1) / E * g.v_columns;
  g.run = 32 / g.per_block * g.qk_columns;
  return (int64_t)((a.n_tokens + g.per_block - 1) / g.per_block) * g.qk_columns + g.v_blocks;
}

hipError_t launch_append(const Args& g, int64_t blocks, hipStream_t stream) {
  if (g.c.type == SI_KV_BF16) hipLaunchKernelGGL(k_append<SI_KV_BF16>, dim3((unsigned)blocks), dim3(THREADS), 0, stream, g);
  else hipLaunchKernelGGL(k_append<SI_KV_E4M3>, dim3((unsigned)blocks), dim3(THREADS), 0, stream, g);
  return hipGetLastError();
}

}  // namespace

int check_cache(const si_cache_t* c, const char* who) {
  if (!c) return set_error(SI_EINVAL, "%s: cache descriptor is NULL", who);
  if (c->type != SI_KV_BF16 && c->type != SI_KV_E4M3) return set_error(SI_EINVAL, "%s: unknown cache type %d", who, c->type);
  const int d = c->head_dim;
  if (!(d == 64 || d == 128 || d == 192 || d == 256 || (d == 96 && c->type == SI_KV_BF16))) return set_error(SI_EINVAL, "%s: head_dim %d of cache type %d", who, d, c->type);
  if (c->page_tokens < 1 || c->page_tokens > (1 << 16) || c->page_tokens % kv_block(c->type) != 0)
    return set_error(SI_EINVAL, "%s: page_tokens %d is not a multiple of %d up to 65536", who, c->page_tokens, kv_block(c->type));
  if (c->n_pages < 1 || c->n_layers < 1 || c->n_kv_heads < 1 || c->n_kv_heads > 1024 || c->n_layers > (1 << 16) || c->n_seqs < 1 || c->max_pages < 1)
    return set_error(SI_EINVAL, "%s: bad n_pages=%d n_layers=%d n_kv_heads=%d n_seqs=%d max_pages=%d", who, c->n_pages, c->n_layers, c->n_kv_heads, c->n_seqs,
                     c->max_pages);
  if ((int64_t)c->max_pages * c->page_tokens > 0x7fff0000) return set_error(SI_EINVAL, "%s: max_pages * page_tokens exceeds 0x7fff0000", who);
  if (!c->pages || !c->table || !c->lens || !c->status) return set_error(SI_EINVAL, "%s: pages, table, lens or status is NULL", who);
  if (misaligned(c->pages, 16)) return set_error(SI_EINVAL, "%s: pages are not aligned to 16 bytes", who);
  if (misaligned(c->table, 4) || misaligned(c->lens, 4) || misaligned(c->refs, 4) || misaligned(c->status, 4) || misaligned(c->scale_k, 4) || misaligned(c->scale_v, 4))
    return set_error(SI_EINVAL, "%s: table, lens, refs, status or a scale is not aligned to 4 bytes", who);
  return SI_OK;
}
int check_layer(const si_cache_t* c, int layer, const char* who) {
  if (layer < 0 || layer >= c->n_layers) return set_error(SI_EINVAL, "%s: layer %d of %d", who, layer, c->n_layers);
  return SI_OK;
}

// Everything but what a launch cannot hold; *nothing: there are no tokens
int check_append(const si_cache_t* c, int layer, const si_append_t* a, const char* who, bool* nothing) {
  *nothing = false;
  if (int rc = check_cache(c, who)) return rc;
  if (int rc = check_layer(c, layer, who)) return rc;
  if (!a) return set_error(SI_EINVAL, "%s: descriptor is NULL", who);
  if (a->n_tokens < 0) return set_error(SI_EINVAL, "%s: n_tokens %d", who, a->n_tokens);
  if ((*nothing = a->n_tokens == 0)) return SI_OK;  // (an empty tensor's address may be NULL)
  if (!a->k || !a->v || !a->seq || !a->pos || (a->q && !a->q_out)) return set_error(SI_EINVAL, "%s: k, v, seq, pos or q_out is NULL", who);
  if (a->q && (a->n_heads < 1 || a->n_heads > 4096 || a->n_heads % c->n_kv_heads != 0))
    return set_error(SI_EINVAL, "%s: n_heads %d is not a multiple of n_kv_heads %d", who, a->n_heads, c->n_kv_heads);
  if (a->rot_dim < 0 || a->rot_dim > c->head_dim || a->rot_dim % 2 != 0) return set_error(SI_EINVAL, "%s: rot_dim %d of head_dim %d", who, a->rot_dim, c->head_dim);
  if (a->rot_dim > 0 && !a->inv_freq) return set_error(SI_EINVAL, "%s: rot_dim without inv_freq", who);
  if (misaligned(a->q, 2) || misaligned(a->k, 2) || misaligned(a->v, 2) || misaligned(a->q_out, 2) || misaligned(a->seq, 4) || misaligned(a->pos, 4) || misaligned(a->inv_freq, 4))
    return set_error(SI_EINVAL, "%s: a pointer is not aligned to its element", who);
  const int64_t row_kv = (int64_t)c->n_kv_heads * c->head_dim, row_q = (int64_t)a->n_heads * c->head_dim;
  auto bad = [&](int64_t stride, int64_t row) { return stride < row && !(a->n_tokens <= 1 && stride == 0); };
  if (bad(a->k_stride, row_kv) || bad(a->v_stride, row_kv) || (a->q && (bad(a->q_stride, row_q) || bad(a->q_out_stride, row_q))))
    return set_error(SI_EINVAL, "%s: a stride is smaller than its row", who);
  if (a->q && a->q_out == a->q && a->q_out_stride != a->q_stride && a->n_tokens > 1) return set_error(SI_EINVAL, "%s: q_out is q, with another stride", who);
  if (a->n_tokens > (1 << 22) || (int64_t)a->n_tokens * row_kv > ((int64_t)1 << 33)) return set_error(SI_EINVAL, "%s: too many tokens in one call (%d)", who, a->n_tokens);
  return SI_OK;
}

}  // namespace si

extern "C" int si_kv_offsets(const si_cache_t* c, int32_t layer, int32_t kv_head, int32_t t_in_page, int32_t dim, int64_t* k_offset, int64_t* v_offset) {
  using namespace si;
  if (int rc = check_cache(c, "si_kv_offsets")) return rc;
  if (int rc = check_layer(c, layer, "si_kv_offsets")) return rc;
  if (kv_head < 0 || kv_head >= c->n_kv_heads || t_in_page < 0 || t_in_page >= c->page_tokens || dim < 0 || dim >= c->head_dim)
    return set_error(SI_EINVAL, "si_kv_offsets: kv_head %d, token %d or element %d outside the page", kv_head, t_in_page, dim);
  const int E = kv_vec(c->type), B = 4 * E;
  const int64_t block = (int64_t)(t_in_page / B) * B * c->head_dim;
  if (k_offset) *k_offset = kv_head_offset(*c, layer, 0, kv_head) + block + kv_k_offset(E, t_in_page % B, dim);
  if (v_offset) *v_offset = kv_head_offset(*c, layer, 1, kv_head) + block + kv_v_offset(E, c->head_dim, t_in_page % B, dim);
  return SI_OK;
}

extern "C" int si_cache_append(const si_cache_t* c, int32_t layer, const si_append_t* a, void* stream) {
  using namespace si;
  const char* who = "si_cache_append";
  bool nothing;
  if (int rc = check_append(c, layer, a, who, &nothing)) return rc;
  if (nothing) return SI_OK;
  Args g{*c, *a, layer, 1, 1, 0, 0, 1};
  const int64_t blocks = cut(g);
  if (blocks >= (1 << 24))  // (a launch has fewer than 2^32 threads)
    return set_error(SI_EINVAL, "%s: too many tokens and heads in one call (%d, %d)", who, a->n_tokens, a->n_heads);
  const hipError_t e = launch_append(g, blocks, (hipStream_t)stream);
  if (e != hipSuccess) return set_error(SI_EHIP, "append launch failed: %s", hipGetErrorString(e));
  return SI_OK;
}
