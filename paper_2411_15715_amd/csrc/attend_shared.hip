// Attention for sequences that share leading pages: which they are, found on the device from the table, and the call's launches.
//
// Softmax splits over positions: with m, l, o of a row over the shared positions and over its own,
//   m' = max m,  l' = sum l 2^(m - m'),  o' = sum o 2^(m - m')
// so neighbours of the list whose tables begin with the same pages attend to these as rows of one sequence, which is read once for all of them and
// fills the matrix instructions, and each to what it alone has.  Three launches: the plan makes pieces of both kinds, shared and own; their
// blocks, one after the other, are cut into equal slices as those of whole sequences are in si_attend; and every row's sums are joined.
#include "si_internal.h"
#include "si_error.h"
#include "attend_device.h"

#include <algorithm>

namespace si {
namespace {

constexpr int THREADS = 256, WAVES = THREADS / 64;

// Pieces as the plan writes them
struct PlanList {
  int slices;
  Piece* pieces;
  SliceStart* starts;
  int2* parted;
};
struct PlanArgs {
  si_cache_t c;
  const int32_t* seqs;
  int n, n_new, per, window, wide_rows, block_rows, chunks;
  uint32_t* count;       // [1], 0 between calls
  int32_t* common;       // [n] full pages that an entry of the list has in common with the one before
  int32_t* tokens_of;    // [n] of a group's first entry: tokens in its shared pages
  int32_t* piece_of;     // [n] of a group's first entry: its first piece, or -1
  PlanList shared, own;  // the groups' pieces, of up to wide_rows rows, and those of each entry's own tokens
  int2* group;           // [n] first piece of an entry's group (-1: none), first entry of it
};

__device__ __forceinline__ int seq_at(const PlanArgs& g, int e) { return g.seqs ? g.seqs[e] : e; }
// tokens of an entry's sequence as the attention counts them
__device__ __forceinline__ int len_at(const PlanArgs& g, int e) {
  const int s = seq_at(g, e);
  return s < 0 || s >= g.c.n_seqs ? 0 : min(max(g.c.lens[s], 0), g.c.max_pages * g.c.page_tokens);
}

// A group ends where two neighbours have nothing in common, or less than half of what one of them has in common with its other neighbour (two prompts
// with the same few words before them are two groups).
__device__ __forceinline__ bool begins(const PlanArgs& g, int e) {
  if (e == 0) return true;
  const int c = __hip_atomic_load(g.common + e, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  const int before = e > 1 ? __hip_atomic_load(g.common + e - 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0;
  const int after = e + 1 < g.n ? __hip_atomic_load(g.common + e + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0;
  return c == 0 || 2ll * c < max(before, after);
}

struct Run {  // of entries of a group so far
  int first, pages, shortest, longest;
};
__device__ __forceinline__ Run joined(const Run& a, const Run& b) {  // b begins no group: a's goes on
  return Run{a.first, min(a.pages, b.pages), min(a.shortest, b.shortest), max(a.longest, b.longest)};
}

// A block for each entry: the pages that it has in common with the one before.  The block that finishes last forms the groups.
__global__ __launch_bounds__(THREADS) void k_share(PlanArgs g) {
  __shared__ int s_first, s_last, s_offset[WAVES];
  __shared__ Run s_run[WAVES];
  __shared__ int s_begins[WAVES];
  __shared__ int64_t s_sum[WAVES];
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64, e = blockIdx.x, B = kv_block(g.c.type);
  if (tid == 0) {
    const int s = seq_at(g, e), bad = s < 0 || s >= g.c.n_seqs ? SI_CACHE_BAD_SEQ : g.c.lens[s] < 0 || g.c.lens[s] > g.c.max_pages * g.c.page_tokens ? SI_CACHE_BAD_LEN : 0;
    if (bad) atomicOr(g.c.status, bad);
  }
  int common = 0;
  if (e > 0) {
    const int most = min(len_at(g, e), len_at(g, e - 1)) / g.c.page_tokens;
    const int32_t *a = g.c.table + (int64_t)max(seq_at(g, e - 1), 0) * g.c.max_pages, *b = g.c.table + (int64_t)max(seq_at(g, e), 0) * g.c.max_pages;
    if (tid == 0) s_first = most;
    for (int j0 = 0; j0 < most; j0 += THREADS) {
      __syncthreads();
      if (s_first < most) break;
      const int j = j0 + tid;
      __syncthreads();
      if (j < most && (a[j] != b[j] || b[j] < 0 || b[j] >= g.c.n_pages)) atomicMin(&s_first, j);
    }
    __syncthreads();
    common = s_first;
  }
  if (tid == 0) {
    __hip_atomic_store(g.common + e, common, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    s_last = __hip_atomic_fetch_add(g.count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)g.n - 1;
    if (s_last) __hip_atomic_store(g.count, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  if (!s_last) return;

  Run carry{0, 0x7fffffff, 0x7fffffff, 0};  // the group that is open before this round
  int n_shared = 0;
  for (int e0 = 0; e0 < g.n; e0 += THREADS) {
    const int i = e0 + tid;
    const bool in = i < g.n;
    bool start = in && begins(g, i);
    Run r{i, 0x7fffffff, 0x7fffffff, 0};
    if (in) {
      const int len = len_at(g, i);
      r.pages = max(0, len - g.n_new + 1) / g.c.page_tokens;  // (what the first of the new tokens sees too)
      if (!start) r.pages = min(r.pages, __hip_atomic_load(g.common + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
      r.shortest = r.longest = len;
    }
    const bool ends = in && (i + 1 == g.n || begins(g, i + 1));
    bool any = start;  // a group begins among the entries that r covers
    for (int d = 1; d < 64; d *= 2) {
      const Run o{__shfl_up(r.first, d), __shfl_up(r.pages, d), __shfl_up(r.shortest, d), __shfl_up(r.longest, d)};
      const bool o_any = __shfl_up((int)any, d);
      if (lane >= d && !any) {
        r = joined(o, r);
        any = o_any;
      }
    }
    __syncthreads();
    if (lane == 63) { s_run[wave] = r; s_begins[wave] = any; }
    __syncthreads();
    Run before = carry;
    for (int w = 0; w < wave; ++w) before = s_begins[w] ? s_run[w] : joined(before, s_run[w]);
    if (!any) r = joined(before, r);
    Run next = carry;
    for (int w = 0; w < WAVES; ++w) next = s_begins[w] ? s_run[w] : joined(next, s_run[w]);
    // (beyond the last entry a run is empty and changes nothing)
    const int members = i - r.first + 1, tokens = ends && members > 1 ? r.pages * g.c.page_tokens : 0, rows = members * g.n_new * g.per;
    const int mine = tokens > 0 ? (rows + g.wide_rows - 1) / g.wide_rows : 0;
    int at = mine;
    for (int d = 1; d < 64; d *= 2) {
      const int o = __shfl_up(at, d);
      if (lane >= d) at += o;
    }
    if (lane == 63) s_offset[wave] = at;
    __syncthreads();
    at += n_shared - mine;
    for (int w = 0; w < WAVES; ++w) {
      if (w < wave) at += s_offset[w];
      n_shared += s_offset[w];
    }
    if (in) g.group[i].y = r.first;
    if (ends) {
      g.tokens_of[r.first] = tokens;
      g.piece_of[r.first] = mine > 0 ? at : -1;
      const int lo = g.window ? min(tokens, max(0, r.shortest - g.n_new + 1 - g.window)) : 0, lo_all = g.window ? min(tokens, max(0, r.longest - g.window)) : 0;
      for (int k = 0; k < mine; ++k)
        g.shared.pieces[at + k] = Piece{seq_at(g, r.first), r.first * g.n_new * g.per + k * g.wide_rows, min(g.wide_rows, rows - k * g.wide_rows), lo, tokens, lo_all, tokens,
                                 lo / B, tokens > lo ? tokens / B - lo / B : 0, -1, 0};
    }
    carry = next;
  }
  __syncthreads();
  const int n_own = g.n * g.chunks, of_entry = g.n_new * g.per;
  for (int k = tid; k < n_own; k += THREADS) {
    const int i = k / g.chunks, row0 = (k - i * g.chunks) * g.block_rows, rows = min(g.block_rows, of_entry - row0), first = g.group[i].y, from = g.tokens_of[first];
    const int sight = len_at(g, i) - g.n_new + 1, t0 = row0 / g.per, t1 = (row0 + rows - 1) / g.per;
    const int hi = max(0, sight + t1), lo = g.window ? max(from, sight + t0 - g.window) : from;
    g.own.pieces[k] = Piece{seq_at(g, i), i * of_entry + row0, rows, lo, hi, g.window ? max(from, sight + t1 - g.window) : from, max(0, sight + t0),
                     lo / B, hi > lo ? (hi + B - 1) / B - lo / B : 0, i, sight};
    if (row0 == 0) g.group[i].x = g.piece_of[first];
  }
  __syncthreads();
  // Equal slices of each list's blocks: slice w is [end(w - 1), end(w)) with end(w) = (w + 1) total / G.  (Quotients by way of double: exact, as the dividends
  // stay below 2^53.)
  auto cut = [&](const PlanList& list, int n) {
    auto scan = [&](auto f) {  // f(piece, its blocks, blocks before it) for all; returns the number of blocks
      int64_t done = 0;
      for (int k0 = 0; k0 < n; k0 += THREADS) {
        const int k = k0 + tid;
        const int64_t mine = k < n ? max(1, list.pieces[k].nb) : 0;
        int64_t x = mine;
        for (int d = 1; d < 64; d *= 2) {
          const int64_t o = __shfl_up(x, d);
          if (lane >= d) x += o;
        }
        __syncthreads();
        if (lane == 63) s_sum[wave] = x;
        __syncthreads();
        x += done - mine;
        for (int w = 0; w < WAVES; ++w) {
          if (w < wave) x += s_sum[w];
          done += s_sum[w];
        }
        if (k < n) f(k, mine, x);
      }
      return done;
    };
    const int64_t total = scan([](int, int64_t, int64_t) {}), G = min<int64_t>(list.slices, total);
    auto quotient = [](int64_t x, int64_t y) { return (int64_t)((double)x / (double)y); };
    auto end = [&](int64_t w) { return quotient((w + 1) * total, G); };
    auto slice_of = [&](int64_t block) { return (int)quotient((block + 1) * G - 1, total); };  // the one whose end is the first beyond the block
    scan([&](int k, int64_t mine, int64_t x) {
      const int first = slice_of(x), last = slice_of(x + mine - 1);
      list.parted[k] = make_int2(first, last - first + 1);
      for (int w = first; w <= last; ++w)  // those that begin in this piece
        if (end(w - 1) >= x) list.starts[w] = SliceStart{k, (int)(end(w - 1) - x), (int)(end(w) - end(w - 1))};
    });
    for (int w = (int)G + tid; w < list.slices; w += THREADS) list.starts[w] = SliceStart{0, 0, 0};
  };
  cut(g.shared, n_shared);
  cut(g.own, n_own);
}

constexpr int WIDE = 128;  // rows of a shared piece

struct Layout {
  AttendCut alone;           // of si_attend
  bool pieces;               // else the call is si_attend
  int block_rows, chunks, shared_slices, own_slices;
  int64_t shared_parted, own_parted, shared_part, own_part, sums, shared, own, shared_starts, own_starts, group, common, tokens_of, piece_of, bytes;
};

Layout lay_out(const si_cache_t& c, const si_attend_t& a) {
  Layout l{};
  l.alone = cut_attend(c, a);
  const int of_entry = a.n_new * (a.n_heads / c.n_kv_heads);
  const int64_t rows = (int64_t)a.n * of_entry;
  l.pieces = a.n > 1 && rows <= 200000;  // (the joining launch has a block for 4 rows and more)
  for (l.block_rows = 16; l.block_rows < of_entry && l.block_rows < 64;) l.block_rows *= 2;
  l.chunks = (of_entry + l.block_rows - 1) / l.block_rows;
  const int64_t each = (a.max_len + kv_block(c.type) - 1) / kv_block(c.type), turns = (rows + WIDE - 1) / WIDE * each * c.n_kv_heads / 256;
  l.shared_slices = std::max(1, (turns > 24 && c.head_dim < 192 ? 512 : 256) / c.n_kv_heads);
  l.own_slices = std::max(1, 256 / c.n_kv_heads);
  const int64_t shared = rows / WIDE + a.n / 2 + 1, own = (int64_t)a.n * l.chunks;
  int64_t at = std::max<int64_t>(l.alone.scratch, ATTEND_COUNTERS * 4);  // (the counters are at the same place in every call's scratch)
  auto take = [&](int64_t bytes) {
    const int64_t q = (at + 15) / 16 * 16;
    at = q + bytes;
    return q;
  };
  l.shared_parted = take(shared * 8);
  l.own_parted = take(own * 8);
  l.shared_part = take((int64_t)c.n_kv_heads * l.shared_slices * 2 * WIDE * (c.head_dim + 4) * 4);
  l.own_part = take((int64_t)c.n_kv_heads * l.own_slices * 2 * std::min(of_entry, l.block_rows) * (c.head_dim + 2) * 4);
  l.sums = take(2 * c.n_kv_heads * rows * (c.head_dim + 4) * 4);
  l.shared = take(shared * (int64_t)sizeof(Piece));
  l.own = take(own * (int64_t)sizeof(Piece));
  l.shared_starts = take(l.shared_slices * (int64_t)sizeof(SliceStart));
  l.own_starts = take(l.own_slices * (int64_t)sizeof(SliceStart));
  l.group = take(a.n * 8ll);
  l.common = take(a.n * 4ll);
  l.tokens_of = take(a.n * 4ll);
  l.piece_of = take(a.n * 4ll);
  l.bytes = (at + 15) / 16 * 16;
  return l;
}

int check(const si_cache_t* c, const si_attend_t* a, const char* who) {
  if (int rc = check_attend_shape(c, a, who)) return rc;
  if ((int64_t)a->n * a->n_new * a->n_heads >= ((int64_t)1 << 31)) return set_error(SI_EINVAL, "%s: n * n_new * n_heads is too large for one call (%d, %d, %d)", who, a->n, a->n_new, a->n_heads);
  return SI_OK;
}

}  // namespace
}  // namespace si

extern "C" int64_t si_attend_shared_scratch_bytes(const si_cache_t* c, const si_attend_t* a) {
  using namespace si;
  if (int rc = check(c, a, "si_attend_shared_scratch_bytes")) return rc;
  return lay_out(*c, *a).bytes;
}

extern "C" int si_attend_shared(const si_cache_t* c, int32_t layer, const si_attend_t* a, void* stream) {
  using namespace si;
  const char* who = "si_attend_shared";
  bool nothing;
  if (int rc = check_attend(c, layer, a, who, &nothing)) return rc;
  if (int rc = check(c, a, who)) return rc;
  if (nothing) return SI_OK;
  const Layout l = lay_out(*c, *a);
  if (!a->scratch || a->scratch_bytes < l.bytes || (reinterpret_cast<uintptr_t>(a->scratch) & 15) != 0)
    return set_error(SI_EINVAL, "%s: %lld bytes of scratch needed, 16-byte aligned", who, (long long)l.bytes);
  char* p = static_cast<char*>(a->scratch);
  AttendArgs g = attend_args(*c, *a, layer, l.alone);
  hipError_t e = hipSuccess;
  if (!l.pieces) {
    e = (c->type == SI_KV_BF16 ? launch_attend_bf16 : launch_attend_e4m3)(g, (hipStream_t)stream);
  } else {
    const auto ints = [&](int64_t at) { return reinterpret_cast<int32_t*>(p + at); };
    const int part_rows = std::min(a->n_new * (a->n_heads / c->n_kv_heads), l.block_rows);
    const PlanList shared{l.shared_slices, reinterpret_cast<Piece*>(p + l.shared), reinterpret_cast<SliceStart*>(p + l.shared_starts), reinterpret_cast<int2*>(p + l.shared_parted)};
    const PlanList mine{l.own_slices, reinterpret_cast<Piece*>(p + l.own), reinterpret_cast<SliceStart*>(p + l.own_starts), reinterpret_cast<int2*>(p + l.own_parted)};
    const PlanArgs plan{*c, a->seqs, a->n, a->n_new, a->n_heads / c->n_kv_heads, a->window, WIDE, l.block_rows, l.chunks, reinterpret_cast<uint32_t*>(p), ints(l.common),
                        ints(l.tokens_of), ints(l.piece_of), shared, mine, reinterpret_cast<int2*>(p + l.group)};
    g.rows = g.block_rows = l.block_rows;
    g.groups = 1;
    g.whole = g.last_joins = 0;
    g.shared = PieceList{l.shared_slices, shared.pieces, shared.starts, shared.parted, reinterpret_cast<float*>(p + l.shared_part), WIDE, c->head_dim + 4};
    g.own = PieceList{l.own_slices, mine.pieces, mine.starts, mine.parted, reinterpret_cast<float*>(p + l.own_part), part_rows, c->head_dim + 2};
    g.sums = reinterpret_cast<float*>(p + l.sums);
    g.group = plan.group;
    g.chunks = l.chunks;
    hipLaunchKernelGGL(k_share, dim3(a->n), dim3(THREADS), 0, (hipStream_t)stream, plan);
    e = hipGetLastError();
    if (e == hipSuccess) e = (c->type == SI_KV_BF16 ? launch_attend_pieces_bf16 : launch_attend_pieces_e4m3)(g, (hipStream_t)stream);
  }
  if (e != hipSuccess) return set_error(SI_EHIP, "attention launch failed: %s", hipGetErrorString(e));
  return SI_OK;
}
