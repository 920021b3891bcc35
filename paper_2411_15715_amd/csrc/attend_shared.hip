// Attention for sequences that share leading pages: which they are, found on the device from the table, and the call's launches.
//
// Softmax splits over positions: with m, l, o of a row over the shared positions and over its own,
//   m' = max m,  l' = sum l 2^(m - m'),  o' = sum o 2^(m - m')
// so neighbours of the list whose tables begin with the same pages attend to these as rows of one sequence, which is read once for all of them and
// fills the matrix instructions, and each to what it alone has.  Three launches: the plan makes pieces of both kinds, shared and own; their
// blocks, one after the other, are cut into equal slices as those of whole sequences are in si_attend; and every row's sums are joined.
// The plan takes 8 to 10 us and the joining 7 to 10 (64 sequences with 8000 shared tokens: 18 MB of sums), whatever the pieces take (attend_wide.h).
#include "si_internal.h"
#include "si_error.h"
#include "attend_device.h"
#include "wave_device.h"

#include <algorithm>
#include <cstdlib>

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
  uint64_t* facts;       // [n] of an entry of the list: tokens of its sequence << 32 | full pages that it has in common with the one before
  int32_t* area;         // [area_words(n, most, chunks)] the forming block's notes, or null where these fit its shared memory
  int most;              // shared pieces that there can be
  PlanList shared, own;  // the groups' pieces, of up to wide_rows rows, and those of each entry's own tokens
  int2* group;           // [n] first piece of an entry's group (-1: none), first entry of it
};

constexpr int AREA = 8192;  // words of notes in shared memory: lists of some 800 sequences
__host__ __device__ inline int64_t area_words(int64_t n, int64_t most, int64_t chunks) { return 2 * (n * chunks + most) + 6 * n; }

__device__ __forceinline__ int seq_at(const PlanArgs& g, int e) { return g.seqs ? g.seqs[e] : e; }
// tokens of a sequence as the attention counts them
__device__ __forceinline__ int len_of(const PlanArgs& g, int s) {
  return s < 0 || s >= g.c.n_seqs ? 0 : min(max(g.c.lens[s], 0), g.c.max_pages * g.c.page_tokens);
}

struct Run {  // of entries of a group so far
  int first, pages, shortest, longest;
};
__device__ __forceinline__ Run joined(const Run& a, const Run& b) {  // b begins no group: a's goes on
  return Run{a.first, min(a.pages, b.pages), min(a.shortest, b.shortest), max(a.longest, b.longest)};
}

// A block for each entry: the pages that it has in common with the one before.  The block that finishes last forms the groups; it alone is what the call
// waits for, so all that it needs again is in shared memory and each list is scanned once (13 to 16 us with scans over lists in memory and a
// thread that wrote the slices of a piece in turn; 8.3 and 10.4 as it is for 64 and 45 sequences, most of it one round trip to memory or one barrier after another).  LOCAL: where the notes are
// is known when this is compiled.  A pointer to either memory would not do: such an address is told by its base before the instruction's
// offset is added, and the compiler may take one from a base that lies below the array.
template <bool LOCAL>
__global__ __launch_bounds__(THREADS) void k_share(PlanArgs g) {
  __shared__ int s_first, s_last, s_offset[WAVES];
  __shared__ Run s_run[WAVES];
  __shared__ int s_begins[WAVES];
  __shared__ int64_t s_sum[2][WAVES];
  __shared__ __align__(8) int32_t s_area[LOCAL ? AREA : 2];
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64, e = blockIdx.x, B = kv_block(g.c.type);
  const int seq = seq_at(g, e), seq_before = e > 0 ? seq_at(g, e - 1) : 0, len = len_of(g, seq), len_before = e > 0 ? len_of(g, seq_before) : 0;
  const int most = min(len, len_before) / g.c.page_tokens;
  if (tid == 0) {
    s_first = most;
    const int bad = seq < 0 || seq >= g.c.n_seqs ? SI_CACHE_BAD_SEQ : g.c.lens[seq] < 0 || g.c.lens[seq] > g.c.max_pages * g.c.page_tokens ? SI_CACHE_BAD_LEN : 0;
    if (bad) atomicOr(g.c.status, bad);
  }
  const int32_t *mine = g.c.table + (int64_t)max(seq, 0) * g.c.max_pages, *before = g.c.table + (int64_t)max(seq_before, 0) * g.c.max_pages;
  for (int j0 = 0; j0 < most; j0 += THREADS) {
    __syncthreads();
    if (s_first < most) break;
    const int j = j0 + tid;
    __syncthreads();
    if (j < most && (before[j] != mine[j] || mine[j] < 0 || mine[j] >= g.c.n_pages)) atomicMin(&s_first, j);
  }
  __syncthreads();
  if (tid == 0) {
    __hip_atomic_store(g.facts + e, (uint64_t)len << 32 | (uint32_t)s_first, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    s_last = __hip_atomic_fetch_add(g.count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)g.n - 1;
    if (s_last) __hip_atomic_store(g.count, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  if (!s_last) return;

  // Notes: blocks of each piece, then the sum of them and of those before; of the entries their facts; of a group's first entry its tokens and first piece
  const int n = g.n, n_own = n * g.chunks, of_entry = g.n_new * g.per;
  int32_t* area;
  if constexpr (LOCAL) area = s_area;
  else area = g.area;
  int64_t *own_to = reinterpret_cast<int64_t*>(area), *shared_to = own_to + n_own;
  int32_t *seqs = reinterpret_cast<int32_t*>(shared_to + g.most), *lens = seqs + n, *common = lens + n, *firsts = common + n, *tokens_of = firsts + n, *piece_of = tokens_of + n;
  for (int i = tid; i < n; i += THREADS) {
    const uint64_t f = __hip_atomic_load(g.facts + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    seqs[i] = seq_at(g, i);
    lens[i] = (int)(f >> 32);
    common[i] = (int)(uint32_t)f;
  }
  __syncthreads();
  // A group ends where two neighbours have nothing in common, or less than half of what one of them has in common with its other neighbour (two
  // prompts with the same few words before them are two groups).
  auto begins = [&](int i) { return i == 0 || common[i] == 0 || 2ll * common[i] < max(i > 1 ? common[i - 1] : 0, i + 1 < n ? common[i + 1] : 0); };

  Run carry{0, 0x7fffffff, 0x7fffffff, 0};  // the group that is open before these entries
  int n_shared = 0;
  for (int e0 = 0; e0 < n; e0 += THREADS) {
    const int i = e0 + tid;
    const bool in = i < n;
    bool any = in && begins(i);  // a group begins among the entries that r covers
    Run r{i, 0x7fffffff, 0x7fffffff, 0};
    if (in) {
      r.shortest = r.longest = lens[i];
      r.pages = max(0, lens[i] - g.n_new + 1) / g.c.page_tokens;  // (what the first of the new tokens sees too)
      if (!any) r.pages = min(r.pages, common[i]);
    }
    const bool ends = in && (i + 1 == n || begins(i + 1));
    auto step = [&](auto ctrl, auto rows, bool there) {  // there: a lane that this one takes a run from
      constexpr int C = decltype(ctrl)::value, M = decltype(rows)::value;
      const Run o{(int)moved<C, M>((uint32_t)r.first), (int)moved<C, M>((uint32_t)r.pages), (int)moved<C, M>((uint32_t)r.shortest), (int)moved<C, M>((uint32_t)r.longest)};
      const bool o_any = moved<C, M>((uint32_t)any) != 0;
      if (there && !any) {
        r = joined(o, r);
        any = o_any;
      }
    };
    step(std::integral_constant<int, SHIFT + 1>{}, std::integral_constant<int, 0xf>{}, lane % 16 >= 1);
    step(std::integral_constant<int, SHIFT + 2>{}, std::integral_constant<int, 0xf>{}, lane % 16 >= 2);
    step(std::integral_constant<int, SHIFT + 4>{}, std::integral_constant<int, 0xf>{}, lane % 16 >= 4);
    step(std::integral_constant<int, SHIFT + 8>{}, std::integral_constant<int, 0xf>{}, lane % 16 >= 8);
    step(std::integral_constant<int, FROM_ROW>{}, std::integral_constant<int, 0xa>{}, lane / 16 % 2 == 1);
    step(std::integral_constant<int, FROM_HALF>{}, std::integral_constant<int, 0xc>{}, lane >= 32);
    __syncthreads();
    if (lane == 63) { s_run[wave] = r; s_begins[wave] = any; }
    __syncthreads();
    Run open = carry;
    for (int w = 0; w < wave; ++w) open = s_begins[w] ? s_run[w] : joined(open, s_run[w]);
    if (!any) r = joined(open, r);
    Run next = carry;
    for (int w = 0; w < WAVES; ++w) next = s_begins[w] ? s_run[w] : joined(next, s_run[w]);
    // (beyond the last entry a run is empty and changes nothing)
    const int members = i - r.first + 1, tokens = ends && members > 1 ? r.pages * g.c.page_tokens : 0, rows = members * of_entry;
    const int pieces = tokens > 0 ? (rows + g.wide_rows - 1) / g.wide_rows : 0;
    int at = (int)scan_wave((uint32_t)pieces);
    if (lane == 63) s_offset[wave] = at;
    __syncthreads();
    at += n_shared - pieces;
    for (int w = 0; w < WAVES; ++w) {
      if (w < wave) at += s_offset[w];
      n_shared += s_offset[w];
    }
    if (in) firsts[i] = r.first;
    if (ends) {
      tokens_of[r.first] = tokens;
      piece_of[r.first] = pieces > 0 ? at : -1;
      const bool windows = g.window > 0 && tokens > 0;  // (all of a group have n_new tokens then: no difference passes 32 bits)
      const int lo = windows ? min(tokens, max(0, r.shortest - g.n_new + 1 - g.window)) : 0, lo_all = windows ? min(tokens, max(0, r.longest - g.window)) : 0;
      const int nb = tokens > lo ? tokens / B - lo / B : 0;
      for (int k = 0; k < pieces; ++k) {
        g.shared.pieces[at + k] = Piece{seqs[r.first], r.first * of_entry + k * g.wide_rows, min(g.wide_rows, rows - k * g.wide_rows), lo, tokens, lo_all, tokens, lo / B, nb, -1, 0};
        shared_to[at + k] = max(1, nb);
      }
    }
    carry = next;
  }
  __syncthreads();
  for (int k = tid; k < n_own; k += THREADS) {
    const int i = k / g.chunks, row0 = (k - i * g.chunks) * g.block_rows, rows = min(g.block_rows, of_entry - row0), first = firsts[i], from = tokens_of[first];
    const int sight = lens[i] - g.n_new + 1, t0 = row0 / g.per, t1 = (row0 + rows - 1) / g.per;
    const int window = g.window < lens[i] ? g.window : 0;  // (sight may be negative: less the longest windows it would pass 32 bits)
    const int hi = max(0, sight + t1), lo = window ? max(from, sight + t0 - window) : from, nb = hi > lo ? (hi + B - 1) / B - lo / B : 0;
    g.own.pieces[k] = Piece{seqs[i], i * of_entry + row0, rows, lo, hi, window ? max(from, sight + t1 - window) : from, max(0, sight + t0), lo / B, nb, i, sight};
    own_to[k] = max(1, nb);
    if (row0 == 0) g.group[i] = make_int2(piece_of[first], first);
  }
  __syncthreads();
  int64_t total[2] = {0, 0};
  for (int k0 = 0; k0 < max(n_own, n_shared); k0 += THREADS) {
    const int k = k0 + tid;
    int64_t x[2] = {k < n_shared ? shared_to[k] : 0, k < n_own ? own_to[k] : 0};
    for (int q = 0; q < 2; ++q) x[q] = (int64_t)scan_wave((uint64_t)x[q]);
    __syncthreads();
    if (lane == 63) { s_sum[0][wave] = x[0]; s_sum[1][wave] = x[1]; }
    __syncthreads();
    for (int q = 0; q < 2; ++q) {
      x[q] += total[q];
      for (int w = 0; w < WAVES; ++w) {
        if (w < wave) x[q] += s_sum[q][w];
        total[q] += s_sum[q][w];
      }
    }
    if (k < n_shared) shared_to[k] = x[0];
    if (k < n_own) own_to[k] = x[1];
  }
  __syncthreads();
  // Equal slices of each list's blocks: slice w is [end(w - 1), end(w)) with end(w) = (w + 1) total / G.  (Quotients by way of double: exact, as the dividends
  // stay below 2^53.)
  auto quotient = [](int64_t x, int64_t y) { return (int64_t)((double)x / (double)y); };
  {
    const int q = wave * 2 / WAVES, id = tid % (THREADS / 2);  // (half of the threads a list)
    const int64_t *to = q ? own_to : shared_to, sum = q ? total[1] : total[0];
    const int pieces = q ? n_own : n_shared, slices = q ? g.own.slices : g.shared.slices, G = (int)min<int64_t>(slices, sum);
    int2* parted = q ? g.own.parted : g.shared.parted;
    SliceStart* starts = q ? g.own.starts : g.shared.starts;
#pragma unroll 1
    for (int k = id; k < pieces; k += THREADS / 2) {
      int of[2];  // the slices of its first and last block: those whose ends are the first beyond them
      for (int h = 0; h < 2; ++h) of[h] = (int)quotient((h ? to[k] : (k > 0 ? to[k - 1] : 0) + 1) * G - 1, sum);
      parted[k] = make_int2(of[0], of[1] - of[0] + 1);
    }
#pragma unroll 1
    for (int w = id; w < slices; w += THREADS / 2) {
      SliceStart start{0, 0, 0};
      if (w < G) {
        const int64_t begin = quotient(w * sum, G), end = quotient((w + 1) * sum, G);
        int k = 0;  // the first piece that ends beyond the slice's begin
        for (int hi = pieces - 1; k < hi;) {
          const int mid = (k + hi) / 2;
          if (to[mid] > begin) hi = mid; else k = mid + 1;
        }
        start = SliceStart{k, (int)(begin - (k > 0 ? to[k - 1] : 0)), (int)(end - begin)};
      }
      starts[w] = start;
    }
  }
}

constexpr int WIDE = 128;  // rows of a shared piece
constexpr int MOST_ROWS = 1 << 16, MOST_SUMS = 1 << 19;  // of a kv head, of all

struct Layout {
  AttendCut alone;           // of si_attend
  bool pieces;               // else the call is si_attend
  bool local;                // the plan's notes fit its shared memory
  int block_rows, chunks, shared_slices, own_slices;
  int64_t shared_parted, own_parted, shared_part, own_part, sums, shared, own, shared_starts, own_starts, group, facts, area, most, bytes;
};

Layout lay_out(const si_cache_t& c, const si_attend_t& a) {
  Layout l{};
  l.alone = cut_attend(c, a);
  const int64_t of_entry = (int64_t)a.n_new * (a.n_heads / c.n_kv_heads);
  // (a block of the joining launch has 4 rows or more, and all rows have two sums; longer lists are si_attend's and need its scratch and that of shorter ones)
  const int n = (int)std::min<int64_t>(a.n, std::min(MOST_ROWS, MOST_SUMS / c.n_kv_heads) / of_entry);
  const int64_t rows = n * of_entry;
  l.bytes = l.alone.scratch;
  if (n < 2) return l;
  // Pieces cost three launches, some 25 us of planning and joining, so calls that are short anyway are si_attend: those that read less than 640 MB even if
  // no page were shared.  Measured with one prompt for all, heads 32 of 8 x 128 bf16, as pieces and as si_attend: 4 x 611 tokens (12 MB) 24 and 14 us,
  // 64 x 1000 (288 MB) 37 and 18, 64 x 2000 (550 MB) 38 and 31, 256 x 512 (642 MB) 57 and 43, 64 x 4000 (1075 MB) 43 and 68, 64 x 8000 50 and 135.
  const double sight = a.window > 0 ? std::min<double>(a.max_len, (double)a.window + a.n_new) : a.max_len, reads = a.n * sight * c.n_kv_heads * c.head_dim * (c.type == SI_KV_BF16 ? 4 : 2);
  l.pieces = n == a.n && (reads >= 640e6 || std::getenv("SI_ATTEND_PIECES"));  // (the variable: tests of the pieces at small sizes)
  for (l.block_rows = 16; l.block_rows < of_entry && l.block_rows < 64;) l.block_rows *= 2;
  l.chunks = (int)((of_entry + l.block_rows - 1) / l.block_rows);
  const int64_t each = (a.max_len + kv_block(c.type) - 1) / kv_block(c.type), turns = (rows + WIDE - 1) / WIDE * each * c.n_kv_heads / 256;
  l.shared_slices = std::max(1, (turns > 32 && c.head_dim < 192 ? 512 : 256) / c.n_kv_heads);
  l.own_slices = std::max(1, std::min(std::max(n * l.chunks, 256 / c.n_kv_heads), 512 / c.n_kv_heads));
  const int64_t shared = rows / WIDE + n / 2 + 1, own = (int64_t)n * l.chunks;
  int64_t at = std::max<int64_t>(l.alone.scratch, ATTEND_COUNTERS * 4);  // (the counters are at the same place in every call's scratch)
  auto take = [&](int64_t bytes) {
    const int64_t q = (at + 15) / 16 * 16;
    at = q + bytes;
    return q;
  };
  l.shared_parted = take(shared * 8);
  l.own_parted = take(own * 8);
  l.shared_part = take((int64_t)c.n_kv_heads * l.shared_slices * 2 * WIDE * (c.head_dim + 4) * 4);
  l.own_part = take((int64_t)c.n_kv_heads * l.own_slices * 2 * std::min<int64_t>(of_entry, l.block_rows) * (c.head_dim + 2) * 4);
  l.sums = take(2 * c.n_kv_heads * rows * (c.head_dim + 4) * 4);
  l.shared = take(shared * (int64_t)sizeof(Piece));
  l.own = take(own * (int64_t)sizeof(Piece));
  l.shared_starts = take(l.shared_slices * (int64_t)sizeof(SliceStart));
  l.own_starts = take(l.own_slices * (int64_t)sizeof(SliceStart));
  l.group = take(n * 8ll);
  l.facts = take(n * 8ll);
  l.most = shared;
  l.local = area_words(n, shared, l.chunks) <= AREA;
  l.area = take(l.local ? 0 : area_words(n, shared, l.chunks) * 4);
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
  if (l.bytes > 0 && (!a->scratch || a->scratch_bytes < l.bytes || (reinterpret_cast<uintptr_t>(a->scratch) & 15) != 0))  // (none needed: an empty tensor's address may be NULL)
    return set_error(SI_EINVAL, "%s: %lld bytes of scratch needed, 16-byte aligned", who, (long long)l.bytes);
  char* p = static_cast<char*>(a->scratch);
  AttendArgs g = attend_args(*c, *a, layer, l.alone);
  hipError_t e = hipSuccess;
  if (!l.pieces) {
    e = (c->type == SI_KV_BF16 ? launch_attend_bf16 : launch_attend_e4m3)(g, (hipStream_t)stream);
  } else {
    const int part_rows = std::min(a->n_new * (a->n_heads / c->n_kv_heads), l.block_rows);
    const PlanList shared{l.shared_slices, reinterpret_cast<Piece*>(p + l.shared), reinterpret_cast<SliceStart*>(p + l.shared_starts), reinterpret_cast<int2*>(p + l.shared_parted)};
    const PlanList mine{l.own_slices, reinterpret_cast<Piece*>(p + l.own), reinterpret_cast<SliceStart*>(p + l.own_starts), reinterpret_cast<int2*>(p + l.own_parted)};
    const PlanArgs plan{*c, a->seqs, a->n, a->n_new, a->n_heads / c->n_kv_heads, a->window, WIDE, l.block_rows, l.chunks, reinterpret_cast<uint32_t*>(p), reinterpret_cast<uint64_t*>(p + l.facts),
                        l.local ? nullptr : reinterpret_cast<int32_t*>(p + l.area), (int)l.most, shared, mine, reinterpret_cast<int2*>(p + l.group)};
    g.rows = g.block_rows = l.block_rows;
    g.groups = 1;
    g.whole = g.last_joins = 0;
    g.shared = PieceList{l.shared_slices, shared.pieces, shared.starts, shared.parted, reinterpret_cast<float*>(p + l.shared_part), WIDE, c->head_dim + 4};
    g.own = PieceList{l.own_slices, mine.pieces, mine.starts, mine.parted, reinterpret_cast<float*>(p + l.own_part), part_rows, c->head_dim + 2};
    g.sums = reinterpret_cast<float*>(p + l.sums);
    g.group = plan.group;
    g.chunks = l.chunks;
    hipLaunchKernelGGL(l.local ? k_share<true> : k_share<false>, dim3(a->n), dim3(THREADS), 0, (hipStream_t)stream, plan);
    e = hipGetLastError();
    if (e == hipSuccess) e = (c->type == SI_KV_BF16 ? launch_attend_pieces_bf16 : launch_attend_pieces_e4m3)(g, (hipStream_t)stream);
  }
  if (e != hipSuccess) return set_error(SI_EHIP, "attention launch failed: %s", hipGetErrorString(e));
  return SI_OK;
}
