// Moves of the cache's pages.  Every decision (which page is free, who shares what) depends on all of the small tables, so a block makes it
// alone, with prefix sums instead of counters.  Where pages are copied, all blocks of a launch make the same decisions, each copies its
// share (into pages that are free: nobody minds, whatever comes after), and the block that finishes last, when nobody reads the tables any
// more, writes them: one launch, and no block waits for another.  (A launch that decides and one that copies: 33 sequences extended
// 13.9 us a call, in one launch 11.7; 48 beams of 5 sources forked 113 and 108.)
// Forking and compacting are bound by memory (beams: 445 MB, 4.3 TB/s; 2.0 GB of a pool packed in 366 us, 5.5 TB/s), extending by the
// chain of a decision: lists, lengths, table, counts, two prefix sums, 9 us in the kernel for 33 sequences.
#include "si_internal.h"
#include "si_error.h"
#include "kv_layout.h"

#include <algorithm>

namespace si {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef i32x4 i32x4_a4 __attribute__((aligned(4)));

constexpr int WAVE = 64;
constexpr int BOOK = 1024;            // threads of the block that keeps the books
constexpr int WAVES = BOOK / WAVE;
constexpr int PER_THREAD = 8;         // pages of a thread in one sweep of the reference counts
constexpr int COPY_THREADS = 256;
constexpr int COPY_BYTES = 65536;     // of a page that a block copies

// scratch of a cache
struct Head { uint32_t arrived; int32_t used, pad[14]; };  // arrived: 0 between calls
struct Scratch {
  Head* head;
  int32_t* list;   // [n_pages] free pages; pages that move: holes
  int32_t* place;  // [n_pages] new number of a page
};
__host__ __device__ inline int64_t round16(int64_t x) { return (x + 15) / 16 * 16; }
int64_t scratch_bytes(const si_cache_t& c) { return sizeof(Head) + 2 * round16(4ll * c.n_pages); }
Scratch scratch_of(const si_cache_t& c) {
  char* p = static_cast<char*>(c.scratch);
  Scratch s;
  s.head = reinterpret_cast<Head*>(p); p += sizeof(Head);
  s.list = reinterpret_cast<int32_t*>(p); p += round16(4ll * c.n_pages);
  s.place = reinterpret_cast<int32_t*>(p);
  return s;
}

__device__ __forceinline__ int ceil_div(int a, int b) { return (a + b - 1) / b; }

// exclusive prefix sum over the block; `total` of all
__device__ __forceinline__ int block_scan(int v, int& total, int (&w)[WAVES]) {
  const int lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE;
  int x = v;
#pragma unroll
  for (int d = 1; d < WAVE; d *= 2) {
    const int y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  __syncthreads();  // (w may still be read from the scan before)
  if (lane == WAVE - 1) w[wave] = x;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int i = 0; i < WAVES; ++i) {
    before += i < wave ? w[i] : 0;
    total += w[i];
  }
  return before + x - v;
}

// reference counts of pages at .. at + 7 (1 beyond the pool): bit i: page at + i is free
__device__ __forceinline__ int free_bits(const int32_t* refs, int n_pages, int at) {
  int bits = 0;
  if (at + PER_THREAD <= n_pages) {
    const i32x4 a = *reinterpret_cast<const i32x4_a4*>(refs + at), b = *reinterpret_cast<const i32x4_a4*>(refs + at + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) bits |= (a[i] <= 0) << i | (b[i] <= 0) << (i + 4);
  } else {
    for (int i = 0; i < PER_THREAD; ++i)
      if (at + i < n_pages && refs[at + i] <= 0) bits |= 1 << i;
  }
  return bits;
}

// The first `need` free pages into `list`; returns how many there are, counted up to at least `need`.  bits: free_bits of the thread's first pages
__device__ int list_free(const si_cache_t& c, int need, int bits, int32_t* list, int (&w)[WAVES]) {
  int found = 0;
  for (int at0 = 0; at0 < c.n_pages && found < need; at0 += BOOK * PER_THREAD) {
    const int at = at0 + threadIdx.x * PER_THREAD;
    if (at0 > 0) bits = at < c.n_pages ? free_bits(c.refs, c.n_pages, at) : 0;
    int total, rank = found + block_scan(__popc(bits), total, w);
    for (; bits && rank < need; bits &= bits - 1, ++rank) list[rank] = at + __ffs(bits) - 1;
    found += total;
  }
  return found;
}

// largest e < n with prefix[e] <= f (entries that add nothing are passed over, as prefix[n] > f)
__device__ __forceinline__ int entry_of(const int* prefix, int n, int f) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (prefix[mid] <= f) lo = mid;
    else hi = mid;
  }
  return lo;
}

static_assert(SI_CACHE_MAX_LIST == BOOK, "a thread for each entry of a list");
constexpr int SHORT_LIST = 4096;  // free pages that are listed in LDS
struct BookLds {
  int w[WAVES];
  int64_t w2[2][WAVES];
  int seq[BOOK], len[BOOK];
  int need[BOOK + 1];     // prefix sums: pages taken
  int put[BOOK + 1];      // tokens added (extend), pages named (fork)
  int src[BOOK];          // page that is copied for the entry, or -1
  int first[BOOK];        // of the entries with this source
  int g_src[BOOK], g_first[BOOK], g_count[BOOK];  // one source each, copied to dst[first] .. dst[first + count - 1]
  int dst[BOOK];
  int list[SHORT_LIST];
  int groups, why;
  uint32_t arrived;
};

// s.need and s.put become the prefix sums of the entries' a and b, with the totals behind them; false where a total does not fit 31 bits
__device__ bool prefix_lists(BookLds& s, int n, int a, int b) {
  const int lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE;
  int64_t x = a, y = b;
#pragma unroll
  for (int d = 1; d < WAVE; d *= 2) {
    const int64_t x2 = __shfl_up(x, d), y2 = __shfl_up(y, d);
    if (lane >= d) { x += x2; y += y2; }
  }
  if (lane == WAVE - 1) { s.w2[0][wave] = x; s.w2[1][wave] = y; }
  __syncthreads();
  int64_t before_x = 0, before_y = 0, all_x = 0, all_y = 0;
  for (int i = 0; i < WAVES; ++i) {
    if (i < wave) { before_x += s.w2[0][i]; before_y += s.w2[1][i]; }
    all_x += s.w2[0][i];
    all_y += s.w2[1][i];
  }
  if (all_x > 0x7fffffff || all_y > 0x7fffffff) return false;
  if ((int)threadIdx.x < n) { s.need[threadIdx.x] = (int)(before_x + x - a); s.put[threadIdx.x] = (int)(before_y + y - b); }
  if (threadIdx.x == 0) { s.need[n] = (int)all_x; s.put[n] = (int)all_y; }
  __syncthreads();
  return true;
}

// Number of entries i < end with v[i] == x
__device__ __forceinline__ int equals(const int* v, int end, int x) {
  int k = 0;
  for (int i = 0; i < end; ++i) k += v[i] == x;
  return k;
}

// Entries with the same source next to each other, so that a source is read once: s.src[e] is copied to `dst` of the thread's entry
__device__ void list_copies(BookLds& s, int n, int dst) {
  const int e = threadIdx.x, src = e < n ? s.src[e] : -1;
  int f = e;
  if (src >= 0)
    for (f = 0; s.src[f] != src; ++f) {}
  if (e < n) s.first[e] = src >= 0 ? f : -1;
  if (e == 0) s.groups = 0;
  __syncthreads();
  if (src >= 0) {
    int before = 0, rank = 0, count = 0, groups_before = 0;
    for (int i = 0; i < n; ++i) {
      const int o = s.first[i];
      before += o >= 0 && o < f;
      groups_before += o == i && o < f;
      count += o == f;
      rank += o == f && i < e;
    }
    s.dst[before + rank] = dst;
    if (f == e) {
      s.g_src[groups_before] = src; s.g_first[groups_before] = before; s.g_count[groups_before] = count;
      atomicAdd(&s.groups, 1);
    }
  }
  __syncthreads();
}

// bytes [at, end) of one page to `count` others; `dst(i)` is the first byte of the i-th
template <int THREADS, class F> __device__ __forceinline__ void copy_run(const char* src, int64_t at, int64_t end, int count, F dst) {
  constexpr int STEP = THREADS * 16, N = 4;
  for (at += threadIdx.x * 16; at < end; at += N * STEP) {
    u32x4 v[N];
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (at + i * STEP < end) v[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src + at + i * STEP));
    for (int k = 0; k < count; ++k) {
      char* to = dst(k);
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (at + i * STEP < end) __builtin_nontemporal_store(v[i], reinterpret_cast<u32x4*>(to + at + i * STEP));
    }
  }
}
// this block's share of the listed copies
__device__ void copy_share(const BookLds& s, char* pages, int64_t page_bytes, int parts) {
  for (int64_t i = blockIdx.x; i < (int64_t)s.groups * parts; i += gridDim.x) {
    const int q = (int)(i / parts), first = s.g_first[q];
    const int64_t at = i % parts * COPY_BYTES;
    copy_run<BOOK>(pages + s.g_src[q] * page_bytes, at, min(page_bytes, at + COPY_BYTES), s.g_count[q], [&](int k) { return pages + s.dst[first + k] * page_bytes; });
  }
}
// the block that finishes last goes on
__device__ bool last_block(BookLds& s, Head* head) {
  __syncthreads();
  if (threadIdx.x == 0) {
    s.arrived = __hip_atomic_fetch_add(&head->arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (s.arrived == gridDim.x - 1) __hip_atomic_store(&head->arrived, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  return s.arrived == gridDim.x - 1;
}

// A wave for each entry of the list; that of a sequence's first entry takes all of its entries, in list order, so that no two waves write to
// a sequence and what is reported does not depend on which comes first.  Each entry that is not left out makes the sequence shorter: the pages
// are dropped together, after the last.
__global__ __launch_bounds__(WAVE) void k_trim(si_cache_t c, const int32_t* __restrict__ seqs, int n, const int32_t* __restrict__ keep) {
  const int e = blockIdx.x, seq = seqs[e], lane = threadIdx.x;
  if (seq < 0 || seq >= c.n_seqs) {
    if (lane == 0) atomicOr(c.status, keep && keep[e] < 0 ? SI_CACHE_BAD_LEN : SI_CACHE_BAD_SEQ);
    return;
  }
  const int old = c.lens[seq];
  bool earlier = false;
  for (int i = lane; i < e; i += WAVE) earlier |= seqs[i] == seq;
  if (__any(earlier)) return;
  int len = old, why = 0;
  for (int i0 = e; i0 < n; i0 += WAVE) {
    const int i = i0 + lane;
    const bool mine = i < n && seqs[i] == seq;
    const int to = mine && keep ? keep[i] : 0;
    for (uint64_t m = __ballot(mine); m; m &= m - 1) {
      const int k = __builtin_amdgcn_readlane(to, __ffsll((unsigned long long)m) - 1);
      if (k < 0 || k > len) why |= SI_CACHE_BAD_LEN;
      else len = k;
    }
  }
  const int most = c.max_pages * c.page_tokens;
  if (old > most) why |= SI_CACHE_BAD_LEN;
  int32_t* row = c.table + (int64_t)seq * c.max_pages;
  for (int j = ceil_div(min(max(len, 0), most), c.page_tokens) + lane; j < ceil_div(min(max(old, 0), most), c.page_tokens); j += WAVE) {
    const int page = row[j];
    row[j] = -1;
    if (page < 0 || page >= c.n_pages) {
      why |= SI_CACHE_BAD_PAGE;
    } else if (atomicSub(c.refs + page, 1) <= 0) {
      atomicAdd(c.refs + page, 1);
      why |= SI_CACHE_BAD_PAGE;
    }
  }
  if (lane == 0 && len != old) c.lens[seq] = len;
  if (why) atomicOr(c.status, why);
}

struct ExtendArgs {
  si_cache_t c;
  Scratch x;
  const int32_t *seqs, *counts;
  int32_t *seq_out, *pos_out;
  int n, n_new, capacity, parts;
  int64_t page_bytes;
};

__global__ __launch_bounds__(BOOK) void k_extend(ExtendArgs g) {
  __shared__ BookLds s;
  const si_cache_t& c = g.c;
  const int e = threadIdx.x, page = c.page_tokens, n = g.n;
  const int bits = e * PER_THREAD < c.n_pages ? free_bits(c.refs, c.n_pages, e * PER_THREAD) : 0;
  if (e == 0) { s.why = 0; s.groups = 0; }
  int why = 0, seq = -1, m = 0, len = 0, need = 0, src = -1, shared = 0;
  if (e < n) {
    seq = g.seqs[e];
    m = g.counts ? g.counts[e] : g.n_new;
    if (seq < 0 || seq >= c.n_seqs) {
      why = SI_CACHE_BAD_SEQ;
    } else {
      len = c.lens[seq];
      if (len < 0 || m < 0 || (int64_t)len + m > (int64_t)c.max_pages * page) {
        why = SI_CACHE_BAD_LEN;
      } else {
        need = ceil_div(len + m, page) - ceil_div(len, page);
        if (m > 0 && len % page > 0) {
          const int last = c.table[(int64_t)seq * c.max_pages + len / page];
          // (a page with a count of 0 counts as free, and would be given away)
          const int count = last < 0 || last >= c.n_pages ? 0 : c.refs[last];
          if (count <= 0) why = SI_CACHE_BAD_PAGE;
          else if ((shared = count - 1) > 0) src = last;
        }
      }
    }
    s.seq[e] = seq; s.len[e] = len; s.src[e] = src;
  }
  const bool some = __syncthreads_or(src >= 0);
  if (e < n && equals(s.seq, e, seq) > 0) why |= SI_CACHE_BAD_SEQ;
  if (some) {
    // a shared last page: whoever comes after all of its other sharers keeps it
    if (src >= 0 && equals(s.src, e, src) >= shared) src = -1;
    __syncthreads();
    if (e < n) s.src[e] = src;
    need += src >= 0;
  }
  if (why) atomicOr(&s.why, why);
  bool ok = prefix_lists(s, n, need, why ? 0 : m);
  why = ok ? 0 : SI_CACHE_NO_ROOM;
  ok = ok && s.why == 0;
  int pages = 0, tokens = 0;
  int32_t* list = s.list;
  if (ok) {
    pages = s.need[n];
    tokens = s.put[n];
    if (pages > SHORT_LIST) list = g.x.list;  // (every block writes the same)
    if (g.seq_out && tokens > g.capacity) { ok = false; why = SI_CACHE_NO_ROOM; }
    else if (pages > 0 && list_free(c, pages, bits, list, s.w) < pages) { ok = false; why = SI_CACHE_NO_PAGES; }
  }
  __syncthreads();
  if (ok && some) {
    list_copies(s, n, e < n ? list[min(s.need[e], pages - 1)] : 0);
    copy_share(s, static_cast<char*>(c.pages), g.page_bytes, g.parts);
  }
  if (!last_block(s, g.x.head)) return;
  if (ok) {
    for (int f = e; f < pages; f += BOOK) {
      const int i = entry_of(s.need, n, f), k = f - s.need[i], p = list[f];
      const int j = s.src[i] >= 0 ? s.len[i] / page + k : ceil_div(s.len[i], page) + k;
      c.table[(int64_t)s.seq[i] * c.max_pages + j] = p;
      c.refs[p] = 1;
      if (s.src[i] >= 0 && k == 0) atomicSub(c.refs + s.src[i], 1);
    }
    if (e < n) c.lens[seq] = len + m;
  } else if (e == 0) {
    atomicOr(c.status, why | s.why);
  }
  if (g.seq_out)
    for (int f = e; f < g.capacity; f += BOOK) {
      int to = -1, pos = -1;
      if (f < tokens && ok) {
        const int i = g.counts ? entry_of(s.put, n, f) : f / g.n_new;
        to = s.seq[i];
        pos = s.len[i] + f - s.put[i];
      }
      g.seq_out[f] = to;
      g.pos_out[f] = pos;
    }
}

struct ForkArgs {
  si_cache_t c;
  Scratch x;
  const int32_t *parents, *children;
  int n, parts;
  int64_t page_bytes;
};

__global__ __launch_bounds__(BOOK) void k_fork(ForkArgs g) {
  __shared__ BookLds s;  // seq: child, len: parent's, put: pages of the parent
  const si_cache_t& c = g.c;
  const int e = threadIdx.x, page = c.page_tokens, n = g.n;
  const int bits = e * PER_THREAD < c.n_pages ? free_bits(c.refs, c.n_pages, e * PER_THREAD) : 0;
  if (e == 0) { s.why = 0; s.groups = 0; }
  int bad_seq = 0, bad_len = 0, bad_page = 0, a = -1, b = -1, len = 0, src = -1;
  if (e < n) {
    a = g.parents[e];
    b = g.children[e];
    bad_seq = a < 0 || a >= c.n_seqs || b < 0 || b >= c.n_seqs;
    if (!bad_seq) {
      len = c.lens[a];
      bad_len = c.lens[b] != 0 || len < 0 || len > c.max_pages * page;
      if (!bad_len && len % page > 0) {
        src = c.table[(int64_t)a * c.max_pages + len / page];
        bad_page = src < 0 || src >= c.n_pages;
      }
      if (bad_len || bad_page) { len = 0; src = -1; }
    }
    s.seq[e] = b; s.len[e] = len; s.src[e] = src;
  }
  __syncthreads();
  if (e < n && !bad_seq) bad_seq = equals(s.seq, e, b) > 0 || equals(s.seq, n, a) > 0;  // named twice, or parent and child
  bad_seq = __syncthreads_or(bad_seq);
  bad_len = __syncthreads_or(bad_len);
  bad_page = __syncthreads_or(bad_page);
  // (sequence numbers, then lengths, then pages: each counts only where what comes before is in order)
  int why = bad_seq ? SI_CACHE_BAD_SEQ : bad_len ? SI_CACHE_BAD_LEN : bad_page ? SI_CACHE_BAD_PAGE : 0;
  bool ok = why == 0;
  int32_t* list = s.list;  // (at most one page an entry)
  int pages = 0, named = 0;
  if (ok) {
    if (e < n) s.first[e] = a;
    ok = prefix_lists(s, n, src >= 0, ceil_div(len, page));
    why = SI_CACHE_NO_PAGES;
  }
  if (ok) {
    pages = s.need[n];
    named = s.put[n];
    for (int f = e; f < named; f += BOOK) {
      const int i = entry_of(s.put, n, f), p = c.table[(int64_t)s.first[i] * c.max_pages + f - s.put[i]];
      if (p < 0 || p >= c.n_pages || c.refs[p] <= 0) bad_page = 1;
    }
    bad_page = __syncthreads_or(bad_page);
    if (bad_page) why = SI_CACHE_BAD_PAGE;
    ok = !bad_page && (pages == 0 || list_free(c, pages, bits, list, s.w) >= pages);
  }
  __syncthreads();
  if (ok && pages > 0) {
    list_copies(s, n, e < n ? list[min(s.need[e], pages - 1)] : 0);
    copy_share(s, static_cast<char*>(c.pages), g.page_bytes, g.parts);
  }
  if (!last_block(s, g.x.head)) return;
  if (!ok) {
    if (e == 0) atomicOr(c.status, why);
    return;
  }
  if (e < n) s.first[e] = a;  // (list_copies has had it)
  __syncthreads();
  for (int f = e; f < named; f += BOOK) {
    const int i = entry_of(s.put, n, f), j = f - s.put[i];
    int p;
    if (j == s.len[i] / page) {
      p = list[s.need[i]];
      c.refs[p] = 1;
    } else {
      p = c.table[(int64_t)s.first[i] * c.max_pages + j];
      atomicAdd(c.refs + p, 1);
    }
    c.table[(int64_t)s.seq[i] * c.max_pages + j] = p;
  }
  if (e < n) c.lens[b] = len;
}

__global__ __launch_bounds__(BOOK) void k_places(si_cache_t c, Scratch x, int room, int32_t* n_used) {
  __shared__ int w[WAVES];
  const int tid = threadIdx.x, n = c.n_pages;
  int mine = 0, used = 0;
  for (int at = tid * PER_THREAD; at < n; at += BOOK * PER_THREAD) mine += min(PER_THREAD, n - at) - __popc(free_bits(c.refs, n, at));
  block_scan(mine, used, w);
  if (tid == 0) {
    x.head->used = used <= room ? used : -1;
    if (n_used) *n_used = used;
    if (used > room) atomicOr(c.status, SI_CACHE_NO_PAGES);
  }
  if (used > room) return;
  int holes = 0, movers = 0;
  for (int at0 = 0; at0 < n; at0 += BOOK * PER_THREAD) {
    const int at = at0 + tid * PER_THREAD, here = max(0, min(PER_THREAD, n - at));
    const int bits = here > 0 ? free_bits(c.refs, n, at) : 0;
    const int low = max(0, min(here, used - at));  // pages of this thread below the border
    int total;
    int hole = holes + block_scan(__popc(bits & ((1 << low) - 1)), total, w);
    holes += total;
    int mover = movers + block_scan(here - low - __popc(bits >> low), total, w);
    movers += total;
    for (int i = 0; i < low; ++i) {
      const bool is_free = bits >> i & 1;
      if (is_free) x.list[hole++] = at + i;
      x.place[at + i] = is_free ? -1 : at + i;
    }
    __syncthreads();
    for (int i = low; i < here; ++i) x.place[at + i] = bits >> i & 1 ? -1 : x.list[mover++];
  }
}

struct CompactArgs {
  si_cache_t c, to;
  Scratch x;
  int parts;         // of a page
  int64_t copy_blocks;
};

__global__ __launch_bounds__(COPY_THREADS) void k_compact(CompactArgs g) {
  const int used = g.x.head->used;
  if (used < 0) return;
  const int64_t page_bytes = kv_page_elems(g.c) * kv_elem_bytes(g.c.type);
  if (blockIdx.x < g.copy_blocks) {
    const int p = blockIdx.x / g.parts, place = g.x.place[p];
    if (place < 0 || (place == p && g.to.pages == g.c.pages)) return;
    const int64_t at = (int64_t)(blockIdx.x % g.parts) * COPY_BYTES;
    char* to = static_cast<char*>(g.to.pages) + place * page_bytes;
    copy_run<COPY_THREADS>(static_cast<const char*>(g.c.pages) + p * page_bytes, at, min(page_bytes, at + COPY_BYTES), 1, [&](int) { return to; });
    return;
  }
  const int64_t first = (blockIdx.x - g.copy_blocks) * COPY_THREADS + threadIdx.x, step = (gridDim.x - g.copy_blocks) * COPY_THREADS;
  for (int64_t i = first; i < (int64_t)g.c.n_seqs * g.c.max_pages; i += step) {
    const int p = g.c.table[i];
    int to = -1;
    if (p >= 0) {
      if (p < g.c.n_pages) to = g.x.place[p];
      if (to < 0) atomicOr(g.c.status, SI_CACHE_BAD_PAGE);
    }
    g.to.table[i] = to;
  }
  for (int64_t i = first; i < g.c.n_seqs; i += step) g.to.lens[i] = g.c.lens[i];
  // in place: the count of a page that moves is read before it becomes 0, by the same thread; it moves to a hole, which no other reads
  for (int64_t i = first; i < max(g.c.n_pages, g.to.n_pages); i += step) {
    if (i < g.c.n_pages && g.x.place[i] >= 0) g.to.refs[g.x.place[i]] = g.c.refs[i];
    if (i >= used && i < g.to.n_pages) g.to.refs[i] = 0;
  }
}

bool misaligned(const void* p, int to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

int check_moves(const si_cache_t* c, const char* who) {
  if (int rc = check_cache(c, who)) return rc;
  if (!c->refs || !c->scratch) return set_error(SI_EINVAL, "%s: refs or scratch of the cache is NULL", who);
  if (misaligned(c->scratch, 16)) return set_error(SI_EINVAL, "%s: scratch is not aligned to 16 bytes", who);
  return SI_OK;
}
int check_list(const int32_t* a, const int32_t* b, bool both, int n, const char* who) {
  if (n < 0 || n > SI_CACHE_MAX_LIST) return set_error(SI_EINVAL, "%s: n %d outside 0 .. %d", who, n, SI_CACHE_MAX_LIST);
  if (n > 0 && (!a || (both && !b))) return set_error(SI_EINVAL, "%s: a list is NULL", who);
  if (misaligned(a, 4) || misaligned(b, 4)) return set_error(SI_EINVAL, "%s: a list is not aligned to 4 bytes", who);
  return SI_OK;
}
int done(const char* who) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SI_OK : set_error(SI_EHIP, "%s: launch failed: %s", who, hipGetErrorString(e));
}
int64_t page_bytes(const si_cache_t& c) { return kv_page_elems(c) * kv_elem_bytes(c.type); }
int parts_of(const si_cache_t& c) { return (int)((page_bytes(c) + COPY_BYTES - 1) / COPY_BYTES); }

// Blocks of a launch that may copy a page for each of n entries: a compute unit each, unless the pages are small
int copy_blocks(const si_cache_t& c, int n) { return (int)std::max<int64_t>(1, std::min<int64_t>(256, (int64_t)n * parts_of(c))); }

}  // namespace
}  // namespace si

using namespace si;

extern "C" int64_t si_cache_scratch_bytes(const si_cache_t* c) {
  if (!c || c->n_seqs < 1 || c->n_pages < 1) return set_error(SI_EINVAL, "si_cache_scratch_bytes: no descriptor, or bad n_seqs or n_pages");
  return scratch_bytes(*c);
}

extern "C" int si_cache_trim(const si_cache_t* c, const int32_t* seqs, int32_t n, const int32_t* keep, void* stream) {
  const char* who = "si_cache_trim";
  if (int rc = check_moves(c, who)) return rc;
  if (int rc = check_list(seqs, keep, false, n, who)) return rc;
  if (n == 0) return SI_OK;
  hipLaunchKernelGGL(k_trim, dim3(n), dim3(WAVE), 0, (hipStream_t)stream, *c, seqs, n, keep);
  return done(who);
}

extern "C" int si_cache_extend(const si_cache_t* c, const int32_t* seqs, int32_t n, const int32_t* counts, int32_t n_new, int32_t* seq_out, int32_t* pos_out,
                               int32_t capacity, void* stream) {
  const char* who = "si_cache_extend";
  if (int rc = check_moves(c, who)) return rc;
  if (int rc = check_list(seqs, counts, false, n, who)) return rc;
  if (!counts && n_new < 0) return set_error(SI_EINVAL, "%s: n_new %d", who, n_new);
  if ((seq_out == nullptr) != (pos_out == nullptr) || misaligned(seq_out, 4) || misaligned(pos_out, 4)) return set_error(SI_EINVAL, "%s: one of seq_out and pos_out is NULL, or misaligned", who);
  if (capacity < 0) return set_error(SI_EINVAL, "%s: capacity %d", who, capacity);
  if (n == 0) return SI_OK;
  ExtendArgs g{*c, scratch_of(*c), seqs, counts, seq_out, pos_out, n, n_new, capacity, parts_of(*c), page_bytes(*c)};
  hipLaunchKernelGGL(k_extend, dim3(std::min(64, copy_blocks(*c, n))), dim3(BOOK), 0, (hipStream_t)stream, g);
  return done(who);
}

extern "C" int si_cache_fork(const si_cache_t* c, const int32_t* parents, const int32_t* children, int32_t n, void* stream) {
  const char* who = "si_cache_fork";
  if (int rc = check_moves(c, who)) return rc;
  if (int rc = check_list(parents, children, true, n, who)) return rc;
  if (n == 0) return SI_OK;
  ForkArgs g{*c, scratch_of(*c), parents, children, n, parts_of(*c), page_bytes(*c)};
  hipLaunchKernelGGL(k_fork, dim3(copy_blocks(*c, n)), dim3(BOOK), 0, (hipStream_t)stream, g);
  return done(who);
}

extern "C" int si_cache_compact(const si_cache_t* c, const si_cache_t* to, int32_t* n_used, void* stream) {
  const char* who = "si_cache_compact";
  if (int rc = check_moves(c, who)) return rc;
  if (int rc = check_cache(to, who)) return rc;
  if (!to->refs || misaligned(n_used, 4)) return set_error(SI_EINVAL, "%s: refs of the target is NULL, or n_used not aligned", who);
  if (to->page_tokens != c->page_tokens || to->n_layers != c->n_layers || to->n_kv_heads != c->n_kv_heads || to->head_dim != c->head_dim || to->type != c->type ||
      to->n_seqs != c->n_seqs || to->max_pages != c->max_pages)
    return set_error(SI_EINVAL, "%s: the target has another shape", who);
  CompactArgs g{*c, *to, scratch_of(*c), parts_of(*c), 0};
  g.copy_blocks = (int64_t)c->n_pages * g.parts;
  const int64_t entries = std::max<int64_t>((int64_t)c->n_seqs * c->max_pages, std::max(c->n_pages, to->n_pages));
  const int64_t blocks = g.copy_blocks + std::min<int64_t>(1024, (entries + COPY_THREADS - 1) / COPY_THREADS);
  if (blocks >= (1 << 24)) return set_error(SI_EINVAL, "%s: a pool of %lld pieces of %d bytes is too large for one call", who, (long long)g.copy_blocks, COPY_BYTES);
  hipLaunchKernelGGL(k_places, dim3(1), dim3(BOOK), 0, (hipStream_t)stream, *c, g.x, to->n_pages, n_used);
  if (int rc = done(who)) return rc;
  hipLaunchKernelGGL(k_compact, dim3((unsigned)blocks), dim3(COPY_THREADS), 0, (hipStream_t)stream, g);
  return done(who);
}
