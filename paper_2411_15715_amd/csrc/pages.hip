// Moves of the cache's pages.  The tables are small and every decision (which page is free, who shares what) depends on all of them, so one
// block makes it, with prefix sums instead of counters, and later launches copy what it has listed.
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
struct Head { int32_t groups, used, pad[14]; };
struct Group { int32_t src, first, count, pad; };  // one page that is copied, to dst[first] .. dst[first + count - 1]
struct Scratch {
  Head* head;
  int32_t* mark;   // [n_seqs] 1: named by the running call; 0 between calls
  Group* group;    // [SI_CACHE_MAX_LIST]
  int32_t* dst;    // [SI_CACHE_MAX_LIST]
  int32_t* list;   // [n_pages] free pages; pages that move: holes
  int32_t* place;  // [n_pages] new number of a page
};
__host__ __device__ inline int64_t round16(int64_t x) { return (x + 15) / 16 * 16; }
int64_t scratch_bytes(const si_cache_t& c) {
  return sizeof(Head) + round16(4ll * c.n_seqs) + SI_CACHE_MAX_LIST * (sizeof(Group) + 4) + 2 * round16(4ll * c.n_pages);
}
Scratch scratch_of(const si_cache_t& c) {
  char* p = static_cast<char*>(c.scratch);
  Scratch s;
  s.head = reinterpret_cast<Head*>(p); p += sizeof(Head);
  s.mark = reinterpret_cast<int32_t*>(p); p += round16(4ll * c.n_seqs);
  s.group = reinterpret_cast<Group*>(p); p += SI_CACHE_MAX_LIST * sizeof(Group);
  s.dst = reinterpret_cast<int32_t*>(p); p += SI_CACHE_MAX_LIST * 4;
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

// The first `need` free pages into `list`; returns how many there are, counted up to at least `need`
__device__ int list_free(const si_cache_t& c, int need, int32_t* list, int (&w)[WAVES]) {
  int found = 0;
  for (int at0 = 0; at0 < c.n_pages && found < need; at0 += BOOK * PER_THREAD) {
    const int at = at0 + threadIdx.x * PER_THREAD;
    int bits = at < c.n_pages ? free_bits(c.refs, c.n_pages, at) : 0, total;
    int rank = found + block_scan(__popc(bits), total, w);
    for (; bits && rank < need; bits &= bits - 1, ++rank) list[rank] = at + __ffs(bits) - 1;
    found += total;
  }
  return found;
}

// largest e < n with prefix[e] <= f, entries that add nothing passed over (prefix[n] > f)
__device__ __forceinline__ int entry_of(const int* prefix, int n, int f) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (prefix[mid] <= f) lo = mid;
    else hi = mid;
  }
  return lo;
}

constexpr int LIST = SI_CACHE_MAX_LIST;
struct BookLds {
  int w[WAVES];
  int seq[LIST], len[LIST];
  int src[LIST];          // page that is copied for the entry, or -1
  int need[LIST + 1];     // prefix sums: pages taken
  int put[LIST + 1];      // tokens added (extend), pages named (fork)
  int first[LIST];
  int why;
};

// exclusive prefix sums of v[0 .. n) in place, v[n] = total; false (and v left as it may be) where a sum passes `most`
__device__ bool prefix_list(int* v, int n, int most, int (&w)[WAVES]) {
  int64_t carry = 0;
  for (int e0 = 0; e0 < n; e0 += BOOK) {
    const int e = e0 + threadIdx.x, x = e < n ? v[e] : 0;
    // (every entry is at most `most`: cut so that a sum over the block stays in 31 bits, and look at the sum in 64)
    int hi_total, lo_total;
    const int hi = block_scan(x >> 12, hi_total, w), lo = block_scan(x & 0xfff, lo_total, w);
    const int64_t at = carry + ((int64_t)hi << 12) + lo;
    carry += ((int64_t)hi_total << 12) + lo_total;
    if (carry > most) return false;
    __syncthreads();
    if (e < n) v[e] = (int)at;
  }
  if (threadIdx.x == 0) v[n] = (int)carry;
  __syncthreads();
  return true;
}

// Entries with the same source next to each other, so that a source is read once: s.src[e] is copied to the page that `dst(e)` names.
template <class F> __device__ void list_copies(BookLds& s, int n, const Scratch& x, F dst) {
  for (int e = threadIdx.x; e < n; e += BOOK) {
    int f = e;
    if (s.src[e] >= 0)
      for (f = 0; s.src[f] != s.src[e]; ++f) {}
    s.first[e] = s.src[e] >= 0 ? f : -1;
  }
  __syncthreads();
  for (int e = threadIdx.x; e < n; e += BOOK) {
    const int mine = s.first[e];
    if (mine < 0) continue;
    int before = 0, rank = 0, count = 0, groups_before = 0;
    for (int i = 0; i < n; ++i) {
      const int f = s.first[i];
      before += f >= 0 && f < mine;
      groups_before += f == i && f < mine;
      count += f == mine;
      rank += f == mine && i < e;
    }
    x.dst[before + rank] = dst(e);
    if (mine == e) x.group[groups_before] = Group{s.src[e], before, count, 0};
  }
  // the number of groups
  int groups = 0, total = 0;
  for (int e0 = 0; e0 < n; e0 += BOOK) {
    const int e = e0 + threadIdx.x;
    block_scan(e < n && s.first[e] == e, total, s.w);
    groups += total;
  }
  if (threadIdx.x == 0) x.head->groups = groups;
}

__global__ __launch_bounds__(WAVE) void k_trim(si_cache_t c, const int32_t* __restrict__ seqs, const int32_t* __restrict__ keep) {
  const int seq = seqs[blockIdx.x], lane = threadIdx.x, to = keep ? keep[blockIdx.x] : 0;
  if (seq < 0 || seq >= c.n_seqs || to < 0) {
    if (lane == 0) atomicOr(c.status, to < 0 ? SI_CACHE_BAD_LEN : SI_CACHE_BAD_SEQ);
    return;
  }
  // (an exchange, so that a sequence named twice loses its pages once)
  int old = lane == 0 ? atomicMin(c.lens + seq, to) : 0;
  old = __builtin_amdgcn_readfirstlane(old);
  int why = old < to ? SI_CACHE_BAD_LEN : 0;
  const int most = c.max_pages * c.page_tokens;
  if (old > most) { old = most; why = SI_CACHE_BAD_LEN; }
  int32_t* row = c.table + (int64_t)seq * c.max_pages;
  for (int j = ceil_div(min(to, most), c.page_tokens) + lane; j < ceil_div(max(old, 0), c.page_tokens); j += WAVE) {
    const int page = row[j];
    row[j] = -1;
    if (page < 0 || page >= c.n_pages) {
      why |= SI_CACHE_BAD_PAGE;
    } else if (atomicSub(c.refs + page, 1) <= 0) {
      atomicAdd(c.refs + page, 1);
      why |= SI_CACHE_BAD_PAGE;
    }
  }
  if (why) atomicOr(c.status, why);
}

struct ExtendArgs {
  si_cache_t c;
  Scratch x;
  const int32_t *seqs, *counts;
  int32_t *seq_out, *pos_out;
  int n, n_new, capacity;
};

__global__ __launch_bounds__(BOOK) void k_extend(ExtendArgs g) {
  __shared__ BookLds s;
  const si_cache_t& c = g.c;
  const int tid = threadIdx.x, page = c.page_tokens;
  if (tid == 0) { s.why = 0; g.x.head->groups = 0; }
  __syncthreads();
  int why = 0;
  for (int e = tid; e < g.n; e += BOOK) {
    const int seq = g.seqs[e], m = g.counts ? g.counts[e] : g.n_new;
    int len = 0, need = 0, src = -1;
    if (seq < 0 || seq >= c.n_seqs) {
      why |= SI_CACHE_BAD_SEQ;
    } else {
      if (atomicExch(g.x.mark + seq, 1) != 0) why |= SI_CACHE_BAD_SEQ;
      len = c.lens[seq];
      if (len < 0 || m < 0 || (int64_t)len + m > (int64_t)c.max_pages * page) {
        why |= SI_CACHE_BAD_LEN;
      } else {
        need = ceil_div(len + m, page) - ceil_div(len, page);
        if (m > 0 && len % page > 0) {
          const int last = c.table[(int64_t)seq * c.max_pages + len / page];
          if (last < 0 || last >= c.n_pages) why |= SI_CACHE_BAD_PAGE;
          else if (c.refs[last] > 1) src = last;
        }
      }
    }
    s.seq[e] = seq; s.len[e] = len; s.need[e] = need; s.put[e] = max(m, 0); s.src[e] = src;
  }
  if (why) atomicOr(&s.why, why);
  __syncthreads();
  // a shared last page: whoever comes after all of its other sharers keeps it
  for (int e = tid; e < g.n; e += BOOK) {
    const int src = s.src[e];
    int before = 0;
    if (src >= 0) {
      for (int i = 0; i < e; ++i) before += s.src[i] == src;
    }
    s.first[e] = src >= 0 && before < c.refs[src] - 1;
  }
  __syncthreads();
  for (int e = tid; e < g.n; e += BOOK) {
    if (s.first[e]) s.need[e] += 1;
    else s.src[e] = -1;
  }
  __syncthreads();
  bool ok = s.why == 0;
  int tokens = 0, pages = 0;
  if (ok && !prefix_list(s.put, g.n, 0x7fffffff, s.w)) { ok = false; why = SI_CACHE_NO_ROOM; }
  if (ok && !prefix_list(s.need, g.n, 0x7fffffff, s.w)) { ok = false; why = SI_CACHE_NO_PAGES; }
  if (ok) {
    tokens = s.put[g.n];
    pages = s.need[g.n];
    if (g.seq_out && tokens > g.capacity) { ok = false; why = SI_CACHE_NO_ROOM; }
    else if (pages > 0 && list_free(c, pages, g.x.list, s.w) < pages) { ok = false; why = SI_CACHE_NO_PAGES; }
  }
  __syncthreads();
  if (ok) {
    for (int f = tid; f < pages; f += BOOK) {
      const int e = entry_of(s.need, g.n, f), k = f - s.need[e], p = g.x.list[f];
      const int j = s.src[e] >= 0 ? s.len[e] / page + k : ceil_div(s.len[e], page) + k;
      c.table[(int64_t)s.seq[e] * c.max_pages + j] = p;
      c.refs[p] = 1;
      if (s.src[e] >= 0 && k == 0) atomicSub(c.refs + s.src[e], 1);
    }
    for (int e = tid; e < g.n; e += BOOK) c.lens[s.seq[e]] = s.len[e] + s.put[e + 1] - s.put[e];
    list_copies(s, g.n, g.x, [&](int e) { return g.x.list[s.need[e]]; });
  } else if (tid == 0) {
    atomicOr(c.status, why | s.why);
  }
  for (int e = tid; e < g.n; e += BOOK)
    if (s.seq[e] >= 0 && s.seq[e] < c.n_seqs) g.x.mark[s.seq[e]] = 0;
  if (g.seq_out)
    for (int f = tid; f < g.capacity; f += BOOK) {
      int seq = -1, pos = -1;
      if (f < tokens && ok) {
        const int e = g.counts ? entry_of(s.put, g.n, f) : f / g.n_new;
        seq = s.seq[e];
        pos = s.len[e] + f - s.put[e];
      }
      g.seq_out[f] = seq;
      g.pos_out[f] = pos;
    }
}

struct ForkArgs {
  si_cache_t c;
  Scratch x;
  const int32_t *parents, *children;
  int n;
};

__global__ __launch_bounds__(BOOK) void k_fork(ForkArgs g) {
  __shared__ BookLds s;  // seq: child, len: parent's, put: pages of the parent
  const si_cache_t& c = g.c;
  const int tid = threadIdx.x, page = c.page_tokens;
  if (tid == 0) { s.why = 0; g.x.head->groups = 0; }
  __syncthreads();
  int why = 0;
  for (int e = tid; e < g.n; e += BOOK) {
    const int a = g.parents[e], b = g.children[e];
    if (a < 0 || a >= c.n_seqs || b < 0 || b >= c.n_seqs || atomicExch(g.x.mark + b, 1) != 0) why = SI_CACHE_BAD_SEQ;
    s.seq[e] = b; s.first[e] = a;
  }
  if (why) atomicOr(&s.why, why);
  __syncthreads();
  // Sequence numbers, then lengths: each is looked at only where what came before is in order, which is the same for all threads
  auto step = [&](auto&& look) {
    const bool go_on = s.why == 0;
    why = 0;
    if (go_on)
      for (int e = tid; e < g.n; e += BOOK) look(e);
    __syncthreads();
    if (why) atomicOr(&s.why, why);
    __syncthreads();
  };
  step([&](int e) {
    if (__hip_atomic_load(g.x.mark + s.first[e], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != 0) why |= SI_CACHE_BAD_SEQ;  // a parent that is a child
  });
  step([&](int e) {
    int len = c.lens[s.first[e]];
    if (c.lens[s.seq[e]] != 0 || len < 0 || len > c.max_pages * page) { why |= SI_CACHE_BAD_LEN; len = 0; }
    s.len[e] = len; s.put[e] = ceil_div(len, page); s.need[e] = len % page > 0; s.src[e] = -1;
  });
  bool ok = s.why == 0;
  int pages = 0, named = 0;
  if (ok && !(prefix_list(s.put, g.n, 0x7fffffff, s.w) && prefix_list(s.need, g.n, 0x7fffffff, s.w))) { ok = false; why = SI_CACHE_NO_PAGES; }
  if (ok) {
    named = s.put[g.n];
    pages = s.need[g.n];
    why = 0;
    for (int f = tid; f < named; f += BOOK) {
      const int e = entry_of(s.put, g.n, f), j = f - s.put[e], p = c.table[(int64_t)s.first[e] * c.max_pages + j];
      if (p < 0 || p >= c.n_pages) why |= SI_CACHE_BAD_PAGE;
      else if (j == s.len[e] / page) s.src[e] = p;
    }
    if (why) atomicOr(&s.why, why);
    __syncthreads();
    ok = s.why == 0;
    if (ok && pages > 0 && list_free(c, pages, g.x.list, s.w) < pages) { ok = false; why = SI_CACHE_NO_PAGES; }
  }
  __syncthreads();
  if (ok) {
    for (int f = tid; f < named; f += BOOK) {
      const int e = entry_of(s.put, g.n, f), j = f - s.put[e];
      int p;
      if (j == s.len[e] / page) {
        p = g.x.list[s.need[e]];
        c.refs[p] = 1;
      } else {
        p = c.table[(int64_t)s.first[e] * c.max_pages + j];
        atomicAdd(c.refs + p, 1);
      }
      c.table[(int64_t)s.seq[e] * c.max_pages + j] = p;
    }
    for (int e = tid; e < g.n; e += BOOK) c.lens[s.seq[e]] = s.len[e];
    __syncthreads();  // (first[] is used anew)
    list_copies(s, g.n, g.x, [&](int e) { return g.x.list[s.need[e]]; });
  } else if (tid == 0) {
    atomicOr(c.status, why | s.why);
  }
  __syncthreads();
  for (int e = tid; e < g.n; e += BOOK)
    if (s.seq[e] >= 0 && s.seq[e] < c.n_seqs) g.x.mark[s.seq[e]] = 0;
}

// bytes [at, end) of one page to `count` others; `dst(i)` is the first byte of the i-th
template <class F> __device__ __forceinline__ void copy_run(const char* src, int64_t at, int64_t end, int count, F dst) {
  constexpr int STEP = COPY_THREADS * 16, N = 4;
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

// grid: parts of a page x groups (any number of blocks along them)
__global__ __launch_bounds__(COPY_THREADS) void k_copy_groups(char* pages, int64_t page_bytes, Scratch x) {
  const int64_t at = (int64_t)blockIdx.x * COPY_BYTES, end = min(page_bytes, at + COPY_BYTES);
  for (int i = blockIdx.y; i < x.head->groups; i += gridDim.y) {
    const Group q = x.group[i];
    copy_run(pages + q.src * page_bytes, at, end, q.count, [&](int k) { return pages + x.dst[q.first + k] * page_bytes; });
  }
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
    copy_run(static_cast<const char*>(g.c.pages) + p * page_bytes, at, min(page_bytes, at + COPY_BYTES), 1, [&](int) { return to; });
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

void copy_groups(const si_cache_t& c, const Scratch& x, int n, hipStream_t stream) {
  const int parts = parts_of(c);
  hipLaunchKernelGGL(k_copy_groups, dim3(parts, std::max(1, std::min(n, 4096 / std::min(parts, 4096)))), dim3(COPY_THREADS), 0, stream, static_cast<char*>(c.pages), page_bytes(c), x);
}

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
  hipLaunchKernelGGL(k_trim, dim3(n), dim3(WAVE), 0, (hipStream_t)stream, *c, seqs, keep);
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
  ExtendArgs g{*c, scratch_of(*c), seqs, counts, seq_out, pos_out, n, n_new, capacity};
  hipLaunchKernelGGL(k_extend, dim3(1), dim3(BOOK), 0, (hipStream_t)stream, g);
  if (int rc = done(who)) return rc;
  copy_groups(*c, g.x, n, (hipStream_t)stream);
  return done(who);
}

extern "C" int si_cache_fork(const si_cache_t* c, const int32_t* parents, const int32_t* children, int32_t n, void* stream) {
  const char* who = "si_cache_fork";
  if (int rc = check_moves(c, who)) return rc;
  if (int rc = check_list(parents, children, true, n, who)) return rc;
  if (n == 0) return SI_OK;
  ForkArgs g{*c, scratch_of(*c), parents, children, n};
  hipLaunchKernelGGL(k_fork, dim3(1), dim3(BOOK), 0, (hipStream_t)stream, g);
  if (int rc = done(who)) return rc;
  copy_groups(*c, g.x, n, (hipStream_t)stream);
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
