// Attention for sequences that share leading pages: which they are, found on the device from the table, and the call's launches.
//
// Softmax splits over positions: with m, l, o of a row over the shared positions and over its own,
//   m' = max m,  l' = sum l 2^(m - m'),  o' = sum o 2^(m - m')
// so neighbours of the list whose tables begin with the same pages attend to these as rows of one sequence, which is read once for all of them and
// fills the matrix instructions, and each to what it alone has.  Launches: the plan, shared pages, own tokens (whose last step adds the
// sums over the shared ones), with a joining launch after either where parts are left.
#include "si_internal.h"
#include "si_error.h"
#include "attend_device.h"

#include <algorithm>

namespace si {
namespace {

constexpr int THREADS = 256, WAVES = THREADS / 64;

struct PlanArgs {
  si_cache_t c;
  const int32_t* seqs;
  int n, n_new, per, window, block_rows;
  uint32_t* count;      // [1], 0 between calls
  int32_t* common;      // [n] full pages that an entry of the list has in common with the one before
  int32_t* first_of;    // [n] first entry of an entry's group
  int32_t* tokens_of;   // [n] of a group's first entry: tokens in its shared pages
  int32_t* n_shared;
  SharedRows* shared;
  int32_t* own_from;    // [n]
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
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64, e = blockIdx.x;
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
    const int mine = tokens > 0 ? (rows + g.block_rows - 1) / g.block_rows : 0;
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
    if (in) g.first_of[i] = r.first;
    if (ends) {
      g.tokens_of[r.first] = tokens;
      for (int k = 0; k < mine; ++k)
        g.shared[at + k] = SharedRows{r.first, r.first * g.n_new * g.per + k * g.block_rows, min(g.block_rows, rows - k * g.block_rows), tokens,
                                      g.window ? max(0, r.shortest - g.n_new + 1 - g.window) : 0, g.window ? max(0, r.longest - g.window) : 0};
    }
    carry = next;
  }
  if (tid == 0) *g.n_shared = n_shared;
  __syncthreads();
  for (int i = tid; i < g.n; i += THREADS) g.own_from[i] = g.tokens_of[g.first_of[i]];
}

struct Layout {
  AttendCut own;
  int block_rows, slices, most;  // of the launch over shared pages; most: SharedRows
  int64_t parted, part, sums, n_shared, shared, own_from, common, first_of, tokens_of, bytes;
};

Layout lay_out(const si_cache_t& c, const si_attend_t& a) {
  Layout l{};
  l.own = cut_attend(c, a);
  const int64_t rows = (int64_t)a.n * a.n_new * (a.n_heads / c.n_kv_heads), each = (a.max_len + kv_block(c.type) - 1) / kv_block(c.type);
  const int wide = c.head_dim <= attend_wide_dim(c.type) ? 128 : 64;
  int most_rows = 16;  // (whatever max_len is)
  while (most_rows < rows && most_rows < wide) most_rows *= 2;
  l.block_rows = each > 20 ? most_rows : std::min(most_rows, 64);
  l.slices = std::max(1, (c.head_dim <= 128 ? 512 : 256) / c.n_kv_heads);
  l.most = (int)(rows / l.block_rows + a.n / 2 + 1);
  const int64_t most = rows / 16 + a.n / 2 + 1;
  int64_t at = std::max<int64_t>(l.own.scratch, ATTEND_COUNTERS * 4);  // (the counters are at the same place in every call's scratch)
  auto take = [&](int64_t bytes) {
    const int64_t q = (at + 15) / 16 * 16;
    at = q + bytes;
    return q;
  };
  l.parted = take(most * c.n_kv_heads * 8);
  l.part = take(l.slices > 1 ? (int64_t)c.n_kv_heads * l.slices * 2 * most_rows * (c.head_dim + 2) * 4 : 0);
  l.sums = take(c.n_kv_heads * rows * (c.head_dim + 4) * 4);
  l.n_shared = take(4);
  l.shared = take(most * (int64_t)sizeof(SharedRows));
  l.own_from = take(a.n * 4ll);
  l.common = take(a.n * 4ll);
  l.first_of = take(a.n * 4ll);
  l.tokens_of = take(a.n * 4ll);
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
  AttendArgs own = attend_args(*c, *a, layer, l.own);
  own.shared_sums = reinterpret_cast<float*>(p + l.sums);
  own.n_shared = reinterpret_cast<int32_t*>(p + l.n_shared);
  own.shared = reinterpret_cast<SharedRows*>(p + l.shared);
  own.own_from = reinterpret_cast<int32_t*>(p + l.own_from);
  AttendArgs shared = own;
  shared.rows = shared.block_rows = shared.part_rows = l.block_rows;
  shared.groups = 1;
  shared.slices = l.slices;
  shared.whole = shared.last_joins = 0;
  shared.joins = std::min(l.most, 8);
  shared.count = reinterpret_cast<uint32_t*>(p);
  shared.parted = reinterpret_cast<int2*>(p + l.parted);
  shared.part = reinterpret_cast<float*>(p + l.part);
  PlanArgs plan{*c, a->seqs, a->n, a->n_new, a->n_heads / c->n_kv_heads, a->window, l.block_rows, reinterpret_cast<uint32_t*>(p),
                reinterpret_cast<int32_t*>(p + l.common), reinterpret_cast<int32_t*>(p + l.first_of), reinterpret_cast<int32_t*>(p + l.tokens_of),
                reinterpret_cast<int32_t*>(p + l.n_shared), reinterpret_cast<SharedRows*>(p + l.shared), reinterpret_cast<int32_t*>(p + l.own_from)};
  hipLaunchKernelGGL(k_share, dim3(a->n), dim3(THREADS), 0, (hipStream_t)stream, plan);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess) e = (c->type == SI_KV_BF16 ? launch_attend_shared_bf16 : launch_attend_shared_e4m3)(shared, own, (hipStream_t)stream);
  if (e != hipSuccess) return set_error(SI_EHIP, "attention launch failed: %s", hipGetErrorString(e));
  return SI_OK;
}
