// Attention over the paged cache: arguments, and how a call is cut into blocks.
#include "si_internal.h"
#include "si_error.h"
#include "attend_device.h"

#include <algorithm>
#include <cmath>

namespace si {
namespace {

constexpr int64_t ATTEND_BLOCKS = 1 << 24;  // (a launch has fewer than 2^32 threads)

struct Cut {
  int block_rows, groups, slices, whole, part_rows, last_joins;
  int64_t scratch, part_at;
};

// Rows of a block, row groups, and the slices that a kv head's cache blocks are cut into.
Cut cut(const si_cache_t& c, const si_attend_t& a) {
  Cut k{};
  const int rows = a.n_new * (a.n_heads / c.n_kv_heads), B = kv_block(c.type);
  int64_t seen = a.max_len;
  if (a.window) seen = std::min<int64_t>(seen, (int64_t)a.window + a.n_new - 1 + B);
  const int64_t each = std::max<int64_t>(1, (seen + B - 1) / B);
  // Blocks of 128 rows read the cache once where two of 64 read it twice (96 rows over 16 x 8000 positions 182 us in blocks of 64, 168 of 128; 640 over
  // 16 x 4000 487 and 443), but short sequences are not bound by that, and with longer heads 32 rows a wave do not fit the registers (e4m3,
  // heads of 128, which also converts its codes there: the first case 153 and 161 us, 160 rows over 16 x 4000 138 and 183).
  const int most_rows = c.head_dim <= attend_wide_dim(c.type) && each > 20 ? 128 : 64;
  for (k.block_rows = 16; k.block_rows < rows && k.block_rows < most_rows;) k.block_rows *= 2;
  k.groups = (rows + k.block_rows - 1) / k.block_rows;
  k.part_rows = std::min(rows, k.block_rows);
  const int64_t units = (int64_t)c.n_kv_heads * k.groups;
  // As many blocks as there are compute units; twice that where a slice holds several sequences (the next one's first loads have nothing beside
  // them: 512 sequences of 64 positions 57 -> 38 us) or the waves of a block share their loads and wait for each other (40 rows over
  // 16 x 8000 positions 119 -> 106 us) and two blocks fit a unit.  Else it is one more round of sums to write and read (131071 positions 86
  // against 88 us).  No slice has fewer than two cache blocks a wave.
  const bool twice = c.head_dim <= 128 && (k.block_rows > 16 || a.n * units > 256);
  const int most = twice ? 512 : 256, streams = std::max(1, 64 / k.block_rows);
  // Short sequences have a block each, without a search and without joining.  How short goes by the turns that a wave then takes and by the
  // number of these blocks: few leave most of the chip idle, many even out by themselves.  8 kv heads, us in slices and whole:
  //   up to 16 rows      1 x 640 (5 turns) 9.0, 8.5;  1 x 900 (8) 9.1, 10.5;  8 x 768 (6) 12.3, 12.3;  8 x 1536 (12) 16.3, 19.9;  32 x 1 .. 2560 (20) 35.7, 35.7;
  //                      64 x 1 .. 3584 (28) 80.8, 89.1
  //   more, whose sums   1 x 300 (20 rows, 5 turns) 13.1, 11.7;  1 x 300 (48 rows, 10) 13.3, 16.5;  4 x 1 .. 512 (20 rows, 8) 22.4, 15.2;  8 x 768 (20 rows, 12) 18.5, 19.8;  8 x 1 .. 512 (48 rows, 16) 21.1, 22.0;
  //   are longer         16 x 1 .. 1792 (20 rows, 28) 36.1, 35.8;  32 x 1280 (48 rows, 40) 52.5, 46.0;  64 x 1 .. 640 (48 rows, 20) 59.4, 33.7
  const int64_t turns = (each + streams - 1) / streams, blocks = a.n * units;
  k.whole = turns <= (k.block_rows > 16 ? std::min<int64_t>(5 + blocks / 8, 40) : std::clamp<int64_t>(blocks / 8, 5, 20));
  // So have so many sequences that a launch could not hold a joining block for each of their rows.
  if (most / units > 1 && blocks * k.part_rows >= ATTEND_BLOCKS) k.whole = 1;
  const int64_t useful = (a.n * each + 2 * streams - 1) / (2 * streams);
  k.slices = k.whole ? std::max(1, a.n) : (int)std::max<int64_t>(1, std::min(most / units, useful));
  const int64_t join_bytes = (k.slices / std::max(1, a.n) + 1) * k.part_rows * (c.head_dim + 2) * 4ll;
  k.last_joins = !k.whole && k.slices > 1 && join_bytes <= 64 * 1024 && blocks <= ATTEND_COUNTERS;
  // Room for as many slices as any call of no more or longer sequences takes, in blocks of up to 64 rows too
  for (int block_rows = std::min(64, k.block_rows); block_rows <= k.block_rows; block_rows *= 2) {
    const int64_t block_units = (int64_t)c.n_kv_heads * ((rows + block_rows - 1) / block_rows), room = std::min((c.head_dim <= 128 ? 512 : 256) / block_units, useful);
    const int64_t part_at = ATTEND_COUNTERS * 4 + (a.n * block_units * 8 + 15) / 16 * 16;
    if (room > 1) k.scratch = std::max(k.scratch, part_at + block_units * room * 2 * std::min(rows, block_rows) * (c.head_dim + 2) * 4);
    if (block_rows == k.block_rows) k.part_at = part_at;
  }
  return k;
}

bool misaligned(const void* p, int to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

int check_shape(const si_cache_t* c, const si_attend_t* a, const char* who) {
  if (int rc = check_cache(c, who)) return rc;
  if (!a) return set_error(SI_EINVAL, "%s: descriptor is NULL", who);
  if (a->n < 0 || a->n > 65535) return set_error(SI_EINVAL, "%s: n %d outside 0 .. 65535", who, a->n);
  if (a->n_new < 1 || a->n_new > 65536) return set_error(SI_EINVAL, "%s: n_new %d outside 1 .. 65536", who, a->n_new);
  if (a->n_heads < 1 || a->n_heads > 4096 || a->n_heads % c->n_kv_heads != 0)
    return set_error(SI_EINVAL, "%s: n_heads %d is not a multiple of n_kv_heads %d", who, a->n_heads, c->n_kv_heads);
  if (a->window < 0 || a->max_len < 0) return set_error(SI_EINVAL, "%s: window %d or max_len %d is negative", who, a->window, a->max_len);
  if (!std::isfinite(a->scale)) return set_error(SI_EINVAL, "%s: scale is not finite", who);
  // (at most so many blocks, in cut() of up to 128 rows, have a slice for each sequence)
  const int64_t groups = ((int64_t)a->n_new * (a->n_heads / c->n_kv_heads) + 63) / 64;
  if (std::max(1, a->n) * c->n_kv_heads * groups >= ATTEND_BLOCKS)
    return set_error(SI_EINVAL, "%s: n * n_new * n_heads is too large for one call (%d, %d, %d)", who, a->n, a->n_new, a->n_heads);
  return SI_OK;
}

}  // namespace
}  // namespace si

extern "C" int64_t si_attend_scratch_bytes(const si_cache_t* c, const si_attend_t* a) {
  using namespace si;
  if (int rc = check_shape(c, a, "si_attend_scratch_bytes")) return rc;
  return cut(*c, *a).scratch;
}

extern "C" int si_attend(const si_cache_t* c, int32_t layer, const si_attend_t* a, void* stream) {
  using namespace si;
  const char* who = "si_attend";
  if (int rc = check_shape(c, a, who)) return rc;
  if (int rc = check_layer(c, layer, who)) return rc;
  if (a->n == 0) return SI_OK;  // (an empty tensor's address may be NULL)
  if (!a->q || !a->out) return set_error(SI_EINVAL, "%s: q or out is NULL", who);
  if (misaligned(a->q, 2) || misaligned(a->out, 2) || misaligned(a->lse, 4) || misaligned(a->seqs, 4)) return set_error(SI_EINVAL, "%s: a pointer is not aligned to its element", who);
  if (!a->seqs && a->n > c->n_seqs) return set_error(SI_EINVAL, "%s: n %d of %d sequences", who, a->n, c->n_seqs);
  const int64_t row = (int64_t)a->n_heads * c->head_dim;
  if (a->q_stride < row || a->out_stride < row) return set_error(SI_EINVAL, "%s: a stride is smaller than its row", who);
  const Cut k = cut(*c, *a);
  if (k.scratch > 0 && (!a->scratch || a->scratch_bytes < k.scratch || misaligned(a->scratch, 16)))
    return set_error(SI_EINVAL, "%s: %lld bytes of scratch needed, 16-byte aligned", who, (long long)k.scratch);
  AttendArgs g{*c, *a, layer, a->n_new * (a->n_heads / c->n_kv_heads), k.groups, k.block_rows, k.slices, k.whole, k.part_rows, k.last_joins, 0.f, nullptr, nullptr, nullptr};
  g.scale2 = (float)((a->scale == 0.f ? 1.0 / std::sqrt((double)c->head_dim) : (double)a->scale) * 1.4426950408889634);
  if (k.scratch > 0) {
    char* p = static_cast<char*>(a->scratch);
    g.count = reinterpret_cast<uint32_t*>(p);
    g.parted = reinterpret_cast<int2*>(p + ATTEND_COUNTERS * 4);
    g.part = reinterpret_cast<float*>(p + k.part_at);
  }
  const hipError_t e = (c->type == SI_KV_BF16 ? launch_attend_bf16 : launch_attend_e4m3)(g, (hipStream_t)stream);
  if (e != hipSuccess) return set_error(SI_EHIP, "attention launch failed: %s", hipGetErrorString(e));
  return SI_OK;
}
