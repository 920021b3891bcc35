/*
 * scheinfer_attention.h - the operators around the feed-forward layer in the generation phase, for one MI355X (gfx950): norms with
 * residual and gate, a paged key-value cache with the attention that reads it, and the moves of its pages.
 *
 * Between two feed-forward layers (scheinfer.h) a serving program calls, on one stream,
 *   si_norm          r' = res_scale r + y_scale gate * N1(y),  out = N2(r')
 *   (its own projection of out to q, k and v)
 *   si_cache_append  rotates q and k, writes k and v into the pages of the cache
 *   si_attend        the new tokens attend to the cache
 *   (its own output projection), si_norm again, then si_layer_forward
 * and, between steps, si_cache_extend / _trim / _fork / _compact.
 *
 * Conventions: those of scheinfer.h (codes, si_last_error, bf16 as bit patterns, stream as void*), and
 *  - every pointer inside the descriptors is a DEVICE address, aligned to its element; the descriptors themselves are HOST and are
 *    read during the call only;
 *  - a call with no rows, tokens, sequences or list entries is a no-op, and the addresses of what is empty may then be NULL;
 *  - no call allocates, copies to or from the host, or waits: every call can be recorded into a HIP graph, and acts on the
 *    descriptors' addresses and on the device's tables as they are when it runs.  Work runs on the current HIP device, which has to be
 *    the one that owns the memory and the stream;
 *  - what only the device can see (a page number outside the pool, a position beyond the table, too few free pages) is never followed:
 *    the call leaves that part out, as its description says, and sets bits of *status, which stay set until the caller clears them.
 */
#ifndef SCHEINFER_ATTENTION_H
#define SCHEINFER_ATTENTION_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* element types of dense operands */
#define SI_F32 0
#define SI_BF16 1

#define SI_NORM_NONE 0 /* N(x) = x */
#define SI_NORM_RMS 1  /* N(x) = x / sqrt(mean(x^2) + eps) * w + b */
#define SI_NORM_MEAN 2 /* N(x) = z / sqrt(mean(z^2) + eps) * w + b,  z = x - mean(x) */
#define SI_NORM_MAX_D 32768

/*
 * One residual step of `rows` rows of d elements:
 *   r' = res_scale * r + y_scale * gate * N1(y)      (the terms whose pointer is NULL left out; gate NULL: 1)
 *   r_out = r',   out = N2(r')                        (either may be NULL, not both)
 * N2 reads r' as formed, not as rounded to r_out's type.  Sums, means and r' are fp32; every output is rounded once.
 * Strides are in elements, between the rows of an operand; an input's stride may be 0 (one row for all of them, e.g. a gate that
 * belongs to the layer), an output's at least d.  r_out and out may be r, y or gate themselves (same address, type and
 * stride; another type or stride there is refused); other overlaps are not allowed.
 * Errors: SI_EINVAL (NULL descriptor, neither r nor y, neither output, unknown type or kind, rows < 0, d outside 1 .. SI_NORM_MAX_D, a stride
 * as above, an address not aligned to its type, eps negative or not finite, post without y).  rows == 0 is a no-op.
 */
typedef struct {
  const void* r;      /* [rows][d] of r_type, or NULL */
  const void* y;      /* [rows][d] of y_type, or NULL */
  const void* gate;   /* [rows][d] of gate_type, or NULL */
  const void* w_post; /* [d] of w_type: weight of N1, NULL: 1 */
  const void* b_post; /* [d] of w_type: bias of N1, NULL: 0 */
  const void* w_pre;  /* the same of N2 */
  const void* b_pre;
  void* r_out;        /* [rows][d] of r_out_type, or NULL */
  void* out;          /* [rows][d] of out_type, or NULL */
  int64_t r_stride, y_stride, gate_stride, r_out_stride, out_stride;
  int32_t rows, d;
  int32_t r_type, y_type, gate_type, w_type, r_out_type, out_type; /* SI_F32 | SI_BF16 */
  int32_t post, pre;                                               /* N1, N2: SI_NORM_* */
  float eps, res_scale, y_scale;
} si_norm_t;
int si_norm(const si_norm_t* desc, void* stream);

/* ------------------------------------------------------------------------------------------------ the cache
 * Keys and values lie in pages of page_tokens tokens each; a page is one contiguous run over all layers, so that a page moves as one:
 *   pages [n_pages][n_layers][2: K, V][n_kv_heads][page_tokens / B blocks]
 * with E = 16 bytes / element size (8 bf16, 16 e4m3) and blocks of B = 4 E tokens, laid out as the matrix instructions take them:
 *   K block [head_dim / E][B slots][E]: elements E c .. E c + E - 1 of the token in a slot; token t of the block is in slot
 *                                       (t % E / 4) * 16 + 4 * (t / E) + t % 4
 *   V block [4][head_dim][E]:           tokens E g .. E g + E - 1 of an element
 * si_kv_offsets gives the place of one element.  A stored e4m3 code (OCP, 448 the largest) stands for code * scale of its head.
 *
 * table [n_seqs][max_pages]: page of each page_tokens tokens of a sequence, -1 where it has none; lens [n_seqs]; refs [n_pages]: how many
 * places of the table name the page, 0: it is free.  The page calls keep the three consistent; a program that starts with an empty
 * cache fills table with -1 and the others with 0.
 */
#define SI_KV_BF16 0
#define SI_KV_E4M3 1

/* bits of *status */
#define SI_CACHE_BAD_SEQ 1   /* a sequence number outside the table, or one that a call may not name (twice) */
#define SI_CACHE_BAD_LEN 2   /* a length or position that is negative, beyond the table, or more than there is */
#define SI_CACHE_BAD_PAGE 4  /* a page number outside the pool (or -1) where a page has to be, or a reference count of a page that does not fit */
#define SI_CACHE_NO_PAGES 8  /* more pages needed than are free */
#define SI_CACHE_NO_ROOM 16  /* more tokens than the output arrays hold */

typedef struct {
  void* pages;            /* the pool, 16-byte aligned */
  const float* scale_k;   /* [n_kv_heads], e4m3 only; NULL: 1 */
  const float* scale_v;
  int32_t* table;         /* [n_seqs][max_pages] */
  int32_t* lens;          /* [n_seqs] */
  int32_t* refs;          /* [n_pages]; may be NULL for si_cache_append and si_attend */
  int32_t* status;        /* [1] */
  void* scratch;          /* si_cache_scratch_bytes bytes, 16-byte aligned, zero before its first use; every call leaves it fit for the next:
                             the page calls only */
  int32_t n_pages;        /* >= 1 */
  int32_t page_tokens;    /* a multiple of B: 32 (bf16) or 64 (e4m3) */
  int32_t n_layers;
  int32_t n_kv_heads;
  int32_t head_dim;       /* bf16: 64, 96, 128, 192 or 256; e4m3: 64, 128, 192 or 256 */
  int32_t type;           /* SI_KV_* */
  int32_t n_seqs, max_pages;
} si_cache_t; /* limits: page_tokens and n_layers up to 65536, n_kv_heads up to 1024, max_pages * page_tokens up to 0x7fff0000 */

/* Element offsets inside a page, from its first: K and V of element `dim` of the token at position t_in_page (host, no GPU needed).
 * Errors: SI_EINVAL (bad descriptor, an index outside it). */
int si_kv_offsets(const si_cache_t* cache, int32_t layer, int32_t kv_head, int32_t t_in_page, int32_t dim, int64_t* k_offset, int64_t* v_offset);

/*
 * New tokens into the cache: for token i, with s = seq[i] and p = pos[i],
 *   q_out[i] = R(p) q[i],   K of (s, p) = R(p) k[i],   V of (s, p) = v[i]
 * R(p) turns the first rot_dim elements of every head by the angles p * inv_freq[j], j < rot_dim / 2, formed in 64 bits: elements j and
 * j + rot_dim / 2, or with rot_pairs elements 2 j and 2 j + 1, become (a cos - b sin, b cos + a sin).  The rest stays as it is.  Everything in
 * fp32, rounded once; e4m3: x / scale of the head, cut to +-448, rounded to nearest even (NaN stays NaN).
 * Nothing else of the cache changes: si_cache_extend has given the tokens their pages and counted them.
 * A token with seq -1 is left out (q_out is 0), so that a recorded graph may have more tokens than a step needs.  So is, with
 * a bit in *status, one whose sequence, position or page is not there.  Each element
 * of a place that two tokens of a call name is that of one of them, and neighbours need not be of the same (si_cache_extend names no place twice).
 * Strides are in elements between tokens, at least the row they stride (or 0 where there is one token); q, k and v may be slices of one
 * projection.  q == NULL: keys and values only.
 * Errors: SI_EINVAL (NULL or misaligned pointer: 2 bytes for rows, 4 for the others; rot_dim odd, negative or beyond head_dim; rot_dim without
 * inv_freq; n_heads not a multiple of n_kv_heads or above 4096; layer outside the cache; bad cache descriptor; more than 2^22 tokens, or more
 * than 2^33 elements of k, or about 2^38 of q and k (2^35 where rot_dim is no multiple of 16), in one call), SI_EHIP.  n_tokens == 0 is a no-op.
 */
typedef struct {
  const void* q;         /* bf16 [n_tokens][n_heads][head_dim], or NULL */
  const void* k;         /* bf16 [n_tokens][n_kv_heads][head_dim] */
  const void* v;
  void* q_out;           /* bf16 [n_tokens][n_heads][head_dim]; may be q, with its stride */
  const int32_t* seq;    /* [n_tokens] */
  const int32_t* pos;
  const float* inv_freq; /* [rot_dim / 2], NULL where rot_dim == 0 */
  int64_t q_stride, k_stride, v_stride, q_out_stride;
  int32_t n_tokens, n_heads, rot_dim, rot_pairs;
} si_append_t;
int si_cache_append(const si_cache_t* cache, int32_t layer, const si_append_t* desc, void* stream);

/*
 * Attention of the last n_new tokens of n sequences over the cache (they are in it: si_cache_append came before).  Row i * n_new + j of q
 * and out is token j of sequence seqs[i], at position lens - n_new + j; it sees the positions p with
 *   p <= lens - n_new + j,  and with window > 0 also  p > lens - n_new + j - window,
 * and for every head h, with kv head h / (n_heads / n_kv_heads):
 *   out = softmax over them of (scale q . K) applied to V,   lse = ln sum exp(scale q . K)
 * Made for a few new tokens over a long cache; whole prompts are taken too.
 * A token that sees nothing (its position is negative: lens < n_new) gets out 0 and lse -infinity, and so does a row all of whose scores are
 * -infinity; a row with a score of +infinity gets out NaN and lse +infinity.  What a token does not see has no part in
 * its output, whatever the pages hold there, NaN and infinities included.  Products are of bf16 operands (e4m3 codes widen to bf16
 * exactly); sums and maxima are fp32, a weight is multiplied as the sum of two bf16 values, 2^-16 of it lost.
 * max_len sizes the launch: an upper bound of lens (a sequence beyond it is still computed, by fewer blocks than it deserves).
 * scratch: si_attend_scratch_bytes of these descriptors or more, 16-byte aligned, zero before its first use; every call leaves it fit for
 * any other call.  Two calls that may run at once need one each.  Results do not depend on the order in which blocks run.
 * Left out with a bit in *status: a sequence outside the table (as if its length were 0), a length that is negative or
 * beyond the table (cut to it), a page outside the pool (its tokens are not seen).
 * Errors: SI_EINVAL (NULL or misaligned pointer: 2 bytes for q and out, 4 for lse and seqs; n_heads not a multiple of n_kv_heads or above 4096;
 * a stride smaller than its row; n negative, above 65535, or above n_seqs without seqs; n_new < 1 or above 65536; n * n_kv_heads *
 * ceil(n_new * n_heads / n_kv_heads / 64) of 2^24 or more; window or max_len negative; scale not finite; scratch_bytes too small; layer outside the
 * cache; bad cache descriptor), SI_EHIP.  n == 0 is a no-op.
 */
typedef struct {
  const void* q;        /* bf16 [n * n_new][n_heads][head_dim] */
  void* out;            /* bf16, the same shape */
  float* lse;           /* [n * n_new][n_heads], or NULL */
  const int32_t* seqs;  /* [n], or NULL: sequences 0 .. n - 1 */
  void* scratch;
  int64_t scratch_bytes;
  int64_t q_stride, out_stride; /* elements between rows */
  int32_t n, n_new, n_heads;
  int32_t window;       /* 0: all */
  int32_t max_len;
  float scale;          /* 0: 1 / sqrt(head_dim) */
} si_attend_t;
int si_attend(const si_cache_t* cache, int32_t layer, const si_attend_t* desc, void* stream);

/* Bytes of scratch that si_attend needs for these descriptors, and for any with a smaller n or max_len; or a negative SI_E* code (host only, no
 * GPU needed; q, out, lse, scratch and scratch_bytes are not looked at). */
int64_t si_attend_scratch_bytes(const si_cache_t* cache, const si_attend_t* desc);

/* ------------------------------------------------------------------------------------------------ moves of pages
 * All act on every layer at once.  `seqs` and the like are DEVICE int32 [n], n <= SI_CACHE_MAX_LIST.  Pages are taken from the free ones (refs
 * 0) in ascending order, in the order of the list and of the positions, so that results do not depend on scheduling.  The list of
 * si_cache_trim is taken sequence by sequence; the other calls do all that they are asked or, with a bit in *status, nothing.
 * cache->refs and cache->scratch are needed.
 * Errors: SI_EINVAL (NULL or misaligned pointer, n negative or above SI_CACHE_MAX_LIST, bad cache descriptor), SI_EHIP.  n == 0 is a no-op.
 */
#define SI_CACHE_MAX_LIST 1024

/* Bytes of cache->scratch, or a negative SI_E* code (host only; pages and tables may be NULL). */
int64_t si_cache_scratch_bytes(const si_cache_t* cache);

/*
 * Cuts sequence seqs[i] to its first keep[i] tokens (keep NULL: to nothing, i.e. frees it): rejected drafts, ended sequences.  Pages
 * that no other sequence shares become free.  A sequence number outside the table or a length above the present one is left out (of a
 * sequence named twice: the length that the entries before have left it).
 */
int si_cache_trim(const si_cache_t* cache, const int32_t* seqs, int32_t n, const int32_t* keep, void* stream);

/*
 * Adds counts[i] tokens (counts NULL: n_new) to sequence seqs[i] and gives them pages.  A partly filled last page that other
 * sequences share is replaced by a copy first (the last of its sharers keeps it).  The new tokens, in list order and ascending
 * positions, are written to seq_out / pos_out, -1 from there to `capacity`: the arrays that si_cache_append takes (both NULL: not wanted).
 * Nothing is done, seq_out is all -1, and *status has bits, where a sequence is outside the table or named twice, a length is bad or grows
 * beyond the table's row, a partly filled last page is outside the pool or has no count, more than `capacity` tokens are added, or pages run out (the
 * last two are looked at where the others are in order).
 */
int si_cache_extend(const si_cache_t* cache, const int32_t* seqs, int32_t n, const int32_t* counts, int32_t n_new, int32_t* seq_out, int32_t* pos_out,
                    int32_t capacity, void* stream);

/*
 * Makes sequence children[i], which has to be empty, a copy of parents[i]: full pages are shared, a partly filled last one is copied (a parent's
 * once read, however many children it has).  A sequence may be the parent of several, but not a parent and a child in one call.
 * Nothing is done, and *status has a bit, where that is not so or a sequence is outside the table, a length is bad, a page of a parent is outside
 * the pool or has no count, or pages run out (looked at in this order).
 */
int si_cache_fork(const si_cache_t* cache, const int32_t* parents, const int32_t* children, int32_t n, void* stream);

/*
 * Packs the pool: of m pages in use, those with a number below m keep it, the others move, in ascending order, into the free places below m.
 * `to` is a cache of the same shape but for n_pages (>= m), whose pages, table, lens and refs are written (its status and scratch are not used), or
 * the same cache: then it is packed in place.  Anything between (some arrays shared, pools that overlap) is allowed for whole arrays
 * only: each of to's four is either the cache's own or memory of its own.  n_used, DEVICE [1] or NULL, receives m.  Where m exceeds to's
 * n_pages, nothing else is written.  (Pools of up to 2^24 pieces of 64 KB, a page counted in whole pieces: SI_EINVAL beyond.)
 */
int si_cache_compact(const si_cache_t* cache, const si_cache_t* to, int32_t* n_used, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* SCHEINFER_ATTENTION_H */
