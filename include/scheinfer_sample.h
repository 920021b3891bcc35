/*
 * scheinfer_sample.h - the next token of each sequence from its logits, for one MI355X (gfx950): the end of a step whose layers scheinfer.h and
 * scheinfer_attention.h run.
 *
 * Conventions: those of scheinfer_attention.h (codes, si_last_error, device addresses in a host descriptor that is read during the call only, stream
 * as void*, no allocation, no copy, no wait: every call can be recorded into a HIP graph; work runs on the current HIP device).
 */
#ifndef SCHEINFER_SAMPLE_H
#define SCHEINFER_SAMPLE_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define SI_SAMPLE_MAX_VOCAB (1 << 20)
#define SI_SAMPLE_MAX_ROWS (1 << 16)

/*
 * One token for each row of logits l, drawn by a given random number u.  With T = temperature, m = max l, and the tokens in the order of
 * (l descending, index ascending):
 *   w = e^((l - m) / T)
 *   top_k  > 0:  the first top_k tokens are left                                           (S_k: the sum of their w)
 *   top_p  < 1:  of these the smallest leading part whose sum of w is at least top_p S_k (one token at least)
 *   min_p  > 0:  of these the tokens with w >= min(min_p, 1)
 *   token: the first, in ascending index, whose sum of w over the tokens left up to it is above u S   (S: the sum of all that are left)
 * so that it is drawn with probability w / S from a u that is uniform in [0, 1).
 * T <= 0 or NaN: the token of the largest logit, the lowest of several; top_k, top_p, min_p and u are not looked at.  A limit that is NaN is none;
 * top_p <= 0 leaves one token; u below 0 or NaN counts as 0, u of 1 or more draws the last token left that has a w.
 * A logit that is NaN counts as -infinity, and tokens of -infinity are never left; where there are tokens of +infinity, only they have a w, of 1.  A
 * row without a token above -infinity gets token -1, prob 0, kept 0.
 * Weights and sums are of 64 bits: w is taken as a multiple of 2^-(62 - ceil(log2(vocab))), so that sums are exact and no result depends on
 * the order in which blocks run; the sum over a whole vocabulary (rows without top_k) is of doubles in a fixed order.
 *
 * scratch: si_sample_scratch_bytes bytes, 16-byte aligned, zero before its first use; every call leaves it fit for any other call that needs no
 * more.  Two calls that may run at once need one each.
 * Errors: SI_EINVAL (NULL descriptor; logits, u, token or scratch NULL; a pointer not aligned to its element, scratch to 16 bytes; unknown type;
 * rows outside 0 .. SI_SAMPLE_MAX_ROWS, vocab outside 1 .. SI_SAMPLE_MAX_VOCAB, rows * ceil(vocab / 8192) of 2^22 or more; stride smaller than vocab (but 0, one row of logits
 * for all, is taken); scratch_bytes too small), SI_EHIP.  rows == 0 is a no-op.
 */
typedef struct {
  const void* logits;         /* [rows][vocab] of type */
  const float* temperature;   /* [rows], or NULL: 1 */
  const int32_t* top_k;       /* [rows], or NULL: no limit; <= 0: none either */
  const float* top_p;         /* [rows], or NULL: no limit */
  const float* min_p;         /* [rows], or NULL: no limit */
  const float* u;             /* [rows] */
  int32_t* token;             /* [rows] */
  float* prob;                /* [rows] w / S of the token, or NULL */
  int32_t* kept;              /* [rows] number of tokens left, or NULL */
  void* scratch;
  int64_t scratch_bytes;
  int64_t stride;             /* elements between rows */
  int32_t rows, vocab;
  int32_t type;               /* SI_F32 | SI_BF16 (scheinfer_attention.h) */
} si_sample_t;
int si_sample(const si_sample_t* desc, void* stream);

/* Bytes of scratch that si_sample needs for this descriptor, and for any with fewer rows or a smaller vocab; or a negative SI_E* code (host only, no
 * GPU needed; the pointers, scratch_bytes and stride are not looked at). */
int64_t si_sample_scratch_bytes(const si_sample_t* desc);

#ifdef __cplusplus
}
#endif
#endif /* SCHEINFER_SAMPLE_H */
