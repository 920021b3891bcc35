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
 * stride); other overlaps are not allowed.
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

#ifdef __cplusplus
}
#endif
#endif /* SCHEINFER_ATTENTION_H */
