// Places in the paged key-value cache, for the host and the kernels (scheinfer_attention.h describes the layout).
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "scheinfer_attention.h"
#include "cc_worker.h"

namespace si {

inline SI_HD int kv_vec(int type) { return type == SI_KV_E4M3 ? 16 : 8; }    // E: elements of 16 bytes
inline SI_HD int kv_block(int type) { return 4 * kv_vec(type); }             // B: tokens of a block
inline SI_HD int kv_elem_bytes(int type) { return type == SI_KV_E4M3 ? 1 : 2; }

inline SI_HD int64_t kv_head_elems(const si_cache_t& c) { return (int64_t)c.page_tokens * c.head_dim; }           // K or V of one head in a page
inline SI_HD int64_t kv_page_elems(const si_cache_t& c) { return 2 * kv_head_elems(c) * c.n_kv_heads * c.n_layers; }
// first element of K (which = 0) or V (1) of a head inside a page
inline SI_HD int64_t kv_head_offset(const si_cache_t& c, int layer, int which, int head) {
  return (((int64_t)layer * 2 + which) * c.n_kv_heads + head) * kv_head_elems(c);
}
// element `dim` of token t of a block, from the block's first element
inline SI_HD int kv_slot(int E, int t) { return t % E / 4 * 16 + 4 * (t / E) + t % 4; }
inline SI_HD int kv_k_offset(int E, int t, int dim) { return dim / E * (4 * E * E) + kv_slot(E, t) * E + dim % E; }
inline SI_HD int kv_v_offset(int E, int head_dim, int t, int dim) { return (t / E * head_dim + dim) * E + t % E; }

// Page that holds position `pos` of sequence `seq`, or -1 and the bits that say why not.  Reads the table inside its bounds only.
inline SI_HD int kv_page_of(const si_cache_t& c, int seq, int pos, int& why) {
  if (seq < 0 || seq >= c.n_seqs) { why |= SI_CACHE_BAD_SEQ; return -1; }
  if (pos < 0 || pos / c.page_tokens >= c.max_pages) { why |= SI_CACHE_BAD_LEN; return -1; }
  const int page = c.table[(int64_t)seq * c.max_pages + pos / c.page_tokens];
  if (page < 0 || page >= c.n_pages) { why |= SI_CACHE_BAD_PAGE; return -1; }
  return page;
}

// append.hip: SI_OK, or an error that names `who`
int check_cache(const si_cache_t* c, const char* who);
int check_layer(const si_cache_t* c, int layer, const char* who);
int check_append(const si_cache_t* c, int layer, const si_append_t* a, const char* who, bool* nothing);

}  // namespace si
