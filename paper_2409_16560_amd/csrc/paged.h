// Paged caches: which sequence a row belongs to, and where a token of a sequence is stored.
#pragma once
#include "common.h"

// Division of numbers below 2^31 by a fixed number: n / d = (n * mul) >> shift, exact because mul = floor(2^shift / d) + 1
// with shift = 31 + ceil(log2 d) misses 2^shift / d by less than 2^(shift - 31).
struct FastDiv {
  uint32_t mul;
  int32_t shift, d;
};
static inline FastDiv fast_div(int32_t d) {
  int l = 0;
  while ((1ll << l) < d) ++l;
  FastDiv f;
  f.d = d; f.shift = 31 + l;
  f.mul = (uint32_t)(((1ull << f.shift) / (uint64_t)d) + 1);
  return f;
}
__device__ __forceinline__ int quotient(const FastDiv& f, int n) {
  return (int)(((unsigned long long)(uint32_t)n * f.mul) >> f.shift);
}

struct PagedArgs {
  const int32_t *page_table, *ctx_len, *q_off;
  long long page_stride, token_stride, head_stride;    // elements
  int n_pages, table_stride, n_seqs, max_new, max_len;
  FastDiv page;                                        // its size
};

// What the host can see of a cache: an error code.
static inline int32_t paged_check(const dsbd_paged_kv* c, int32_t n_rows, int32_t Hkv) {
  if (c->n_seqs < 0 || c->n_pages < 0 || c->page_size < 1 || c->table_stride < 0 || c->max_new < 0 || c->max_len < 0 ||
      n_rows < 0 || Hkv < 1) return DSBD_ERR_INVALID;
  if (c->page_stride < 0 || c->token_stride < 0 || c->head_stride < 0) return DSBD_ERR_INVALID;
  if (c->page_size > (1 << 30) || c->max_len > (1 << 30) || c->n_seqs > (1 << 30)) return DSBD_ERR_UNSUPPORTED;
  if ((c->page_stride | c->token_stride | c->head_stride) & 7) return DSBD_ERR_UNSUPPORTED;
  if (n_rows == 0 || c->n_seqs == 0) return DSBD_OK;
  if (!c->ctx_len || !c->q_off) return DSBD_ERR_INVALID;
  if (c->table_stride > 0 && !c->page_table) return DSBD_ERR_INVALID;
  if (c->n_pages > 0 && (!c->k_pages || !c->v_pages)) return DSBD_ERR_INVALID;
  if ((reinterpret_cast<uintptr_t>(c->k_pages) | reinterpret_cast<uintptr_t>(c->v_pages)) & 15) return DSBD_ERR_INVALID;
  return DSBD_OK;
}
static inline PagedArgs paged_args(const dsbd_paged_kv* c) {
  PagedArgs p;
  p.page_table = c->page_table; p.ctx_len = c->ctx_len; p.q_off = c->q_off;
  p.page_stride = c->page_stride; p.token_stride = c->token_stride; p.head_stride = c->head_stride;
  p.n_pages = c->n_pages; p.table_stride = c->table_stride; p.n_seqs = c->n_seqs;
  p.max_new = c->max_new; p.max_len = c->max_len;
  p.page = fast_div(c->page_size);
  return p;
}

// The last of the n entries of `off` (ascending) whose key(entry, index) is at most x, or -1: 64 pivots at a time, one per
// lane, so two trips to memory for 4096 entries.  All lanes of a wave take part.  Never reads outside [0, n), whatever the
// entries are.
template <typename Key>
__device__ __forceinline__ int last_at_most(const int32_t* __restrict__ off, int n, int x, Key key) {
  const int lane = threadIdx.x & 63;
  int lo = 0;
  bool first = true;
  while (n > 0) {
    const int step = (n + 63) >> 6, i = lane * step;
    const bool in = i < n && key(off[lo + min(i, n - 1)], lo + min(i, n - 1)) <= x;
    const unsigned long long m = __ballot(in);
    if (m == 0ull) return first ? -1 : lo;
    const int l = 63 - __builtin_clzll(m);
    lo += l * step;
    n = min(step, n - l * step);
    if (step == 1) break;
    first = false;
  }
  return lo;
}
