// Index arithmetic of the paged K/V cache: where a token's key and value lie, which
// page ids and lengths may be used, and how the attention shares its work out.  No
// HIP in here, so that all of it can be checked on a machine without a GPU.
#pragma once

#include <stddef.h>
#include <stdint.h>

#ifdef __HIP__
#define UAD_HD __host__ __device__ inline
#else
#define UAD_HD inline
#endif

namespace uad {

// The cache of one layer: K pages [page][KV head][token][head dim], V pages transposed,
// [page][KV head][head dim][token].  Transposed V is what the attention's P V product
// consumes (8 consecutive keys of one column per lane), so that both go from global
// memory to registers without a stop in LDS.
struct PagedDims {
  int n_pages, page_shift;  // page size 2^page_shift, 16 .. 256
  int n_kv_heads, head_dim;
};

// First element of a page's head, of K and of V alike.  Pools pass 2^31 elements.
UAD_HD size_t page_base(const PagedDims &d, int page, int head) {
  return (((size_t)page * d.n_kv_heads + head) * d.head_dim) << d.page_shift;
}
UAD_HD size_t k_in_page(const PagedDims &d, int off, int col) { return (size_t)off * d.head_dim + col; }
UAD_HD size_t v_in_page(const PagedDims &d, int off, int col) { return ((size_t)col << d.page_shift) + off; }

// A page id from the caller's table: usable, or an error (and no access).
UAD_HD bool page_ok(const PagedDims &d, int page) { return page >= 0 && page < d.n_pages; }

// A sequence's length from the caller's memory, cut to what its row of the page table
// can address; *bad is set where it had to be.
UAD_HD int usable_length(int len, int pages_per_seq, int page_shift, bool *bad) {
  const int64_t cap = (int64_t)pages_per_seq << page_shift;
  if (len < 0) {
    *bad = true;
    return 0;
  }
  if (len > cap) {
    *bad = true;
    return (int)cap;
  }
  return len;
}

// Elements (a, b) that rotation pair p of a head turns, p < head_dim / 2; pairs from
// rope_dim / 2 on are left as they are.
UAD_HD void rope_pair(int p, int rope_dim, bool neighbours, int *a, int *b) {
  if (p < rope_dim / 2 && !neighbours) {
    *a = p;
    *b = p + rope_dim / 2;
  } else {
    *a = 2 * p;
    *b = 2 * p + 1;
  }
}

}  // namespace uad
