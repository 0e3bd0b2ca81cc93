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

// ---------------------------------------------------------------------------
// The attention's work: unit u of sequence b is (KV head, run of up to 16 query heads)
// u, read in tiles of `tile` keys; a sequence without keys counts one tile, so that
// somebody writes its zeros.  All tiles of all units stand in one row, sequences
// outermost, and each workgroup takes an equal run of it, whatever the lengths are.
// ---------------------------------------------------------------------------
UAD_HD int tiles_of_length(int len, int tile) { return len > tile ? (int)(((int64_t)len + tile - 1) / tile) : 1; }

// Workgroups that take part: at least min_tiles tiles each, where there are as many.
UAD_HD int sharing_wgs(int64_t total, int grid, int min_tiles) {
  const int64_t n = (total + min_tiles - 1) / min_tiles;
  return n < grid ? (int)n : grid;
}
// First tile of workgroup w (and, for w + 1, the end of w's run).
UAD_HD int64_t share_begin(int64_t total, int wgs, int w) {
  if (total < ((int64_t)1 << 32) / 4096 && wgs <= 4096) return (uint32_t)total * (uint32_t)w / (uint32_t)wgs;
  return total * w / wgs;
}
// The workgroup whose run holds tile t.
UAD_HD int share_holding(int64_t total, int wgs, int64_t t) {
  if (total < ((int64_t)1 << 32) / 4096 && wgs <= 4096)
    return (int)(((uint32_t)(t + 1) * (uint32_t)wgs - 1) / (uint32_t)total);
  return (int)(((t + 1) * wgs - 1) / total);
}

}  // namespace uad
