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

// The same, where a length that cannot be used counts as none.
UAD_HD int length_or_none(int len, int pages_per_seq, int page_shift, bool *bad) {
  bool cut = false;
  const int usable = usable_length(len, pages_per_seq, page_shift, &cut);
  *bad |= cut;
  return cut ? 0 : usable;
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
// Appends of many rows go by tiles: runs of up to kAppendTile cache positions that start
// at a multiple of their size and lie in one page.
// ---------------------------------------------------------------------------
constexpr int kAppendTile = 64;

UAD_HD int append_tile_shift(int page_shift) { return page_shift < 6 ? page_shift : 6; }
// Tiles that positions [from, to) touch.
UAD_HD int append_tiles(int from, int to, int shift) { return to > from ? ((to - 1) >> shift) - (from >> shift) + 1 : 0; }
// At most as many workgroups: every tile holds a row, and a sequence's first and last
// tile may be shorter than the others.
UAD_HD int64_t append_grid(int n_rows, int n_seqs, int shift) {
  const int64_t most = ((int64_t)n_rows >> shift) + 2 * (int64_t)n_seqs;
  return most < n_rows ? most : n_rows;
}
// New rows of a sequence at row_start[b] .. row_start[b + 1]: usable, or an error.
UAD_HD bool rows_ok(int from, int to, int n_rows) { return from >= 0 && from <= to && to <= n_rows; }
// The same of sequence b whose length with them is `len`: all of its new rows can be
// used, or none.
UAD_HD bool sequence_ok(int b, int from, int to, int n_rows, int len, int pages_per_seq, int page_shift) {
  bool bad = false;
  const int usable = usable_length(len, pages_per_seq, page_shift, &bad);
  return !bad && rows_ok(from, to, n_rows) && to - from <= usable && (b > 0 || from == 0);
}

// ---------------------------------------------------------------------------
// The attention's work.  Unit u of sequence b is a KV head with up to 16 of its query
// heads, read in tiles of `tile` keys; a sequence without keys counts one tile, so that
// somebody writes its zeros.  Every unit of a sequence of more than `whole` tiles is cut
// into the same number of splits of at most `share` tiles, one workgroup each; up to
// `whole` the join would cost more than the shorter read gains.  The lengths are known
// on the device alone, and every workgroup works the plan out for itself.
// ---------------------------------------------------------------------------
constexpr int kMaxSplits = 512;   // of a unit
constexpr int kJoinFan = 16;      // splits that one workgroup joins; above 2 * kJoinFan of them in two levels

UAD_HD int tiles_of_length(int len, int tile) { return len > tile ? (int)(((uint32_t)len + tile - 1) / tile) : 1; }

// Tiles of a workgroup for `total` tiles on `target` workgroups that run at once.
UAD_HD int first_share(int64_t total, int target, int min_tiles) {
  const int64_t s = total < (1 << 30) ? ((uint32_t)total + (uint32_t)target - 1) / (uint32_t)target : (total + target - 1) / target;
  return s < min_tiles ? min_tiles : s > (1 << 30) ? 1 << 30 : (int)s;
}
// With fewer units than workgroups that run at once, the splits' remainders may take
// more than those: then the next larger share is tried, a few times (what is over
// runs in a second round).
constexpr int kShareTries = 6;
UAD_HD int next_share(int share) { return share + (share >> 4) + 1; }

UAD_HD int splits_of(int tiles, int share, int whole) {
  if (tiles <= whole) return 1;
  const int s = (int)(((uint32_t)tiles + (uint32_t)share - 1) / (uint32_t)share);
  return s < kMaxSplits ? s : kMaxSplits;
}
// First tile of split s of n (and, for s + 1, the end of s).
UAD_HD int split_begin(int tiles, int n, int s) {
  const int each = (int)((uint32_t)tiles / (uint32_t)n), more = tiles - each * n;
  return each * s + (s < more ? s : more);
}

// Workgroups in units that are split: a unit of more than `share` tiles has fewer than
// twice tiles / share of them, and total / share is at most `target`.
UAD_HD int max_slots(int target) { return 2 * target; }

}  // namespace uad
