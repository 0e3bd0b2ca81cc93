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

// Turns per position in units of 2^-64, whole turns left out (53 bits of it matter; more
// than 2^53 turns, which no position makes sense with, count as none).
inline uint64_t steps_of(double turns) {
  const double whole = turns < 9007199254740992.0 ? (double)(int64_t)turns : turns;
  const double high = (turns - whole) * 4294967296.0, low = high - (double)(uint32_t)high;
  return ((uint64_t)(uint32_t)high << 32) + (uint64_t)(low * 4294967296.0);
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
// Whether all sequences together can have more tiles than 32 bits count: only where starts
// fall, so that several take the same rows, and a page table has 2^29 entries or more.
UAD_HD bool append_tiles_overflow(int n_rows, int n_seqs, int pages_per_seq, int page_shift) {
  const int64_t tokens = (int64_t)pages_per_seq << page_shift, rows = tokens < n_rows ? tokens : n_rows;
  return n_seqs * ((rows >> append_tile_shift(page_shift)) + 2) > 0x7FFFFFFF;
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

// ---------------------------------------------------------------------------
// The same for new rows.  A sequence's rows are units of up to `cols` (row, query head) pairs
// of a KV head, its tiles those that any of its rows sees.  The launch knows bounds of the
// units and tiles only, the plan on the device what they are: what both decide by is here, so
// that no workgroup that a plan counts on is left out of a launch.
// ---------------------------------------------------------------------------
// What differs between the kernels (constants there: from functions, as a variable's would be
// loaded, for 0.4 to 0.9 us a call).
struct RowsKind {
  int tile, cols, whole, min_tiles;
  bool one_round;  // with idle workgroups, no splits that all of them together could not take
};
constexpr int kUncut = 1 << 30;  // a share that no unit is more than

UAD_HD int runs_of(int rows, int group, int cols) { return (int)(((int64_t)rows * group + cols - 1) / cols); }
// Whether some of the workgroups that run at once would have no unit.
UAD_HD bool leaves_idle(int64_t units, int target) { return units < target; }
// Splits of a sequence's units; one_round: a remainder of less than half a share is not worth
// a join.
UAD_HD int rows_splits(const RowsKind &k, int tiles, int share) {
  const int rest = share + (share >> 1);
  return splits_of(tiles, share, k.one_round && rest > k.whole ? rest : k.whole);
}
// The plan's share of `units` units, from `share` on, the first or that of a launch without
// splits; count(share) gives the workgroups.
template <class Count>
UAD_HD int rows_share(const RowsKind &k, int share, int units, int target, Count count) {
  for (int i = 0;; ++i) {
    if (count(share) <= target || !leaves_idle(units, target)) return share;
    if (i < kShareTries) share = next_share(share);
    else if (k.one_round && share < kUncut) share = kUncut;
    else return share;
  }
}
// Workgroups to launch: a unit more for every sequence, whose last may have fewer columns, and
// a split more for each of the slots.
struct RowsGrid {
  int64_t wgs;
  bool unsplit;  // no sequence can have a split
};
UAD_HD RowsGrid rows_grid(const RowsKind &k, int n_rows, int n_seqs, bool starts, int n_kv_heads, int group, int64_t max_tokens,
                          int window, int sinks, int target, int slots) {
  const int64_t units = n_kv_heads * (starts ? (int64_t)n_rows * group / k.cols + n_seqs : (int64_t)n_seqs * runs_of(1, group, k.cols));
  int64_t tiles = tiles_of_length((int)(max_tokens < 0x7FFFFFFF ? max_tokens : 0x7FFFFFFF), k.tile);
  // a window's, of up to all the rows, and the sinks', each in a tile more than they fill
  const int64_t seen = ((int64_t)window + (starts ? n_rows : 1)) / k.tile + sinks / k.tile + 4;
  if (window > 0 && seen < tiles) tiles = seen;
  const int64_t splits = splits_of((int)tiles, k.min_tiles, k.whole);
  const int64_t most = k.one_round && leaves_idle(units, target) ? target : units + slots;
  return {units * splits < most ? units * splits : most, splits == 1};
}

// ---------------------------------------------------------------------------
// 8-bit pools with scales of their own: one for K and one for V of every kScaleBlock
// tokens of a page's head, [page][KV head][page size / kScaleBlock].
// ---------------------------------------------------------------------------
constexpr int kScaleBlock = 16;

UAD_HD size_t scale_index(const PagedDims &d, int page, int head, int off) {
  return (((((size_t)page * d.n_kv_heads + head) << d.page_shift) + off)) / kScaleBlock;
}

// The least power of two by which magnitudes up to one of these bits (finite, no sign) lie
// within 448 = 1.75 * 2^8, from 2^-100 (blocks of zeros) up to 2^119, whose product with
// 448 is finite (larger values are cut): its bits.
UAD_HD uint32_t scale_bits(uint32_t most) {
  int e = (int)(most >> 23) - 127 - 8 + ((most & 0x7FFFFFu) > 0x600000u);
  e = e < -100 ? -100 : e > 119 ? 119 : e;
  return (uint32_t)(e + 127) << 23;
}

// ---------------------------------------------------------------------------
// Attention of new rows: what a row at cache position p of a sequence of `len` tokens
// sees, keys [lo, hi) and those before `first`.  window 0: no window.
// ---------------------------------------------------------------------------
UAD_HD int seen_from(int p, int window) { return window > 0 && p >= window ? p - window + 1 : 0; }
UAD_HD int seen_to(int p, int len, int window, bool causal) {
  return causal ? p + 1 : window > 0 && window < len - p ? p + window : len;
}

UAD_HD int seen_first(int p, int len, int sinks, bool causal) {
  const int most = causal ? p + 1 : len;
  return sinks < most ? sinks : most;
}

// The tiles of `tile` keys that rows see of which the first sees from `lo`, counted
// without the gap behind the sinks: tile i of them is tile i + (i < first ? 0 : gap).
struct SeenTiles {
  int first, gap, count;
};
UAD_HD SeenTiles seen_tiles(int len, int lo, int sinks, int tile) {
  const int from = (int)((uint32_t)lo / (uint32_t)tile), s = sinks < lo ? sinks : lo;
  const int t = (int)(((uint32_t)s + tile - 1) / tile);
  SeenTiles r;
  r.first = t < from ? t : from;
  r.gap = from - r.first;
  r.count = tiles_of_length(len, tile) - r.gap;
  return r;
}
UAD_HD int seen_tile(const SeenTiles &s, int i) { return i < s.first ? i : i + s.gap; }

// Bits from .. to-1 of a lane's run of `n` keys (n <= 32), whatever lies outside of it.
UAD_HD uint32_t run_bits(int from, int to, int n) {
  from = from < 0 ? 0 : from;
  to = to > n ? n : to;
  return to <= from ? 0u : (0xFFFFFFFFu >> (32 - (to - from))) << from;
}

// ---------------------------------------------------------------------------
// Pages of new tokens.  Sequence b holds `len` tokens and gets n more: it needs pages
// pages_of(len) .. pages_of(len + n) - 1 of its table row.
// ---------------------------------------------------------------------------
UAD_HD int pages_of(int len, int page_shift) { return (int)(((uint32_t)len + (1u << page_shift) - 1) >> page_shift); }
UAD_HD bool growth_ok(int len, int n, int pages_per_seq, int page_shift) {
  return len >= 0 && n >= 0 && (int64_t)len + n <= (int64_t)pages_per_seq << page_shift;
}
// Whether page i of a sequence of `len` tokens holds one that a later token sees, or is the
// one, not full, that the next token goes to.
UAD_HD bool page_in_use(int i, int len, int window, int sinks, int page_shift) {
  const int64_t from = (int64_t)i << page_shift, to = from + ((int64_t)1 << page_shift);
  return from < len && (from < sinks || window == 0 || to > (int64_t)len - window + 1);
}

}  // namespace uad
