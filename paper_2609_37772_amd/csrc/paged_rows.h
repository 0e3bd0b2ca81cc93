// What the kernels of new rows' attention share: a call's sequences, and values that are
// not finite.
#pragma once

#include "paged_device.h"

namespace uad {

// A sequence's new rows from `from` on, its length with them, its units, and the tiles that
// any of its rows sees.
struct RowsSeq {
  int from, n, len, units;
  SeenTiles tiles;
};

// Sequence b; one that cannot be used has no units.
__device__ __forceinline__ RowsSeq rows_of(RowsKind k, const KvRowsArgs &a, int b, bool *bad, bool *falls) {
  RowsSeq s{b, 1, 0, 0, {}};
  if (a.row_start) {
    s.from = a.row_start[b];
    const int to = a.row_start[b + 1], len = a.lens[b];
    *falls |= s.from > to;
    const bool ok = sequence_ok(b, s.from, to, a.n_rows, len, a.pages_per_seq, a.d.page_shift);
    *bad |= !ok;
    s.n = ok ? to - s.from : 0;
    s.len = ok ? len : 0;
  } else {
    s.len = length_or_none(a.lens[b], a.pages_per_seq, a.d.page_shift, bad);
  }
  s.units = a.d.n_kv_heads * runs_of(s.n, a.group, k.cols);
  s.tiles = seen_tiles(s.len, seen_from(s.len - s.n, a.window), a.sinks, k.tile);
  return s;
}

// What workgroup `wg` does: split `split` of `splits` of a unit, whose slots begin at `slot`;
// false if it has nothing to do.  A sequence's units have as many splits as its tiles ask for
// (see rows_share), and share out the tiles that they see themselves.  one_round: the longest
// sequences' come first.
struct RowsWork {
  RowsSeq s;
  int b, unit, split, splits, slot;
  // Of a unit that sees `tiles` tiles; a split that is not needed is not done.
  __device__ __forceinline__ bool of_unit(int tiles) {
    const int each = (int)(((unsigned)s.tiles.count + splits - 1) / (unsigned)splits);
    splits = max(1, min(splits, (int)(((unsigned)tiles + each - 1) / (unsigned)each)));
    return split < splits;
  }
};

template <int NW>
__device__ __forceinline__ bool plan_rows(RowsKind k, const KvRowsArgs &a, int wg, int *lds, RowsWork *w) {
  bool bad = false, falls = false;
  if (a.unsplit && !a.row_start) {  // no sequence can have a split: a workgroup per unit
    const int units = a.d.n_kv_heads * runs_of(1, a.group, k.cols);
    *w = RowsWork{};
    w->b = (unsigned)wg / (unsigned)units;
    w->unit = wg - w->b * units;
    w->s = rows_of(k, a, w->b, &bad, &falls);
    w->splits = 1;
    if (bad && threadIdx.x == 0) raise_status(a.status, kStatusPage);
    return true;
  }
  PlanScan<NW> scan(a.n_seqs, lds);
  const int b0 = scan.me * scan.per;
  RowsSeq s0{};
  if (b0 < a.n_seqs) s0 = rows_of(k, a, b0, &bad, &falls);
  int seq = b0;  // whose s0 is
  if (k.one_round && !scan.block && __ballot(b0 < a.n_seqs && s0.tiles.count != __builtin_amdgcn_readfirstlane(s0.tiles.count))) {
    // the longest first, so that none of theirs is left for the end (16 sequences of up to
    // 1024 rows: 109 -> 91 us; where they differ little it costs up to 4 of 100)
    const int key = s0.tiles.count << 6 | (63 - scan.me);  // below 2^31: such tiles have 64 keys
    int rank = 0;
    for (int j = 0; j < a.n_seqs; ++j) rank += __builtin_amdgcn_readlane(key, j) > key;
    seq = __builtin_amdgcn_ds_permute(4 * (scan.me < a.n_seqs ? rank : scan.me), scan.me);
    for (int *v : {&s0.from, &s0.n, &s0.len, &s0.units, &s0.tiles.first, &s0.tiles.gap, &s0.tiles.count}) *v = __shfl(*v, seq);
  }
  // f over this thread's sequences, of which the first is kept
  auto each = [&](auto f) {
    if (b0 < a.n_seqs) f(s0);
    for (int i = 1; i < scan.per; ++i)
      if (b0 + i < a.n_seqs) f(rows_of(k, a, b0 + i, &bad, &falls));
  };
  int64_t n = 0;
  int my_units = 0, units, hi, lo, mine, upto, wgs, all;
  each([&](const RowsSeq &s) {
    n += (int64_t)s.units * s.tiles.count;
    my_units += s.units;
  });
  if (bad && wg == 0) raise_status(a.status, kStatusPage);
  auto count = [&](int share) {  // workgroups of this thread's sequences, up to them, and all
    mine = 0;
    each([&](const RowsSeq &s) { mine += rows_splits(k, s.tiles.count, share) * s.units; });
    upto = scan(mine, &wgs);
    return wgs;
  };
  // Sequences whose starts fall share rows with others, which may be more than the launch is
  // for: units stay whole then, so that none is begun without an end.
  const bool any_falls = a.row_start && (scan.block ? __syncthreads_or(falls) != 0 : __ballot(falls) != 0);
  int share = kUncut;
  if (!a.unsplit && !any_falls) {
    scan((int)(n >> 22), &hi);
    scan((int)(n & 0x3FFFFF), &lo);
    share = first_share(((int64_t)hi << 22) + lo, a.target, k.min_tiles);
  }
  scan(my_units, &units);
  share = rows_share(k, share, units, a.target, count);
  if (wg >= wgs) return false;
  int in_slots = 0;  // workgroups in split units, for the slots
  each([&](const RowsSeq &s) {
    const int splits = rows_splits(k, s.tiles.count, share);
    if (splits > 1) in_slots += splits * s.units;
  });
  int slot = scan(in_slots, &all) - in_slots, start = upto - mine, b = b0;
  if (!scan.block) {
    b = __builtin_ctzll(__ballot(upto > wg));
    start = __builtin_amdgcn_readlane(start, b);
    slot = __builtin_amdgcn_readlane(slot, b);
    w->b = __builtin_amdgcn_readlane(seq, b);
    w->s.from = __builtin_amdgcn_readlane(s0.from, b);
    w->s.n = __builtin_amdgcn_readlane(s0.n, b);
    w->s.len = __builtin_amdgcn_readlane(s0.len, b);
    w->s.units = __builtin_amdgcn_readlane(s0.units, b);
    w->s.tiles.first = __builtin_amdgcn_readlane(s0.tiles.first, b);
    w->s.tiles.gap = __builtin_amdgcn_readlane(s0.tiles.gap, b);
    w->s.tiles.count = __builtin_amdgcn_readlane(s0.tiles.count, b);
  } else {
    if (upto > wg && start <= wg) {  // one thread: it looks for the sequence among its own
      RowsSeq s = s0;
      for (;;) {
        const int splits = rows_splits(k, s.tiles.count, share);
        if (start + splits * s.units > wg) break;
        start += splits * s.units;
        if (splits > 1) slot += splits * s.units;
        if (++b >= min(b0 + scan.per, a.n_seqs)) break;
        s = rows_of(k, a, b, &bad, &falls);
      }
      const int found[3] = {b, start, slot};
#pragma unroll
      for (int i = 0; i < 3; ++i) scan.lds[i] = found[i];
    }
    __syncthreads();
    b = __builtin_amdgcn_readfirstlane(scan.lds[0]);
    start = __builtin_amdgcn_readfirstlane(scan.lds[1]);
    slot = __builtin_amdgcn_readfirstlane(scan.lds[2]);
    // only if the caller's arrays change while this runs, or starts fall so often that sums overflow
    if ((unsigned)b >= (unsigned)a.n_seqs) return false;
    w->b = b;
    w->s = rows_of(k, a, b, &bad, &falls);
  }
  w->splits = rows_splits(k, w->s.tiles.count, share);
  w->unit = (unsigned)(wg - start) / (unsigned)w->splits;
  if ((unsigned)w->unit >= (unsigned)w->s.units) return false;  // likewise
  w->split = wg - start - w->unit * w->splits;
  w->slot = slot + w->unit * w->splits;
  if (w->splits > 1 && w->slot + w->splits > a.slots) return false;  // likewise
  return true;
}

// 16-byte pieces of V that hold a value that is not finite: those become zeros in v, and
// ones in the bf16 operand that is returned (its other elements zero).
template <bool F8>
__device__ __forceinline__ bool not_finite(u32x4_t v) {
  bool any = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (F8) {
#pragma unroll
      for (int k = 0; k < 4; ++k) any |= (v[i] >> (8 * k) & 0x7F) == 0x7F;
    } else {
      any |= (v[i] & 0x7F80u) == 0x7F80u || (v[i] & 0x7F800000u) == 0x7F800000u;
    }
  }
  return any;
}
template <bool F8>
__device__ __forceinline__ bf16x8 take_not_finite(u32x4_t &v, int u) {
  union {
    bf16x8 h;
    uint16_t e[8];
  } o;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int i = F8 ? 2 * u + e / 4 : e / 2, shift = F8 ? 8 * (e % 4) : 16 * (e % 2);
    const uint32_t top = F8 ? 0x7Fu : 0x7F80u, whole = F8 ? 0xFFu : 0xFFFFu;
    const bool odd = (v[i] >> shift & top) == top;
    o.e[e] = odd ? 0x3F80u : 0u;
    if (odd) v[i] &= ~(whole << shift);
  }
  return o.h;
}

}  // namespace uad
