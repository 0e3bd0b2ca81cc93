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

__device__ __forceinline__ int runs_of(int rows, int group) { return (int)(((int64_t)rows * group + 15) / 16); }

// Sequence b; one that cannot be used has no units.
template <int TILE>
__device__ __forceinline__ RowsSeq rows_of(const KvRowsArgs &a, int b, bool *bad) {
  RowsSeq s{b, 1, 0, 0, {}};
  if (a.row_start) {
    s.from = a.row_start[b];
    const int to = a.row_start[b + 1], len = a.lens[b];
    const bool ok = sequence_ok(b, s.from, to, a.n_rows, len, a.pages_per_seq, a.d.page_shift);
    *bad |= !ok;
    s.n = ok ? to - s.from : 0;
    s.len = ok ? len : 0;
  } else {
    s.len = length_or_none(a.lens[b], a.pages_per_seq, a.d.page_shift, bad);
  }
  s.units = a.d.n_kv_heads * runs_of(s.n, a.group);
  s.tiles = seen_tiles(s.len, seen_from(s.len - s.n, a.window), a.sinks, TILE);
  return s;
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
