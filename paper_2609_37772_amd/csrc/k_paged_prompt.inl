// Attention of many new rows over a paged K/V cache.
#include "paged_rows.h"

namespace uad {

// ---------------------------------------------------------------------------
// Many rows: bound by the matrix instructions.  A unit is a KV head of a sequence with up
// to 128 (row, query head) pairs, 32 columns to each of four waves (or 64, where two waves
// share 32 columns and take half of every tile's keys each: for calls with too few units
// to fill the chip).  S^T = K Q^T and O^T = V^T P^T with v_mfma_f32_32x32x16_bf16: row i of
// the 32-key product is key 16 (i / 4 % 2) + 4 (i / 8) + i % 4, so that a half wave ends
// with the scores of 16 consecutive keys, which are its operand of the P V product as they
// stand.  Tiles of 64 keys go from memory to LDS past the registers, the next one while
// this one is worked on; a 16-byte piece p of a row lies at piece p ^ (a few bits of the row),
// so that the rows that a read takes at once do not meet in a bank.  The query is held in
// registers, rotated in fp32 on the way.
//
// Precision: the query and the weights enter as bf16 terms, two (16 bits) for bf16 rows and
// three for fp32 rows; keys and values as stored.  One term would halve the time and add
// as much error again as the output's one rounding to bf16 has, twice over: once for the
// query, whose error the scores take in, and once for the weights.
// ---------------------------------------------------------------------------
constexpr int kPromptTile = 64;

// LDS: two buffers of a tile's K and V^T; before that the query in fp32, after it, where two
// waves share columns, one's outputs, maxima and sums.
template <int HD, bool F8, int KW>
constexpr int prompt_lds_bytes() {
  constexpr int buffers = 2 * 2 * kPromptTile * HD * (F8 ? 1 : 2), query = 128 / KW * HD * 4;
  constexpr int meeting = KW == 2 ? 64 * HD * 4 + 2 * 2 * 64 * 4 : 0;
  constexpr int most = buffers > query ? buffers : query;
  return most > meeting ? most : meeting;
}
// Waves per SIMD: outputs and query take 32 columns x head dim x (4 + 2 TERMS) bytes.
template <int HD, bool F32>
constexpr int kPromptPerSimd = HD == 256 || (HD == 128 && F32) ? 1 : 2;

typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16;

// 16 bytes per lane from memory to LDS at `to` + 16 * lane.  The compiler would wait for
// each before the next read of LDS: the kernel waits itself, once per tile.
__device__ __forceinline__ void load_to_lds(const void *from, uint32_t to) {
  uint32_t kept;  // m0 is the compiler's
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, off\n\ts_mov_b32 m0, %0"
               : "=&s"(kept) : "s"(to), "v"(from) : "memory");
}

template <int HD, bool F32, bool F8, int KW>
__global__ __launch_bounds__(256, (kPromptPerSimd<HD, F32>)) void kv_prompt_kernel(KvRowsArgs a) {
  constexpr int TILE = kPromptTile, COLS = 128 / KW, NS = 2 / KW;  // NS: 32-key parts of a tile that a wave takes
  constexpr int KS = HD / 16, NT = HD / 32, TERMS = F32 ? 3 : 2, ESZ = F8 ? 1 : 2;
  constexpr int KP = HD * ESZ / 16, VP = TILE * ESZ / 16;          // 16-byte pieces of a row of K, of V^T
  constexpr int KBYTES = TILE * HD * ESZ, BUF = 2 * KBYTES;
  constexpr int RUN = 16 / ESZ;                                    // keys of a piece of V^T
  extern __shared__ __align__(16) uint8_t lds_bytes[];
  __shared__ int plan[4 * 4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 31, h = lane >> 5;
  const int cw = wave / KW, kw = wave % KW;

  // the unit: sequences' units side by side, a sequence's last rows first (where rows are
  // causal they see the most), its KV heads next to each other
  const int group = a.group;
  RowsSeq sq;
  int b, unit;
  {
    PlanScan<4> scan(a.n_seqs, plan);
    const int b0 = scan.me * scan.per;
    bool bad = false;
    auto units_of = [&](int i) {
      const RowsSeq s = rows_of<TILE>(a, i, &bad);
      return a.d.n_kv_heads * (int)(((int64_t)s.n * group + COLS - 1) / COLS);
    };
    int mine = 0, all;
    for (int i = 0; i < scan.per; ++i)
      if (b0 + i < a.n_seqs) mine += units_of(b0 + i);
    if (bad && blockIdx.x == 0) raise_status(a.status, kStatusPage);
    const int upto = scan(mine, &all), wg = blockIdx.x;
    if (wg >= all) return;
    int start = upto - mine;
    if (!scan.block) {
      b = __builtin_ctzll(__ballot(upto > wg));
      start = __builtin_amdgcn_readlane(start, b);
    } else {
      if (upto > wg && start <= wg) {
        int i = b0;
        for (; i < min(b0 + scan.per, a.n_seqs) - 1; ++i) {
          const int k = units_of(i);
          if (start + k > wg) break;
          start += k;
        }
        scan.lds[0] = i;
        scan.lds[1] = start;
      }
      __syncthreads();
      b = __builtin_amdgcn_readfirstlane(scan.lds[0]);
      start = __builtin_amdgcn_readfirstlane(scan.lds[1]);
    }
    sq = rows_of<TILE>(a, b, &bad);
    unit = wg - start;
  }
  const int runs = (int)(((int64_t)sq.n * group + COLS - 1) / COLS);
  const int run = runs - 1 - unit / a.d.n_kv_heads, kvh = unit % a.d.n_kv_heads;
  if (run < 0) return;  // only if the caller's arrays change while this runs
  const int m0 = run * COLS, cols = min(COLS, sq.n * group - m0);
  const int last = sq.len - 1, mask = (1 << a.d.page_shift) - 1, pos0 = sq.len - sq.n;
  const int32_t *table = a.table + (int64_t)b * a.pages_per_seq;
  auto row_of = [&](int m) { return (int)((unsigned)m / (unsigned)group); };
  auto from_at = [&](int p) { return seen_from(p, a.window); };
  auto to_at = [&](int p) { return min(seen_to(p, sq.len, a.window, a.causal), sq.len); };
  auto first_at = [&](int p) { return seen_first(p, sq.len, a.sinks, a.causal); };
  const int p_min = pos0 + row_of(m0), p_max = pos0 + row_of(m0 + cols - 1), p_mine = pos0 + row_of(m0 + min(32 * cw + c, cols - 1));
  const int lo = from_at(p_mine), hi = to_at(p_mine), first = first_at(p_mine);
  const int lo_min = from_at(p_min), lo_max = from_at(p_max), hi_min = to_at(p_min), hi_max = to_at(p_max);
  const int first_min = first_at(p_min), first_max = first_at(p_max);
  const SeenTiles tiles = seen_tiles(max(hi_max, first_max), lo_min, a.sinks, TILE);
  auto tile_at = [&](int i) { return seen_tile(tiles, i) * TILE; };
  auto seen_by_any = [&](int key, int n) { return run_bits(lo_min - key, hi_max - key, n) | run_bits(-key, first_max - key, n); };
  auto seen_by_mine = [&](int key, int n) { return run_bits(lo - key, hi - key, n) | run_bits(-key, first - key, n); };
  bool bad = false;

  // Page ids of a tile's four runs of 16 keys, in lanes 0 .. 3 (and every four more).
  auto page_ids = [&](int i) { return table[min(tile_at(i) + 16 * (lane & 3), last) >> a.d.page_shift]; };
  auto checked = [&](int id, int i) {
    if (seen_by_any(tile_at(i) + 16 * (lane & 3), 16) == 0) return 0;  // not looked at
    const bool ok = page_ok(a.d, id);
    bad |= !ok;
    return ok ? id : 0;
  };
  int next_ids = tiles.count > 0 ? page_ids(0) : 0;

  // The query: rotated and scaled in fp32, so that scores are in powers of two, through LDS
  // into operands.
  bf16x8 qf[TERMS][KS];
  {
    float *q32 = (float *)lds_bytes;  // [COLS][HD], 16-byte piece p of column i at p ^ (i % 8)
    constexpr int HP = HD / 2, AT_ONCE = 256 / HP, BATCH = 8;
    const int p = threadIdx.x % HP;
    int ea, eb;
    rope_pair(p, a.rope_dim, a.rope_pairs != 0, &ea, &eb);
    const bool turned = p < a.rope_dim / 2;
    const double turns = a.turns[p];  // 128 of them are allocated
    auto at = [&](int col, int e) { return col * HD + (((e >> 2) ^ (col & 7)) << 2) + (e & 3); };
    for (int i0 = threadIdx.x / HP; i0 < COLS; i0 += AT_ONCE * BATCH) {
      uint32_t x[BATCH], y[BATCH];
      int position[BATCH];
#pragma unroll
      for (int i = 0; i < BATCH; ++i) {
        const int m = m0 + min(i0 + i * AT_ONCE, cols - 1), j = row_of(m);
        const int64_t qi = (int64_t)(sq.from + j) * a.ldq + (int64_t)(kvh * group + m - j * group) * HD;
        position[i] = a.positions ? a.positions[sq.from + j] : pos0 + j;
        x[i] = load_raw<F32>(a.q, qi + ea);
        y[i] = load_raw<F32>(a.q, qi + eb);
      }
#pragma unroll
      for (int i = 0; i < BATCH; ++i) {
        const int col = i0 + i * AT_ONCE;
        float sn = 0.f, cs = 1.f;
        if (turned) turn_of(turns, position[i], &sn, &cs);
        const float u = col < cols ? value_of<F32>(x[i]) : 0.f, v = col < cols ? value_of<F32>(y[i]) : 0.f;
        if (col < COLS) {
          q32[at(col, ea)] = (turned ? u * cs - v * sn : u) * a.scale_log2;
          q32[at(col, eb)] = (turned ? v * cs + u * sn : v) * a.scale_log2;
        }
      }
    }
    __syncthreads();
    const int col = 32 * cw + c;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const int d0 = F8 ? (ks >> 1) * 32 + 16 * h + 8 * (ks & 1) : 16 * ks + 8 * h;
      const f32x4 v[2] = {*(const f32x4 *)(q32 + at(col, d0)), *(const f32x4 *)(q32 + at(col, d0 + 4))};
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float x = v[e / 4][e % 4];
#pragma unroll
        for (int t = 0; t < TERMS; ++t) {
          qf[t][ks][e] = (__bf16)x;
          x -= (float)qf[t][ks][e];
        }
      }
    }
    __syncthreads();
  }

  // Loads of a tile into buffer `to`.  K: thread t of pass n takes piece 256 n + t, of a row
  // whose 16-key run is one for the wave; V^T: a column each, the same keys in every pass.
  constexpr int K_PASSES = TILE * KP / 256, V_PASSES = HD * VP / 256, V_ROWS = 256 / VP;
  auto k_bits = [&](int key) { return KP == 4 ? (key >> 1 & 1) | (key >> 4 & 1) << 1 : (key & 3) | (key >> 4 & 1) << 2; };
  auto v_bits = [&](int d) { return VP == 4 ? d >> 1 & 3 : d & 7; };
  const int v_row = threadIdx.x / VP, v_key = ((threadIdx.x % VP) ^ v_bits(v_row)) * RUN;
  auto load_tile = [&](int i, int ids, uint32_t to) {
    const int k0 = tile_at(i);
#pragma unroll
    for (int n = 0; n < K_PASSES; ++n) {
      const int piece = n * 256 + threadIdx.x, row = piece / KP, p = piece % KP;
      const int page = __builtin_amdgcn_readlane(ids, (n * 256 + wave * 64) / KP / 16);
      const size_t at = page_base(a.d, page, kvh) + k_in_page(a.d, (k0 + row) & mask, 0);
      load_to_lds((const char *)a.kp + at * ESZ + (p ^ k_bits(row)) * 16, to + n * 4096 + wave * 1024);
    }
    const int run16 = v_key >> 4;
    const int id0 = __builtin_amdgcn_readlane(ids, 0), id1 = __builtin_amdgcn_readlane(ids, 1);
    const int id2 = __builtin_amdgcn_readlane(ids, 2), id3 = __builtin_amdgcn_readlane(ids, 3);
    const int page = run16 == 0 ? id0 : run16 == 1 ? id1 : run16 == 2 ? id2 : id3;
    const char *src = (const char *)a.vp + (page_base(a.d, page, kvh) + v_in_page(a.d, (k0 + v_key) & mask, v_row)) * ESZ;
#pragma unroll
    for (int n = 0; n < V_PASSES; ++n)
      load_to_lds(src + ((size_t)(n * V_ROWS) << a.d.page_shift) * ESZ, to + KBYTES + n * 4096 + wave * 1024);
  };
  // scales of the blocks that this lane's scores and weights lie in
  float ks_[NS], vs_[NS], next_ks[NS], next_vs[NS];
  auto load_scales = [&](int i, int ids) {
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      next_ks[s] = next_vs[s] = 1.f;
      if constexpr (F8)
        if (a.k_scales) {
          const int part = KW == 1 ? s : kw, key = tile_at(i) + 32 * part + 16 * h;
          const int lower = __builtin_amdgcn_readlane(ids, 2 * part), upper = __builtin_amdgcn_readlane(ids, 2 * part + 1);
          const size_t at = scale_index(a.d, h ? upper : lower, kvh, key & mask);
          if (seen_by_any(key, 16) != 0) {  // else it may be anything
            next_ks[s] = a.k_scales[at];
            next_vs[s] = a.v_scales[at];
          }
        }
    }
  };

  // the 16 bytes of K that are operand ks of part `part` of a tile (and the next one in 8 bits)
  const int k_row = 16 * (c >> 2 & 1) + 4 * (c >> 3) + (c & 3);
  auto k_piece = [&](const uint8_t *buf, int part, int ks) {
    return *(const u32x4_t *)(buf + (32 * part + k_row) * (KP * 16) + (((F8 ? ks & ~1 : 2 * ks) + h) ^ k_bits(k_row)) * 16);
  };
  // the 16 bytes of V^T that are operand u of part `part` of a tile for columns 32 n .. (both
  // operands of it in 8 bits)
  auto v_piece = [&](const uint8_t *buf, int n, int part, int u) {
    const int d = 32 * n + c;
    return *(const u32x4_t *)(buf + KBYTES + d * (VP * 16) + ((F8 ? 2 * part + h : 4 * part + 2 * h + u) ^ v_bits(d)) * 16);
  };

  f32x16 o[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[n][r] = 0.f;
  float m = -INFINITY, l = 0.f;
  uint32_t nans[NT / 2] = {};  // 16 bits for each of o
  const uint32_t lds0 = (uint32_t)(uintptr_t)lds_bytes;
  int ids = checked(next_ids, 0);
  load_tile(0, ids, lds0);
  load_scales(0, ids);
  if (tiles.count > 1) next_ids = page_ids(1);
  for (int i = 0; i < tiles.count; ++i) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();  // this tile is there, and everyone is done with the other buffer
    uint8_t *buf = lds_bytes + (i & 1) * BUF;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      ks_[s] = next_ks[s];
      vs_[s] = next_vs[s];
    }
    if (i + 1 < tiles.count) {
      ids = checked(next_ids, i + 1);
      load_tile(i + 1, ids, lds0 + ((i + 1) & 1) * BUF);
      load_scales(i + 1, ids);
      if (i + 2 < tiles.count) next_ids = page_ids(i + 2);
    }
    const int k0 = tile_at(i);
    const bool edge = (k0 < lo_max || k0 + TILE > hi_min) && k0 + TILE > first_min;
    uint32_t seen[NS];  // of this lane's scores
#pragma unroll
    for (int s = 0; s < NS; ++s) seen[s] = edge ? seen_by_mine(k0 + 32 * (KW == 1 ? s : kw) + 16 * h, 16) : 0xFFFFu;
    if (edge) {
      // What no column sees may be anything, and becomes zero: a thread looks at the pieces
      // of V^T that it loaded.  What only some see must not reach the others as 0 * NaN.
      u32x4_t *mine = (u32x4_t *)(buf + KBYTES + threadIdx.x * 16);
      const uint32_t any = seen_by_any(k0 + v_key, RUN);
      u32x4_t keep = {0, 0, 0, 0};
#pragma unroll
      for (int e = 0; e < RUN; ++e) keep[e * ESZ / 4] |= (any >> e & 1) ? (F8 ? 0xFFu : 0xFFFFu) << (e * ESZ % 4 * 8) : 0u;
      bool odd = false;
#pragma unroll
      for (int n = 0; n < V_PASSES; ++n) {
        const u32x4_t v = mine[n * 256] & keep;
        odd |= not_finite<F8>(v);
        mine[n * 256] = v;
      }
      if (__syncthreads_or(odd)) {  // columns that see such a value become NaN at the end, and it a zero
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            union {
              bf16x8 v;
              uint16_t e[8];
            } sees;
#pragma unroll
            for (int e = 0; e < 8; ++e) sees.e[e] = seen[s] >> (8 * u + e) & 1 ? 0x3F80u : 0u;
#pragma unroll 1  // rare: registers count for more
            for (int n = 0; n < NT; ++n) {
              u32x4_t raw = v_piece(buf, n, KW == 1 ? s : kw, u);
              f32x16 hits;
#pragma unroll
              for (int r = 0; r < 16; ++r) hits[r] = 0.f;
              hits = __builtin_amdgcn_mfma_f32_32x32x16_bf16(take_not_finite<F8>(raw, F8 ? u : 0), sees.v, hits, 0, 0, 0);
              uint32_t bits = 0;
#pragma unroll
              for (int r = 0; r < 16; ++r) bits |= hits[r] > 0.f ? 1u << r : 0u;
#pragma unroll
              for (int k = 0; k < NT / 2; ++k) nans[k] |= n / 2 == k ? bits << (n % 2 * 16) : 0u;
            }
          }
        __syncthreads();
#pragma unroll
        for (int n = 0; n < V_PASSES; ++n) {
          u32x4_t v = mine[n * 256];
#pragma unroll
          for (int u = 0; u < (F8 ? 2 : 1); ++u) (void)take_not_finite<F8>(v, u);
          mine[n * 256] = v;
        }
        __syncthreads();
      }
    }
    // scores, in powers of two
    f32x16 sc[NS];
    u32x4_t raw[NS];
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
      for (int r = 0; r < 16; ++r) sc[s][r] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        if (!F8 || ks % 2 == 0) raw[s] = k_piece(buf, KW == 1 ? s : kw, ks);
        const bf16x8 kf = operand_of<F8>(raw[s], ks & 1);
#pragma unroll
        for (int t = TERMS - 1; t >= 0; --t) sc[s] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[t][ks], sc[s], 0, 0, 0);
      }
    if constexpr (F8)
      if (a.k_scales) {
#pragma unroll
        for (int s = 0; s < NS; ++s) sc[s] *= ks_[s];
      }
    if (edge) {
      asm volatile("");  // a branch: the other tiles are spared three instructions a score
#pragma unroll
      for (int s = 0; s < NS; ++s)
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[s][r] = seen[s] >> r & 1 ? sc[s][r] : -INFINITY;
    }
    float mt = -INFINITY;
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
      for (int r = 0; r < 16; ++r) mt = fmaxf(mt, sc[s][r]);
    mt = max_pair32(mt);
    if (__ballot(mt > m + kKvRescale || m == -INFINITY)) {
      const float m1 = fmaxf(m, mt), f = m == m1 ? 1.f : __builtin_amdgcn_exp2f(m - m1);
      m = m1;
      l *= f;
#pragma unroll
      for (int n = 0; n < NT; ++n) o[n] *= f;
    }
    const float base = m == -INFINITY ? 0.f : m;  // nothing seen yet: every weight is 2^-inf
    // weights and outputs, 8 keys a lane at a time
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        bf16x8 pf[TERMS];
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float p = __builtin_amdgcn_exp2f(sc[s][8 * u + e] - base);
          sum[e & 1] += p;
          if constexpr (F8) {  // weights that are not seen stay zero whatever the scale is
            p *= vs_[s];
            if (edge) p = seen[s] >> (8 * u + e) & 1 ? p : 0.f;
          }
#pragma unroll
          for (int t = 0; t < TERMS; ++t) {
            pf[t][e] = (__bf16)p;
            p -= (float)pf[t][e];
          }
        }
        l += sum[0] + sum[1];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const bf16x8 vf = operand_of<F8>(v_piece(buf, n, KW == 1 ? s : kw, u), F8 ? u : 0);
#pragma unroll
          for (int t = TERMS - 1; t >= 0; --t) o[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[t], o[n], 0, 0, 0);
        }
      }
  }
  if (bad) raise_status(a.status, kStatusPage);
  l = sum_pair32(l);
  uint32_t any_nan = 0;
#pragma unroll
  for (int k = 0; k < NT / 2; ++k) any_nan |= nans[k];
  if (__ballot(any_nan != 0)) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[n][r] = nans[n / 2] >> (n % 2 * 16 + r) & 1 ? NAN : o[n][r];
  }

  // two waves with the same columns meet in LDS, the second's values in units of its maximum
  if constexpr (KW == 2) {
    __syncthreads();
    f32x4 *part = (f32x4 *)lds_bytes + cw * (NT * 4 * 64);
    float *ml = (float *)(lds_bytes + 64 * HD * 4) + cw * 128;
    if (kw == 1) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int k = 0; k < 4; ++k) part[(n * 4 + k) * 64 + lane] = f32x4{o[n][4 * k], o[n][4 * k + 1], o[n][4 * k + 2], o[n][4 * k + 3]};
      ml[lane] = m;
      ml[64 + lane] = l;
    }
    __syncthreads();
    if (kw == 1) return;
    const float m1 = ml[lane], l1 = ml[64 + lane], mx = fmaxf(m, m1);
    const float f0 = l != 0.f ? __builtin_amdgcn_exp2f(m - mx) : 0.f, f1 = l1 != 0.f ? __builtin_amdgcn_exp2f(m1 - mx) : 0.f;
    l = l * f0 + l1 * f1;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const f32x4 v = part[(n * 4 + k) * 64 + lane];
#pragma unroll
        for (int r = 0; r < 4; ++r) o[n][4 * k + r] = o[n][4 * k + r] * f0 + v[r] * f1;
      }
  }
  const int col = 32 * cw + c;
  if (col >= cols) return;
  const float scale = l != 0.f ? a.v_scale / l : 0.f;
  const int j = row_of(m0 + col);
  const int64_t oi = (int64_t)(sq.from + j) * a.ldo + (int64_t)(kvh * group + m0 + col - j * group) * HD + 4 * h;
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int64_t at = oi + 32 * n + 8 * k;
      const f32x4 v = f32x4{o[n][4 * k], o[n][4 * k + 1], o[n][4 * k + 2], o[n][4 * k + 3]} * scale;
      if (a.out_vec) {
        if constexpr (F32) *(f32x4 *)((float *)a.out + at) = v;
        else *(bf16x4 *)((__bf16 *)a.out + at) = bf16x4{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r) store_elem<F32>(a.out, at + r, v[r]);
      }
    }
}

template <int HD, bool F32, bool F8, int KW>
static hipError_t prompt_attr() {
  return hipFuncSetAttribute((const void *)kv_prompt_kernel<HD, F32, F8, KW>, hipFuncAttributeMaxDynamicSharedMemorySize,
                             prompt_lds_bytes<HD, F8, KW>());
}
template <int HD, bool F32, bool F8>
static hipError_t prompt_attrs() {
  const hipError_t e = prompt_attr<HD, F32, F8, 1>();
  return e == hipSuccess ? prompt_attr<HD, F32, F8, 2>() : e;
}
template <int HD>
static hipError_t prompt_attrs_of() {
  hipError_t e = prompt_attrs<HD, true, true>();
  if (e == hipSuccess) e = prompt_attrs<HD, true, false>();
  if (e == hipSuccess) e = prompt_attrs<HD, false, true>();
  if (e == hipSuccess) e = prompt_attrs<HD, false, false>();
  return e;
}
hipError_t kv_prompt_init(int head_dim) {
  return head_dim == 64 ? prompt_attrs_of<64>() : head_dim == 128 ? prompt_attrs_of<128>() : prompt_attrs_of<256>();
}

template <int HD, bool F32, bool F8, int KW>
static hipError_t launch_prompt_type(const KvRowsArgs &a, hipStream_t s) {
  // as many workgroups as any starts could need
  const int64_t grid = a.d.n_kv_heads * ((int64_t)a.n_rows * a.group / (128 / KW) + a.n_seqs);
  hipLaunchKernelGGL((kv_prompt_kernel<HD, F32, F8, KW>), dim3((unsigned)grid), dim3(256), (prompt_lds_bytes<HD, F8, KW>()), s, a);
  return hipGetLastError();
}
template <int HD, int KW>
static hipError_t launch_prompt_hd(const KvRowsArgs &a, bool f32, bool f8, hipStream_t s) {
  if (f32) return f8 ? launch_prompt_type<HD, true, true, KW>(a, s) : launch_prompt_type<HD, true, false, KW>(a, s);
  return f8 ? launch_prompt_type<HD, false, true, KW>(a, s) : launch_prompt_type<HD, false, false, KW>(a, s);
}

hipError_t launch_kv_prompt(const KvRowsArgs &a, int key_waves, bool f32, bool f8, hipStream_t s) {
  if (a.d.head_dim == 64) return key_waves == 1 ? launch_prompt_hd<64, 1>(a, f32, f8, s) : launch_prompt_hd<64, 2>(a, f32, f8, s);
  if (a.d.head_dim == 128) return key_waves == 1 ? launch_prompt_hd<128, 1>(a, f32, f8, s) : launch_prompt_hd<128, 2>(a, f32, f8, s);
  if (a.d.head_dim == 256) return key_waves == 1 ? launch_prompt_hd<256, 1>(a, f32, f8, s) : launch_prompt_hd<256, 2>(a, f32, f8, s);
  return hipErrorInvalidValue;
}

}  // namespace uad
