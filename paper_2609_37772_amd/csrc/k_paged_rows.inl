// Attention of new rows over a paged K/V cache: a prompt's, a few more of a conversation,
// or a single token of each sequence, with a sliding window and sinks; pools in bf16, or
// in 8 bits with one scale or one for every block of tokens.  What a row sees is in
// paged.h.
#include "paged_rows.h"

namespace uad {

// ---------------------------------------------------------------------------
// Few rows: the attention of one token (k_paged.inl) with other columns.  A unit is a KV
// head of a sequence with up to 16 (row, query head) pairs in the order of the rows, the
// 16 columns of the matrix instruction; each column has its own range of keys.  A
// sequence's tiles are those that any of its rows sees, counted without the gap that a
// window leaves behind the sinks, and are shared out in splits like the other's.
//
// Masks.  A tile that every column sees whole takes no part in them.  In any other, a
// score that its column does not see becomes -inf; what no column of the unit sees may be
// anything (slots never written, pages given back) and is zero in V.  A value that some
// columns see and others do not must not reach the others through 0 * NaN: values that
// are not finite are taken out, and the columns that see them become NaN.
//
// Precision: query and weights enter the matrix instructions as three bf16 terms (24 bits,
// all of an fp32 value); there is time for them while keys and values arrive.
//
// Bound by memory where there is much to read: a token of 64 sequences, window 4096, 32/8
// heads of 128, blocks of 8 bits: 547 MB in 105 us, 5.2 TB/s of the 6.2 that reads alone
// reach; 48 uneven ones of up to 16383 tokens 2.8 TB/s in 22.5 us, where the fixed cost of
// split units (plan, first loads, meeting, join: 7 to 8 us) does not overlap the reading.
// Else by that chain: a token with a window of 512 at head dim 256 12.0 us, up to 61 rows
// each on 20000 tokens of 5 sequences with a window of 1000 10.1.
// ---------------------------------------------------------------------------

template <int HD, bool F8>
__host__ __device__ constexpr RowsKind few_rows() { return {kTileKeys<F8>, 16, kAttendWhole<HD, F8>, kAttendMinTiles, false}; }

// SINGLE: a row for every sequence, so that all columns of a unit see the same keys.
template <int HD, bool F32, bool F8, bool SINGLE>
__global__ __launch_bounds__(64 * kAttendWaves, kAttendPerCu<HD> * kAttendWaves / 4) void kv_rows_kernel(KvRowsArgs a) {
  constexpr int TILE = kTileKeys<F8>, NT = TILE / 16, KPL = 4 * NT;
  constexpr int KS = HD / 32;           // k steps of Q K^T
  constexpr int KL = F8 ? HD / 64 : KS; // 16-byte loads of a key row per lane
  constexpr int NTO = HD / 16;          // 16-column tiles of the output
  constexpr int TERMS = kTerms;
  constexpr int NW = kAttendWaves;
  constexpr int ESZ = F8 ? 1 : 2;
  extern __shared__ __align__(16) float lds[];
  __bf16 *qf = (__bf16 *)lds;                       // [TERMS][KS][64][8]
  f32x4 *obuf = (f32x4 *)(lds + kQueryFloats<HD>);  // [NW][NTO][64]
  float *ml = (float *)(obuf + NW * NTO * 64);      // [NW or slots][16][2]
  float *top = ml + kAttendMl, *word = top + 32;
  static_assert((kPlanScans + 1) * NW + 3 <= kAttendMl, "the plan fits the slots' weights");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, g = lane >> 4;
  constexpr int HP = HD / 2, RS = 64 * NW / HP, QN = (16 + RS - 1) / RS;
  const int p = threadIdx.x % HP;
  int ea, eb;
  rope_pair(p, a.rope_dim, a.rope_pairs != 0, &ea, &eb);
  const bool turned = p < a.rope_dim / 2;
  const double turns = a.turns[p];  // 128 of them are allocated

  RowsWork w;
  if (!plan_rows<NW>(few_rows<HD, F8>(), a, blockIdx.x, (int *)ml, &w)) return;
  const int runs = w.s.units / a.d.n_kv_heads;
  const int kvh = w.unit / runs, m0 = (w.unit - kvh * runs) * 16, cols = min(16, w.s.n * a.group - m0);
  const int last = w.s.len - 1, mask = (1 << a.d.page_shift) - 1;
  const int32_t *table = a.table + (int64_t)w.b * a.pages_per_seq;
  // column m of the unit's sequence: row m / group, query head kvh * group + m % group
  auto row_of = [&](int m) { return SINGLE ? 0 : (int)((unsigned)m / (unsigned)a.group); };
  const int pos0 = w.s.len - w.s.n;  // of the sequence's first row
  auto from_of = [&](int col) { return seen_from(pos0 + row_of(m0 + col), a.window); };
  auto to_of = [&](int col) { return min(seen_to(pos0 + row_of(m0 + col), w.s.len, a.window, a.causal), w.s.len); };
  auto first_of = [&](int col) { return seen_first(pos0 + row_of(m0 + col), w.s.len, a.sinks, a.causal); };
  const int my_col = min(c, cols - 1), lo = from_of(my_col), hi = to_of(my_col), first = first_of(my_col);
  const int lo_min = from_of(0), lo_max = from_of(cols - 1), hi_min = to_of(0), hi_max = to_of(cols - 1);
  const int first_min = first_of(0), first_max = first_of(cols - 1);
  const SeenTiles tiles = SINGLE ? w.s.tiles : seen_tiles(max(hi_max, first_max), lo_min, a.sinks, TILE);
  if (!SINGLE && !w.of_unit(tiles.count)) return;
  auto tile_at = [&](int i) { return seen_tile(tiles, i) * TILE; };  // its first key
  // keys key .. key + n - 1 that some column sees, or this lane's column does, as bits
  auto seen_by_any = [&](int key, int n) { return run_bits(lo_min - key, hi_max - key, n) | run_bits(-key, first_max - key, n); };
  auto seen_by_mine = [&](int key, int n) { return run_bits(lo - key, hi - key, n) | run_bits(-key, first - key, n); };
  bool bad = false;

  // Loads are waited for in the order of their issue: page ids and the query's values
  // first, then the keys and values, which arrive while the query is rotated.
  auto page_ids = [&](int i, int &kp, int &vp) {
    const int k0 = tile_at(i);
    kp = table[min(k0 + KPL * (c >> 2), last) >> a.d.page_shift];
    vp = table[min(k0 + KPL * g, last) >> a.d.page_shift];
  };
  auto checked = [&](int page, int key) {  // of a run of keys; one that nobody sees is not looked at
    if (seen_by_any(key, KPL) == 0) return 0;
    const bool ok = page_ok(a.d, page);
    bad |= !ok;
    return ok ? page : 0;
  };
  u32x4_t kr[NT][KL], vr[NTO];
  float ks = 1.f, vs = 1.f, next_ks = 1.f, next_vs = 1.f;  // scales of the lane group's run
  auto load_k = [&](int i, int page, int v_page) {
    const int k0 = tile_at(i);
    const char *src = (const char *)a.kp + (page_base(a.d, checked(page, k0 + KPL * (c >> 2)), kvh) + (F8 ? 16 : 8) * g) * ESZ;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int off = min(k0 + KPL * (c >> 2) + 4 * t + (c & 3), last) & mask;
#pragma unroll
      for (int j = 0; j < KL; ++j) kr[t][j] = *(const u32x4_t *)(src + (unsigned)(off * HD * ESZ) + j * 64);
    }
    if constexpr (F8)
      if (a.k_scales) {
        const int key = k0 + KPL * g;
        const size_t at = scale_index(a.d, checked(v_page, key), kvh, min(key, last) & mask);
        const bool seen = seen_by_any(key, KPL) != 0;  // else the scale may be anything
        next_ks = seen ? a.k_scales[at] : 1.f;
        next_vs = seen ? a.v_scales[at] : 1.f;
      }
  };
  auto load_v = [&](int i, int page) {
    const int key = tile_at(i) + KPL * g, off = min(key, last & ~(KPL - 1)) & mask;
    const char *src = (const char *)a.vp + (page_base(a.d, checked(page, key), kvh) + off + (c << a.d.page_shift)) * ESZ;
#pragma unroll
    for (int n = 0; n < NTO; ++n) vr[n] = *(const u32x4_t *)(src + (unsigned)((n * 16 << a.d.page_shift) * ESZ));
  };

  const int t0 = split_begin(tiles.count, w.splits, w.split);
  int tile = t0 + wave;
  const int t1 = last >= 0 ? split_begin(tiles.count, w.splits, w.split + 1) : 0;
  int kp = 0, vp = 0, next_kp = 0, next_vp = 0;
  if (tile < t1) page_ids(tile, kp, vp);
  if (tile + NW < t1) page_ids(tile + NW, next_kp, next_vp);
  uint32_t qx[QN], qy[QN];
  int position[QN];
#pragma unroll
  for (int i = 0; i < QN; ++i) {
    const int m = m0 + min((int)threadIdx.x / HP + i * RS, cols - 1), j = row_of(m);
    const int64_t qi = (int64_t)(w.s.from + j) * a.ldq + (int64_t)(kvh * a.group + m - j * a.group) * HD;
    position[i] = a.positions ? a.positions[w.s.from + j] : pos0 + j;
    qx[i] = load_raw<F32>(a.q, qi + ea);
    qy[i] = load_raw<F32>(a.q, qi + eb);
  }
  if (tile < t1) {
    load_k(tile, kp, vp);
    load_v(tile, vp);
  }

  // the query, rotated, as bf16 terms in operand order; columns past the unit's are zero
  {
    auto at = [&](int e, int row) {  // operand element of column e
      if constexpr (F8) return (((e >> 6) * 2 + ((e >> 3) & 1)) * 64 + ((e >> 4) & 3) * 16 + row) * 8 + (e & 7);
      else return ((e >> 5) * 64 + ((e >> 3) & 3) * 16 + row) * 8 + (e & 7);
    };
#pragma unroll
    for (int i = 0; i < QN; ++i) {
      const int col = threadIdx.x / HP + i * RS;
      if (col >= 16) break;
      float sn = 0.f, cs = 1.f;
      if (turned) turn_of(turns, position[i], &sn, &cs);
      const float x = col < cols ? value_of<F32>(qx[i]) : 0.f, y = col < cols ? value_of<F32>(qy[i]) : 0.f;
      float v0 = turned ? x * cs - y * sn : x, v1 = turned ? y * cs + x * sn : y;
#pragma unroll
      for (int t = 0; t < TERMS; ++t) {
        const __bf16 h0 = (__bf16)v0, h1 = (__bf16)v1;
        qf[t * KS * 512 + at(ea, col)] = h0;
        qf[t * KS * 512 + at(eb, col)] = h1;
        v0 -= (float)h0;
        v1 -= (float)h1;
      }
    }
  }
  __syncthreads();

  f32x4 o[NTO];
#pragma unroll
  for (int n = 0; n < NTO; ++n) o[n] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  for (; tile < t1; tile += NW) {
    // the query's operands are read anew for every tile: kept, they would take up to 96
    // registers from the tiles in flight
    asm volatile("" ::: "memory");
    f32x4 s[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kb = 0; kb < KS; ++kb) {
      bf16x8 qt[TERMS];
#pragma unroll
      for (int i = 0; i < TERMS; ++i) qt[i] = *(const bf16x8 *)(qf + ((i * KS + kb) * 64 + lane) * 8);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const bf16x8 kf = operand_of<F8>(kr[t][F8 ? kb / 2 : kb], kb & 1);
#pragma unroll
        for (int i = TERMS - 1; i >= 0; --i) s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qt[i], s[t], 0, 0, 0);
      }
    }
    ks = next_ks;
    vs = next_vs;
    vp = next_vp;
    const bool more = tile + NW < t1;
    if (more) {
      kp = next_kp;
      if (tile + 2 * NW < t1) page_ids(tile + 2 * NW, next_kp, next_vp);
      load_k(tile + NW, kp, vp);
    }
    // scores in powers of two, keys that the column does not see masked
    const int k0 = tile_at(tile), key0 = k0 + KPL * g;
    const bool edge = (k0 < lo_max || k0 + TILE > hi_min) && k0 + TILE > first_min;
    const uint32_t seen = !edge ? 0xFFFFFFFFu : SINGLE ? seen_by_any(key0, KPL) : seen_by_mine(key0, KPL);
    const float to_log2 = F8 ? a.scale_log2 * ks : a.scale_log2;
    float mt = -INFINITY;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float v = s[t][r] * to_log2;
        if (edge && !(seen >> (4 * t + r) & 1)) v = -INFINITY;
        s[t][r] = v;
        mt = fmaxf(mt, v);
      }
    mt = max_pair32(max_pair16(mt));
    // the running maximum is raised when it is passed by more than 2^8 (the weights
    // stay below that); all lanes of a query agree
    if (__ballot(mt > m + kKvRescale || m == -INFINITY)) {
      const float m1 = fmaxf(m, mt), f = m == m1 ? 1.f : __builtin_amdgcn_exp2f(m - m1);
      m = m1;
      l *= f;
#pragma unroll
      for (int n = 0; n < NTO; ++n) o[n] *= f;
    }
    const float unit = m == -INFINITY ? 0.f : m;  // nothing seen yet: every weight is 2^-inf
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        s[t][r] = __builtin_amdgcn_exp2f(s[t][r] - unit);
        l += s[t][r];
        if constexpr (F8) {  // weights that are not seen stay zero whatever the scale is
          const float v = s[t][r] * vs;
          s[t][r] = edge && !(seen >> (4 * t + r) & 1) ? 0.f : v;
        }
      }
    bool odd = false;
    if (edge) {
      constexpr int PER = F8 ? 4 : 2;  // elements of a register
      const uint32_t any = seen_by_any(key0, KPL);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t keep = 0;
#pragma unroll
        for (int e = 0; e < PER; ++e) keep |= (any >> (i * PER + e) & 1) ? (F8 ? 0xFFu : 0xFFFFu) << (e * 32 / PER) : 0u;
#pragma unroll
        for (int k = 0; k < NTO; ++k) vr[k][i] &= keep;
      }
      if constexpr (!SINGLE) {
#pragma unroll
        for (int k = 0; k < NTO; ++k) odd |= not_finite<F8>(vr[k]);
        odd = __ballot(odd) != 0;
      }
    }
#pragma unroll
    for (int u = 0; u < NT / 2; ++u) {  // 8 weights of the lane, as terms
      if (!SINGLE && odd) {
        union {
          bf16x8 v;
          uint16_t e[8];
        } sees;
#pragma unroll
        for (int e = 0; e < 8; ++e) sees.e[e] = seen >> (8 * u + e) & 1 ? 0x3F80u : 0u;
#pragma unroll
        for (int n = 0; n < NTO; ++n) {
          const bf16x8 vf = take_not_finite<F8>(vr[n], u);
          const f32x4 hits = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, sees.v, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
          for (int r = 0; r < 4; ++r) o[n][r] = hits[r] > 0.f ? NAN : o[n][r];
        }
      }
      union {
        bf16x8 v;
        __bf16 e[8];
      } pf[TERMS];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float q = s[2 * u + e / 4][e % 4];
#pragma unroll
        for (int i = 0; i < TERMS; ++i) {
          pf[i].e[e] = (__bf16)q;
          q -= (float)pf[i].e[e];
        }
      }
#pragma unroll
      for (int n = 0; n < NTO; ++n) {
        const bf16x8 vf = operand_of<F8>(vr[n], u);
#pragma unroll
        for (int i = TERMS - 1; i >= 0; --i) o[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[i].v, o[n], 0, 0, 0);
      }
    }
    if (more) load_v(tile + NW, vp);
  }
  if (bad) raise_status(a.status, kStatusPage);

  // The waves meet: maxima, sums and outputs, each in units of its wave's maximum, of half
  // the waves where no others had a tile.
  const bool all = t1 - t0 > NW / 2;
  l = sum_pair32(sum_pair16(l));
  if (g == 0) {
    ml[(wave * 16 + c) * 2] = m;
    ml[(wave * 16 + c) * 2 + 1] = l;
  }
  if (c < cols && (all || wave < NW / 2))
#pragma unroll
    for (int n = 0; n < NTO; ++n) obuf[(wave * NTO + n) * 64 + lane] = o[n];
  __syncthreads();
  float mx = -INFINITY, sum = 0.f, f[NW];
#pragma unroll
  for (int i = 0; i < NW; ++i) mx = fmaxf(mx, ml[(i * 16 + c) * 2]);
#pragma unroll
  for (int i = 0; i < NW; ++i) {
    const float li = ml[(i * 16 + c) * 2 + 1];
    f[i] = li != 0.f ? __builtin_amdgcn_exp2f(ml[(i * 16 + c) * 2] - mx) : 0.f;
    sum += li * f[i];
  }
  const bool vec = a.out_vec;
  auto put_out = [&](int col, int e, f32x4 v, float total) {
    const float scale = total != 0.f ? a.v_scale / total : 0.f;
    const int j = row_of(m0 + col);
    const int64_t oi = (int64_t)(w.s.from + j) * a.ldo + (int64_t)(kvh * a.group + m0 + col - j * a.group) * HD + e;
    v *= scale;
    if (vec) {
      if constexpr (F32) *(f32x4 *)((float *)a.out + oi) = v;
      else *(bf16x4 *)((__bf16 *)a.out + oi) = bf16x4{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r) store_elem<F32>(a.out, oi + r, v[r]);
    }
  };
  const int slot = w.slot + w.split;
  const auto slots = slots_of(a, 16 * HD);
  if (c < cols) {
    for (int n = wave; n < NTO; n += NW) {
      f32x4 v = obuf[n * 64 + lane] * f[0];
#pragma unroll
      for (int i = 1; i < NW / 2; ++i) v += obuf[(i * NTO + n) * 64 + lane] * f[i];
      if (all)
#pragma unroll
        for (int i = NW / 2; i < NW; ++i) v += obuf[(i * NTO + n) * 64 + lane] * f[i];
      if (w.splits == 1) put_out(c, 16 * n + 4 * g, v, sum);
      else put_slot(slots, (slot * 16 + c) * HD + 16 * n + 4 * g, v);
    }
    if (w.splits > 1 && wave == 0 && g == 0)
      __hip_atomic_store(a.part_ml + (size_t)slot * 16 + c, pair_of(mx, sum), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  if (w.splits == 1) return;

  // many splits: runs of kJoinFan first, into the first slot of each
  bool final = w.splits <= 2 * kJoinFan;
  for (;;) {
    const int run = w.split / kJoinFan * kJoinFan;
    const int from = final ? w.slot : w.slot + run, step = final && w.splits > 2 * kJoinFan ? kJoinFan : 1;
    const int n = !final ? min(kJoinFan, w.splits - run) : (w.splits + step - 1) / step;
    if (!last_to_arrive(a.arrived + (final ? a.slots : 0) + from, n, word)) return;
    join_slots<HD>(a, cols, 16, from, step, n, ml, top, obuf, [&](int col, int e, f32x4 v, float total) {
      if (final) put_out(col, e, v, total);
      else put_slot(slots, (from * 16 + col) * HD + e, v);
    });
    if (final) return;
    if ((int)threadIdx.x < cols)
      __hip_atomic_store(a.part_ml + (size_t)from * 16 + threadIdx.x,
                         pair_of(top[2 * threadIdx.x], top[2 * threadIdx.x + 1]), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    final = true;
  }
}

template <int HD, bool F32, bool F8>
static hipError_t rows_attr() {
  hipError_t e = hipSuccess;
  for (const void *f : {(const void *)kv_rows_kernel<HD, F32, F8, false>, (const void *)kv_rows_kernel<HD, F32, F8, true>})
    if (e == hipSuccess) e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, attend_lds_floats<HD>() * 4);
  return e;
}
template <int HD>
static hipError_t rows_attrs() {
  hipError_t e = rows_attr<HD, true, true>();
  if (e == hipSuccess) e = rows_attr<HD, true, false>();
  if (e == hipSuccess) e = rows_attr<HD, false, true>();
  if (e == hipSuccess) e = rows_attr<HD, false, false>();
  return e;
}
hipError_t kv_rows_init(int head_dim) {
  const hipError_t e = head_dim == 64 ? rows_attrs<64>() : head_dim == 128 ? rows_attrs<128>() : rows_attrs<256>();
  return e == hipSuccess ? kv_prompt_init(head_dim) : e;
}

template <int HD, bool F32, bool F8>
static hipError_t launch_rows_type(KvRowsArgs a, hipStream_t s) {
  const RowsGrid grid = rows_grid(few_rows<HD, F8>(), a.n_rows, a.n_seqs, a.row_start != nullptr, a.d.n_kv_heads, a.group,
                                  (int64_t)a.pages_per_seq << a.d.page_shift, a.window, a.sinks, a.target, a.slots);
  a.unsplit = grid.unsplit;
  const dim3 wgs((unsigned)grid.wgs), wg(64 * kAttendWaves);
  constexpr int lds = attend_lds_floats<HD>() * 4;
  if (a.row_start) hipLaunchKernelGGL((kv_rows_kernel<HD, F32, F8, false>), wgs, wg, lds, s, a);
  else hipLaunchKernelGGL((kv_rows_kernel<HD, F32, F8, true>), wgs, wg, lds, s, a);
  return hipGetLastError();
}

template <int HD>
static hipError_t launch_rows_hd(const KvRowsArgs &a, bool f32, bool f8, hipStream_t s) {
  if (f32) return f8 ? launch_rows_type<HD, true, true>(a, s) : launch_rows_type<HD, true, false>(a, s);
  return f8 ? launch_rows_type<HD, false, true>(a, s) : launch_rows_type<HD, false, false>(a, s);
}

// Which kernel: 0: that of few rows; else the waves that share a column of that of many.
// The kernel of few rows reads a KV head's cache for every 16 columns, that of many for 64
// or 128, with more to do before and after: the one loses from a size of the query on, the
// sooner the longer the histories are, which the launch does not know.  us, few rows / many
// (two waves a column): one causal sequence with nothing, 1500 and 8000 tokens before its
// rows, 16/2 heads of 256 and 32/8 of 128 and 64; last, their ratio over these, 8 sequences of
// an eighth of the rows, and other heads (8/1, 12/2, 4/4):
//   query    bf16                                          8 bits
//   256
//    65k     11.9 / 15.5   25.1 / 27.4   40.3 / 48.3  0.90  14.7 / 15.8   22.0 / 29.0   32.9 / 50.1  0.83
//   130k     12.1 / 15.4   27.8 / 28.3   60.4 / 44.1  1.05  14.7 / 15.9   22.8 / 29.7   44.1 / 47.7  0.91
//   260k     12.9 / 15.5   36.8 / 29.3  100.8 / 45.4  1.35  15.0 / 16.0   29.7 / 31.9   67.3 / 49.7  1.07
//   520k     15.3 / 17.8   53.3 / 29.5  182.9 / 65.1  1.68  15.8 / 19.0   41.0 / 32.5  115.1 / 70.1  1.23
//   128
//   130k      7.6 / 11.0   17.9 / 20.9   40.6 / 31.0  0.92   9.4 / 11.1   17.5 / 21.8   30.8 / 33.8  0.84
//   260k      8.0 / 11.1   24.2 / 21.3   68.9 / 43.1  1.07   9.4 / 11.2   21.2 / 22.8   45.1 / 46.8  0.87
//   520k      8.9 / 12.6   33.5 / 24.5  122.9 / 66.1  1.33   9.8 / 13.4   24.5 / 28.0   72.4 / 76.3  0.93
//  1040k     20.8 / 16.2   64.0 / 34.6  241.7 / 117   1.75  19.2 / 17.7   43.6 / 39.9  139.2 / 137.6 1.16
//   64
//   130k      6.4 /  8.7   16.4 / 19.4   39.0 / 30.7  0.94   7.7 /  8.8   17.3 / 20.3   31.3 / 33.8  0.85
//   260k      6.8 / 10.0   22.2 / 20.0   67.9 / 41.6  1.15   7.8 / 10.3   21.8 / 21.7   50.8 / 47.9  0.96
//   520k     10.6 / 12.5   31.9 / 23.7  122.9 / 69.1  1.37  10.4 / 13.6   27.1 / 26.6   87.8 / 80.6  1.02
// The kernel of many takes over where that ratio passes 1.  Prompts without a history lose by
// that up to a million elements, 3 to 5 us of 9 to 18.
// With few columns a sequence its units would be mostly empty.  64 sequences with 1000 tokens
// before their rows, few / many: of 16 columns 54.1 / 83.9 (32/8 heads of 128), 35.3 / 44.6 (of
// 64), 50.8 / 37.6 (16/2 of 256); of 32 96.8 / 85.9, 46.4 / 45.9, 118 / 39; in 8 bits of 32 76 /
// 93, 39.1 / 50.6, 52.4 / 42.0; of 64 141 / 99, 69.5 / 53.3, 97.9 / 52.
// Two waves share a column where units of 128 columns would be half empty or too few to fill
// the chip: from 256 full ones on one wave a column is as fast or faster, but for a single
// sequence's causal rows at 256 of them (two waves / one: 256, 400 and 1024 units of 16/2 heads
// of 256, one sequence with 1500 tokens before its rows 222 / 242, 456 / 386, 1795 / 1560; of
// 32/8 of 128 124 / 139, 247 / 189, 785 / 600; of 64 71 / 80, 128 / 118, 408 / 343; 16
// sequences of 32/8 of 128 104 / 96, 194 / 138, 404 / 291; below 256 of them, 128 full ones, 61
// / 113).
static int prompt_key_waves(const KvRowsArgs &a, bool f8) {
  const int64_t columns = (int64_t)a.n_rows * a.group;
  const int64_t few = a.d.head_dim == 256 ? (f8 ? 200000 : 130000) : !f8 ? 250000 : a.d.head_dim == 128 ? 650000 : 500000;
  const int least = a.d.head_dim == 256 ? 16 : f8 ? 33 : 17;  // columns of a sequence, on average
  if (!a.row_start || columns < least * (int64_t)a.n_seqs || columns * a.d.n_kv_heads * a.d.head_dim < few) return 0;
  return columns < 128 * (int64_t)a.n_seqs || columns / 128 * a.d.n_kv_heads < 256 ? 2 : 1;
}

hipError_t launch_kv_rows(const KvRowsArgs &a, bool f32, bool f8, hipStream_t s) {
  if (a.n_seqs < 1 || a.n_rows < 1 || a.group < 1 || a.n_heads != a.group * a.d.n_kv_heads || a.pages_per_seq < 1 ||
      a.target < 1 || a.slots < max_slots(a.target) || a.d.page_shift < 4 || a.window < 0 || a.sinks < 0 ||
      (!a.row_start && a.n_rows != a.n_seqs) || (!f8 && a.k_scales))
    return hipErrorInvalidValue;
  const int key_waves = prompt_key_waves(a, f8);
  if (key_waves) return launch_kv_prompt(a, key_waves, f32, f8, s);
  if (a.d.head_dim == 64) return launch_rows_hd<64>(a, f32, f8, s);
  if (a.d.head_dim == 128) return launch_rows_hd<128>(a, f32, f8, s);
  if (a.d.head_dim == 256) return launch_rows_hd<256>(a, f32, f8, s);
  return hipErrorInvalidValue;
}

}  // namespace uad
