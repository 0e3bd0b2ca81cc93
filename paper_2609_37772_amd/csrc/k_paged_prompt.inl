// Attention of many new rows over a paged K/V cache.
#include "paged_rows.h"

namespace uad {

// ---------------------------------------------------------------------------
// Many rows: bound by the matrix instructions.  A unit is a KV head of a sequence with up
// to 128 (row, query head) pairs, its columns; each of its waves takes 32 of them (or 16,
// where 32 columns' outputs and query would leave a SIMD one wave).  For calls with too few
// units to fill the chip a unit has 64 columns, and two waves share theirs and take half of
// every tile's keys each.
//
// S^T = K Q^T and O^T = V^T P^T with v_mfma_f32_32x32x16_bf16 (16x16x32): rows of K enter in
// an order in which each group of lanes ends with the scores of 16 (8) consecutive keys,
// which are its operand of the P V product as they stand.  Tiles of 64 keys go from memory
// to LDS past the registers, the next one while this one is worked on; a 16-byte piece p
// of a row lies at piece p ^ (a few bits of the row), so that rows that are read at once do
// not meet in a bank.  The query is held in registers, rotated and scaled in fp32 on the way.
//
// Precision: the query and the weights enter as three bf16 terms (24 bits, all of an fp32
// value), as in the kernel of few rows: a row is held in no fewer bits for others that its
// call has.  Keys and values as stored.
//
// Measured: one causal prompt of 8191 rows, 32/8 heads of 128: 1300 to 1360 us, with three
// terms 1.2 to 1.27 PFLOP/s of the 1.3 to 1.4 that a library's large products reach; 816 rows
// that all see each other, 8/1 heads of 256: 35 us; 16 prompts of up to 1024 rows in 8 bits,
// 12/2 heads of 128: 91 us, not much more than the one unit with the most tiles takes.
//
// Masks as in the kernel of few rows: what no column sees is zero in V, and values that are
// not finite where some columns do not see them are taken out of LDS and noted for those
// that do.
// ---------------------------------------------------------------------------
constexpr int kPromptTile = 64;
// Tiles of a split at least, and those up to which a unit stays whole: a split costs the query
// anew and a join, which take as long as 3 tiles.  102 units of 13 tiles at head dim 256:
// 43.6 us whole, 35.1 us in two; 32 units of 63: 158 whole, 46 split.
template <int KW>
__host__ __device__ constexpr RowsKind many_rows() { return {kPromptTile, 128 / KW, 6, 3, true}; }

// Columns of a wave: outputs and query take it columns x head dim x (4 + 2 terms) bytes,
// and two waves are to share a SIMD's 512 registers.  At head dim 128 32 columns leave 18 of
// the query's registers (28 with 8-bit pools) to be read again from memory for every tile, and
// are faster all the same than 16, which read each operand from LDS for half as many columns:
// a prompt of 8191 rows 1357 us for 1433, 16 of up to 1024 rows in 8 bits 92 for 99.  Where
// workgroups are too few to fill the chip, 16 columns give each of them twice the waves: 8
// sequences of 64 rows in 8 bits 73 us for 81; at 64 a tile of 8 bits has fewer pieces than
// twice the threads.
template <int HD, int KW>
constexpr int kPromptCols = (KW == 2 && HD == 128) || HD == 256 ? 16 : 32;
template <int HD, int KW>
constexpr int kPromptThreads = 64 * 128 / kPromptCols<HD, KW>;

// LDS: two buffers of a tile's K and V^T; before that the query in fp32 (in the first buffer
// and where two waves share columns, which are calls that wait for latency, no further, so
// that the first tile can be on its way to the second), after it, where waves share
// columns, one's outputs, maxima and sums.
template <int HD, bool F8, int KW>
struct PromptLds {
  static constexpr int buffer = 2 * kPromptTile * HD * (F8 ? 1 : 2), query = 128 / KW * HD * 4;
  static constexpr int second = KW == 2 && query > buffer ? query : buffer;  // where the second buffer lies
  static constexpr int meeting = KW == 2 ? 64 * HD * 4 + 4 * 2 * 64 * 4 : 0;
  static constexpr int tiles = second + buffer, most = tiles > query ? tiles : query;
  static constexpr int bytes = most > meeting ? most : meeting;
};

typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16;

// The matrix instruction of a wave with C columns: rows x C results, lane (c, g) has those
// of column c and rows 4 g + 4 GROUPS k + r at 4 k + r.
template <int C>
struct Product;
template <>
struct Product<32> {
  typedef f32x16 acc;
  static constexpr int values = 16;
  static __device__ __forceinline__ acc of(bf16x8 a, bf16x8 b, acc c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Product<16> {
  typedef f32x4 acc;
  static constexpr int values = 4;
  static __device__ __forceinline__ acc of(bf16x8 a, bf16x8 b, acc c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};

// 16 bytes per lane from memory to LDS at `to` + 16 * lane, by the lanes of `mask` (all or
// none: a branch would part the instructions that these loads are to lie between).  The
// compiler would wait for each before the next read of LDS: the kernel waits itself, once
// per tile.  No reads of LDS are held back by it either: they are on the other side of a
// barrier, or of the other buffer.
__device__ __forceinline__ void load_to_lds(const void *from, uint32_t to, uint64_t mask) {
  uint32_t kept;  // m0 and exec are the compiler's
  uint64_t lanes;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b64 %1, exec\n\ts_mov_b32 m0, %2\n\ts_mov_b64 exec, %4\n\ts_nop 0\n\t"
               "global_load_lds_dwordx4 %3, off\n\ts_mov_b64 exec, %1\n\ts_mov_b32 m0, %0"
               : "=&s"(kept), "=&s"(lanes) : "s"(to), "v"(from), "s"(mask));
}
// The same from an address that is one for the wave and an offset below 2^31.
__device__ __forceinline__ void load_to_lds(const void *base, uint32_t offset, uint32_t to, uint64_t mask) {
  uint32_t kept;
  uint64_t lanes;
  const uint64_t at = (uint64_t)base;
  base = (const void *)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(at >> 32)) << 32 |
                        (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)at));
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b64 %1, exec\n\ts_mov_b32 m0, %2\n\ts_mov_b64 exec, %5\n\ts_nop 0\n\t"
               "global_load_lds_dwordx4 %3, %4\n\ts_mov_b64 exec, %1\n\ts_mov_b32 m0, %0"
               : "=&s"(kept), "=&s"(lanes) : "s"(to), "v"(offset), "s"(base), "s"(mask));
}

template <int HD, bool F32, bool F8, int KW>
__global__ __launch_bounds__((kPromptThreads<HD, KW>), 2) void kv_prompt_kernel(KvRowsArgs a) {
  using Lds = PromptLds<HD, F8, KW>;
  constexpr int C = kPromptCols<HD, KW>, THREADS = kPromptThreads<HD, KW>, NW = THREADS / 64;
  using Mul = Product<C>;
  typedef typename Mul::acc acc;
  constexpr int VAL = Mul::values, GROUPS = 64 / C;   // results a lane; groups of lanes
  constexpr int TILE = kPromptTile, COLS = 128 / KW, NS = 2 / KW;  // NS: 32-key parts of a tile that a wave takes
  constexpr int RUN = 32 / GROUPS;                    // consecutive keys of a part that a lane has
  constexpr int MK = 32 / C;                          // products of a part: 32 keys in rows of C
  constexpr int K = 8 * GROUPS, KS = HD / K;          // depth of a product, steps of Q K^T
  constexpr int NT = HD / C;                          // output tiles
  constexpr int TERMS = kTerms, ESZ = F8 ? 1 : 2;
  constexpr int KP = HD * ESZ / 16, VP = TILE * ESZ / 16;  // 16-byte pieces of a row of K, of V^T
  constexpr int KBYTES = TILE * HD * ESZ, PIECE = 16 / ESZ;  // keys of a piece of V^T
  extern __shared__ __align__(16) uint8_t lds_bytes[];
  __shared__ int plan[(kPlanScans + 2) * NW + 3];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane % C, g = lane / C;
  const int cw = wave / KW, kw = wave % KW;

  // the unit: sequences' units side by side, a sequence's last rows first (where rows are
  // causal they see the most), its KV heads next to each other
  const int group = a.group;
  constexpr bool SPLITS = KW == 2;
  RowsWork w;
  if (!plan_rows<NW>(many_rows<KW>(), a, blockIdx.x, plan, &w)) return;
  const RowsSeq sq = w.s;
  const int runs = sq.units / a.d.n_kv_heads;
  const int run = runs - 1 - w.unit / a.d.n_kv_heads, kvh = w.unit % a.d.n_kv_heads;
  const int m0 = run * COLS, cols = min(COLS, sq.n * group - m0);
  const int last = sq.len - 1, mask = (1 << a.d.page_shift) - 1, pos0 = sq.len - sq.n;
  const int32_t *table = a.table + (int64_t)w.b * a.pages_per_seq;
  auto row_of = [&](int m) { return (int)((unsigned)m / (unsigned)group); };
  auto from_at = [&](int p) { return seen_from(p, a.window); };
  auto to_at = [&](int p) { return min(seen_to(p, sq.len, a.window, a.causal), sq.len); };
  auto first_at = [&](int p) { return seen_first(p, sq.len, a.sinks, a.causal); };
  const int p_min = pos0 + row_of(m0), p_max = pos0 + row_of(m0 + cols - 1), p_mine = pos0 + row_of(m0 + min(C * cw + c, cols - 1));
  const int lo = from_at(p_mine), hi = to_at(p_mine), first = first_at(p_mine);
  const int lo_min = from_at(p_min), lo_max = from_at(p_max), hi_min = to_at(p_min), hi_max = to_at(p_max);
  const int first_min = first_at(p_min), first_max = first_at(p_max);
  const SeenTiles tiles = seen_tiles(max(hi_max, first_max), lo_min, a.sinks, TILE);
  if (SPLITS && !w.of_unit(tiles.count)) return;
  const int t0 = SPLITS ? split_begin(tiles.count, w.splits, w.split) : 0;
  const int n_tiles = SPLITS ? split_begin(tiles.count, w.splits, w.split + 1) - t0 : tiles.count;
  auto tile_at = [&](int i) { return seen_tile(tiles, t0 + i) * TILE; };
  auto seen_by_any = [&](int key, int n) { return run_bits(lo_min - key, hi_max - key, n) | run_bits(-key, first_max - key, n); };
  auto seen_by_mine = [&](int key, int n) { return run_bits(lo - key, hi - key, n) | run_bits(-key, first - key, n); };
  bool bad = false;

  // Page ids of a tile's four runs of 16 keys, in lanes 0 .. 3 (and every four more).
  auto page_ids = [&](int i) { return table[min(tile_at(i) + 16 * (lane & 3), last) >> a.d.page_shift]; };
  auto checked = [&](int id, int i) {
    const int k0 = tile_at(i);
    const bool whole = k0 >= lo_min && k0 + TILE <= hi_max;
    if (!whole && seen_by_any(k0 + 16 * (lane & 3), 16) == 0) return 0;  // not looked at
    const bool ok = page_ok(a.d, id);
    bad |= !ok;
    return ok ? id : 0;
  };

  // Loads of a tile into the buffer at `to`.  K: thread t of pass n takes piece n * THREADS + t,
  // of a row whose run of 16 is one for the wave; V^T: the same keys of other columns in every
  // pass.
  constexpr int K_PASSES = TILE * KP / THREADS, V_PASSES = HD * VP / THREADS, V_ROWS = THREADS / VP;
  static_assert(K_PASSES > 0 && V_PASSES > 0 && V_ROWS % 8 == 0, "every thread has a piece in every pass");
  auto k_bits = [&](int key) {  // of the 8 rows that are read at once
    const int far = key >> (C == 32 ? 4 : 3) & 1;
    return KP == 4 ? (key >> 1 & 1) | far << 1 : (key & 3) | far << 2;
  };
  auto v_bits = [&](int d) { return VP == 4 ? d >> 1 & 3 : d & 7; };
  const int v_row = threadIdx.x / VP, v_key = ((threadIdx.x % VP) ^ v_bits(v_row)) * PIECE;
  const uint32_t v_offset = (((uint32_t)v_row << a.d.page_shift) + (v_key & 15)) * ESZ;
  // The loads of a tile are shared out over the products of the one before: issued all at
  // once they held a wave up for 1000 to 1800 clocks a tile.
  int next_k0 = 0, next_pages = 0;  // pages in lanes 0 .. 3
  const char *next_v = nullptr;     // this thread's first piece of V^T
  uint32_t next_to = 0;
  uint64_t next_mask = 0;
  auto plan_tile = [&](int i, int ids, uint32_t to, int real) __attribute__((always_inline)) {
    next_k0 = __builtin_amdgcn_readfirstlane(tile_at(i));
    next_pages = ids;
    const int r = v_key >> 4, page = __shfl(ids, r);
    next_v = (const char *)a.vp + (page_base(a.d, page, kvh) + ((next_k0 + 16 * r) & mask)) * ESZ + v_offset;
    next_to = __builtin_amdgcn_readfirstlane(to);
    next_mask = (uint64_t)(int64_t)__builtin_amdgcn_readfirstlane(real >> 31);
  };
  auto load_k = [&](int n) __attribute__((always_inline)) {
    const int row = (n * THREADS + (int)threadIdx.x) / KP, p = (n * THREADS + (int)threadIdx.x) % KP;
    const int r = (n * THREADS + wave * 64) / KP / 16;  // one for the wave
    load_to_lds((const char *)a.kp + (page_base(a.d, __builtin_amdgcn_readlane(next_pages, r), kvh) + k_in_page(a.d, (next_k0 + 16 * r) & mask, 0)) * ESZ,
                (uint32_t)((row & 15) * HD * ESZ + (p ^ k_bits(row)) * 16), next_to + (n * THREADS + wave * 64) * 16, next_mask);
  };
  auto load_v = [&](int n) __attribute__((always_inline)) {
    load_to_lds(next_v + ((size_t)(n * V_ROWS) << a.d.page_shift) * ESZ, next_to + KBYTES + (n * THREADS + wave * 64) * 16, next_mask);
  };
  // scales of the blocks that this lane's scores and weights lie in
  float ks_[NS], vs_[NS], next_ks[NS], next_vs[NS];
  auto load_scales = [&](int i, int ids) {
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      next_ks[s] = next_vs[s] = 1.f;
      if constexpr (F8)
        if (a.k_scales) {
          const int part = KW == 1 ? s : kw, key = tile_at(i) + 32 * part + RUN * g;
          const int lower = __builtin_amdgcn_readlane(ids, 2 * part), upper = __builtin_amdgcn_readlane(ids, 2 * part + 1);
          const size_t at = scale_index(a.d, RUN * g >= 16 ? upper : lower, kvh, key & mask);
          if (seen_by_any(key & ~15, 16) != 0) {  // else it may be anything
            next_ks[s] = a.k_scales[at];
            next_vs[s] = a.v_scales[at];
          }
        }
    }
  };
  const uint32_t lds0 = (uint32_t)(uintptr_t)lds_bytes;
  // tile i's buffer: where two waves share columns the first tile takes the second one
  constexpr int FLIP = KW == 2 ? 1 : 0;
  auto buffer_of = [&](int i) { return ((i + FLIP) & 1) * Lds::second; };

  int next_ids = n_tiles > 0 ? page_ids(0) : 0, ids = 0;
  auto first_tile = [&]() __attribute__((always_inline)) {
    plan_tile(0, ids, lds0 + buffer_of(0), -1);
#pragma unroll
    for (int n = 0; n < K_PASSES; ++n) load_k(n);
#pragma unroll
    for (int n = 0; n < V_PASSES; ++n) load_v(n);
  };
  // The query: rotated and scaled in fp32, so that scores are in powers of two, through LDS
  // into operands.  A thread takes the same 16 elements, two pieces of 8 that are turned
  // with each other, of consecutive columns, whose rows are mostly one, and so is the turn.
  bf16x8 qf[TERMS][KS];
  {
    float *q32 = (float *)lds_bytes;  // [COLS][HD], 16-byte piece p of column i at p ^ (i % 8)
    constexpr int ITEMS = HD / 16, N = COLS * ITEMS / THREADS;  // of a column; columns of a thread
    const int i = threadIdx.x % ITEMS, col0 = threadIdx.x / ITEMS * N, half = a.rope_dim / 16;
    const bool apart = !a.rope_pairs && i < half;
    const int x = apart ? i : 2 * i, y = apart ? i + half : 2 * i + 1;
    const int64_t per16 = F32 ? 4 : 8;
    const bool vec = ((uintptr_t)a.q & 15) == 0 && a.ldq % per16 == 0;
    Raw8<F32> rx[N], ry[N];
    int row[N];
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int m = m0 + min(col0 + n, cols - 1);
      row[n] = row_of(m);
      const int64_t at = (int64_t)(sq.from + row[n]) * a.ldq + (int64_t)(kvh * group + m - row[n] * group) * HD;
      rx[n].load(a.q, at + 8 * x, vec);
      ry[n].load(a.q, at + 8 * y, vec);
    }
    if (KW == 2 && n_tiles > 0) {
      ids = checked(next_ids, 0);
      first_tile();
      load_scales(0, ids);
      if (n_tiles > 1) next_ids = page_ids(1);
    }
    auto put = [&](int col, int piece, const float *v) {  // 8 elements
      f32x4 *at = (f32x4 *)(q32 + col * HD);
#pragma unroll
      for (int k = 0; k < 2; ++k) at[(2 * piece + k) ^ (col & 7)] = f32x4{v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]} * a.scale_log2;
    };
    float sn[8], cs[8];
    int turned = -1;  // the row whose turn they are
#pragma unroll
    for (int n = 0; n < N; ++n) {
      float u[8], w[8];
      const bool real = col0 + n < cols;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        u[e] = real ? rx[n].value(e) : 0.f;
        w[e] = real ? ry[n].value(e) : 0.f;
      }
      if (i < half) {
        if (row[n] != turned) {
          turned = row[n];
          const int position = a.positions ? a.positions[sq.from + turned] : pos0 + turned;
#pragma unroll
          for (int e = 0; e < 8; ++e) turn_of(a.turns[8 * i + e], position, &sn[e], &cs[e]);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if (a.rope_pairs) {  // elements 16 i + 2 e and the next
            float &p = e < 4 ? u[2 * e] : w[2 * e - 8], &q = e < 4 ? u[2 * e + 1] : w[2 * e - 7];
            const float p0 = p, q0 = q;
            p = p0 * cs[e] - q0 * sn[e];
            q = q0 * cs[e] + p0 * sn[e];
          } else {
            const float p0 = u[e], q0 = w[e];
            u[e] = p0 * cs[e] - q0 * sn[e];
            w[e] = q0 * cs[e] + p0 * sn[e];
          }
        }
      }
      put(col0 + n, x, u);
      put(col0 + n, y, w);
    }
    __syncthreads();
    const int col = C * cw + c;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      // the 8 dims of this lane: a 16-byte piece of a row of K, or half of one of 8 bits
      const int d0 = F8 ? (ks >> 1) * 2 * K + 16 * g + 8 * (ks & 1) : K * ks + 8 * g;
      f32x4 v[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) v[k] = ((const f32x4 *)(q32 + col * HD))[(d0 / 4 + k) ^ (col & 7)];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float z = v[e / 4][e % 4];
#pragma unroll
        for (int t = 0; t < TERMS; ++t) {
          qf[t][ks][e] = (__bf16)z;
          z -= (float)qf[t][ks][e];
        }
      }
    }
    __syncthreads();
  }

  // the 16 bytes of K that are operand ks of product k of part `part` (and the next one in 8 bits)
  auto k_piece = [&](const uint8_t *buf, int part, int k, int ks) {
    // row c of the product is the key whose score ends with lanes (, c / 4 % GROUPS) as number 4 k + c % 4, or 4 (c / 8) + c % 4
    const int key = 32 * part + RUN * (c / 4 % GROUPS) + 4 * (C == 32 ? c >> 3 : k) + (c & 3);
    return *(const u32x4_t *)(buf + key * (KP * 16) + (((F8 ? (ks >> 1) : ks) * GROUPS + g) ^ k_bits(key)) * 16);
  };
  // operand u of part `part` of V^T for output tile n: keys 32 part + RUN g + 8 u ..
  auto v_operand = [&](const uint8_t *buf, int n, int part, int u) {
    const int d = C * n + c, key = 32 * part + RUN * g + 8 * u;
    const uint8_t *at = buf + KBYTES + d * (VP * 16) + ((key / PIECE) ^ v_bits(d)) * 16;
    u32x4_t r;
    if constexpr (F8) {
      typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
      const u32x2_t w = *(const u32x2_t *)(at + key % PIECE);
      r[0] = w[0];
      r[1] = w[1];
    } else {
      r = *(const u32x4_t *)at;
    }
    return operand_of<F8>(r, 0);
  };

  acc o[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int r = 0; r < VAL; ++r) o[n][r] = 0.f;
  float m = -INFINITY, l = 0.f;
  uint32_t nans[(NT * VAL + 31) / 32] = {};  // a bit for each value of o
  if (KW == 1 && n_tiles > 0) {
    ids = checked(next_ids, 0);
    first_tile();
    load_scales(0, ids);
    if (n_tiles > 1) next_ids = page_ids(1);
  }
  for (int i = 0; i < n_tiles; ++i) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();  // this tile is there, and everyone is done with the other buffer
    uint8_t *buf = lds_bytes + buffer_of(i);
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      ks_[s] = next_ks[s];
      vs_[s] = next_vs[s];
    }
    if (i + 1 < n_tiles) {
      ids = checked(next_ids, i + 1);
      load_scales(i + 1, ids);
      if (i + 2 < n_tiles) next_ids = page_ids(i + 2);
    }
    plan_tile(min(i + 1, n_tiles - 1), ids, lds0 + buffer_of(i + 1), i + 1 - n_tiles);
    const int k0 = tile_at(i);
    const bool edge = (k0 < lo_max || k0 + TILE > hi_min) && k0 + TILE > first_min;
    uint32_t seen[NS];  // of this lane's scores
#pragma unroll
    for (int s = 0; s < NS; ++s) seen[s] = edge ? seen_by_mine(k0 + 32 * (KW == 1 ? s : kw) + RUN * g, RUN) : 0xFFFFu;
    if (edge) {
      // What no column sees may be anything, and becomes zero: a thread looks at the pieces
      // of V^T that it loaded.  What only some see must not reach the others as 0 * NaN.
      u32x4_t *mine = (u32x4_t *)(buf + KBYTES + threadIdx.x * 16);
      const uint32_t any = seen_by_any(k0 + v_key, PIECE);
      u32x4_t keep = {0, 0, 0, 0};
#pragma unroll
      for (int e = 0; e < PIECE; ++e) keep[e * ESZ / 4] |= (any >> e & 1) ? (F8 ? 0xFFu : 0xFFFFu) << (e * ESZ % 4 * 8) : 0u;
      bool odd = false;
#pragma unroll
      for (int n = 0; n < V_PASSES; ++n) {
        const u32x4_t v = mine[n * THREADS] & keep;
        odd |= not_finite<F8>(v);
        mine[n * THREADS] = v;
      }
      if (__syncthreads_or(odd)) {  // columns that see such a value become NaN at the end, and it a zero
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
          for (int u = 0; u < RUN / 8; ++u) {
            union {
              bf16x8 v;
              uint16_t e[8];
            } sees;
#pragma unroll
            for (int e = 0; e < 8; ++e) sees.e[e] = seen[s] >> (8 * u + e) & 1 ? 0x3F80u : 0u;
#pragma unroll 1  // rare: registers count for more
            for (int n = 0; n < NT; ++n) {
              union {
                bf16x8 v;
                u32x4_t w;
              } vf{v_operand(buf, n, KW == 1 ? s : kw, u)};
              acc hits;
#pragma unroll
              for (int r = 0; r < VAL; ++r) hits[r] = 0.f;
              hits = Mul::of(take_not_finite<false>(vf.w, 0), sees.v, hits);
              uint32_t bits = 0;
#pragma unroll
              for (int r = 0; r < VAL; ++r) bits |= hits[r] > 0.f ? 1u << r : 0u;
#pragma unroll
              for (int k = 0; k < (NT * VAL + 31) / 32; ++k) nans[k] |= n * VAL / 32 == k ? bits << (n * VAL % 32) : 0u;
            }
          }
        __syncthreads();
#pragma unroll
        for (int n = 0; n < V_PASSES; ++n) {
          u32x4_t v = mine[n * THREADS];
#pragma unroll
          for (int u = 0; u < (F8 ? 2 : 1); ++u) (void)take_not_finite<F8>(v, u);
          mine[n * THREADS] = v;
        }
        __syncthreads();
      }
    }
    // scores, in powers of two
    acc sc[NS][MK];
    u32x4_t raw[NS][MK];
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
      for (int k = 0; k < MK; ++k)
#pragma unroll
        for (int r = 0; r < VAL; ++r) sc[s][k][r] = 0.f;
    static_assert(KS % K_PASSES == 0 && NT % V_PASSES == 0, "loads between the products");
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      if (ks % (KS / K_PASSES) == 0) load_k(ks / (KS / K_PASSES));
#pragma unroll
      for (int s = 0; s < NS; ++s)
#pragma unroll
        for (int k = 0; k < MK; ++k) {
          if (!F8 || ks % 2 == 0) raw[s][k] = k_piece(buf, KW == 1 ? s : kw, k, ks);
          const bf16x8 kf = operand_of<F8>(raw[s][k], ks & 1);
#pragma unroll
          for (int t = TERMS - 1; t >= 0; --t) sc[s][k] = Mul::of(kf, qf[t][ks], sc[s][k]);
        }
    }
    if constexpr (F8)
      if (a.k_scales) {
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
          for (int k = 0; k < MK; ++k) sc[s][k] *= ks_[s];
      }
    if (edge) {
      asm volatile("");  // a branch: the other tiles are spared three instructions a score
#pragma unroll
      for (int s = 0; s < NS; ++s)
#pragma unroll
        for (int e = 0; e < RUN; ++e) sc[s][e / VAL][e % VAL] = seen[s] >> e & 1 ? sc[s][e / VAL][e % VAL] : -INFINITY;
    }
    float mt = -INFINITY;
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
      for (int e = 0; e < RUN; ++e) mt = fmaxf(mt, sc[s][e / VAL][e % VAL]);
    if constexpr (C == 16) mt = max_pair16(mt);
    mt = max_pair32(mt);
    // the running maximum is raised when it is passed by more than 2^8 (the weights
    // stay below that); all lanes of a column agree
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
      for (int u = 0; u < RUN / 8; ++u) {
        bf16x8 pf[TERMS];
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float p = __builtin_amdgcn_exp2f(sc[s][(8 * u + e) / VAL][(8 * u + e) % VAL] - base);
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
          if (s == 0 && u == 0 && n % (NT / V_PASSES) == 0) load_v(n / (NT / V_PASSES));
          const bf16x8 vf = v_operand(buf, n, KW == 1 ? s : kw, u);
#pragma unroll
          for (int t = TERMS - 1; t >= 0; --t) o[n] = Mul::of(vf, pf[t], o[n]);
        }
      }
  }
  if (bad) raise_status(a.status, kStatusPage);
  if constexpr (C == 16) l = sum_pair16(l);
  l = sum_pair32(l);
  uint32_t any_nan = 0;
#pragma unroll
  for (int k = 0; k < (NT * VAL + 31) / 32; ++k) any_nan |= nans[k];
  if (__ballot(any_nan != 0)) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int r = 0; r < VAL; ++r) o[n][r] = nans[n * VAL / 32] >> (n * VAL % 32 + r) & 1 ? NAN : o[n][r];
  }

  // two waves with the same columns meet in LDS, the second's values in units of its maximum
  constexpr int QUADS = VAL / 4;
  if constexpr (KW == 2) {
    __syncthreads();
    f32x4 *part = (f32x4 *)lds_bytes + cw * (NT * QUADS * 64);
    float *ml = (float *)(lds_bytes + 64 * HD * 4) + cw * 128;
    if (kw == 1) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int k = 0; k < QUADS; ++k)
          part[(n * QUADS + k) * 64 + lane] = f32x4{o[n][4 * k], o[n][4 * k + 1], o[n][4 * k + 2], o[n][4 * k + 3]};
      ml[lane] = m;
      ml[64 + lane] = l;
    }
    __syncthreads();
    if (kw == 0) {
      const float m1 = ml[lane], l1 = ml[64 + lane], mx = fmaxf(m, m1);
      const float f0 = l != 0.f ? __builtin_amdgcn_exp2f(m - mx) : 0.f, f1 = l1 != 0.f ? __builtin_amdgcn_exp2f(m1 - mx) : 0.f;
      l = l * f0 + l1 * f1;
      m = mx;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int k = 0; k < QUADS; ++k) {
          const f32x4 v = part[(n * QUADS + k) * 64 + lane];
#pragma unroll
          for (int r = 0; r < 4; ++r) o[n][4 * k + r] = o[n][4 * k + r] * f0 + v[r] * f1;
        }
    }
  }
  const int col = C * cw + c, j = row_of(m0 + min(col, cols - 1));
  const int64_t oi = (int64_t)(sq.from + j) * a.ldo + (int64_t)(kvh * group + m0 + col - j * group) * HD + 4 * g;
  auto put_out = [&](int n, int k, f32x4 v) {
    const int64_t at = oi + C * n + 4 * GROUPS * k;
    if (a.out_vec) {
      if constexpr (F32) *(f32x4 *)((float *)a.out + at) = v;
      else *(bf16x4 *)((__bf16 *)a.out + at) = bf16x4{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r) store_elem<F32>(a.out, at + r, v[r]);
    }
  };
  if (!SPLITS || w.splits == 1) {
    if (kw == 1 || col >= cols) return;
    const float scale = l != 0.f ? a.v_scale / l : 0.f;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int k = 0; k < QUADS; ++k)
        put_out(n, k, f32x4{o[n][4 * k], o[n][4 * k + 1], o[n][4 * k + 2], o[n][4 * k + 3]} * scale);
    return;
  }
  if constexpr (SPLITS) {
    // a slot: a wave's outputs as it holds them, and a maximum and a sum a column
    const auto slots = slots_of(a, COLS * HD);
    auto at = [&](int slot, int n, int k) { return (unsigned)((slot * (COLS / C) + cw) * (NT * QUADS) + n * QUADS + k) * 256 + 4 * lane; };
    const int mine = w.slot + w.split;
    if (kw == 0 && col < cols) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int k = 0; k < QUADS; ++k) put_slot(slots, at(mine, n, k), f32x4{o[n][4 * k], o[n][4 * k + 1], o[n][4 * k + 2], o[n][4 * k + 3]});
      if (g == 0) __hip_atomic_store(a.part_ml + (size_t)mine * COLS + col, pair_of(m, l), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    if (!last_to_arrive(a.arrived + w.slot, w.splits, (float *)plan)) return;
    // the last to arrive joins the splits in their order; two waves with the same columns
    // take half of the outputs each
    if (col >= cols) return;
    constexpr int HALF = NT * QUADS / 2;
    f32x4 sum[HALF];
    float total = 0.f, top = -INFINITY;
#pragma unroll
    for (int n = 0; n < HALF; ++n) sum[n] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < w.splits; ++s) {
      const uint64_t pair = __hip_atomic_load(a.part_ml + (size_t)(w.slot + s) * COLS + col, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      f32x4 v[HALF];
#pragma unroll
      for (int n = 0; n < HALF; ++n) v[n] = get_slot(slots, at(w.slot + s, 0, kw * HALF + n));
      const float ms = __uint_as_float((uint32_t)pair), ls = __uint_as_float((uint32_t)(pair >> 32)), mx = fmaxf(top, ms);
      const float f0 = total != 0.f ? __builtin_amdgcn_exp2f(top - mx) : 0.f, f1 = ls != 0.f ? __builtin_amdgcn_exp2f(ms - mx) : 0.f;
      total = total * f0 + ls * f1;
      top = mx;
#pragma unroll
      for (int n = 0; n < HALF; ++n) sum[n] = sum[n] * f0 + v[n] * f1;
    }
    const float scale = total != 0.f ? a.v_scale / total : 0.f;
#pragma unroll
    for (int n = 0; n < HALF; ++n) put_out((kw * HALF + n) / QUADS, (kw * HALF + n) % QUADS, sum[n] * scale);
  }
}

template <int HD, bool F32, bool F8, int KW>
static hipError_t prompt_attr() {
  return hipFuncSetAttribute((const void *)kv_prompt_kernel<HD, F32, F8, KW>, hipFuncAttributeMaxDynamicSharedMemorySize,
                             (PromptLds<HD, F8, KW>::bytes));
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
static hipError_t launch_prompt_type(KvRowsArgs a, hipStream_t s) {
  constexpr RowsKind kind = many_rows<KW>();
  // units of 128 columns are not split
  const int64_t tokens = KW == 2 ? (int64_t)a.pages_per_seq << a.d.page_shift : kind.tile;
  const RowsGrid grid = rows_grid(kind, a.n_rows, a.n_seqs, true, a.d.n_kv_heads, a.group, tokens, a.window, a.sinks, a.target, a.slots);
  a.unsplit = grid.unsplit;
  hipLaunchKernelGGL((kv_prompt_kernel<HD, F32, F8, KW>), dim3((unsigned)grid.wgs), dim3(kPromptThreads<HD, KW>), ((PromptLds<HD, F8, KW>::bytes)), s, a);
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
