// Paged K/V cache: append with rotation, attention of one token per sequence, and
// the expert's prefix from pages.  Layouts and checks in paged.h.
#include "paged_device.h"

namespace uad {

// ---------------------------------------------------------------------------
// Append of few rows: one workgroup per new row, a thread per pair of columns and as
// many heads at once as there are threads.  Bound by the launch and three dependent
// loads (length, page id, store): 2.0 us for a token of 1 x 256, 3.1 us for 64 tokens of
// 2 x 128 in e4m3 (kernel time; 2.7 and 3.1 a call in a graph of them).
// ---------------------------------------------------------------------------
template <bool F32, bool F8>
__device__ __forceinline__ void append_row(const KvAppendArgs &a, int r) {
  int b = r, j = 0, n_b = 1;
  bool bad = false;
  if (a.row_start) {
    b = sequence_of_row(a.row_start, a.n_seqs, r);
    if (b >= a.n_seqs) return;  // a row behind the last sequence
    int lo = 0, hi = 0;
    if (b >= 0) {
      lo = a.row_start[b];
      hi = a.row_start[b + 1];
    }
    bad = b < 0 || r < lo || r >= hi;
    j = r - lo;
    n_b = hi - lo;
    if (!bad) bad = !sequence_ok(b, lo, hi, a.n_rows, a.lens[b], a.pages_per_seq, a.d.page_shift);
  }
  int pos = 0, page = 0;
  if (!bad) {
    pos = length_or_none(a.lens[b], a.pages_per_seq, a.d.page_shift, &bad) - n_b + j;
    bad |= pos < 0;
  }
  if (!bad) {
    page = a.table[(int64_t)b * a.pages_per_seq + (pos >> a.d.page_shift)];
    bad = !page_ok(a.d, page);
  }
  if (bad) {
    if (threadIdx.x == 0) raise_status(a.status, kStatusPage);
    return;
  }
  const int off = pos & ((1 << a.d.page_shift) - 1);
  const int half = a.d.head_dim / 2;
  const int p = threadIdx.x % half, heads_at_once = blockDim.x / half;
  int ea, eb;
  rope_pair(p, a.rope_dim, a.rope_pairs != 0, &ea, &eb);
  float s = 0.f, c = 1.f;
  if (p < a.rope_dim / 2) turn_of(a.turns[p], a.positions ? a.positions[r] : pos, &s, &c);
  for (int h = threadIdx.x / half; h < a.d.n_kv_heads; h += heads_at_once) {
    const int64_t col = (int64_t)h * a.d.head_dim;
    const float x = load_elem<F32>(a.k, r * a.ldk + col + ea), y = load_elem<F32>(a.k, r * a.ldk + col + eb);
    const float u = load_elem<F32>(a.v, r * a.ldv + col + 2 * p), w = load_elem<F32>(a.v, r * a.ldv + col + 2 * p + 1);
    const size_t base = page_base(a.d, page, h);
    const float kx = p < a.rope_dim / 2 ? x * c - y * s : x, ky = p < a.rope_dim / 2 ? y * c + x * s : y;
    store_pool<F8>(a.kp, base + k_in_page(a.d, off, ea), F8 ? quotient(kx, a.k_scale, a.k_inv) : kx);
    store_pool<F8>(a.kp, base + k_in_page(a.d, off, eb), F8 ? quotient(ky, a.k_scale, a.k_inv) : ky);
    store_pool<F8>(a.vp, base + v_in_page(a.d, off, 2 * p), F8 ? quotient(u, a.v_scale, a.v_inv) : u);
    store_pool<F8>(a.vp, base + v_in_page(a.d, off, 2 * p + 1), F8 ? quotient(w, a.v_scale, a.v_inv) : w);
  }
}

template <bool F32, bool F8>
__global__ __launch_bounds__(256) void kv_append_kernel(KvAppendArgs a) {
  const int r = a.row0 + blockIdx.x;
  if (!a.row_start) {
    append_row<F32, F8>(a, r);
    return;
  }
  // every sequence is looked at, those too in which no row lands: loaded before the row
  // is dealt with, looked at after it
  unsigned i = blockIdx.x * 256 + threadIdx.x;
  const int at = min(i, (unsigned)a.n_seqs - 1), from = a.row_start[at], to = a.row_start[at + 1], len = a.lens[at];
  append_row<F32, F8>(a, r);
  bool odd = i < (unsigned)a.n_seqs && !sequence_ok(at, from, to, a.n_rows, len, a.pages_per_seq, a.d.page_shift);
  for (i += gridDim.x * 256; i < (unsigned)a.n_seqs; i += gridDim.x * 256)
    odd |= !sequence_ok(i, a.row_start[i], a.row_start[i + 1], a.n_rows, a.lens[i], a.pages_per_seq, a.d.page_shift);
  if (odd) raise_status(a.status, kStatusPage);
}

// ---------------------------------------------------------------------------
// Append of many rows: one workgroup per tile (see paged.h), KV head, pool and up to 128
// columns, so that pages are written 16 bytes at a time: bound by memory; a row by
// itself would scatter its values over a transposed page two bytes at a time.  K: a
// thread rotates 16 elements of a row, the pieces of 8 that are turned with each other.
// V: through LDS, whose 16-byte pieces are swizzled by the token's chunk, so that the
// lanes that read 8 (or 16) tokens of a column do not meet in a bank.  64 prompts of 816
// rows, 1 x 256 bf16 (104 MB): 28.9 us, with non-temporal stores of the pages 19.3 us
// (5.4 TB/s; a device copy of as much 22.4 us); the workgroups of a tile next to each
// other instead of K's first and V's last: 24.7 us.  Row by row: 118 us.
// ---------------------------------------------------------------------------
template <int HD, bool F32, bool F8>
__global__ __launch_bounds__(256) void kv_append_tile_kernel(KvAppendArgs a) {
  constexpr int ESZ = F8 ? 1 : 2;
  constexpr int WIDE = kAppendWide<HD>;               // columns of this workgroup
  constexpr int PIECES = WIDE / 8;                    // of 8 elements of a row
  constexpr int ROUNDS = kAppendTile * PIECES / 2 / 256;  // of 256 threads with two pieces each, at most
  constexpr int N = ROUNDS > 1 ? ROUNDS : 1;
  __shared__ __align__(16) uint8_t lds[kAppendTile * WIDE * ESZ];
  __shared__ int plan[kPlanScans * 4];
  AppendTile t;
  if (!plan_append<4>(a, blockIdx.x, plan, &t)) return;
  const int head = blockIdx.y, part = blockIdx.z >> 1, mask = (1 << a.d.page_shift) - 1;
  const int page = a.table[(int64_t)t.b * a.pages_per_seq + (t.first >> a.d.page_shift)];  // looked at when the rows are on their way
  const int tokens = t.last - t.first + 1, items = tokens * (PIECES / 2);
  const int tile_off = (t.first & mask) & ~(kAppendTile - 1);  // offset in the page of the tile's first slot
  const bool is_v = blockIdx.z & 1;
  const void *src = is_v ? a.v : a.k;
  const int64_t ld = is_v ? a.ldv : a.ldk;
  // an item: pieces x and y of a token; for K the ones that are turned with each other
  // (piece p with p + rope_dim / 16, or neighbours, as which all pieces count for V, for
  // rotated neighbours and behind rope_dim)
  const int half = a.rope_dim / 16;
  auto pieces = [&](int i, int *x, int *y) {
    if (!is_v && !a.rope_pairs && i < half) {
      *x = i;
      *y = i + half;
    } else {
      *x = 2 * i;
      *y = 2 * i + 1;
    }
  };
  Raw8<F32> rx[N], ry[N];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int item = min((int)threadIdx.x + n * 256, items - 1), token = item / (PIECES / 2);
    int x, y;
    pieces(part * (PIECES / 2) + item % (PIECES / 2), &x, &y);
    const int64_t at = (t.row + token) * ld + (int64_t)head * HD;
    rx[n].load(src, at + 8 * x, a.in_vec);
    ry[n].load(src, at + 8 * y, a.in_vec);
  }
  if (!page_ok(a.d, page)) {
    if (threadIdx.x == 0) raise_status(a.status, kStatusPage);
    return;
  }
  const size_t base = page_base(a.d, page, head);
  if (!is_v) {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int item = threadIdx.x + n * 256, token = item / (PIECES / 2);
      const int i = part * (PIECES / 2) + item % (PIECES / 2);
      if (item >= items) break;
      float u[8], w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        u[e] = rx[n].value(e);
        w[e] = ry[n].value(e);
      }
      int x, y;
      pieces(i, &x, &y);
      if (i < half) {
        const int position = a.positions ? a.positions[t.row + token] : t.first + token;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float s, c;
          turn_of(a.turns[8 * i + e], position, &s, &c);
          if (a.rope_pairs) {  // elements 16 i + 2 e and the next
            float &p = e < 4 ? u[2 * e] : w[2 * e - 8], &q = e < 4 ? u[2 * e + 1] : w[2 * e - 7];
            const float p0 = p, q0 = q;
            p = p0 * c - q0 * s;
            q = q0 * c + p0 * s;
          } else {
            const float p0 = u[e], q0 = w[e];
            u[e] = p0 * c - q0 * s;
            w[e] = q0 * c + p0 * s;
          }
        }
      }
      if constexpr (F8)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          u[e] = quotient(u[e], a.k_scale, a.k_inv);
          w[e] = quotient(w[e], a.k_scale, a.k_inv);
        }
      char *dst = (char *)a.kp + (base + k_in_page(a.d, (t.first & mask) + token, 0)) * ESZ;
      Pool8<F8> o;
      o.set(u);
      o.put_page(dst + 8 * x * ESZ);
      o.set(w);
      o.put_page(dst + 8 * y * ESZ);
    }
    return;
  }
  // V: tokens x WIDE in pool type, a token's 8-element piece p at place p ^ (token / RUN)
  constexpr int RUN = F8 ? 16 : 8;  // tokens of a 16-byte store
  const int lead = (t.first & mask) - tile_off;  // slots of the tile before the first row
  auto place = [&](int slot, int piece) { return (slot * PIECES + (piece ^ ((slot / RUN) & (PIECES - 1)))) * 8 * ESZ; };
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int item = threadIdx.x + n * 256, token = item / (PIECES / 2), i = item % (PIECES / 2);
    if (item >= items) break;
    float u[8], w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      u[e] = F8 ? quotient(rx[n].value(e), a.v_scale, a.v_inv) : rx[n].value(e);
      w[e] = F8 ? quotient(ry[n].value(e), a.v_scale, a.v_inv) : ry[n].value(e);
    }
    Pool8<F8> o;
    o.set(u);
    o.put(lds + place(lead + token, 2 * i));
    o.set(w);
    o.put(lds + place(lead + token, 2 * i + 1));
  }
  __syncthreads();
  // columns in words (2 of bf16, 4 of e4m3), runs of RUN slots
  constexpr int COLS = 4 / ESZ, WORDS = WIDE / COLS;
  const int run0 = lead / RUN, runs = (lead + tokens - 1) / RUN - run0 + 1;
  char *vp = (char *)a.vp + (base + v_in_page(a.d, tile_off, part * WIDE)) * ESZ;
  for (int item = threadIdx.x; item < WORDS * runs; item += 256) {
    const int run = run0 + item % runs, word = item / runs, slot0 = run * RUN;
    uint32_t v[RUN];
#pragma unroll
    for (int e = 0; e < RUN; ++e)
      v[e] = *(const uint32_t *)(lds + place(slot0 + e, word * COLS / 8) + (word * COLS % 8) * ESZ);
    char *dst = vp + (((size_t)(word * COLS) << a.d.page_shift) + slot0) * ESZ;
    const size_t next = ((size_t)1 << a.d.page_shift) * ESZ;  // from a column to the next
    uint32_t o[COLS][4];
#pragma unroll
    for (int col = 0; col < COLS; ++col)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if constexpr (F8)
          o[col][k] = (v[4 * k] >> (8 * col) & 0xFF) | (v[4 * k + 1] >> (8 * col) & 0xFF) << 8 |
                      (v[4 * k + 2] >> (8 * col) & 0xFF) << 16 | (v[4 * k + 3] >> (8 * col)) << 24;
        else
          o[col][k] = (v[2 * k] >> (16 * col) & 0xFFFF) | (v[2 * k + 1] >> (16 * col)) << 16;
      }
    if (slot0 >= lead && slot0 + RUN <= lead + tokens) {
#pragma unroll
      for (int col = 0; col < COLS; ++col)
        __builtin_nontemporal_store(u32x4_t{o[col][0], o[col][1], o[col][2], o[col][3]}, (u32x4_t *)(dst + col * next));
    } else {  // a sequence's first or last run: whole words, then what is left of them
      const int from = lead - slot0, to = lead + tokens - slot0;  // slots of the run that have rows
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (COLS * k >= from && COLS * (k + 1) <= to) {
#pragma unroll
          for (int col = 0; col < COLS; ++col) *(uint32_t *)(dst + col * next + 4 * k) = o[col][k];
        } else if (COLS * (k + 1) > from && COLS * k < to) {
#pragma unroll
          for (int e = 0; e < COLS; ++e)
            if (COLS * k + e >= from && COLS * k + e < to)
#pragma unroll
              for (int col = 0; col < COLS; ++col) {
                if constexpr (F8) *(uint8_t *)(dst + col * next + 4 * k + e) = (uint8_t)(o[col][k] >> (8 * e));
                else *(uint16_t *)(dst + col * next + 4 * k + 2 * e) = (uint16_t)(o[col][k] >> (16 * e));
              }
        }
      }
    }
  }
}

// Mean rows per sequence from which an append goes by tiles: 64 sequences, 1 x 256
// bf16, 4 rows each row by row 3.8, by tiles 4.0 us; 8 rows 4.6, 4.4; 32 rows 7.7, 5.1.
constexpr int kAppendTileRows = 8;

template <bool F32, bool F8>
static hipError_t launch_append_type(const KvAppendArgs &a, hipStream_t s) {
  constexpr int kMaxWgs = 1 << 23;  // work items of a grid stay below 2^32
  const int64_t tiles = append_grid(a.n_rows, a.n_seqs, append_tile_shift(a.d.page_shift));
  if (a.row_start && (int64_t)a.n_seqs * kAppendTileRows <= a.n_rows && tiles <= kMaxWgs && a.d.n_kv_heads <= 65535) {
    const dim3 grid((unsigned)tiles, a.d.n_kv_heads, a.d.head_dim > 128 ? 4 : 2), wg(256);
    if (a.d.head_dim == 64) hipLaunchKernelGGL((kv_append_tile_kernel<64, F32, F8>), grid, wg, 0, s, a);
    else if (a.d.head_dim == 128) hipLaunchKernelGGL((kv_append_tile_kernel<128, F32, F8>), grid, wg, 0, s, a);
    else hipLaunchKernelGGL((kv_append_tile_kernel<256, F32, F8>), grid, wg, 0, s, a);
    return hipGetLastError();
  }
  for (int64_t r = 0; r < a.n_rows; r += kMaxWgs) {
    KvAppendArgs p = a;
    p.row0 = (int)r;
    const dim3 grid((unsigned)(a.n_rows - r < kMaxWgs ? a.n_rows - r : kMaxWgs)), wg(256);
    hipLaunchKernelGGL((kv_append_kernel<F32, F8>), grid, wg, 0, s, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_kv_append(const KvAppendArgs &a, bool f32, bool f8, hipStream_t s) {
  if (a.n_rows < 1 || a.n_seqs < 1 || (a.d.head_dim != 64 && a.d.head_dim != 128 && a.d.head_dim != 256) ||
      a.d.page_shift < 4 || a.rope_dim % 16 || a.rope_dim > a.d.head_dim)
    return hipErrorInvalidValue;
  if (a.k_scales) return f8 ? launch_kv_append_blocks(a, f32, s) : hipErrorInvalidValue;
  if (f32) return f8 ? launch_append_type<true, true>(a, s) : launch_append_type<true, false>(a, s);
  return f8 ? launch_append_type<false, true>(a, s) : launch_append_type<false, false>(a, s);
}

// ---------------------------------------------------------------------------
// Attention of one token per sequence.
//
// Bound by reading K and V once.  A unit is a KV head of a sequence with up to 16 of
// its query heads, the 16 columns of the matrix instruction: S^T = K Q^T and
// O^T = V^T P^T with v_mfma_f32_16x16x32_bf16, whose time is a tenth of the read's, so
// that operands can be split into bf16 terms (a value = hi + lo + rest, each the bf16
// of what is left): the rotated query and the weights keep their 24 bits, so that a bf16
// result too is one of fp32, rounded once.  Two terms of 16 bits for bf16 results put
// seven times as many of them on the other side of a rounding; 817 keys of 1 x 256 took
// 11.2 instead of 11.5 us, 48 uneven sequences of 2 x 128 in e4m3 19.8 instead of 20.9.
//
// A wave takes tiles of kTileKeys keys.  Row i of the t-th 16-key product is key
// KPL * (i / 4) + 4 t + i % 4, so that lane group g ends with the scores of the
// KPL = 4 * kTileKeys / 16 consecutive keys KPL * g.., which are the k index of its
// operand of the P V product, and the keys of one 16-byte load of a transposed V page:
// K and V go from memory to the matrix instructions' registers, with no LDS between.
// Loads of the next K tile are issued when this one's scores are done, of the next V
// tile when this one's products are.  The waves of a workgroup take every
// kAttendWaves-th tile with running maxima and sums of their own and meet in LDS.  A
// unit's splits meet in slots of the workspace: the last workgroup to arrive joins
// them, in the order of the keys.
//
// One sequence of 131071 keys, 32/8 heads of 128 in bf16 (537 MB): 98 - 100 us, 5.4 -
// 5.5 TB/s, where a kernel that only reads takes 85; 8 x 4001 keys of 16 x 64 (127 MB)
// 30; 64 x 900 keys of 1 x 256 (58 MB) 20.5; 817 keys of 1 x 256 11.5 us, of which
// the launch, the plan, the meeting in LDS and the join take about 7.  More splits than
// workgroups run at once cost their prologues (twice as many, with two terms: 109, 37
// and 27 us).
// ---------------------------------------------------------------------------
// What a workgroup does: tiles t0 .. t1-1 of a unit of sequence b; split `split` of
// `splits`, whose slots start at `slot`.
struct AttendWork {
  int b, unit, len, t0, t1, split, splits, slot;
};

// The plan (see paged.h).
template <int HD, bool F8>
__device__ __forceinline__ bool plan_attend(const KvAttendArgs &a, int units, int wg, int *lds, AttendWork *w) {
  constexpr int TILE = kTileKeys<F8>;
  bool bad = false;
  if (a.unsplit) {  // the page table holds too few keys for a split: a workgroup per unit
    *w = AttendWork{};
    w->b = (unsigned)wg / (unsigned)units;
    w->unit = wg - w->b * units;
    w->len = length_or_none(a.lens[w->b], a.pages_per_seq, a.d.page_shift, &bad);
    w->t1 = tiles_of_length(w->len, TILE);
    w->splits = 1;
    if (bad && threadIdx.x == 0) raise_status(a.status, kStatusPage);
    return true;
  }
  auto length = [&](int b) { return length_or_none(a.lens[b], a.pages_per_seq, a.d.page_shift, &bad); };
  const bool spare = (int64_t)a.n_seqs * units < a.target;  // fewer units than run at once
  int start, slot, b, tiles, splits;
  if (a.n_seqs <= 64) {  // each wave for itself, a sequence per lane
    const int lane = threadIdx.x & 63;
    const bool have = lane < a.n_seqs;
    const int len = have ? length(lane) : 0;
    if (bad && wg == 0) raise_status(a.status, kStatusPage);
    const int my_tiles = have ? tiles_of_length(len, TILE) : 0;
    int64_t total;
    if (a.few_tiles) {
      total = last_lane(scan_wave64(my_tiles * units));
    } else {
      const int64_t n = (int64_t)my_tiles * units;
      total = ((int64_t)last_lane(scan_wave64((int)(n >> 22))) << 22) + last_lane(scan_wave64((int)(n & 0x3FFFFF)));
    }
    int share = first_share(total, a.target, kAttendMinTiles);
    int my_splits = have ? splits_of(my_tiles, share, kAttendWhole<HD, F8>) : 0, upto = scan_wave64(my_splits * units);
    for (int i = 0; spare && i < kShareTries && last_lane(upto) > a.target; ++i) {
      share = next_share(share);
      my_splits = have ? splits_of(my_tiles, share, kAttendWhole<HD, F8>) : 0;
      upto = scan_wave64(my_splits * units);
    }
    if (wg >= last_lane(upto)) return false;
    const int mine = my_splits * units, in_slots = my_splits > 1 ? mine : 0, slot_upto = scan_wave64(in_slots);
    b = __builtin_ctzll(__ballot(upto > wg));
    start = __builtin_amdgcn_readlane(upto - mine, b);
    slot = __builtin_amdgcn_readlane(slot_upto - in_slots, b);
    tiles = __builtin_amdgcn_readlane(my_tiles, b);
    splits = __builtin_amdgcn_readlane(my_splits, b);
    w->len = __builtin_amdgcn_readlane(len, b);
  } else {
    PlanScan<kAttendWaves> scan(a.n_seqs, lds);
    // f(length) over this thread's sequences, of which the first is kept
    const int b0 = scan.me * scan.per;
    const int my_len = b0 < a.n_seqs ? length(b0) : 0;
    auto each = [&](auto f) {
      if (b0 < a.n_seqs) f(my_len);
      for (int i = 1; i < scan.per; ++i)
        if (b0 + i < a.n_seqs) f(length(b0 + i));
    };
    int64_t n = 0;
    each([&](int len) { n += tiles_of_length(len, TILE); });
    if (bad && wg == 0) raise_status(a.status, kStatusPage);
    n *= units;
    int hi, lo, mine, upto, wgs, all;
    scan((int)(n >> 22), &hi);
    scan((int)(n & 0x3FFFFF), &lo);
    int share = first_share(((int64_t)hi << 22) + lo, a.target, kAttendMinTiles);
    auto count = [&]() {  // workgroups of this thread's sequences, and up to them
      mine = 0;
      each([&](int len) { mine += splits_of(tiles_of_length(len, TILE), share, kAttendWhole<HD, F8>) * units; });
      upto = scan(mine, &wgs);
    };
    count();
    for (int i = 0; spare && i < kShareTries && wgs > a.target; ++i) {
      share = next_share(share);
      count();
    }
    if (wg >= wgs) return false;
    int in_slots = 0;  // workgroups in split units, for the slots
    each([&](int len) {
      const int s = splits_of(tiles_of_length(len, TILE), share, kAttendWhole<HD, F8>);
      if (s > 1) in_slots += s * units;
    });
    const int slot_upto = scan(in_slots, &all);
    start = upto - mine;
    if (upto > wg && start <= wg) {  // one thread: it looks for the sequence among its own
      int len = my_len;
      slot = slot_upto - in_slots;
      for (b = b0;;) {
        const int s = splits_of(tiles_of_length(len, TILE), share, kAttendWhole<HD, F8>);
        if (start + s * units > wg) break;
        start += s * units;
        if (s > 1) slot += s * units;
        if (++b >= a.n_seqs) break;
        len = length(b);
      }
      const int found[4] = {b, len, start, slot};
#pragma unroll
      for (int i = 0; i < 4; ++i) scan.lds[i] = found[i];
    }
    __syncthreads();
    b = __builtin_amdgcn_readfirstlane(scan.lds[0]);
    w->len = __builtin_amdgcn_readfirstlane(scan.lds[1]);
    start = __builtin_amdgcn_readfirstlane(scan.lds[2]);
    slot = __builtin_amdgcn_readfirstlane(scan.lds[3]);
    if (b >= a.n_seqs) return false;  // only if the lengths change while this runs
    tiles = tiles_of_length(w->len, TILE);
    splits = splits_of(tiles, share, kAttendWhole<HD, F8>);
  }
  w->b = b;
  w->splits = splits;
  w->unit = splits == 1 ? wg - start : (unsigned)(wg - start) / (unsigned)splits;
  if (w->unit >= units) return false;  // likewise
  w->split = wg - start - w->unit * splits;
  w->slot = slot + w->unit * splits;
  if (splits > 1 && w->slot + splits > a.slots) return false;  // likewise
  w->t0 = splits == 1 ? 0 : split_begin(tiles, splits, w->split);
  w->t1 = splits == 1 ? tiles : split_begin(tiles, splits, w->split + 1);
  return true;
}

template <int HD, bool F32, bool F8>
__global__ __launch_bounds__(64 * kAttendWaves, kAttendPerCu<HD> * kAttendWaves / 4) void kv_attend_kernel(KvAttendArgs a) {
  constexpr int TILE = kTileKeys<F8>, NT = TILE / 16, KPL = 4 * NT;
  constexpr int KS = HD / 32;           // k steps of Q K^T
  constexpr int KL = F8 ? HD / 64 : KS; // 16-byte loads of a key row per lane
  constexpr int NTO = HD / 16;          // 16-column tiles of the output
  constexpr int TERMS = kTerms;
  constexpr int NW = kAttendWaves;
  constexpr int ESZ = F8 ? 1 : 2;
  extern __shared__ __align__(16) float lds[];
  __bf16 *qf = (__bf16 *)lds;                      // [TERMS][KS][64][8]
  f32x4 *obuf = (f32x4 *)(lds + kQueryFloats<HD>);  // [NW][NTO][64]
  float *ml = (float *)(obuf + NW * NTO * 64);     // [NW or slots][16][2]
  float *top = ml + kAttendMl, *word = top + 32;
  static_assert(TERMS * KS * 64 * 8 * 2 == kQueryFloats<HD> * 4, "the query's terms");
  static_assert(NW * 16 * 2 <= kAttendMl && kPlanScans * NW <= kAttendMl, "the waves' maxima and the plan fit the slots' weights");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, g = lane >> 4;
  const int runs = (a.group + 15) / 16, units = a.d.n_kv_heads * runs;
  const int rows_max = a.group < 16 ? a.group : 16;
  // the turns per position of this thread's pair of columns
  constexpr int HP = HD / 2, RS = 64 * NW / HP, QN = (16 + RS - 1) / RS;
  const int p = threadIdx.x % HP;
  int ea, eb;
  rope_pair(p, a.rope_dim, a.rope_pairs != 0, &ea, &eb);
  const bool turned = p < a.rope_dim / 2;
  const double turns = a.turns[p];  // 128 of them are allocated

  AttendWork w;
  if (!plan_attend<HD, F8>(a, units, blockIdx.x, (int *)ml, &w)) return;
  const int kvh = w.unit / runs, head0 = kvh * a.group + (w.unit - kvh * runs) * 16;
  const int rows = min(16, (kvh + 1) * a.group - head0);
  const int last = w.len - 1, mask = (1 << a.d.page_shift) - 1;
  const int32_t *table = a.table + (int64_t)w.b * a.pages_per_seq;
  bool bad = false;

  // Loads are waited for in the order of their issue: page ids and the query's values
  // first, then the keys and values, which arrive while the query is rotated.
  auto page_ids = [&](int tile, int &kp, int &vp) {
    kp = table[min(tile * TILE + KPL * (c >> 2), last) >> a.d.page_shift];
    vp = table[min(tile * TILE + KPL * g, last) >> a.d.page_shift];
  };
  auto checked = [&](int page) {
    const bool ok = page_ok(a.d, page);
    bad |= !ok;
    return ok ? page : 0;
  };
  u32x4_t kr[NT][KL], vr[NTO];
  auto load_k = [&](int tile, int page) {
    const char *src = (const char *)a.kp + (page_base(a.d, checked(page), kvh) + (F8 ? 16 : 8) * g) * ESZ;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int off = min(tile * TILE + KPL * (c >> 2) + 4 * t + (c & 3), last) & mask;
#pragma unroll
      for (int j = 0; j < KL; ++j) kr[t][j] = *(const u32x4_t *)(src + (unsigned)(off * HD * ESZ) + j * 64);
    }
  };
  auto load_v = [&](int tile, int page) {
    const int off = min(tile * TILE + KPL * g, last & ~(KPL - 1)) & mask;
    const char *src = (const char *)a.vp + (page_base(a.d, checked(page), kvh) + off + (c << a.d.page_shift)) * ESZ;
#pragma unroll
    for (int n = 0; n < NTO; ++n) vr[n] = *(const u32x4_t *)(src + (unsigned)((n * 16 << a.d.page_shift) * ESZ));
  };

  int tile = w.t0 + wave;
  const int t1 = last >= 0 ? w.t1 : 0;
  int kp = 0, vp = 0, next_kp = 0, next_vp = 0;
  if (tile < t1) page_ids(tile, kp, vp);
  if (tile + NW < t1) page_ids(tile + NW, next_kp, next_vp);
  int position = last;
  if (a.positions) position = a.positions[w.b];
  uint32_t qx[QN], qy[QN];
#pragma unroll
  for (int i = 0; i < QN; ++i) {
    const int row = min((int)threadIdx.x / HP + i * RS, rows - 1);
    const int64_t qi = w.b * a.ldq + (int64_t)(head0 + row) * HD;
    qx[i] = load_raw<F32>(a.q, qi + ea);
    qy[i] = load_raw<F32>(a.q, qi + eb);
  }
  if (tile < t1) {
    load_k(tile, kp);
    load_v(tile, vp);
  }

  // the query, rotated, as bf16 terms in operand order; rows past the group are zero
  {
    float sn = 0.f, cs = 1.f;
    if (turned) turn_of(turns, position, &sn, &cs);
    auto at = [&](int e, int row) {  // operand element of column e
      if constexpr (F8) return (((e >> 6) * 2 + ((e >> 3) & 1)) * 64 + ((e >> 4) & 3) * 16 + row) * 8 + (e & 7);
      else return ((e >> 5) * 64 + ((e >> 3) & 3) * 16 + row) * 8 + (e & 7);
    };
#pragma unroll
    for (int i = 0; i < QN; ++i) {
      const int row = threadIdx.x / HP + i * RS;
      if (row >= 16) break;
      const float x = row < rows ? value_of<F32>(qx[i]) : 0.f, y = row < rows ? value_of<F32>(qy[i]) : 0.f;
      float v0 = turned ? x * cs - y * sn : x, v1 = turned ? y * cs + x * sn : y;
#pragma unroll
      for (int t = 0; t < TERMS; ++t) {
        const __bf16 h0 = (__bf16)v0, h1 = (__bf16)v1;
        qf[t * KS * 512 + at(ea, row)] = h0;
        qf[t * KS * 512 + at(eb, row)] = h1;
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
    vp = next_vp;
    const bool more = tile + NW < t1;
    if (more) {
      kp = next_kp;
      if (tile + 2 * NW < t1) page_ids(tile + 2 * NW, next_kp, next_vp);
      load_k(tile + NW, kp);
    }
    // scores in powers of two, keys from the end on masked
    const int key0 = tile * TILE + KPL * g;
    const bool tail = tile * TILE + TILE > w.len;
    float mt = -INFINITY;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float v = s[t][r] * a.scale_log2;
        if (tail && key0 + 4 * t + r > last) v = -INFINITY;
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
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        s[t][r] = __builtin_amdgcn_exp2f(s[t][r] - m);
        l += s[t][r];
      }
    if (tail) {  // what lies behind the last key may be anything, NaN included
      constexpr int PER = F8 ? 4 : 2;  // elements of a register
      const int keep = max(w.len - key0, 0);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int n = min(max(keep - i * PER, 0), PER);
        const uint32_t bits = n == PER ? 0xFFFFFFFFu : (1u << (n * (32 / PER))) - 1;
#pragma unroll
        for (int k = 0; k < NTO; ++k) vr[k][i] &= bits;
      }
    }
#pragma unroll
    for (int u = 0; u < NT / 2; ++u) {  // 8 weights of the lane, as terms
      union {
        bf16x8 v;
        __bf16 e[8];
      } pf[TERMS];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float p = s[2 * u + e / 4][e % 4];
#pragma unroll
        for (int i = 0; i < TERMS; ++i) {
          pf[i].e[e] = (__bf16)p;
          p -= (float)pf[i].e[e];
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
  // the waves where no others had a tile. The readers weigh them, so that one barrier does;
  // with a common unit agreed on first, in the query's place, calls took 0.1-0.3 us longer.
  const bool all = t1 - w.t0 > NW / 2;
  l = sum_pair32(sum_pair16(l));
  if (g == 0) {
    ml[(wave * 16 + c) * 2] = m;
    ml[(wave * 16 + c) * 2 + 1] = l;
  }
  if (c < rows && (all || wave < NW / 2))
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
  auto put_out = [&](int row, int col, f32x4 v, float total) {
    const float scale = total != 0.f ? a.v_scale / total : 0.f;
    const int64_t oi = w.b * a.ldo + (int64_t)(head0 + row) * HD + col;
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
  const auto slots = slots_of(a, rows_max * HD);
  if (c < rows) {
    for (int n = wave; n < NTO; n += NW) {
      f32x4 v = obuf[n * 64 + lane] * f[0];
#pragma unroll
      for (int i = 1; i < NW / 2; ++i) v += obuf[(i * NTO + n) * 64 + lane] * f[i];
      if (all)
#pragma unroll
        for (int i = NW / 2; i < NW; ++i) v += obuf[(i * NTO + n) * 64 + lane] * f[i];
      if (w.splits == 1) put_out(c, 16 * n + 4 * g, v, sum);
      else put_slot(slots, (slot * rows_max + c) * HD + 16 * n + 4 * g, v);
    }
    if (w.splits > 1 && wave == 0 && g == 0)
      __hip_atomic_store(a.part_ml + (size_t)slot * rows_max + c, pair_of(mx, sum), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  if (w.splits == 1) return;

  // many splits: runs of kJoinFan first, into the first slot of each
  bool final = w.splits <= 2 * kJoinFan;
  for (;;) {
    const int run = w.split / kJoinFan * kJoinFan;
    const int first = final ? w.slot : w.slot + run, step = final && w.splits > 2 * kJoinFan ? kJoinFan : 1;
    const int n = !final ? min(kJoinFan, w.splits - run) : (w.splits + step - 1) / step;
    if (!last_to_arrive(a.arrived + (final ? a.slots : 0) + first, n, word)) return;
    join_slots<HD>(a, rows, rows_max, first, step, n, ml, top, obuf, [&](int row, int col, f32x4 v, float total) {
      if (final) put_out(row, col, v, total);
      else put_slot(slots, (first * rows_max + row) * HD + col, v);
    });
    if (final) return;
    if ((int)threadIdx.x < rows)
      __hip_atomic_store(a.part_ml + (size_t)first * rows_max + threadIdx.x,
                         pair_of(top[2 * threadIdx.x], top[2 * threadIdx.x + 1]), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    final = true;
  }
}

int kv_attend_target(int n_cu, int head_dim) {
  return n_cu * (head_dim == 256 ? kAttendPerCu<256> : head_dim == 128 ? kAttendPerCu<128> : kAttendPerCu<64>);
}

template <int HD, bool F32, bool F8>
static hipError_t attend_attr() {
  return hipFuncSetAttribute((const void *)kv_attend_kernel<HD, F32, F8>, hipFuncAttributeMaxDynamicSharedMemorySize,
                             attend_lds_floats<HD>() * 4);
}
template <int HD>
static hipError_t attend_attrs() {
  hipError_t e = attend_attr<HD, true, true>();
  if (e == hipSuccess) e = attend_attr<HD, true, false>();
  if (e == hipSuccess) e = attend_attr<HD, false, true>();
  if (e == hipSuccess) e = attend_attr<HD, false, false>();
  return e;
}
hipError_t kv_attend_init(int head_dim) {
  const hipError_t e = head_dim == 64 ? attend_attrs<64>() : head_dim == 128 ? attend_attrs<128>() : attend_attrs<256>();
  return e == hipSuccess ? kv_rows_init(head_dim) : e;
}

template <int HD, bool F32, bool F8>
static hipError_t launch_attend_type(KvAttendArgs a, hipStream_t s) {
  const int64_t units = (int64_t)a.n_seqs * a.d.n_kv_heads * ((a.group + 15) / 16);
  // the plan's workgroups: one for each unit, more where units are split, which are no
  // more than the slots, nor than the page table gives tiles
  const int64_t tiles = tiles_of_length((int)std::min<int64_t>((int64_t)a.pages_per_seq << a.d.page_shift, 0x7FFFFFFF), kTileKeys<F8>);
  const int64_t splits = splits_of((int)tiles, kAttendMinTiles, kAttendWhole<HD, F8>);
  const int64_t grid = std::min(units * splits, units + a.slots);
  a.unsplit = splits == 1;
  a.few_tiles = tiles < ((int64_t)1 << 31) / units;
  hipLaunchKernelGGL((kv_attend_kernel<HD, F32, F8>), dim3((unsigned)grid), dim3(64 * kAttendWaves),
                     (attend_lds_floats<HD>() * 4), s, a);
  return hipGetLastError();
}

template <int HD>
static hipError_t launch_attend_hd(const KvAttendArgs &a, bool f32, bool f8, hipStream_t s) {
  if (f32) return f8 ? launch_attend_type<HD, true, true>(a, s) : launch_attend_type<HD, true, false>(a, s);
  return f8 ? launch_attend_type<HD, false, true>(a, s) : launch_attend_type<HD, false, false>(a, s);
}

hipError_t launch_kv_attend(const KvAttendArgs &a, bool f32, bool f8, hipStream_t s) {
  if (a.n_seqs < 1 || a.group < 1 || a.n_heads != a.group * a.d.n_kv_heads || a.pages_per_seq < 1 || a.target < 1 ||
      a.slots < max_slots(a.target) || a.d.page_shift < 4)
    return hipErrorInvalidValue;
  if (a.k_scales) {  // a row for every sequence, which sees all of its keys
    KvRowsArgs r{};
    (KvAttendArgs &)r = a;
    r.n_rows = a.n_seqs;
    r.causal = true;
    return launch_kv_rows(r, f32, f8, s);
  }
  if (a.d.head_dim == 64) return launch_attend_hd<64>(a, f32, f8, s);
  if (a.d.head_dim == 128) return launch_attend_hd<128>(a, f32, f8, s);
  if (a.d.head_dim == 256) return launch_attend_hd<256>(a, f32, f8, s);
  return hipErrorInvalidValue;
}

// ---------------------------------------------------------------------------
// The expert's prefix from the pages, one 32-key block of one (layer, environment,
// KV head) per workgroup; bound by memory.  K rows are copied; a 16-byte chunk of the
// V^T store is two runs of four keys (vt_key_pos), which the transposed page holds
// side by side, so V needs no LDS.  Keys from n_keys on are zeros, as with
// prefix_pack_kernel.
// ---------------------------------------------------------------------------
// N (4 or 8) pool elements as bf16 bits, from an offset that is a multiple of N.
template <bool F8, int N>
__device__ __forceinline__ void load_run(const char *p, float scale, uint16_t *o) {
  typedef uint32_t words __attribute__((ext_vector_type(N / (F8 ? 4 : 2))));
  const words r = *(const words *)p;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    if constexpr (F8) {
      const float v = __builtin_amdgcn_cvt_f32_fp8((int)(r[e / 4] >> (8 * (e % 4))), 0) * scale;
      o[e] = __builtin_bit_cast(uint16_t, (__bf16)v);
    } else {
      o[e] = (uint16_t)(r[e / 2] >> (16 * (e % 2)));
      if ((o[e] & 0x7FFFu) > 0x7F80u) o[e] |= 0x40u;  // a signalling NaN turns quiet, as in prefix_pack_kernel
    }
  }
}

template <int HD, bool F8>
__global__ __launch_bounds__(256) void kv_prefix_kernel(KvPrefixArgs a) {
  const int blk = blockIdx.x, b = a.env0 + blockIdx.y / a.d.n_kv_heads, g = blockIdx.y % a.d.n_kv_heads;
  const size_t eh = (size_t)b * a.d.n_kv_heads + g;
  const size_t src = blockIdx.z * a.src_layer;
  bool bad = false;
  const int len = length_or_none(a.lens[b], a.pages_per_seq, a.d.page_shift, &bad);
  bad |= len < a.n_keys;
  const int n_keys = min(len, a.n_keys);
  constexpr int ESZ = F8 ? 1 : 2;
  const char *kp = (const char *)a.kp + src * ESZ, *vp = (const char *)a.vp + src * ESZ;
  __bf16 *kd = a.kc + blockIdx.z * a.dst_layer + (eh * a.s_alloc + (size_t)blk * 32) * HD;
  __bf16 *vd = a.vtc + blockIdx.z * a.dst_layer + vt_index(eh, blk * 32, 0, HD, a.s_alloc);
  const int mask = (1 << a.d.page_shift) - 1;
  // the block's 32 keys lie in one page, or in two of 16
  const int32_t *row = a.table + (int64_t)b * a.pages_per_seq;
  int page[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int s = blk * 32 + 16 * h;
    page[h] = s < n_keys ? row[s >> a.d.page_shift] : -1;
    if (s < n_keys && !page_ok(a.d, page[h])) {
      bad = true;
      page[h] = -1;
    }
  }
  // 8-bit values of a block times its scale
  const float *ks = nullptr, *vs = nullptr;
  if constexpr (F8)
    if (a.k_scales) {
      ks = a.k_scales + blockIdx.z * a.scale_layer;
      vs = a.v_scales + blockIdx.z * a.scale_layer;
    }
  float k_scale[2] = {a.k_scale, a.k_scale}, v_scale[2] = {a.v_scale, a.v_scale};  // of the block's two runs of 16
  if constexpr (F8)
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (ks && page[h] >= 0) {
        const size_t at = scale_index(a.d, page[h], g, (blk * 32 + 16 * h) & mask);
        k_scale[h] = ks[at];
        v_scale[h] = vs[at];
      }
  typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
#pragma unroll
  for (int it = 0; it < HD / 64; ++it) {
    const int q = it * 256 + threadIdx.x;
    const int key = q / (HD / 8), c = (q % (HD / 8)) * 8, s = blk * 32 + key, h = key >> 4;
    uint16_t o[8] = {};
    if (s < n_keys && page[h] >= 0) load_run<F8, 8>(kp + (page_base(a.d, page[h], g) + k_in_page(a.d, s & mask, c)) * ESZ, h ? k_scale[1] : k_scale[0], o);
    *(u16x8 *)(kd + key * HD + c) = u16x8{o[0], o[1], o[2], o[3], o[4], o[5], o[6], o[7]};
  }
#pragma unroll
  for (int it = 0; it < HD / 64; ++it) {
    const int q = it * 256 + threadIdx.x, c = q >> 2, ch = q & 3;
    uint16_t o[8] = {};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int s = blk * 32 + 16 * h + 4 * ch;  // four keys of one page
      if (s < n_keys && page[h] >= 0) {
        load_run<F8, 4>(vp + (page_base(a.d, page[h], g) + v_in_page(a.d, s & mask, c)) * ESZ, v_scale[h], o + 4 * h);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (s + e >= n_keys) o[4 * h + e] = 0;
      }
    }
    *(u16x8 *)(vd + c * 32 + ch * 8) = u16x8{o[0], o[1], o[2], o[3], o[4], o[5], o[6], o[7]};
  }
  if (bad) {
    raise_status(a.status, kStatusPage);
    raise_status(a.ctx_status, kStatusPage);
  }
}

template <int HD, bool F8>
static void launch_prefix_grid(const KvPrefixArgs &a, dim3 grid, hipStream_t s) {
  hipLaunchKernelGGL((kv_prefix_kernel<HD, F8>), grid, dim3(256), 0, s, a);
}

hipError_t launch_kv_prefix(const KvPrefixArgs &a, int batch, int n_layers, bool f8, hipStream_t s) {
  if (batch < 1 || n_layers < 1 || a.s_alloc < 32 || a.s_alloc % 32 || a.n_keys > a.s_alloc) return hipErrorInvalidValue;
  if (a.d.n_kv_heads > 65535 || (a.k_scales && !f8)) return hipErrorInvalidValue;
  const int envs = 65535 / a.d.n_kv_heads;  // grid dimensions y and z take 65535 at most
  for (int l = 0; l < n_layers; l += 32768)
    for (int b = 0; b < batch; b += envs) {
      KvPrefixArgs p = a;
      p.env0 = b;
      p.kp = (const char *)a.kp + l * a.src_layer * (f8 ? 1 : 2);
      p.vp = (const char *)a.vp + l * a.src_layer * (f8 ? 1 : 2);
      if (a.k_scales) {
        p.k_scales = a.k_scales + l * a.scale_layer;
        p.v_scales = a.v_scales + l * a.scale_layer;
      }
      p.kc = a.kc + l * a.dst_layer;
      p.vtc = a.vtc + l * a.dst_layer;
      const int n = batch - b < envs ? batch - b : envs, z = n_layers - l < 32768 ? n_layers - l : 32768;
      const dim3 grid(a.s_alloc / 32, n * a.d.n_kv_heads, z);
      if (a.d.head_dim == 64) f8 ? launch_prefix_grid<64, true>(p, grid, s) : launch_prefix_grid<64, false>(p, grid, s);
      else if (a.d.head_dim == 128) f8 ? launch_prefix_grid<128, true>(p, grid, s) : launch_prefix_grid<128, false>(p, grid, s);
      else if (a.d.head_dim == 256) f8 ? launch_prefix_grid<256, true>(p, grid, s) : launch_prefix_grid<256, false>(p, grid, s);
      else return hipErrorInvalidValue;
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
  return hipSuccess;
}

}  // namespace uad
