// Append to 8-bit pools with a scale for every block of 16 tokens and KV head, and the page
// tables of a paged K/V cache.  Layouts and rules in paged.h.
#include "paged_device.h"

namespace uad {

// ---------------------------------------------------------------------------
// Append with scales for blocks: a wave (two at head dim 256, whose registers four on a
// SIMD would not hold) per block of 16 tokens, KV head and pool, so that who finds a block's
// largest magnitude also writes it; a workgroup for the blocks of a tile of up to 64 cache
// positions (see paged.h), or for the token of a sequence.  Rows are loaded once and kept in
// registers.  Scales are powers of two: values are divided exactly, and what a block holds
// already, rounded anew where its scale must grow, changes only where it falls below e4m3's
// normal range.  V goes to its transposed page through LDS, so that it leaves in pieces of
// 64 bytes a column.
//
// Bound by memory with many rows: 64 prompts of 816 rows, head dim 256, read 53 MB and write
// 27 in 21.4 us, 3.8 TB/s of the 5.4 that a copy reaches.  A block's rows must all be there
// before the first is stored, and the table's entry before that.  Of the 1660 workgroups with
// work two are on a CU at once (115 registers: four waves on a SIMD), so three to four come
// one after the other, each with that whole chain; the next block's rows, on their way
// meanwhile, would be 16 registers more (32 of fp32) and leave one workgroup a CU.  With few
// rows, by the chain of loads (length, page, rows): 64 sequences with a token each 4.1 us, 16
// uneven prompts of 64 columns 5.2.
// ---------------------------------------------------------------------------
// 4 e4m3 values times `ratio`, rounded anew.
__device__ __forceinline__ uint32_t rescaled4(uint32_t w, float ratio) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  const int x = __builtin_amdgcn_cvt_pk_fp8_f32(lo[0] * ratio, lo[1] * ratio, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(hi[0] * ratio, hi[1] * ratio, x, true);
}
__device__ __forceinline__ u32x4_t rescaled16(u32x4_t w, float ratio) {
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = rescaled4(w[i], ratio);
  return w;
}
// The first n (0 .. 16) bytes of a, the others of b.
__device__ __forceinline__ u32x4_t first_bytes(u32x4_t a, u32x4_t b, int n) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t bits = run_bits(0, 8 * (n - 4 * i), 32);
    a[i] = (a[i] & bits) | (b[i] & ~bits);
  }
  return a;
}

// 4 x 4 bytes: byte i of each of four words.
__device__ __forceinline__ void transpose4(uint32_t a, uint32_t b, uint32_t c, uint32_t d, uint32_t *o) {
  const uint32_t ab = __builtin_amdgcn_perm(b, a, 0x05010400u), cd = __builtin_amdgcn_perm(d, c, 0x05010400u);  // a0 b0 a1 b1
  const uint32_t ef = __builtin_amdgcn_perm(b, a, 0x07030602u), gh = __builtin_amdgcn_perm(d, c, 0x07030602u);  // a2 b2 a3 b3
  o[0] = __builtin_amdgcn_perm(cd, ab, 0x05040100u);
  o[1] = __builtin_amdgcn_perm(cd, ab, 0x07060302u);
  o[2] = __builtin_amdgcn_perm(gh, ef, 0x05040100u);
  o[3] = __builtin_amdgcn_perm(gh, ef, 0x07060302u);
}

template <int HD, bool F32, int BLOCKS, int PARTS>
__global__ __launch_bounds__(64 * BLOCKS * PARTS) void kv_append_blocks_kernel(KvAppendArgs a) {
  constexpr int WAVES = BLOCKS * PARTS, PIECES = HD / 8;  // of 8 elements of a row
  constexpr int PAIRS = PIECES / 2 / PARTS;               // of them, of a wave and token
  constexpr int N = kScaleBlock * PAIRS / 64;             // of a lane
  __shared__ __align__(16) uint8_t lds[BLOCKS * kScaleBlock * HD];
  __shared__ int plan[(kPlanScans + 1) * WAVES];
  __shared__ float most_of[2 * WAVES];
  const int lane = threadIdx.x & 63, wave = (threadIdx.x >> 6) / PARTS, part = (threadIdx.x >> 6) % PARTS;
  const int head = blockIdx.y, shift = a.d.page_shift, mask = (1 << shift) - 1;
  const bool is_v = blockIdx.z != 0;
  const int wg = a.row0 + blockIdx.x;
  AppendTile t;
  if constexpr (BLOCKS == 1) {
    bool bad = false;
    t.b = t.row = wg;
    t.first = t.last = length_or_none(a.lens[t.b], a.pages_per_seq, shift, &bad) - 1;
    if (t.first < 0) {  // no room for a new token, or none that can be used
      if (threadIdx.x == 0) raise_status(a.status, kStatusPage);
      return;
    }
  } else {
    if (!plan_append<WAVES>(a, wg, plan, &t)) return;
  }
  // this wave's block of the tile, and its tokens first .. last that get rows
  const int block0 = t.first & ~(kScaleBlock - 1), block = block0 + kScaleBlock * wave;
  const int first = max(t.first, block), last = min(t.last, block + kScaleBlock - 1), tokens = max(last - first + 1, 0);
  const int page = a.table[(int64_t)t.b * a.pages_per_seq + (t.first >> shift)];  // looked at when the rows are on their way
  const int held = first - block, items = tokens * PAIRS;  // tokens that the block has already
  const void *src = is_v ? a.v : a.k;
  const int64_t ld = is_v ? a.ldv : a.ldk;
  const int row0 = t.row + first - t.first;
  // an item: pieces x and y of a token, for K the ones that are turned with each other
  const int half = a.rope_dim / 16;
  auto pieces = [&](int i, int *x, int *y) {
    const bool apart = !is_v && !a.rope_pairs && i < half;
    *x = apart ? i : 2 * i;
    *y = apart ? i + half : 2 * i + 1;
  };
  // an item: a lane's pair of pieces, of a token for each round (behind the last one: of it)
  static_assert(64 % PAIRS == 0, "the same pieces in every round");
  const int mine = part * PAIRS + lane % PAIRS;
  auto token_of = [&](int n) { return min((lane + n * 64) / PAIRS, tokens - 1); };
  int px, py;
  pieces(mine, &px, &py);
  uint64_t step[8] = {};
  if (!is_v && mine < half) {
#pragma unroll
    for (int e = 0; e < 8; ++e) step[e] = a.steps[8 * mine + e];
  }
  Raw8<F32> rx[N], ry[N];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    if (n * 64 >= items) break;
    const int64_t at = (int64_t)(row0 + token_of(n)) * ld + (int64_t)head * HD;
    rx[n].load(src, at + 8 * px, a.in_vec);
    ry[n].load(src, at + 8 * py, a.in_vec);
  }
  if (!page_ok(a.d, page)) {  // the whole tile's
    if (lane == 0) raise_status(a.status, kStatusPage);
    return;
  }
  float *scales = (is_v ? a.v_scales : a.k_scales) + scale_index(a.d, page, head, block0 & mask) + wave;
  const float was = tokens && held ? *scales : 0.f;
  float u[N][8], w[N][8], most = 0.f;
  uint32_t turn[8] = {};  // of the lane's pairs at the last item's token
#pragma unroll
  for (int n = 0; n < N; ++n) {
    if (n * 64 >= items) break;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      u[n][e] = rx[n].value(e);
      w[n][e] = ry[n].value(e);
    }
    if (!is_v && mine < half) {
      const int position = a.positions ? a.positions[row0 + token_of(n)] : first + token_of(n);
      float s[8], c[8];
      // the next round's token is as many further, up to the last one
      if (n == 0 || a.positions || lane + n * 64 >= items) {
#pragma unroll
        for (int e = 0; e < 8; ++e) turn[e] = turned(step[e], position);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) turn[e] += (uint32_t)(step[e] * (64 / PAIRS) >> 32);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) sine_of(turn[e], &s[e], &c[e]);
      if (a.rope_pairs) {  // elements 16 i + 2 e and the next
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float &p = e < 4 ? u[n][2 * e] : w[n][2 * e - 8], &q = e < 4 ? u[n][2 * e + 1] : w[n][2 * e - 7];
          const float p0 = p, q0 = q;
          p = p0 * c[e] - q0 * s[e];
          q = q0 * c[e] + p0 * s[e];
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float p0 = u[n][e], q0 = w[n][e];
          u[n][e] = p0 * c[e] - q0 * s[e];
          w[n][e] = q0 * c[e] + p0 * s[e];
        }
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) most = fmaxf(most, fmaxf(fabsf(u[n][e]), fabsf(w[n][e])));  // which passes a NaN over
  }
  auto over_block = [&](float m, int k) {
    m = max_pair32(max_pair16(max_row16(m)));
    if constexpr (PARTS > 1) {  // the waves of a block
      if (lane == 0) most_of[k * WAVES + (threadIdx.x >> 6)] = m;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < PARTS; ++i) m = fmaxf(m, most_of[k * WAVES + wave * PARTS + i]);
    }
    return m;
  };
  most = over_block(most, 0);
  const float most_any = most;
  bool infinite = __builtin_amdgcn_readfirstlane(__float_as_int(most)) == 0x7F800000;
  if constexpr (PARTS > 1) {  // in any block: all waves take part
#pragma unroll
    for (int i = 0; i < WAVES; ++i) infinite |= most_of[i] == INFINITY;
  }
  if (infinite) {  // of the finite ones
    most = 0.f;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      if (n * 64 >= items) break;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = fabsf(u[n][e]), y = fabsf(w[n][e]);
        most = fmaxf(most, fmaxf(x < INFINITY ? x : 0.f, y < INFINITY ? y : 0.f));
      }
    }
    most = over_block(most, 1);
  }
  float scale = __uint_as_float(scale_bits(__float_as_uint(most)));
  if (held) scale = fmaxf(scale, was);
  const bool grows = held && scale > was;
  const float ratio = grows ? was / scale : 1.f, inv = 1.f / scale;
  if (lane == 0 && part == 0 && tokens && (!held || grows)) *scales = scale;
  const size_t base = page_base(a.d, page, head);
  // nothing to cut and a power of two: the quotients are products, exactly
  const bool plain = __builtin_amdgcn_readfirstlane(most_any <= 448.f * scale && most_any < INFINITY && (__float_as_uint(scale) & 0x7FFFFFu) == 0) != 0;
  auto quantised = [&](float *x) {
    if (plain) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] *= inv;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)  // infinities apart: of a scale that the caller has set, 448 times it may be one too
        x[e] = fabsf(x[e]) == INFINITY ? copysignf(448.f, x[e]) : quotient(x[e], scale, inv);
    }
  };
  if (!is_v) {
    if (!tokens) return;
    uint8_t *dst = (uint8_t *)a.kp + base + k_in_page(a.d, block & mask, 0);  // the block's rows lie side by side
    if (grows)
      for (int i = part * 64 + lane; i < held * (HD / 16); i += 64 * PARTS) {
        u32x4_t *p = (u32x4_t *)dst + i;
        *p = rescaled16(*p, ratio);
      }
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int item = lane + n * 64;
      if (item >= items) break;
      quantised(u[n]);
      quantised(w[n]);
      uint8_t *to = dst + (held + token_of(n)) * HD;
      Pool8<true> o;
      o.set(u[n]);
      o.put_page(to + 8 * px);
      o.set(w[n]);
      o.put_page(to + 8 * py);
    }
    return;
  }
  // V: the tile's tokens in LDS, a token's 8-byte piece p at place p ^ token, then a block of
  // four columns a thread, the tile's blocks of a column next to each other
  __shared__ int held_of[BLOCKS], tokens_of[BLOCKS];
  __shared__ float ratio_of[BLOCKS];
  auto place = [&](int token, int piece) { return (token * PIECES + (piece ^ (token & (PIECES - 1)))) * 8; };
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int item = lane + n * 64, token = kScaleBlock * wave + held + token_of(n);
    if (item >= items) break;
    quantised(u[n]);
    quantised(w[n]);
    Pool8<true> o;
    o.set(u[n]);
    o.put(lds + place(token, 2 * mine));
    o.set(w[n]);
    o.put(lds + place(token, 2 * mine + 1));
  }
  if (lane == 0 && part == 0) {
    held_of[wave] = held;
    tokens_of[wave] = tokens;
    ratio_of[wave] = ratio;
  }
  __syncthreads();
  const int blocks = (t.last - block0) / kScaleBlock + 1;
  uint8_t *vp = (uint8_t *)a.vp + base + v_in_page(a.d, block0 & mask, 0);
  for (int item = threadIdx.x; item < HD / 4 * blocks; item += 64 * WAVES) {
    const int blk = item % blocks, word = item / blocks;
    const int old_tokens = held_of[blk], new_tokens = tokens_of[blk];
    const float by = ratio_of[blk];
    uint32_t v[kScaleBlock];
#pragma unroll
    for (int e = 0; e < kScaleBlock; ++e) v[e] = *(const uint32_t *)(lds + place(kScaleBlock * blk + e, word / 2) + (word & 1) * 4);
    u32x4_t cols[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      uint32_t x[4];
      transpose4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3], x);
#pragma unroll
      for (int col = 0; col < 4; ++col) cols[col][k] = x[col];
    }
#pragma unroll
    for (int col = 0; col < 4; ++col) {
      u32x4_t o = cols[col];
      u32x4_t *dst = (u32x4_t *)(vp + ((size_t)(4 * word + col) << shift) + kScaleBlock * blk);
      if (new_tokens < kScaleBlock) {  // what is held, and what lies behind the last token
        const u32x4_t old = *dst;
        o = first_bytes(by != 1.f ? rescaled16(old, by) : old, first_bytes(o, old, old_tokens + new_tokens), old_tokens);
      }
      __builtin_nontemporal_store(o, dst);
    }
  }
}

template <int HD, bool F32>
static hipError_t launch_append_blocks_type(const KvAppendArgs &a, hipStream_t s) {
  constexpr int64_t kMaxWgs = 1 << 21;  // work items of a grid stay below 2^32
  const int64_t tiles = a.row_start ? append_grid(a.n_rows, a.n_seqs, append_tile_shift(a.d.page_shift)) : a.n_rows;
  for (int64_t r = 0; r < tiles; r += kMaxWgs) {
    KvAppendArgs p = a;
    p.row0 = (int)r;
    const dim3 grid((unsigned)std::min(tiles - r, kMaxWgs), a.d.n_kv_heads, 2);
    constexpr int BLOCKS = kAppendTile / kScaleBlock, PARTS = HD > 128 ? 2 : 1;
    if (!a.row_start) hipLaunchKernelGGL((kv_append_blocks_kernel<HD, F32, 1, 1>), grid, dim3(64), 0, s, p);
    else hipLaunchKernelGGL((kv_append_blocks_kernel<HD, F32, BLOCKS, PARTS>), grid, dim3(BLOCKS * PARTS * 64), 0, s, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_kv_append_blocks(const KvAppendArgs &a, bool f32, hipStream_t s) {
  if (a.n_rows < 1 || a.n_seqs < 1 || a.d.page_shift < 4 || a.rope_dim % 16 || a.rope_dim > a.d.head_dim || !a.k_scales ||
      !a.v_scales || a.d.n_kv_heads > 65535 || (!a.row_start && a.n_rows != a.n_seqs))
    return hipErrorInvalidValue;
  if (a.d.head_dim == 64) return f32 ? launch_append_blocks_type<64, true>(a, s) : launch_append_blocks_type<64, false>(a, s);
  if (a.d.head_dim == 128) return f32 ? launch_append_blocks_type<128, true>(a, s) : launch_append_blocks_type<128, false>(a, s);
  if (a.d.head_dim == 256) return f32 ? launch_append_blocks_type<256, true>(a, s) : launch_append_blocks_type<256, false>(a, s);
  return hipErrorInvalidValue;
}

// ---------------------------------------------------------------------------
// Pages of new tokens.  Every workgroup works out the sums over all sequences for itself,
// into LDS (up to kSumEntries of them; with more sequences an entry stands for a run), and
// fills its share of the table's entries and of the slots, eight rows a thread.  Lengths
// and the free pages' number may be written where the others read them: then by the last
// workgroup to be done.  64 sequences with a token each: 4.5 us a call in a graph: lengths,
// the ids for the table and then, though they need not wait for those, the ids for the slots,
// between four scans (without slots 0.8 us less).  1024 prompts with 484 176 rows: 10.1 us; as
// many sequences with a row each take 6.5, the same rows of 8 sequences 8.9, the slots' 3.9 MB
// at a copy's rate 0.8.  Without slots the launch has no measure of the rows, and a few
// workgroups fill all of the table: 30 000 entries 65 us.
// ---------------------------------------------------------------------------
constexpr int kSumEntries = 2048, kSumsPerThread = kSumEntries / 256;

// Sums of two values over the threads, each within 31 bits in all.
struct SumScan {
  int *lds;  // [8] for each scan
  // Sums of the threads before this one, and of all.
  __device__ __forceinline__ void operator()(int x, int y, int *x_before, int *x_all, int *y_before, int *y_all) {
    const int x_upto = scan_wave64(x), y_upto = scan_wave64(y), wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 63) {
      lds[wave] = x_upto;
      lds[4 + wave] = y_upto;
    }
    __syncthreads();
    *x_before = x_upto - x;
    *y_before = y_upto - y;
    *x_all = *y_all = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      *x_before += w < wave ? lds[w] : 0;
      *y_before += w < wave ? lds[4 + w] : 0;
      *x_all += lds[w];
      *y_all += lds[4 + w];
    }
    lds += 8;
  }
};
// The first entry whose sum is above i.
__device__ __forceinline__ int entry_of(const int *upto, int n, int i) {
  int lo = 0;
  for (int step = n > 0 ? 1 << (31 - __builtin_clz(n)) : 0; step > 0; step /= 2)
    if (lo + step <= n && upto[lo + step - 1] <= i) lo += step;
  return lo;
}

// Slots of runs of RUN rows; `begin` and `next` walk the sequences from an entry on.
template <int RUN, class Begin, class Next>
__device__ __forceinline__ void fill_slots(const KvReserveArgs &a, int me, int everyone, int total_rows, int n_free, int entries,
                                           const int *rows_upto, Begin begin, Next next, bool *odd) {
  const bool wide = RUN > 1 && ((uintptr_t)a.slots & 15) == 0;
  for (int64_t r0 = (int64_t)me * RUN; r0 < a.n_rows; r0 += (int64_t)everyone * RUN) {
    int64_t slot[RUN];
    int id[RUN], off[RUN];
#pragma unroll
    for (int k = 0; k < RUN; ++k) slot[k] = -1;
    if (r0 < total_rows) {
      auto s = begin(entry_of(rows_upto, entries - 1, (int)r0));
#pragma unroll
      for (int k = 0; k < RUN; ++k) {
        const int r = min((int)r0 + k, total_rows - 1);
        while (s.b < a.n_seqs - 1 && r >= s.row + s.n) next(&s);  // the last at the latest
        const int p = s.len + r - s.row, i = (p >> a.page_shift) - pages_of(s.len, a.page_shift);
        off[k] = p & ((1 << a.page_shift) - 1);
        // below 0: the page that the sequence's last token is in
        const int32_t *at = i < 0 ? a.table + (int64_t)s.b * a.pages_per_seq + (p >> a.page_shift) : a.free_pages + (n_free - 1 - (s.page + i));
        id[k] = *at;
      }
#pragma unroll
      for (int k = 0; k < RUN; ++k) {
        const bool fine = id[k] >= 0 && id[k] < a.n_pages;
        *odd |= !fine;
        if (fine && r0 + k < total_rows) slot[k] = ((int64_t)id[k] << a.page_shift) + off[k];
      }
    }
    if (wide && r0 + RUN <= a.n_rows) {
      typedef int64_t i64x2_t __attribute__((ext_vector_type(2)));
#pragma unroll
      for (int k = 0; k + 1 < RUN; k += 2) *(i64x2_t *)(a.slots + r0 + k) = i64x2_t{slot[k], slot[k + 1]};
    } else {
#pragma unroll
      for (int k = 0; k < RUN; ++k)
        if (r0 + k < a.n_rows) a.slots[r0 + k] = slot[k];
    }
  }
}

__global__ __launch_bounds__(256) void kv_reserve_kernel(KvReserveArgs a) {
  __shared__ int scans[2 * 8], rows_upto[kSumEntries], pages_upto[kSumEntries], lens[kSumEntries], word[1];
  SumScan scan{scans};
  const int per = (a.n_seqs + kSumEntries - 1) / kSumEntries, entries = (a.n_seqs + per - 1) / per;  // sequences of an entry
  const int mine = (entries + 255) / 256, e0 = threadIdx.x * mine;                                  // entries of a thread
  auto tokens = [&](int b) { return a.new_tokens ? a.new_tokens[b] : 1; };
  auto pages = [&](int len, int n) { return pages_of(len + n, a.page_shift) - pages_of(len, a.page_shift); };
  const int n_free = *a.n_free;
  bool bad = false;
  int64_t rows = 0;
  int row_sum[kSumsPerThread], page_sum[kSumsPerThread], need = 0;  // up to and with each entry; checked before they count
  auto count = [&](int len, int n) {
    if (growth_ok(len, n, a.pages_per_seq, a.page_shift)) {
      rows += n;
      need += pages(len, n);
    } else {
      bad = true;
    }
  };
  if (per == 1) {
    int len[kSumsPerThread], n[kSumsPerThread];  // all on their way at once
#pragma unroll
    for (int k = 0; k < kSumsPerThread; ++k) {
      const int b = min(e0 + min(k, mine - 1), a.n_seqs - 1);
      len[k] = a.lens[b];
      n[k] = tokens(b);
    }
#pragma unroll
    for (int k = 0; k < kSumsPerThread; ++k) {
      if (k < mine && e0 + k < a.n_seqs) {
        lens[e0 + k] = len[k];
        count(len[k], n[k]);
      }
      row_sum[k] = (int)rows;
      page_sum[k] = need;
    }
  } else {
#pragma unroll
    for (int k = 0; k < kSumsPerThread; ++k) {
      if (k < mine)
        for (int b = (e0 + k) * per; b < min((e0 + k + 1) * per, a.n_seqs); ++b) count(a.lens[b], tokens(b));
      row_sum[k] = (int)rows;
      page_sum[k] = need;
    }
  }
  int hi, lo, none[2];
  scan((int)(rows >> 22), (int)(rows & 0x3FFFFF), &none[0], &hi, &none[1], &lo);
  const int64_t all_rows = ((int64_t)hi << 22) + lo;
  bad |= all_rows > 0x7FFFFFFF || (a.slots && all_rows > a.n_rows) || n_free < 0 || n_free > a.n_pages;
  bad = __syncthreads_or(bad);
  // sums fit from here on; a page that is needed gets a row at least
  int rows_before, total_rows, pages_before, total;
  scan(bad ? 0 : (int)rows, bad ? 0 : need, &rows_before, &total_rows, &pages_before, &total);
  bad |= total > n_free;
#pragma unroll
  for (int k = 0; k < kSumsPerThread; ++k)
    if (k < mine && e0 + k < entries) {
      rows_upto[e0 + k] = rows_before + row_sum[k];
      pages_upto[e0 + k] = pages_before + page_sum[k];
    }
  __syncthreads();
  // Nothing that may be written in place is read from here on, but for lengths with more
  // sequences than entries: that this workgroup has got here can be told at once.
  const bool early = per == 1 && gridDim.x > 1;
  unsigned arrived = 0;
  if (early && threadIdx.x == 0) arrived = __hip_atomic_fetch_add(a.arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  // the first workgroups fill the slots, the others the table, or each does both
  const bool apart = a.slot_wgs < (int)gridDim.x, slots = a.slots && (int)blockIdx.x < a.slot_wgs, table = !apart || (int)blockIdx.x >= a.slot_wgs;
  const int me = blockIdx.x * 256 + threadIdx.x, slot_threads = a.slot_wgs * 256;
  const int table_me = apart ? me - slot_threads : me, table_threads = apart ? (int)gridDim.x * 256 - slot_threads : slot_threads;
  if (bad) {
    if (me == 0) raise_status(a.status, kStatusPage);
    if (a.row_start && blockIdx.x == 0)
      for (int b = threadIdx.x; b <= a.n_seqs; b += 256) a.row_start[b] = 0;
    if (slots)
      for (int64_t r = me; r < a.n_rows; r += slot_threads) a.slots[r] = -1;
  } else {
    bool odd = false;
    // sequences from entry e on: what comes before sequence b, and its length and new rows
    struct At {
      int e, b, row, page, len, n;
    };
    auto enter = [&](At *s) {
      if (per == 1) {
        s->len = lens[s->b];
        s->n = rows_upto[s->b] - s->row;
      } else {
        s->len = a.lens[s->b];
        s->n = tokens(s->b);
      }
    };
    auto begin = [&](int e) {
      At s{e, e * per, e ? rows_upto[e - 1] : 0, e ? pages_upto[e - 1] : 0, 0, 0};
      enter(&s);
      return s;
    };
    auto next = [&](At *s) {
      s->row += s->n;
      s->page += pages(s->len, s->n);
      ++s->b;
      enter(s);
    };
    for (int i = table_me; table && i < total; i += table_threads) {
      At s = begin(entry_of(pages_upto, entries - 1, i));
      while (s.b < a.n_seqs - 1 && i >= s.page + pages(s.len, s.n)) next(&s);  // the last at the latest
      const int id = a.free_pages[n_free - 1 - i];
      a.table[(int64_t)s.b * a.pages_per_seq + pages_of(s.len, a.page_shift) + i - s.page] = id;
      odd |= id < 0 || id >= a.n_pages;
    }
    if (slots && a.n_rows <= slot_threads) {
      fill_slots<1>(a, me, slot_threads, total_rows, n_free, entries, rows_upto, begin, next, &odd);
    } else if (slots) {
      fill_slots<8>(a, me, slot_threads, total_rows, n_free, entries, rows_upto, begin, next, &odd);
    }
    if (odd) raise_status(a.status, kStatusPage);
  }
  // row_start and, where it lies apart, lens_out are the first workgroup's
  const bool in_place = a.lens_out == a.lens;
  auto finish = [&](bool starts, bool lengths) {
    int at = rows_before;
    for (int b = e0 * per; b < min((e0 + mine) * per, a.n_seqs); ++b) {
      const int len = per == 1 ? lens[b] : a.lens[b], n = bad ? 0 : per == 1 ? rows_upto[b] - at : tokens(b);
      if (starts) a.row_start[b] = at;
      at += n;
      if (lengths) a.lens_out[b] = len + n;
    }
  };
  const bool starts = a.row_start && !bad;
  if (blockIdx.x == 0) {
    if (starts || !in_place) finish(starts, !in_place);
    if (starts && threadIdx.x == 0) a.row_start[a.n_seqs] = total_rows;
  }
  if (early) {
    if (threadIdx.x == 0) {
      word[0] = arrived == gridDim.x - 1;
      if (word[0]) __hip_atomic_store(a.arrived, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (!word[0]) return;
  } else if (gridDim.x > 1) {
    if (!last_to_arrive(a.arrived, gridDim.x, (float *)word)) return;
  } else {
    __syncthreads();
  }
  if (in_place && !bad) finish(false, true);
  if (threadIdx.x == 0) *a.n_free_out = bad ? n_free : n_free - total;
}

// Pages that no later token sees: counted by a wave per sequence, then moved to the free
// ones by the same waves, in the order of the table.
__device__ __forceinline__ bool gone(const KvReleaseArgs &a, int len, int i, int id, bool *odd) {
  if (id < 0 || page_in_use(i, len, a.window, a.sinks, a.page_shift)) return false;
  *odd |= id >= a.n_pages;
  return id < a.n_pages;
}

__global__ __launch_bounds__(256) void kv_count_gone_kernel(KvReleaseArgs a) {
  const int lane = threadIdx.x & 63;
  bool odd = false;
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.n_free_was = *a.n_free;  // which the other kernel reads and writes
  for (int b = blockIdx.x * 4 + (threadIdx.x >> 6); b < a.n_seqs; b += gridDim.x * 4) {
    const int len = a.lens[b];
    const int32_t *row = a.table + (int64_t)b * a.pages_per_seq;
    constexpr int AHEAD = 4;
    int n = 0;
    odd |= len < 0;
    for (int i0 = 0; len >= 0 && i0 < a.pages_per_seq; i0 += 64 * AHEAD) {
      int id[AHEAD];
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) id[k] = row[min(i0 + 64 * k + lane, a.pages_per_seq - 1)];
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) {
        const int i = i0 + 64 * k + lane;
        n += __popcll(__ballot(i < a.pages_per_seq && gone(a, len, i, id[k], &odd)));
      }
    }
    if (lane == 0) a.counts[b] = n;
  }
  if (odd) raise_status(a.status, kStatusPage);
}

__global__ __launch_bounds__(256) void kv_release_kernel(KvReleaseArgs a) {
  __shared__ int scans[2 * 8], upto[kSumEntries];
  SumScan scan{scans};
  const int per = (a.n_seqs + kSumEntries - 1) / kSumEntries, entries = (a.n_seqs + per - 1) / per;
  const int mine = (entries + 255) / 256, e0 = threadIdx.x * mine;
  const int n_free = *a.n_free_was;
  int64_t pages = 0;  // at most as many as the pool has, else nothing is done
  int sums[kSumsPerThread], first[kSumsPerThread];
#pragma unroll
  for (int k = 0; k < kSumsPerThread; ++k) first[k] = a.counts[min((e0 + min(k, mine - 1)) * per, a.n_seqs - 1)];
#pragma unroll
  for (int k = 0; k < kSumsPerThread; ++k) {
    if (k < mine && (e0 + k) * per < a.n_seqs) {
      pages += first[k];
      for (int b = (e0 + k) * per + 1; b < min((e0 + k + 1) * per, a.n_seqs); ++b) pages += a.counts[b];
    }
    sums[k] = (int)pages;
  }
  int big, before, total, none[3];
  const bool many = pages > a.n_pages;
  scan(many ? 1 << 22 : (int)(pages >> 10), 0, &none[0], &big, &none[1], &none[2]);  // in units of 2^10, so that they fit
  bool bad = __syncthreads_or(many) || big > (a.n_pages >> 10) + 1 || n_free < 0 || n_free > a.n_pages;
  scan(bad ? 0 : (int)pages, 0, &before, &total, &none[0], &none[1]);
  bad |= (int64_t)n_free + total > a.n_pages;
#pragma unroll
  for (int k = 0; k < kSumsPerThread; ++k)
    if (k < mine && e0 + k < entries) upto[e0 + k] = before + sums[k];
  __syncthreads();
  if (!bad) {
    const int lane = threadIdx.x & 63;
    for (int b = blockIdx.x * 4 + (threadIdx.x >> 6); b < a.n_seqs; b += gridDim.x * 4) {
      if (a.counts[b] == 0) continue;
      const int len = a.lens[b], e = b / per;
      int at = n_free + (e ? upto[e - 1] : 0);
      for (int x = e * per; x < b; ++x) at += a.counts[x];
      int32_t *row = a.table + (int64_t)b * a.pages_per_seq;
      constexpr int AHEAD = 4;
      for (int i0 = 0; i0 < a.pages_per_seq; i0 += 64 * AHEAD) {
        int id[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) id[k] = row[min(i0 + 64 * k + lane, a.pages_per_seq - 1)];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
          const int i = i0 + 64 * k + lane;
          bool odd = false;
          const bool go = i < a.pages_per_seq && gone(a, len, i, id[k], &odd);
          const uint64_t goes = __ballot(go);
          if (go) {
            const int to = at + __popcll(goes & ((1ull << lane) - 1));
            if (to < a.n_pages) a.free_pages[to] = id[k];  // always, unless the caller's arrays change while this runs
            row[i] = -1;
          }
          at += __popcll(goes);
        }
      }
    }
  } else if (blockIdx.x == 0 && threadIdx.x == 0) {
    raise_status(a.status, kStatusPage);
  }
  if (blockIdx.x == 0 && threadIdx.x == 0 && !bad) *a.n_free = n_free + total;
}

hipError_t launch_kv_reserve(const KvReserveArgs &a, hipStream_t s) {
  if (a.n_seqs < 1 || a.pages_per_seq < 1 || a.page_shift < 4 || a.n_pages < 1 || a.n_rows < 0) return hipErrorInvalidValue;
  // a workgroup for every 2048 slots, up to two a CU, and from four of them on others for
  // the table
  KvReserveArgs p = a;
  const int64_t items = std::max<int64_t>(a.slots ? a.n_rows : 0, (int64_t)a.n_seqs * 8);
  p.slot_wgs = (int)std::min<int64_t>((items + 2047) / 2048, 512);
  hipLaunchKernelGGL(kv_reserve_kernel, dim3(p.slot_wgs < 4 ? p.slot_wgs : p.slot_wgs + std::min(p.slot_wgs / 2, 128)), dim3(256), 0, s, p);
  return hipGetLastError();
}

hipError_t launch_kv_release(const KvReleaseArgs &a, hipStream_t s) {
  if (a.n_seqs < 1 || a.pages_per_seq < 1 || a.page_shift < 4 || a.n_pages < 1) return hipErrorInvalidValue;
  const unsigned grid = (unsigned)std::min<int64_t>(((int64_t)a.n_seqs + 3) / 4, 512);
  hipLaunchKernelGGL(kv_count_gone_kernel, dim3(grid), dim3(256), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kv_release_kernel, dim3(grid), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace uad
