// Append to 8-bit pools with a scale for every block of 16 tokens and KV head, and the page
// tables of a paged K/V cache.  Layouts and rules in paged.h.
#include "paged_device.h"

namespace uad {

// ---------------------------------------------------------------------------
// Append with scales for blocks: a wave per block of 16 tokens, KV head and pool, so that
// who finds a block's largest magnitude also writes it; as many waves to a workgroup as
// blocks in a tile of up to 64 cache positions (see paged.h), or one for the token of a
// sequence.  Rows are loaded once and kept in registers.  Scales are powers of two: values
// are divided exactly, and what a block holds already, rounded anew where its scale must
// grow, changes only where it falls below e4m3's normal range.  V goes to its transposed
// page through LDS, 16 bytes a column.
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

template <int HD, bool F32, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void kv_append_blocks_kernel(KvAppendArgs a) {
  constexpr int PIECES = HD / 8, ITEMS = kScaleBlock * PIECES / 2;  // of 8 elements of a row; pairs of a block
  constexpr int N = ITEMS / 64;                                     // of a lane
  __shared__ __align__(16) uint8_t lds[WAVES * kScaleBlock * HD];
  __shared__ int plan[kPlanScans * 4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int head = blockIdx.y, shift = a.d.page_shift, mask = (1 << shift) - 1;
  const bool is_v = blockIdx.z != 0;
  AppendTile t;
  if constexpr (WAVES == 1) {
    bool bad = false;
    t.b = t.row = a.row0 + blockIdx.x;
    t.first = t.last = length_or_none(a.lens[t.b], a.pages_per_seq, shift, &bad) - 1;
    if (t.first < 0) {  // no room for a new token, or none that can be used
      if (threadIdx.x == 0) raise_status(a.status, kStatusPage);
      return;
    }
  } else {
    if (!plan_append(a, a.row0 + blockIdx.x, plan, &t)) return;
  }
  // this wave's block of the tile, and its tokens first .. last that get rows
  const int block = (t.first & ~(kScaleBlock - 1)) + kScaleBlock * wave;
  const int first = max(t.first, block), last = min(t.last, block + kScaleBlock - 1), tokens = last - first + 1;
  if (tokens <= 0) return;  // no barrier follows
  const int page = a.table[(int64_t)t.b * a.pages_per_seq + (block >> shift)];  // looked at when the rows are on their way
  const int held = first - block, items = tokens * (PIECES / 2);                // tokens that the block has already
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
  Raw8<F32> rx[N], ry[N];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    if (n * 64 >= items) break;
    const int item = min(lane + n * 64, items - 1);
    int x, y;
    pieces(item % (PIECES / 2), &x, &y);
    const int64_t at = (int64_t)(row0 + item / (PIECES / 2)) * ld + (int64_t)head * HD;
    rx[n].load(src, at + 8 * x, a.in_vec);
    ry[n].load(src, at + 8 * y, a.in_vec);
  }
  if (!page_ok(a.d, page)) {
    if (lane == 0) raise_status(a.status, kStatusPage);
    return;
  }
  const size_t scale_at = scale_index(a.d, page, head, block & mask);
  float *scales = is_v ? a.v_scales : a.k_scales;
  const float was = held ? scales[scale_at] : 0.f;
  float u[N][8], w[N][8], most = 0.f;
#pragma unroll
  for (int n = 0; n < N; ++n) {
    if (n * 64 >= items) break;
    const int item = min(lane + n * 64, items - 1), i = item % (PIECES / 2);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      u[n][e] = rx[n].value(e);
      w[n][e] = ry[n].value(e);
    }
    if (!is_v && i < half) {
      const int token = item / (PIECES / 2), position = a.positions ? a.positions[row0 + token] : first + token;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float s, c;
        turn_of(a.turns[8 * i + e], position, &s, &c);
        if (a.rope_pairs) {  // elements 16 i + 2 e and the next
          float &p = e < 4 ? u[n][2 * e] : w[n][2 * e - 8], &q = e < 4 ? u[n][2 * e + 1] : w[n][2 * e - 7];
          const float p0 = p, q0 = q;
          p = p0 * c - q0 * s;
          q = q0 * c + p0 * s;
        } else {
          const float p0 = u[n][e], q0 = w[n][e];
          u[n][e] = p0 * c - q0 * s;
          w[n][e] = q0 * c + p0 * s;
        }
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {  // the largest finite magnitude
      const float x = fabsf(u[n][e]), y = fabsf(w[n][e]);
      most = fmaxf(most, fmaxf(x < INFINITY ? x : 0.f, y < INFINITY ? y : 0.f));
    }
  }
  most = max_pair32(max_pair16(max_row16(most)));
  float scale = __uint_as_float(scale_bits(__float_as_uint(most)));
  if (held) scale = fmaxf(scale, was);
  const bool grows = held && scale > was;
  const float ratio = grows ? was / scale : 1.f, inv = 1.f / scale;
  if (lane == 0 && (!held || grows)) scales[scale_at] = scale;
  const size_t base = page_base(a.d, page, head);
  auto quantised = [&](float *x) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = quotient(x[e], scale, inv);
  };
  if (!is_v) {
    uint8_t *dst = (uint8_t *)a.kp + base + k_in_page(a.d, block & mask, 0);  // the block's rows lie side by side
    if (grows)
      for (int i = lane; i < held * (HD / 16); i += 64) {
        u32x4_t *p = (u32x4_t *)dst + i;
        *p = rescaled16(*p, ratio);
      }
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int item = lane + n * 64;
      if (item >= items) break;
      int x, y;
      pieces(item % (PIECES / 2), &x, &y);
      quantised(u[n]);
      quantised(w[n]);
      uint8_t *to = dst + (held + item / (PIECES / 2)) * HD;
      Pool8<true> o;
      o.set(u[n]);
      o.put_page(to + 8 * x);
      o.set(w[n]);
      o.put_page(to + 8 * y);
    }
    return;
  }
  // V: the block's tokens in LDS, a token's 8-byte piece p at place p ^ token, then four
  // columns a lane
  uint8_t *mine = lds + wave * kScaleBlock * HD;
  auto place = [&](int token, int piece) { return (token * PIECES + (piece ^ (token & (PIECES - 1)))) * 8; };
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int item = lane + n * 64, token = item / (PIECES / 2), i = item % (PIECES / 2);
    if (item >= items) break;
    quantised(u[n]);
    quantised(w[n]);
    Pool8<true> o;
    o.set(u[n]);
    o.put(mine + place(held + token, 2 * i));
    o.set(w[n]);
    o.put(mine + place(held + token, 2 * i + 1));
  }
  __builtin_amdgcn_wave_barrier();
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // a wave's own LDS: nobody else is waited for
  uint8_t *vp = (uint8_t *)a.vp + base + v_in_page(a.d, block & mask, 0);
  if (lane >= HD / 4) return;
  uint32_t v[kScaleBlock];
#pragma unroll
  for (int e = 0; e < kScaleBlock; ++e) v[e] = *(const uint32_t *)(mine + place(e, lane / 2) + (lane & 1) * 4);
#pragma unroll
  for (int col = 0; col < 4; ++col) {
    u32x4_t o;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      o[k] = (v[4 * k] >> (8 * col) & 0xFF) | (v[4 * k + 1] >> (8 * col) & 0xFF) << 8 | (v[4 * k + 2] >> (8 * col) & 0xFF) << 16 |
             (v[4 * k + 3] >> (8 * col) & 0xFF) << 24;
    u32x4_t *dst = (u32x4_t *)(vp + ((size_t)(4 * lane + col) << shift));
    if (tokens < kScaleBlock) {  // what is held, and what lies behind the last token
      const u32x4_t old = *dst;
      o = first_bytes(grows ? rescaled16(old, ratio) : old, first_bytes(o, old, held + tokens), held);
    }
    __builtin_nontemporal_store(o, dst);
  }
}

template <int HD, bool F32>
static hipError_t launch_append_blocks_type(const KvAppendArgs &a, hipStream_t s) {
  constexpr int64_t kMaxWgs = 1 << 22;  // work items of a grid stay below 2^32
  const int64_t tiles = a.row_start ? append_grid(a.n_rows, a.n_seqs, append_tile_shift(a.d.page_shift)) : a.n_rows;
  for (int64_t r = 0; r < tiles; r += kMaxWgs) {
    KvAppendArgs p = a;
    p.row0 = (int)r;
    const dim3 grid((unsigned)std::min(tiles - r, kMaxWgs), a.d.n_kv_heads, 2);
    if (!a.row_start) hipLaunchKernelGGL((kv_append_blocks_kernel<HD, F32, 1>), grid, dim3(64), 0, s, p);
    else hipLaunchKernelGGL((kv_append_blocks_kernel<HD, F32, kAppendTile / kScaleBlock>), grid, dim3(kAppendTile / kScaleBlock * 64), 0, s, p);
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
// Pages of new tokens.  Every workgroup works out the sums over all sequences for itself
// (a run of them per thread, see PlanScan) and fills its share of the table's entries and
// of the slots; the last to be done writes lengths and the free pages' number, which may
// be where the others read them.
// ---------------------------------------------------------------------------
// The run of sequences (a thread's of the scan) that item i falls to, of sums up to and
// with each: the first above i.
__device__ __forceinline__ int run_of(const int *upto, int n, int i) {
  int lo = 0;
  for (int step = n / 2; step > 0; step /= 2)
    if (upto[lo + step - 1] <= i) lo += step;
  return lo;
}

__global__ __launch_bounds__(256) void kv_reserve_kernel(KvReserveArgs a) {
  __shared__ int plan[6 * 4], rows_upto[256], pages_upto[256], word[1];
  PlanScan<4> scan(a.n_seqs, plan);
  const int threads = scan.block ? 256 : 64, b0 = scan.me * scan.per;
  auto tokens = [&](int b) { return a.new_tokens ? a.new_tokens[b] : 1; };
  bool bad = false;
  int64_t rows = 0;
  for (int b = b0; b < min(b0 + scan.per, a.n_seqs); ++b) {
    const int len = a.lens[b], n = tokens(b);
    if (growth_ok(len, n, a.pages_per_seq, a.page_shift)) rows += n;
    else bad = true;
  }
  int hi, lo;
  scan((int)(rows >> 22), &hi);
  scan((int)(rows & 0x3FFFFF), &lo);
  const int64_t all_rows = ((int64_t)hi << 22) + lo;
  bad |= all_rows > 0x7FFFFFFF || (a.slots && all_rows > a.n_rows);
  bad = __syncthreads_or(bad);
  // sums fit from here on; a page that is needed gets a row at least
  int need = 0, total_rows = 0, total = 0, my_rows = bad ? 0 : (int)rows;
  for (int b = b0; !bad && b < min(b0 + scan.per, a.n_seqs); ++b) {
    const int len = a.lens[b];
    need += pages_of(len + tokens(b), a.page_shift) - pages_of(len, a.page_shift);
  }
  const int rows_to = scan(my_rows, &total_rows), pages_to = scan(need, &total);
  const int n_free = *a.n_free;
  bad |= n_free < 0 || n_free > a.n_pages || total > n_free;
  if (threadIdx.x < (unsigned)threads) {
    rows_upto[threadIdx.x] = rows_to;
    pages_upto[threadIdx.x] = pages_to;
  }
  __syncthreads();
  const int me = blockIdx.x * 256 + threadIdx.x, everyone = gridDim.x * 256;
  if (bad) {
    if (me == 0) raise_status(a.status, kStatusPage);
    if (a.row_start)
      for (int b = me; b <= a.n_seqs; b += everyone) a.row_start[b] = 0;
    if (a.slots)
      for (int64_t r = me; r < a.n_rows; r += everyone) a.slots[r] = -1;
  } else {
    bool odd = false;
    auto page = [&](int i) {  // the i-th that is taken
      return a.free_pages[n_free - 1 - i];
    };
    // the sequence of row or page i: its first row or page, and its tokens before
    auto walk = [&](const int *upto, int i, bool by_rows, int *first) {
      const int run = run_of(upto, threads, i);
      int b = run * scan.per, at = run ? upto[run - 1] : 0;
      for (; b < a.n_seqs - 1; ++b) {  // the last at the latest
        const int len = a.lens[b], n = tokens(b);
        const int k = by_rows ? n : pages_of(len + n, a.page_shift) - pages_of(len, a.page_shift);
        if (i < at + k) break;
        at += k;
      }
      *first = at;
      return b;
    };
    for (int i = me; i < total; i += everyone) {
      int first;
      const int b = walk(pages_upto, i, false, &first), id = page(i);
      a.table[(int64_t)b * a.pages_per_seq + pages_of(a.lens[b], a.page_shift) + i - first] = id;
      odd |= id < 0 || id >= a.n_pages;
    }
    if (a.slots)
      for (int64_t r = me; r < a.n_rows; r += everyone) {
        int64_t slot = -1;
        if (r < total_rows) {
          int first, first_page = 0;
          const int b = walk(rows_upto, (int)r, true, &first), len = a.lens[b], p = len + (int)r - first;
          const int i = (p >> a.page_shift) - pages_of(len, a.page_shift);
          int id;
          if (i < 0) {  // the page that the sequence's last token is in
            id = a.table[(int64_t)b * a.pages_per_seq + (p >> a.page_shift)];
          } else {
            const int run = b / scan.per;
            first_page = run ? pages_upto[run - 1] : 0;
            for (int x = run * scan.per; x < b; ++x)
              first_page += pages_of(a.lens[x] + tokens(x), a.page_shift) - pages_of(a.lens[x], a.page_shift);
            id = page(first_page + i);
          }
          const bool fine = id >= 0 && id < a.n_pages;
          odd |= !fine;
          if (fine) slot = ((int64_t)id << a.page_shift) + (p & ((1 << a.page_shift) - 1));
        }
        a.slots[r] = slot;
      }
    if (odd) raise_status(a.status, kStatusPage);
  }
  if (gridDim.x > 1 && !last_to_arrive(a.arrived, gridDim.x, (float *)word)) return;
  __syncthreads();
  if (scan.block || threadIdx.x < 64) {
    int at = rows_to - my_rows;
    for (int b = b0; b < min(b0 + scan.per, a.n_seqs); ++b) {
      const int len = a.lens[b], n = bad ? 0 : tokens(b);
      if (a.row_start && !bad) a.row_start[b] = at;
      at += n;
      a.lens_out[b] = len + n;
    }
  }
  if (threadIdx.x == 0) {
    if (a.row_start && !bad) a.row_start[a.n_seqs] = total_rows;
    *a.n_free_out = bad ? n_free : n_free - total;
  }
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
  for (int b = blockIdx.x * 4 + (threadIdx.x >> 6); b < a.n_seqs; b += gridDim.x * 4) {
    const int len = a.lens[b];
    const int32_t *row = a.table + (int64_t)b * a.pages_per_seq;
    int n = 0;
    odd |= len < 0;
    for (int i0 = 0; len >= 0 && i0 < a.pages_per_seq; i0 += 64) {
      const int i = i0 + lane;
      n += __popcll(__ballot(i < a.pages_per_seq && gone(a, len, i, row[min(i, a.pages_per_seq - 1)], &odd)));
    }
    if (lane == 0) a.counts[b] = n;
  }
  if (odd) raise_status(a.status, kStatusPage);
}

__global__ __launch_bounds__(256) void kv_release_kernel(KvReleaseArgs a) {
  __shared__ int plan[2 * 4], upto[256], word[1];
  PlanScan<4> scan(a.n_seqs, plan);
  const int b0 = scan.me * scan.per;
  int mine = 0, total;  // pages: at most as many as the pool has, else nothing is done
  int64_t all = 0;
  for (int b = b0; b < min(b0 + scan.per, a.n_seqs); ++b) all += a.counts[b];
  const int n_free = *a.n_free;
  mine = all > a.n_pages ? a.n_pages : (int)all;
  bool bad = n_free < 0 || n_free > a.n_pages || all > a.n_pages;
  // up to 256 runs of up to 2^31 pages: in units of 2^10 first
  int big;
  scan(mine >> 10, &big);
  bad |= big > (a.n_pages >> 10) + 1;
  bad = __syncthreads_or(bad);
  const int to = scan(bad ? 0 : mine, &total);
  bad |= (int64_t)n_free + total > a.n_pages;
  if (scan.block || threadIdx.x < 64) upto[scan.me] = to;
  __syncthreads();
  if (!bad) {
    const int lane = threadIdx.x & 63;
    for (int b = blockIdx.x * 4 + (threadIdx.x >> 6); b < a.n_seqs; b += gridDim.x * 4) {
      if (a.counts[b] == 0) continue;
      const int len = a.lens[b], run = b / scan.per;
      int at = n_free + (run ? upto[run - 1] : 0);
      for (int x = run * scan.per; x < b; ++x) at += a.counts[x];
      int32_t *row = a.table + (int64_t)b * a.pages_per_seq;
      for (int i0 = 0; i0 < a.pages_per_seq; i0 += 64) {
        const int i = i0 + lane, id = row[min(i, a.pages_per_seq - 1)];
        bool odd = false;
        const bool go = i < a.pages_per_seq && gone(a, len, i, id, &odd);
        const uint64_t goes = __ballot(go);
        if (go) {
          const int to_i = at + __popcll(goes & ((1ull << lane) - 1));
          if (to_i < a.n_pages) a.free_pages[to_i] = id;  // always, unless the caller's arrays change while this runs
          row[i] = -1;
        }
        at += __popcll(goes);
      }
    }
  } else if (blockIdx.x == 0 && threadIdx.x == 0) {
    raise_status(a.status, kStatusPage);
  }
  if (gridDim.x > 1 && !last_to_arrive(a.arrived, gridDim.x, (float *)word)) return;
  if (threadIdx.x == 0 && !bad) *a.n_free = n_free + total;
}

hipError_t launch_kv_reserve(const KvReserveArgs &a, hipStream_t s) {
  if (a.n_seqs < 1 || a.pages_per_seq < 1 || a.page_shift < 4 || a.n_pages < 1 || a.n_rows < 0) return hipErrorInvalidValue;
  // a workgroup for every 2048 slots, up to two a CU
  const int64_t items = std::max<int64_t>(a.slots ? a.n_rows : 0, (int64_t)a.n_seqs * 8);
  const unsigned grid = (unsigned)std::min<int64_t>((items + 2047) / 2048, 512);
  hipLaunchKernelGGL(kv_reserve_kernel, dim3(grid), dim3(256), 0, s, a);
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
