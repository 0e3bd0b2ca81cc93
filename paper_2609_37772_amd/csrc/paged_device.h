// What the kernels of the paged K/V cache share: element types, rotation, scans of the
// plans, operands of the matrix instructions, and the join of an attention's splits.
#pragma once

#include "kv_internal.h"

namespace uad {

// The running maximum of a query is raised only when a tile passes it by more than
// this (a power of two), which spares most tiles the rescaling.
constexpr float kKvRescale = 8.0f;

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;

// ---------------------------------------------------------------------------
// Element types
// ---------------------------------------------------------------------------
template <bool F32>
__device__ __forceinline__ float load_elem(const void *p, int64_t i) {
  if constexpr (F32) return ((const float *)p)[i];
  else return __uint_as_float((uint32_t)((const uint16_t *)p)[i] << 16);
}
// The same in two steps, so that a load can be in flight before it is looked at.
template <bool F32>
__device__ __forceinline__ uint32_t load_raw(const void *p, int64_t i) {
  if constexpr (F32) return ((const uint32_t *)p)[i];
  else return ((const uint16_t *)p)[i];
}
template <bool F32>
__device__ __forceinline__ float value_of(uint32_t raw) {
  return __uint_as_float(F32 ? raw : raw << 16);
}
template <bool F32>
__device__ __forceinline__ void store_elem(void *p, int64_t i, float v) {
  if constexpr (F32) ((float *)p)[i] = v;
  else ((__bf16 *)p)[i] = (__bf16)v;
}
// What an 8-bit pool holds of x: x / scale, cut to +-448 (before the division, so that
// it never meets an infinity; both comparisons keep a NaN).  The remainder makes the
// product with the rounded reciprocal the quotient, so that a value halfway between two
// of e4m3 stays there and goes to the even one; a zero keeps its sign.  16 uneven
// prompts, 2 x 128: 4.9 us, by the compiler's division 5.3, by the product alone, which
// moves such values, 4.75.
__device__ __forceinline__ float quotient(float x, float scale, float inv) {
  const float most = 448.f * scale;
  x = x > most ? most : x < -most ? -most : x;
  const float q = x * inv;
  return fmaf(-fmaf(q, scale, -x), inv, q);
}
__device__ __forceinline__ uint8_t to_f8(float v) { return (uint8_t)(__builtin_amdgcn_cvt_pk_fp8_f32(v, 0.f, 0, false) & 0xFF); }

template <bool F8>
__device__ __forceinline__ void store_pool(void *p, size_t i, float v) {
  if constexpr (F8) ((uint8_t *)p)[i] = to_f8(v);
  else ((__bf16 *)p)[i] = (__bf16)v;
}
// Sine and cosine of `position` times a pair's turns: the whole turns go in 64 bits
// (a position of 10^6 leaves 36 bits of the fraction), the rest in fp32 to the
// instructions that take turns, off by at most 1.3e-7 within half a turn either way
// (measured on 2^20 points; sincospif's 5e-8 took one prompt's append 4.6 instead of
// 4.1 us).
__device__ __forceinline__ void turn_of(double turns, int position, float *s, float *c) {
  const double t = turns * (double)position;
  const float f = (float)(t - rint(t));
  *s = __builtin_amdgcn_sinf(f);
  *c = __builtin_amdgcn_cosf(f);
}

// The same in whole numbers, without 64-bit floats, for those who turn much: a turn is 2^64
// steps, of which a product with the position keeps the rest (`steps`), and 2^32 of
// `turned`, off by one at most.
__device__ __forceinline__ uint32_t turned(uint64_t steps, int position) {
  const uint32_t lo = (uint32_t)steps, hi = (uint32_t)(steps >> 32), p = (uint32_t)position;
  return __umulhi(p, lo) + p * hi - (position < 0 ? lo : 0u);
}
__device__ __forceinline__ void sine_of(uint32_t turned, float *s, float *c) {
  const float f = (float)(int)turned * 0x1p-32f;
  *s = __builtin_amdgcn_sinf(f);
  *c = __builtin_amdgcn_cosf(f);
}

// Inclusive sum over the lanes of a wave, by DPP: within rows of 16, then across them.
template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp_i(int v) {
  return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xF, true);
}
__device__ __forceinline__ int scan_wave64(int v) {
  v += dpp_i<0x111, 0xF>(v);  // row_shr 1, 2, 4, 8
  v += dpp_i<0x112, 0xF>(v);
  v += dpp_i<0x114, 0xF>(v);
  v += dpp_i<0x118, 0xF>(v);
  v += dpp_i<0x142, 0xA>(v);  // the last lane of rows 0 and 2 to rows 1 and 3
  v += dpp_i<0x143, 0xC>(v);  // lane 31 to rows 2 and 3
  return v;
}
__device__ __forceinline__ int last_lane(int v) { return __builtin_amdgcn_readlane(v, 63); }

// A workgroup's plan looks at every sequence: by each wave for itself where lanes are
// enough, else by the whole workgroup, a run of sequences per thread.
template <int WAVES>
struct PlanScan {
  const bool block;
  const int me, per;  // this thread's sequences: me * per .. me * per + per - 1
  int *lds;           // [WAVES] for each scan, only where the whole workgroup scans
  __device__ __forceinline__ PlanScan(int n_seqs, int *lds_)
      : block(n_seqs > 64), me(block ? threadIdx.x : threadIdx.x & 63), per(block ? (n_seqs + 64 * WAVES - 1) / (64 * WAVES) : 1),
        lds(lds_) {}
  // Inclusive sum over the threads, and the sum of all.
  __device__ __forceinline__ int operator()(int v, int *all) {
    v = scan_wave64(v);
    *all = last_lane(v);
    if (block) {
      if ((threadIdx.x & 63) == 63) lds[threadIdx.x >> 6] = v;
      __syncthreads();
      *all = 0;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        if (w == (int)(threadIdx.x >> 6)) v += *all;
        *all += lds[w];
      }
      lds += WAVES;  // the next scan's, which spares a barrier
    }
    return v;
  }
};
constexpr int kPlanScans = 4 + kShareTries;  // of one plan at most

// The sequence of a new row: how many of row_start[0 .. n_seqs] are at most r, minus
// one; with more than 64, of every 64th first.  Called by whole waves; r is the same in
// all lanes.
__device__ __forceinline__ int sequence_of_row(const int32_t *row_start, int n_seqs, int r) {
  const int lane = threadIdx.x & 63;
  int base = 0;
  if (n_seqs >= 64) {
    int n = 0;
    for (int i0 = 0; i0 <= n_seqs; i0 += 64 * 64) {
      const int i = i0 + 64 * lane;
      n += __popcll(__ballot(i <= n_seqs && row_start[min(i, n_seqs)] <= r));
    }
    base = 64 * max(n - 1, 0);
  }
  return base + __popcll(__ballot(base + lane <= n_seqs && row_start[min(base + lane, n_seqs)] <= r)) - 1;
}

// Columns of a workgroup: 128 of 256, so that its LDS and its share of the work allow
// eight on a CU.
template <int HD>
constexpr int kAppendWide = HD < 128 ? HD : 128;

struct AppendTile {
  int b, first, last;  // tile's cache positions that get a row: first .. last
  int row;             // row of the first
};

template <int WAVES>
__device__ __forceinline__ bool plan_append(const KvAppendArgs &a, int wg, int *lds, AppendTile *t) {
  PlanScan<WAVES> scan(a.n_seqs, lds);
  const int shift = append_tile_shift(a.d.page_shift);
  bool bad = false;
  // positions [from, to) and rows of a sequence; none where they cannot be used
  auto span = [&](int b, int *from, int *to, int *row) {
    const int lo = a.row_start[b], hi = a.row_start[b + 1];
    const int len = a.lens[b];
    const bool ok = sequence_ok(b, lo, hi, a.n_rows, len, a.pages_per_seq, a.d.page_shift);
    bad |= !ok;
    *row = lo;
    *to = ok ? len : 0;
    *from = ok ? len - (hi - lo) : 0;
  };
  int mine = 0, from = 0, to = 0, row = 0, all;
  for (int i = 0; i < scan.per; ++i)
    if (scan.me * scan.per + i < a.n_seqs) {
      span(scan.me * scan.per + i, &from, &to, &row);
      mine += append_tiles(from, to, shift);
    }
  if (bad && wg == 0) raise_status(a.status, kStatusPage);
  const int upto = scan(mine, &all);
  if (wg >= all) return false;
  int start = upto - mine, b = scan.me;
  if (scan.block) {
    if (upto > wg && start <= wg) {  // one thread: it looks for the sequence among its own
      for (b = scan.me * scan.per;; ++b) {
        if (b < a.n_seqs) span(b, &from, &to, &row);
        const int n = append_tiles(from, to, shift);
        if (b >= a.n_seqs || start + n > wg) break;
        start += n;
      }
      const int found[5] = {b, start, from, to, row};
#pragma unroll
      for (int i = 0; i < 5; ++i) scan.lds[i] = found[i];
    }
    __syncthreads();
    b = __builtin_amdgcn_readfirstlane(scan.lds[0]);
    start = __builtin_amdgcn_readfirstlane(scan.lds[1]);
    from = __builtin_amdgcn_readfirstlane(scan.lds[2]);
    to = __builtin_amdgcn_readfirstlane(scan.lds[3]);
    row = __builtin_amdgcn_readfirstlane(scan.lds[4]);
    if (b >= a.n_seqs) return false;  // only if the caller's arrays change while this runs
  } else {
    b = __builtin_ctzll(__ballot(upto > wg));
    start = __builtin_amdgcn_readlane(start, b);
    from = __builtin_amdgcn_readlane(from, b);
    to = __builtin_amdgcn_readlane(to, b);
    row = __builtin_amdgcn_readlane(row, b);
  }
  const int tile = (from >> shift) + wg - start;
  t->b = b;
  t->first = max(from, tile << shift);
  t->last = min(to, (tile + 1) << shift) - 1;
  t->row = row + t->first - from;
  return t->first <= t->last;
}

// 8 consecutive elements of a row as they are loaded; values of them.
template <bool F32>
struct Raw8 {
  u32x4_t r[F32 ? 2 : 1];
  __device__ __forceinline__ void load(const void *p, int64_t i, bool vec) {
    if (vec) {
#pragma unroll
      for (int k = 0; k < (F32 ? 2 : 1); ++k) r[k] = ((const u32x4_t *)((const char *)p + i * (F32 ? 4 : 2)))[k];
    } else if constexpr (F32) {
#pragma unroll
      for (int e = 0; e < 8; ++e) r[e / 4][e % 4] = ((const uint32_t *)p)[i + e];
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        r[0][e] = ((const uint16_t *)p)[i + 2 * e] | (uint32_t)((const uint16_t *)p)[i + 2 * e + 1] << 16;
    }
  }
  __device__ __forceinline__ float value(int e) const {
    if constexpr (F32) return __uint_as_float(r[e / 4][e % 4]);
    else return __uint_as_float(e & 1 ? r[0][e / 2] & 0xFFFF0000u : r[0][e / 2] << 16);
  }
};

// 8 pool elements: 16 bytes of bf16, 8 of e4m3.
template <bool F8>
struct Pool8 {
  uint32_t w[F8 ? 2 : 4];
  __device__ __forceinline__ void set(const float *v) {
#pragma unroll
    for (int i = 0; i < (F8 ? 2 : 4); ++i) {
      if constexpr (F8) {
        int x = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i], v[4 * i + 1], 0, false);
        w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i + 2], v[4 * i + 3], x, true);
      } else {
        union {
          bf16x2 h;
          uint32_t u;
        } x{bf16x2{(__bf16)v[2 * i], (__bf16)v[2 * i + 1]}};
        w[i] = x.u;
      }
    }
  }
  __device__ __forceinline__ void put(void *p) const {
    if constexpr (F8) *(uint64_t *)p = (uint64_t)w[0] | (uint64_t)w[1] << 32;
    else *(u32x4_t *)p = u32x4_t{w[0], w[1], w[2], w[3]};
  }
  // past the caches: pages are not read again by this kernel
  __device__ __forceinline__ void put_page(void *p) const {
    if constexpr (F8) __builtin_nontemporal_store((uint64_t)w[0] | (uint64_t)w[1] << 32, (uint64_t *)p);
    else __builtin_nontemporal_store(u32x4_t{w[0], w[1], w[2], w[3]}, (u32x4_t *)p);
  }
};

// Tiles of a split, where a unit has as many: fewer leave more to join, more keep a CU
// reading, which takes in 15 to 26 bytes a clock of these loads (26 tiles of 1 x 256: 2
// tiles 12.3 us, 4 tiles 11.9, 8 tiles 14.2; 24 tiles of 2 x 128: 4 tiles 8.8, 8 tiles
// 10.4).
constexpr int kAttendMinTiles = 4;
// Tiles up to which a unit stays whole, where reading it and joining it cost the same
// (one sequence, whole / split): head dim 256, 8 tiles 10.9 / 11.2 us, 10 tiles 11.8 /
// 11.2; 128, 12 tiles 8.5 / 8.8, 16 tiles 9.6 / 8.9; 64, 20 tiles 7.6 / 8.0, 24 tiles
// 8.3 / 8.0.  E4m3, whose tiles take longer to widen: 256, 6 tiles 12.2 / 12.2; 128, 8
// tiles 8.8 / 9.6, 10 tiles 9.9 / 9.6; 64, 12 tiles 7.2 / 8.1, 16 tiles 8.4 / 8.3.
template <int HD, bool F8>
constexpr int kAttendWhole = (HD == 256 ? 8 : HD == 128 ? 12 : 20) * (F8 ? 3 : 4) / 4;
constexpr int kAttendWaves = 8;
// Workgroups per CU: the tiles in flight, the outputs and their operands take a wave up
// to 256 registers at head dim 256 (two waves per SIMD) and 160 at 128; for 128, three
// workgroups of four waves, which fit too, spilled or read slower (131071 keys, 32/8
// heads: 108.9 us, two of them 104.1, one of eight waves 100.8).
template <int HD>
constexpr int kAttendPerCu = HD == 64 ? 2 : 1;

template <bool F8>
constexpr int kTileKeys = F8 ? 64 : 32;  // keys of 16-byte V^T loads by the four lane groups

// 8 bf16 of a 16-byte load (u: which half of an 8-bit one); e4m3 widens exactly, its
// scale goes into the scores' and the outputs'.
template <bool F8>
__device__ __forceinline__ bf16x8 operand_of(u32x4_t r, int u) {
  union {
    bf16x8 v;
    bf16x2 p[4];
    uint32_t w[4];
  } o;
  if constexpr (F8) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      o.p[2 * i] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(r[2 * u + i], 1.0f, false);
      o.p[2 * i + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(r[2 * u + i], 1.0f, true);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) o.w[i] = r[i];
  }
  return o.v;
}

__device__ __forceinline__ float max_row16(float v) {
  v = fmaxf(v, dpp_f<0xB1>(v));
  v = fmaxf(v, dpp_f<0x4E>(v));
  v = fmaxf(v, dpp_f<0x141>(v));
  v = fmaxf(v, dpp_f<0x140>(v));
  return v;
}

// A slot's values cross the XCDs' L2 caches: 16-byte accesses that are written through
// and read past them (cache policy sc1, device scope; the compiler waits for the loads).
constexpr int kDeviceScope = 16;
__device__ __forceinline__ __amdgpu_buffer_rsrc_t slots_of(const KvAttendArgs &a, int floats) {
  return __builtin_amdgcn_make_buffer_rsrc(a.part, 0, a.slots * floats * 4, 0x00027000);  // raw buffer, below 2^31 bytes
}
__device__ __forceinline__ void put_slot(__amdgpu_buffer_rsrc_t slots, unsigned i, f32x4 v) {
  __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, v), slots, (int)(i * 4), 0, kDeviceScope);
}
__device__ __forceinline__ f32x4 get_slot(__amdgpu_buffer_rsrc_t slots, unsigned i) {
  return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(slots, (int)(i * 4), 0, kDeviceScope));
}
__device__ __forceinline__ uint64_t pair_of(float m, float l) {
  return (uint64_t)__float_as_uint(m) | ((uint64_t)__float_as_uint(l) << 32);
}

// LDS of the attention: the query's bf16 terms, the waves' outputs, their maxima and sums
// (before that the plan, later the slots' weights), the joint ones and a word; 158 of a
// CU's 160 KB at head dim 256.
constexpr int kAttendMl = 2 * kJoinFan * 16;  // floats
constexpr int kTerms = 3;
template <int HD>
constexpr int kQueryFloats = kTerms * HD / 32 * 256;
template <int HD>
constexpr int attend_lds_floats() {
  return kQueryFloats<HD> + kAttendWaves * 16 * HD + kAttendMl + 16 * 2 + 4;
}

// The last of `n` workgroups to get here carries on; all of this workgroup's slot
// values have arrived in memory by then.
__device__ __forceinline__ bool last_to_arrive(unsigned *counter, int n, float *word) {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0) {
    const bool last = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (unsigned)(n - 1);
    if (last) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *(int *)word = last;
  }
  __syncthreads();
  return *(int *)word != 0;
}

// Joins slots first, first + step, .. (n of them, at most 2 * kJoinFan): sums go to
// put(row, column, sum of outputs, sum of weights); top [16][2] holds the joint maximum
// and sum of each row.  The outputs are on their way while 16 lanes a row work the
// weights out; threads that the outputs leave over take a part of the slots.
template <int HD, class Put>
__device__ __forceinline__ void join_slots(const KvAttendArgs &a, int rows, int rows_max, int first, int step, int n,
                                           float *weight, float *top, f32x4 *shared, Put put) {
  constexpr int VEC = HD / 4, THREADS = 64 * kAttendWaves, RUN = 8;
  const int items = rows * VEC;
  const int groups = min(n, max(1, THREADS / items)), mine = threadIdx.x / items;  // slots mine, mine + groups, ..
  const int per = (n - mine + groups - 1) / groups;
  const unsigned slot_floats = rows_max * HD;
  const auto slots = slots_of(a, slot_floats);
  f32x4 v[RUN];
  auto fetch = [&](int item, int i0) {
#pragma unroll
    for (int i = 0; i < RUN; ++i) v[i] = get_slot(slots, (first + min(mine + (i0 + i) * groups, n - 1) * step) * slot_floats + item * 4);
  };
  const int row = threadIdx.x >> 4, i = threadIdx.x & 15;
  uint64_t pair[2] = {pair_of(-INFINITY, 0.f), pair_of(-INFINITY, 0.f)};
  if (row < rows)
#pragma unroll
    for (int k = 0; k < 2; ++k)
      if (i + 16 * k < n)
        pair[k] = __hip_atomic_load(a.part_ml + (size_t)(first + (i + 16 * k) * step) * rows_max + row, __ATOMIC_RELAXED,
                                    __HIP_MEMORY_SCOPE_AGENT);
  const int item0 = threadIdx.x - mine * items;  // groups > 1: the only one
  if (mine < groups) fetch(item0, 0);
  if (row < 16) {
    const float m0 = __uint_as_float((uint32_t)pair[0]), m1 = __uint_as_float((uint32_t)pair[1]);
    const float l0 = __uint_as_float((uint32_t)(pair[0] >> 32)), l1 = __uint_as_float((uint32_t)(pair[1] >> 32));
    const float mx = max_row16(fmaxf(m0, m1));
    const float f0 = l0 != 0.f ? __builtin_amdgcn_exp2f(m0 - mx) : 0.f, f1 = l1 != 0.f ? __builtin_amdgcn_exp2f(m1 - mx) : 0.f;
    const float sum = sum_row16(l0 * f0 + l1 * f1);
    weight[i * 16 + row] = f0;
    weight[(i + 16) * 16 + row] = f1;
    if (i == 0) {
      top[2 * row] = mx;
      top[2 * row + 1] = sum;
    }
  }
  __syncthreads();
  auto sum_of = [&](int item) {
    const int r = item / VEC;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int i0 = 0;;) {
#pragma unroll
      for (int k = 0; k < RUN; ++k)
        if (i0 + k < per) o += v[k] * weight[(mine + (i0 + k) * groups) * 16 + r];
      i0 += RUN;
      if (i0 >= per) return o;
      fetch(item, i0);
    }
  };
  if (groups > 1) {  // the groups' sums meet, in order
    if (mine < groups) shared[threadIdx.x] = sum_of(item0);
    __syncthreads();
    if (mine == 0) {
      f32x4 o = shared[item0];
      for (int g = 1; g < groups; ++g) o += shared[g * items + item0];
      put(item0 / VEC, item0 % VEC * 4, o, top[2 * (item0 / VEC) + 1]);
    }
  } else {
    for (int item = threadIdx.x; item < items; item += THREADS) {
      if (item >= THREADS) fetch(item, 0);
      put(item / VEC, item % VEC * 4, sum_of(item), top[2 * (item / VEC) + 1]);
    }
  }
}

}  // namespace uad
