// Paged K/V cache: append with rotation, attention of one token per sequence, and
// the expert's prefix from pages.  Layouts and checks in paged.h.
#include "kv_internal.h"

namespace uad {

// ---------------------------------------------------------------------------
// Element types
// ---------------------------------------------------------------------------
template <bool F32>
__device__ __forceinline__ float load_elem(const void *p, int64_t i) {
  if constexpr (F32) return ((const float *)p)[i];
  else return __uint_as_float((uint32_t)((const uint16_t *)p)[i] << 16);
}
template <bool F32>
__device__ __forceinline__ void store_elem(void *p, int64_t i, float v) {
  if constexpr (F32) ((float *)p)[i] = v;
  else ((__bf16 *)p)[i] = (__bf16)v;
}
// fp32 to e4m3, cut to +-448 (the cut keeps a NaN: both comparisons fail)
__device__ __forceinline__ float cut_f8(float v) { return v > 448.f ? 448.f : v < -448.f ? -448.f : v; }
__device__ __forceinline__ uint8_t to_f8(float v) {
  return (uint8_t)(__builtin_amdgcn_cvt_pk_fp8_f32(cut_f8(v), 0.f, 0, false) & 0xFF);
}
__device__ __forceinline__ float from_f8(uint8_t b) { return __builtin_amdgcn_cvt_f32_fp8((int)b, 0); }

template <bool F8>
__device__ __forceinline__ void store_pool(void *p, size_t i, float v) {
  if constexpr (F8) ((uint8_t *)p)[i] = to_f8(v);
  else ((__bf16 *)p)[i] = (__bf16)v;
}
template <bool F8>
__device__ __forceinline__ float load_pool(const void *p, size_t i) {
  if constexpr (F8) return from_f8(((const uint8_t *)p)[i]);
  else return __uint_as_float((uint32_t)((const uint16_t *)p)[i] << 16);
}

// Sine and cosine of `position` times a pair's turns: the whole turns go in 64 bits
// (a position of 10^6 leaves 36 bits of the fraction), the rest in fp32.
__device__ __forceinline__ void turn_of(double turns, int position, float *s, float *c) {
  const double t = turns * (double)position;
  sincospif(2.0f * (float)(t - rint(t)), s, c);
}

// The sequence of a new row: how many of row_start[0 .. n_seqs] are at most r, minus
// one.  Called by whole waves; r is the same in all lanes.
__device__ __forceinline__ int sequence_of_row(const int32_t *row_start, int n_seqs, int r) {
  const int lane = threadIdx.x & 63;
  int n = 0;
  for (int i0 = 0; i0 <= n_seqs; i0 += 64)
    n += __popcll(__ballot(i0 + lane <= n_seqs && row_start[min(i0 + lane, n_seqs)] <= r));
  return n - 1;
}

// ---------------------------------------------------------------------------
// Append: one workgroup per new row.
// ---------------------------------------------------------------------------
template <bool F32, bool F8>
__global__ __launch_bounds__(256) void kv_append_kernel(KvAppendArgs a) {
  const int r = a.row0 + blockIdx.x;
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
    bad = b < 0 || lo < 0 || hi > a.n_rows || r >= hi;
    j = r - lo;
    n_b = hi - lo;
  }
  int pos = 0, page = 0;
  if (!bad) {
    const int len = usable_length(a.lens[b], a.pages_per_seq, a.d.page_shift, &bad);
    pos = len - n_b + j;
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
    store_pool<F8>(a.kp, base + k_in_page(a.d, off, ea), F8 ? kx * a.k_inv : kx);
    store_pool<F8>(a.kp, base + k_in_page(a.d, off, eb), F8 ? ky * a.k_inv : ky);
    store_pool<F8>(a.vp, base + v_in_page(a.d, off, 2 * p), F8 ? u * a.v_inv : u);
    store_pool<F8>(a.vp, base + v_in_page(a.d, off, 2 * p + 1), F8 ? w * a.v_inv : w);
  }
}

hipError_t launch_kv_append(const KvAppendArgs &a, bool f32, bool f8, hipStream_t s) {
  if (a.n_rows < 1 || a.n_seqs < 1 || a.d.head_dim > 512 || a.d.head_dim < 2) return hipErrorInvalidValue;
  constexpr int kMaxRows = 1 << 23;  // work items of a grid stay below 2^32
  for (int64_t r = 0; r < a.n_rows; r += kMaxRows) {
    KvAppendArgs p = a;
    p.row0 = (int)r;
    const dim3 grid((unsigned)(a.n_rows - r < kMaxRows ? a.n_rows - r : kMaxRows)), wg(256);
    if (f32 && f8) hipLaunchKernelGGL((kv_append_kernel<true, true>), grid, wg, 0, s, p);
    else if (f32) hipLaunchKernelGGL((kv_append_kernel<true, false>), grid, wg, 0, s, p);
    else if (f8) hipLaunchKernelGGL((kv_append_kernel<false, true>), grid, wg, 0, s, p);
    else hipLaunchKernelGGL((kv_append_kernel<false, false>), grid, wg, 0, s, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// ---------------------------------------------------------------------------
// Attention of one token: one workgroup per sequence and query head, four waves
// that take every fourth key with a running maximum and sum, joined in LDS.
// ---------------------------------------------------------------------------
template <int HD, bool F32, bool F8>
__global__ __launch_bounds__(256) void kv_attend_kernel(KvAttendArgs a) {
  constexpr int E = HD / 64;
  __shared__ float qs[HD], o_s[4][HD], ml[4][2];
  const int b = blockIdx.x, head = blockIdx.y, g = head / a.group;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  bool bad = false;
  const int len = usable_length(a.lens[b], a.pages_per_seq, a.d.page_shift, &bad);
  const int64_t qi = b * a.ldq + (int64_t)head * HD;
  for (int p = threadIdx.x; p < HD / 2; p += 256) {
    int ea, eb;
    rope_pair(p, a.rope_dim, a.rope_pairs != 0, &ea, &eb);
    const float x = load_elem<F32>(a.q, qi + ea), y = load_elem<F32>(a.q, qi + eb);
    float s = 0.f, c = 1.f;
    const bool turned = p < a.rope_dim / 2;
    if (turned) turn_of(a.turns[p], a.positions ? a.positions[b] : len - 1, &s, &c);
    qs[ea] = turned ? x * c - y * s : x;
    qs[eb] = turned ? y * c + x * s : y;
  }
  __syncthreads();
  float q[E], o[E], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    q[e] = qs[lane * E + e];
    o[e] = 0.f;
  }
  for (int key = wave; key < len; key += 4) {
    const int page = a.table[(int64_t)b * a.pages_per_seq + (key >> a.d.page_shift)];
    if (!page_ok(a.d, page)) {
      bad = true;
      continue;
    }
    const int off = key & ((1 << a.d.page_shift) - 1);
    const size_t base = page_base(a.d, page, g);
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) s += q[e] * load_pool<F8>(a.kp, base + k_in_page(a.d, off, lane * E + e));
    s = sum_wave64(s) * a.scale_log2;
    const float m1 = fmaxf(m, s), f = exp2f(m - m1), p = exp2f(s - m1);
    l = l * f + p;
#pragma unroll
    for (int e = 0; e < E; ++e)
      o[e] = o[e] * f + p * load_pool<F8>(a.vp, base + v_in_page(a.d, off, lane * E + e));
    m = m1;
  }
  if (bad && lane == 0) raise_status(a.status, kStatusPage);
  if (lane == 0) {
    ml[wave][0] = m;
    ml[wave][1] = l;
  }
#pragma unroll
  for (int e = 0; e < E; ++e) o_s[wave][lane * E + e] = o[e];
  __syncthreads();
  float mx = -INFINITY;
  for (int w = 0; w < 4; ++w) mx = fmaxf(mx, ml[w][0]);
  for (int c = threadIdx.x; c < HD; c += 256) {
    float num = 0.f, den = 0.f;
    for (int w = 0; w < 4; ++w)
      if (ml[w][1] > 0.f) {
        const float f = exp2f(ml[w][0] - mx);
        num += f * o_s[w][c];
        den += f * ml[w][1];
      }
    store_elem<F32>(a.out, b * a.ldo + (int64_t)head * HD + c, den > 0.f ? num / den * a.v_scale : 0.f);
  }
}

template <int HD>
static hipError_t launch_attend_hd(const KvAttendArgs &a, bool f32, bool f8, hipStream_t s) {
  const dim3 grid(a.n_seqs, a.n_heads), wg(256);
  if (f32 && f8) hipLaunchKernelGGL((kv_attend_kernel<HD, true, true>), grid, wg, 0, s, a);
  else if (f32) hipLaunchKernelGGL((kv_attend_kernel<HD, true, false>), grid, wg, 0, s, a);
  else if (f8) hipLaunchKernelGGL((kv_attend_kernel<HD, false, true>), grid, wg, 0, s, a);
  else hipLaunchKernelGGL((kv_attend_kernel<HD, false, false>), grid, wg, 0, s, a);
  return hipGetLastError();
}

hipError_t launch_kv_attend(const KvAttendArgs &a, bool f32, bool f8, hipStream_t s) {
  if (a.n_seqs < 1 || a.group < 1 || a.n_heads != a.group * a.d.n_kv_heads) return hipErrorInvalidValue;
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
template <bool F8, int N>
struct PoolRun {  // N consecutive pool elements as bf16
  __device__ static __forceinline__ void load(const void *p, size_t i, float scale, __bf16 *o) {
#pragma unroll
    for (int e = 0; e < N; ++e) o[e] = (__bf16)(F8 ? load_pool<true>(p, i + e) * scale : load_pool<false>(p, i + e));
  }
};

template <int HD, bool F8>
__global__ __launch_bounds__(256) void kv_prefix_kernel(KvPrefixArgs a) {
  const int blk = blockIdx.x, b = a.env0 + blockIdx.y / a.d.n_kv_heads, g = blockIdx.y % a.d.n_kv_heads;
  const size_t eh = (size_t)b * a.d.n_kv_heads + g;
  const size_t src = blockIdx.z * a.src_layer;
  bool bad = false;
  const int len = usable_length(a.lens[b], a.pages_per_seq, a.d.page_shift, &bad);
  bad |= len < a.n_keys;
  const int n_keys = min(len, a.n_keys);
  const size_t esz = F8 ? 1 : 2;
  const char *kp = (const char *)a.kp + src * esz, *vp = (const char *)a.vp + src * esz;
  __bf16 *kd = a.kc + blockIdx.z * a.dst_layer + (eh * a.s_alloc + (size_t)blk * 32) * HD;
  __bf16 *vd = a.vtc + blockIdx.z * a.dst_layer + vt_index(eh, blk * 32, 0, HD, a.s_alloc);
  const int32_t *row = a.table + (int64_t)b * a.pages_per_seq;
  const int mask = (1 << a.d.page_shift) - 1;
  for (int q = threadIdx.x; q < 32 * HD / 8; q += 256) {
    const int key = q / (HD / 8), c = (q % (HD / 8)) * 8, s = blk * 32 + key;
    __bf16 o[8] = {};
    if (s < n_keys) {
      const int page = row[s >> a.d.page_shift];
      if (page_ok(a.d, page)) PoolRun<F8, 8>::load(kp, page_base(a.d, page, g) + k_in_page(a.d, s & mask, c), a.k_scale, o);
      else bad = true;
    }
    *(bf16x8 *)(kd + key * HD + c) = bf16x8{o[0], o[1], o[2], o[3], o[4], o[5], o[6], o[7]};
  }
  for (int q = threadIdx.x; q < HD * 4; q += 256) {
    const int c = q >> 2, ch = q & 3;
    __bf16 o[8] = {};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int s = blk * 32 + 16 * h + 4 * ch;  // four keys of one page
      if (s < n_keys) {
        const int page = row[s >> a.d.page_shift];
        if (page_ok(a.d, page)) {
          PoolRun<F8, 4>::load(vp, page_base(a.d, page, g) + v_in_page(a.d, s & mask, c), a.v_scale, o + 4 * h);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (s + e >= n_keys) o[4 * h + e] = (__bf16)0.f;
        } else {
          bad = true;
        }
      }
    }
    *(bf16x8 *)(vd + c * 32 + ch * 8) = bf16x8{o[0], o[1], o[2], o[3], o[4], o[5], o[6], o[7]};
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
  if (a.d.n_kv_heads > 65535) return hipErrorInvalidValue;
  const int envs = 65535 / a.d.n_kv_heads;  // grid dimensions y and z take 65535 at most
  for (int l = 0; l < n_layers; l += 32768)
    for (int b = 0; b < batch; b += envs) {
      KvPrefixArgs p = a;
      p.env0 = b;
      p.kp = (const char *)a.kp + l * a.src_layer * (f8 ? 1 : 2);
      p.vp = (const char *)a.vp + l * a.src_layer * (f8 ? 1 : 2);
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
