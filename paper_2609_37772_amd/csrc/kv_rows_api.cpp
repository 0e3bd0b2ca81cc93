// C ABI of the paged K/V cache, continued: scales for blocks of 8-bit pools, attention of
// new rows, page tables.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "kv_call.h"

using namespace uad;

namespace {

// (row, query head) pairs of a call: the attention's units and their work items fit a grid.
constexpr int64_t kMaxColumns = (int64_t)1 << 25;
// Windows and sinks beyond any length count as this.
constexpr int kMaxSeen = 1 << 30;

// What the page tables' calls check alike.
uad_status check_pages(uad_kv *kv, const char *fn, const void *lens, const void *table, const void *free_pages,
                       const void *n_free, int pages_per_seq, int n_seqs) {
  if (n_seqs < 0 || pages_per_seq < 1) return kv_fail(kv, UAD_E_INVALID, fn, "n_seqs must be >= 0, pages_per_seq >= 1");
  if (n_seqs > kv->cfg.max_seqs) return kv_fail(kv, UAD_E_SHAPE, fn, "n_seqs > max_seqs");
  if ((int64_t)pages_per_seq * kv->cfg.page_size > kMaxTokens)
    return kv_fail(kv, UAD_E_SHAPE, fn, "a page table of more than 2^30 tokens per sequence");
  if (n_seqs > 0 && (!lens || !table || !free_pages || !n_free)) return kv_fail(kv, UAD_E_INVALID, fn, "null pointer");
  return UAD_OK;
}

}  // namespace

extern "C" {

uad_status uad_kv_set_block_scales(uad_kv *kv, float *k_scales, float *v_scales) {
  if (!kv) return UAD_E_INVALID;
  const char *fn = "uad_kv_set_block_scales";
  if (!k_scales != !v_scales) return kv_fail(kv, UAD_E_INVALID, fn, "scales of K and of V, or neither");
  if (k_scales) {
    if (kv->cfg.dtype != UAD_DTYPE_F8) return kv_fail(kv, UAD_E_INVALID, fn, "scales are for pools of UAD_DTYPE_F8");
    if (kv->cfg.k_scale != 1.f || kv->cfg.v_scale != 1.f)
      return kv_fail(kv, UAD_E_INVALID, fn, "a handle with scales for blocks takes k_scale and v_scale 1");
    if (kv->cfg.n_kv_heads > 65535) return kv_fail(kv, UAD_E_UNSUPPORTED, fn, "n_kv_heads must be at most 65535");
    if (!aligned(k_scales, 4) || !aligned(v_scales, 4)) return kv_fail(kv, UAD_E_INVALID, fn, "scales not aligned to their type");
    OnDevice on(kv->device);
    if (on.err() != hipSuccess) return kv_hip_fail(kv, on.err(), fn, "hipSetDevice");
    const size_t bytes = kv->layer_elems / kv->cfg.head_dim / kScaleBlock * kv->cfg.n_layers * sizeof(float);
    if (!device_range(kv->device, k_scales, bytes) || !device_range(kv->device, v_scales, bytes))
      return kv_fail(kv, UAD_E_SHAPE, fn, "scales are not device memory of this device for their whole length");
  }
  kv->k_scales = k_scales;
  kv->v_scales = v_scales;
  return UAD_OK;
}

uad_status uad_kv_attend_rows(uad_kv *kv, int32_t layer, const void *q, void *out, int32_t dtype, int64_t ldq, int64_t ldo,
                              int32_t n_rows, const int32_t *row_start, const int32_t *lens, const int32_t *positions,
                              const int32_t *page_table, int32_t pages_per_seq, int32_t n_seqs, float scale,
                              int32_t window, int32_t n_sinks, int32_t causal) {
  if (!kv) return UAD_E_INVALID;
  const char *fn = "uad_kv_attend_rows";
  const bool none = n_rows == 0;
  uad_status st = check_call(kv, fn, layer, dtype, none ? kv->cfg.k : q, none ? kv->cfg.k : out, lens, page_table,
                             pages_per_seq, n_seqs);
  if (st != UAD_OK) return st;
  if (n_rows < 0) return kv_fail(kv, UAD_E_INVALID, fn, "n_rows must be >= 0");
  const int64_t row = (int64_t)kv->cfg.n_heads * kv->cfg.head_dim;
  if (ldq < row || ldo < row || ldq > kMaxLd || ldo > kMaxLd)
    return kv_fail(kv, UAD_E_INVALID, fn, "ldq / ldo below n_heads * head_dim or above 2^30");
  if (!row_start && n_rows != n_seqs) return kv_fail(kv, UAD_E_SHAPE, fn, "n_rows != n_seqs without row_start");
  if ((int64_t)n_rows * kv->cfg.n_heads > kMaxColumns) return kv_fail(kv, UAD_E_SHAPE, fn, "n_rows * n_heads above 2^25");
  if (window < 0 || n_sinks < 0 || (n_sinks > 0 && window == 0))
    return kv_fail(kv, UAD_E_INVALID, fn, "window and n_sinks must be >= 0, and n_sinks 0 without a window");
  if (causal != 0 && causal != 1) return kv_fail(kv, UAD_E_INVALID, fn, "causal must be 0 or 1");
  const float scale_log2 = (float)((double)scale * kv->cfg.k_scale * 1.4426950408889634);
  if (!std::isfinite(scale_log2)) return kv_fail(kv, UAD_E_INVALID, fn, "scale must be finite, times k_scale too");
  if (none || n_seqs == 0) return UAD_OK;
  OnDevice on(kv->device);
  if (on.err() != hipSuccess) return kv_hip_fail(kv, on.err(), fn, "hipSetDevice");
  KvRowsArgs a{};
  a.d = dims_of(kv);
  a.q = q; a.out = out; a.ldq = ldq; a.ldo = ldo;
  a.kp = layer_of(kv, kv->cfg.k, layer); a.vp = layer_of(kv, kv->cfg.v, layer);
  a.lens = lens; a.positions = positions; a.table = page_table;
  a.n_seqs = n_seqs; a.n_heads = kv->cfg.n_heads; a.group = kv->cfg.n_heads / kv->cfg.n_kv_heads;
  a.pages_per_seq = pages_per_seq;
  a.turns = kv->turns; a.rope_dim = kv->cfg.rope_dim; a.rope_pairs = kv->cfg.rope_pairs;
  a.scale_log2 = scale_log2;
  a.v_scale = kv->cfg.v_scale;
  a.k_scales = scales_of(kv, kv->k_scales, layer); a.v_scales = scales_of(kv, kv->v_scales, layer);
  a.status = kv->status;
  a.part = kv->part; a.part_ml = kv->part_ml; a.arrived = kv->arrived; a.slots = kv->slots;
  a.target = kv_attend_target(kv->n_cu, kv->cfg.head_dim);
  const size_t four = dtype == UAD_DTYPE_F32 ? 16 : 8;
  a.out_vec = aligned(out, four) && ldo % 4 == 0;
  a.row_start = row_start; a.n_rows = n_rows;
  a.window = std::min(window, kMaxSeen); a.sinks = std::min(n_sinks, kMaxSeen); a.causal = causal != 0;
  const hipError_t e = launch_kv_rows(a, dtype == UAD_DTYPE_F32, kv->cfg.dtype == UAD_DTYPE_F8, kv->stream);
  return e == hipSuccess ? UAD_OK : kv_hip_fail(kv, e, fn, "launch");
}

uad_status uad_kv_reserve(uad_kv *kv, const int32_t *lens, const int32_t *new_tokens, int32_t *lens_out, int32_t *page_table,
                          int32_t pages_per_seq, int32_t n_seqs, const int32_t *free_pages, const int32_t *n_free,
                          int32_t *n_free_out, int32_t *row_start, int64_t *slots, int32_t n_rows) {
  if (!kv) return UAD_E_INVALID;
  const char *fn = "uad_kv_reserve";
  uad_status st = check_pages(kv, fn, lens, page_table, free_pages, n_free, pages_per_seq, n_seqs);
  if (st != UAD_OK) return st;
  if (n_seqs > 0 && (!lens_out || !n_free_out)) return kv_fail(kv, UAD_E_INVALID, fn, "null pointer");
  if (n_rows < 0) return kv_fail(kv, UAD_E_INVALID, fn, "n_rows must be >= 0");
  if (!aligned(slots, 8)) return kv_fail(kv, UAD_E_INVALID, fn, "data not aligned to its type");
  if (n_seqs == 0) return UAD_OK;
  OnDevice on(kv->device);
  if (on.err() != hipSuccess) return kv_hip_fail(kv, on.err(), fn, "hipSetDevice");
  KvReserveArgs a{};
  a.lens = lens; a.new_tokens = new_tokens; a.lens_out = lens_out; a.table = page_table;
  a.pages_per_seq = pages_per_seq; a.n_seqs = n_seqs;
  a.free_pages = free_pages; a.n_free = n_free; a.n_free_out = n_free_out;
  a.row_start = row_start; a.slots = slots; a.n_rows = slots ? n_rows : 0;
  a.n_pages = kv->cfg.n_pages; a.page_shift = dims_of(kv).page_shift;
  a.status = kv->status; a.arrived = kv->pages_arrived;
  const hipError_t e = launch_kv_reserve(a, kv->stream);
  return e == hipSuccess ? UAD_OK : kv_hip_fail(kv, e, fn, "launch");
}

uad_status uad_kv_release(uad_kv *kv, const int32_t *lens, int32_t *page_table, int32_t pages_per_seq, int32_t n_seqs,
                          int32_t *free_pages, int32_t *n_free, int32_t window, int32_t n_sinks) {
  if (!kv) return UAD_E_INVALID;
  const char *fn = "uad_kv_release";
  uad_status st = check_pages(kv, fn, lens, page_table, free_pages, n_free, pages_per_seq, n_seqs);
  if (st != UAD_OK) return st;
  if (window < 0 || n_sinks < 0 || (n_sinks > 0 && window == 0))
    return kv_fail(kv, UAD_E_INVALID, fn, "window and n_sinks must be >= 0, and n_sinks 0 without a window");
  if (n_seqs == 0) return UAD_OK;
  OnDevice on(kv->device);
  if (on.err() != hipSuccess) return kv_hip_fail(kv, on.err(), fn, "hipSetDevice");
  KvReleaseArgs a{};
  a.lens = lens; a.table = page_table; a.pages_per_seq = pages_per_seq; a.n_seqs = n_seqs;
  a.free_pages = free_pages; a.n_free = n_free;
  a.window = std::min(window, kMaxSeen); a.sinks = std::min(n_sinks, kMaxSeen);
  a.n_pages = kv->cfg.n_pages; a.page_shift = dims_of(kv).page_shift;
  a.n_free_was = kv->page_counts; a.counts = kv->page_counts + 1;
  a.status = kv->status;
  const hipError_t e = launch_kv_release(a, kv->stream);
  return e == hipSuccess ? UAD_OK : kv_hip_fail(kv, e, fn, "launch");
}

}  // extern "C"
