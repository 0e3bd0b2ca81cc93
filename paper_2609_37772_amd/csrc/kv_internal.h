// Internal declarations of the paged K/V cache (see the uad_kv entry points in
// include/uad.h): kernel arguments, launchers and the handle.
#pragma once

#include <string>

#include "paged.h"
#include "uad_internal.h"

namespace uad {

struct KvAppendArgs {
  PagedDims d;
  const void *k, *v;      // new rows [n_rows][n_kv_heads][head_dim], fp32 or bf16
  int64_t ldk, ldv;       // elements from one row to the next
  void *kp, *vp;          // the layer's pools
  const int32_t *row_start;  // [n_seqs + 1] or null: row b belongs to sequence b
  const int32_t *lens;       // [n_seqs] lengths with the new tokens
  const int32_t *positions;  // [n_rows] rotation positions, or null: the cache positions
  const int32_t *table;      // [n_seqs][pages_per_seq]
  int n_rows, n_seqs, pages_per_seq;
  int row0;               // first row of this launch
  bool in_vec;            // rows can be loaded 16 bytes at a time
  const double *turns;    // [rope_dim / 2] turns per position
  const uint64_t *steps;  // the same in units of 2^-64 turns, whole turns left out
  int rope_dim, rope_pairs;
  float k_scale, v_scale, k_inv, v_inv;  // 8-bit pools hold value / scale; 1 / scale
  float *k_scales, *v_scales;  // the layer's, of every block of tokens (see paged.h), or null
  unsigned *status;
};

struct KvAttendArgs {
  PagedDims d;
  const void *q;          // [n_seqs][n_heads][head_dim], fp32 or bf16
  void *out;              // like q
  int64_t ldq, ldo;
  const void *kp, *vp;
  const int32_t *lens, *positions, *table;
  int n_seqs, n_heads, group, pages_per_seq;
  const double *turns;
  int rope_dim, rope_pairs;
  float scale_log2;       // log2(e) * softmax scale * K scale
  float v_scale;
  const float *k_scales, *v_scales;  // the layer's, of every block of tokens, or null (then the above are 1)
  unsigned *status;
  // joins of units that several workgroups share: a slot for each, of up to 64 rows
  // (min(16, group) for a single token, 16 for a few) of unnormalised outputs [rows][head_dim] and a
  // (max, sum) pair per row, and two arrival counters (zero between launches: the last
  // to arrive clears them)
  float *part;
  uint64_t *part_ml;
  unsigned *arrived;      // [2][slots]
  int slots;
  int target;             // workgroups that run at once
  bool out_vec;           // four outputs can be stored at once
  // set by the launcher:
  bool unsplit;           // no sequence can have more tiles than a split takes
  bool few_tiles;         // all tiles count in 32 bits
};

// Attention of new rows: q and out are [n_rows][n_heads][head_dim], positions [n_rows].
struct KvRowsArgs : KvAttendArgs {
  const int32_t *row_start;  // [n_seqs + 1], or null: row b belongs to sequence b
  int n_rows;
  int window, sinks;         // 0, 0: every key; at most 2^30
  bool causal;
};

// Page tables (see uad_kv_reserve and uad_kv_release).
struct KvReserveArgs {
  const int32_t *lens, *new_tokens;  // [n_seqs]; new_tokens null: one each
  int32_t *lens_out;                 // may be lens
  int32_t *table;
  int pages_per_seq, n_seqs;
  const int32_t *free_pages, *n_free;
  int32_t *n_free_out;               // may be n_free
  int32_t *row_start;                // [n_seqs + 1] or null
  int64_t *slots;                    // [n_rows] or null
  int n_rows;
  int n_pages, page_shift;
  unsigned *status, *arrived;        // arrived: zero between launches
  int slot_wgs;                      // set by the launcher: workgroups that fill slots
};
struct KvReleaseArgs {
  const int32_t *lens;
  int32_t *table;
  int pages_per_seq, n_seqs;
  int32_t *free_pages, *n_free;
  int window, sinks;
  int n_pages, page_shift;
  int32_t *counts, *n_free_was;      // [n_seqs], [1]: workspace
  unsigned *status;
};

// The expert's prefix from the pages (stores as in PrefixArgs).
struct KvPrefixArgs {
  PagedDims d;
  const void *kp, *vp;    // pools of the first layer
  size_t src_layer;       // pool elements per layer
  const int32_t *lens, *table;
  int pages_per_seq;
  int n_keys, s_alloc, env0;
  size_t dst_layer;
  __bf16 *kc, *vtc;
  float k_scale, v_scale;
  const float *k_scales, *v_scales;  // the first layer's, of every block of tokens, or null
  size_t scale_layer;     // scales per layer
  unsigned *status, *ctx_status;
};

// Attention workgroups that run at once, and the kernels' LDS limits raised (once per
// handle).
int kv_attend_target(int n_cu, int head_dim);
hipError_t kv_attend_init(int head_dim);
hipError_t launch_kv_append(const KvAppendArgs &a, bool f32, bool f8, hipStream_t s);
hipError_t launch_kv_attend(const KvAttendArgs &a, bool f32, bool f8, hipStream_t s);
hipError_t launch_kv_prefix(const KvPrefixArgs &a, int batch, int n_layers, bool f8, hipStream_t s);
// In code objects of their own: new rows, and what 8-bit pools with scales for blocks take
// of append and attend (which go there by themselves).
hipError_t kv_rows_init(int head_dim);
hipError_t launch_kv_rows(const KvRowsArgs &a, bool f32, bool f8, hipStream_t s);
hipError_t kv_prompt_init(int head_dim);
hipError_t launch_kv_prompt(const KvRowsArgs &a, int key_waves, bool f32, bool f8, hipStream_t s);
hipError_t launch_kv_append_blocks(const KvAppendArgs &a, bool f32, hipStream_t s);
hipError_t launch_kv_reserve(const KvReserveArgs &a, hipStream_t s);
hipError_t launch_kv_release(const KvReleaseArgs &a, hipStream_t s);

}  // namespace uad

struct uad_kv {
  uad_kv_config cfg{};
  int device = 0;
  hipStream_t stream = nullptr;
  std::string err;
  int n_cu = 0;
  size_t layer_elems = 0;  // pool elements per layer
  float *k_scales = nullptr, *v_scales = nullptr;  // the caller's, of every block of tokens (uad_kv_set_block_scales)
  void *buf = nullptr;     // status word, turns, workspace
  unsigned *status = nullptr;
  double *turns = nullptr;
  uint64_t *steps = nullptr;
  float *part = nullptr;
  uint64_t *part_ml = nullptr;
  unsigned *arrived = nullptr;
  int slots = 0;
  unsigned *pages_arrived = nullptr;  // of the page tables' calls
  int32_t *page_counts = nullptr;     // [1 + max_seqs], likewise
  hipEvent_t ev = nullptr;  // orders the cache's stream and an expert's
};
