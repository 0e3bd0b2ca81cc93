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
  int rope_dim, rope_pairs;
  float k_scale, v_scale, k_inv, v_inv;  // 8-bit pools hold value / scale; 1 / scale
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
  unsigned *status;
  // joins of units that several workgroups share: a slot for each, of min(16, group)
  // rows of unnormalised outputs [rows][head_dim] and a (max, sum) pair per row, and
  // two arrival counters (zero between launches: the last to arrive clears them)
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
  unsigned *status, *ctx_status;
};

// Attention workgroups that run at once, and the kernels' LDS limits raised (once per
// handle).
int kv_attend_target(int n_cu, int head_dim);
hipError_t kv_attend_init(int head_dim);
hipError_t launch_kv_append(const KvAppendArgs &a, bool f32, bool f8, hipStream_t s);
hipError_t launch_kv_attend(const KvAttendArgs &a, bool f32, bool f8, hipStream_t s);
hipError_t launch_kv_prefix(const KvPrefixArgs &a, int batch, int n_layers, bool f8, hipStream_t s);

}  // namespace uad

struct uad_kv {
  uad_kv_config cfg{};
  int device = 0;
  hipStream_t stream = nullptr;
  std::string err;
  int n_cu = 0;
  size_t layer_elems = 0;  // pool elements per layer
  void *buf = nullptr;     // status word, turns, workspace
  unsigned *status = nullptr;
  double *turns = nullptr;
  float *part = nullptr;
  uint64_t *part_ml = nullptr;
  unsigned *arrived = nullptr;
  int slots = 0;
  hipEvent_t ev = nullptr;  // orders the cache's stream and an expert's
};
