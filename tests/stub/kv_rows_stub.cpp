// Launchers of the paged cache's other entry points, beside kv_stub.cpp: they note what they
// were given.
#include <cstdio>
#include <string>

#include "../../paper_2609_37772_amd/csrc/kv_internal.h"

namespace {
std::string g_rows, g_rows_text;
hipError_t g_rows_launch = hipSuccess;
}  // namespace

extern "C" {
void kv_rows_stub_reset(int fail) { g_rows.clear(); g_rows_launch = fail ? hipErrorLaunchFailure : hipSuccess; }
const char *kv_rows_stub_calls() { g_rows_text = g_rows; return g_rows_text.c_str(); }
int kv_stub_has_scales(const uad_kv *kv) { return kv->k_scales != nullptr; }
}  // extern "C"

namespace uad {
hipError_t launch_kv_rows(const KvRowsArgs &a, bool f32, bool f8, hipStream_t) {
  char t[200];
  std::snprintf(t, sizeof t, "rows %d %d %d %d %d %d %d %d %d;", a.n_rows, a.n_seqs, a.row_start != nullptr, f32, f8, a.window, a.sinks,
                a.causal, a.k_scales != nullptr);
  g_rows += t;
  return g_rows_launch;
}
hipError_t launch_kv_reserve(const KvReserveArgs &a, hipStream_t) {
  char t[200];
  std::snprintf(t, sizeof t, "reserve %d %d %d %d %d;", a.n_seqs, a.n_rows, a.slots != nullptr, a.n_pages, a.page_shift);
  g_rows += t;
  return g_rows_launch;
}
hipError_t launch_kv_release(const KvReleaseArgs &a, hipStream_t) {
  char t[200];
  std::snprintf(t, sizeof t, "release %d %d %d %d;", a.n_seqs, a.window, a.sinks, a.n_pages);
  g_rows += t;
  return g_rows_launch;
}
}  // namespace uad
