// What the paged cache's host code needs beside hip_stub.cpp: the current device, and
// launchers that note what they were given.
#include <cstdio>
#include <cstring>
#include <string>

#include "../../paper_2609_37772_amd/csrc/kv_internal.h"

namespace {
int g_current = 3;
std::string g_calls, g_text;
hipError_t g_launch = hipSuccess;
}  // namespace

extern "C" {
void kv_stub_reset(int fail) { g_calls.clear(); g_launch = fail ? hipErrorLaunchFailure : hipSuccess; }
const char *kv_stub_calls() { g_text = g_calls; return g_text.c_str(); }
int kv_stub_current_device() { return g_current; }
void kv_stub_status(uad_kv *kv, unsigned w) { *kv->status = w; }
void kv_stub_ctx_status(uad_ctx *c, unsigned w) { *c->status = w; }
int kv_stub_prefix_set(const uad_ctx *c) { return c->prefix_set ? c->prefix_len : -1; }
hipError_t hipGetDevice(int *d) { *d = g_current; return hipSuccess; }
hipError_t hipMemsetAsync(void *p, int v, size_t n, hipStream_t) { std::memset(p, v, n); return hipSuccess; }
hipError_t kv_set_device(int d) { g_current = d; return hipSuccess; }
}  // extern "C"

namespace uad {
int kv_attend_target(int n_cu, int) { return n_cu; }
hipError_t kv_attend_init(int) { return hipSuccess; }
hipError_t launch_kv_append(const KvAppendArgs &a, bool f32, bool f8, hipStream_t) {
  char t[160];
  std::snprintf(t, sizeof t, "append %d %d %d %d %lld %lld %d;", a.n_rows, a.n_seqs, f32, f8, (long long)a.ldk,
                (long long)a.ldv, a.d.page_shift);
  g_calls += t;
  return g_launch;
}
hipError_t launch_kv_attend(const KvAttendArgs &a, bool f32, bool f8, hipStream_t) {
  char t[160];
  std::snprintf(t, sizeof t, "attend %d %d %d %d %d;", a.n_seqs, a.n_heads, a.group, f32, f8);
  g_calls += t;
  return g_launch;
}
hipError_t launch_kv_prefix(const KvPrefixArgs &a, int batch, int n_layers, bool, hipStream_t) {
  char t[160];
  std::snprintf(t, sizeof t, "prefix %d %d %d;", batch, n_layers, a.n_keys);
  g_calls += t;
  return g_launch;
}
}  // namespace uad
