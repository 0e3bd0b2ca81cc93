// C ABI of the paged K/V cache: handle, argument checks, kernel arguments.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <new>
#include <string>

#include "kv_internal.h"

using namespace uad;

namespace {

thread_local std::string g_kv_create_err;

// Every entry point leaves the calling thread's device as it found it, and lets no
// exception (of a message's allocation, say) out into the caller's C.
class OnDevice {
 public:
  explicit OnDevice(int device) {
    err_ = hipGetDevice(&was_);
    if (err_ == hipSuccess && was_ != device) {
      err_ = hipSetDevice(device);
      back_ = err_ == hipSuccess;
    }
  }
  ~OnDevice() {
    if (back_) (void)hipSetDevice(was_);
  }
  hipError_t err() const { return err_; }

 private:
  int was_ = 0;
  bool back_ = false;
  hipError_t err_ = hipSuccess;
};

uad_status kv_fail(uad_kv *kv, uad_status st, const char *fn, const char *what) {
  try {
    kv->err = std::string(fn) + ": " + what;
  } catch (...) {
    kv->err.clear();
  }
  return st;
}

uad_status kv_hip_fail(uad_kv *kv, hipError_t e, const char *fn, const char *what) {
  (void)hipGetLastError();
  try {
    kv->err = std::string(fn) + ": " + what + ": " + hipGetErrorString(e);
  } catch (...) {
    kv->err.clear();
  }
  return UAD_E_HIP;
}

uad_status ctx_fail(uad_ctx *c, uad_status st, const char *what) {
  try {
    c->err = std::string("uad_set_prefix_paged: ") + what;
  } catch (...) {
    c->err.clear();
  }
  return st;
}

// Whether `bytes` from p on are device memory of `device`, in one allocation or in
// adjacent ones: a kernel would read and write past a shorter one.
bool device_range(int device, const void *p, size_t bytes) {
  const char *at = (const char *)p, *const end = at + bytes;
  while (at < end) {
    hipPointerAttribute_t pa{};
    hipDeviceptr_t base = nullptr;
    size_t size = 0;
    if (hipPointerGetAttributes(&pa, at) != hipSuccess || pa.type != hipMemoryTypeDevice || pa.device != device ||
        hipMemGetAddressRange(&base, &size, (hipDeviceptr_t)at) != hipSuccess || (const char *)base + size <= at) {
      (void)hipGetLastError();
      return false;
    }
    at = (const char *)base + size;
  }
  return true;
}

PagedDims dims_of(const uad_kv *kv) {
  PagedDims d{};
  d.n_pages = kv->cfg.n_pages;
  while ((1 << d.page_shift) < kv->cfg.page_size) ++d.page_shift;
  d.n_kv_heads = kv->cfg.n_kv_heads;
  d.head_dim = kv->cfg.head_dim;
  return d;
}

size_t pool_esz(const uad_kv *kv) { return kv->cfg.dtype == UAD_DTYPE_F8 ? 1 : 2; }
void *layer_of(const uad_kv *kv, void *pool, int layer) { return (char *)pool + layer * kv->layer_elems * pool_esz(kv); }

// Row strides (elements) and tokens of a sequence: products with row numbers stay
// within 64 bits, positions and the tiles behind the last one within 32.
constexpr int64_t kMaxLd = (int64_t)1 << 30, kMaxTokens = (int64_t)1 << 30;

bool aligned(const void *p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

// What append and attend check alike.
uad_status check_call(uad_kv *kv, const char *fn, int layer, int dtype, const void *a, const void *b, const void *lens,
                      const void *table, int pages_per_seq, int n_seqs) {
  if (layer < 0 || layer >= kv->cfg.n_layers) return kv_fail(kv, UAD_E_INVALID, fn, "no such layer");
  if (dtype != UAD_DTYPE_F32 && dtype != UAD_DTYPE_BF16) return kv_fail(kv, UAD_E_INVALID, fn, "bad dtype");
  if (n_seqs < 0 || pages_per_seq < 1) return kv_fail(kv, UAD_E_INVALID, fn, "n_seqs must be >= 0, pages_per_seq >= 1");
  if (n_seqs > kv->cfg.max_seqs) return kv_fail(kv, UAD_E_SHAPE, fn, "n_seqs > max_seqs");
  if ((int64_t)pages_per_seq * kv->cfg.page_size > kMaxTokens)
    return kv_fail(kv, UAD_E_SHAPE, fn, "a page table of more than 2^30 tokens per sequence");
  if (n_seqs > 0 && (!a || !b || !lens || !table)) return kv_fail(kv, UAD_E_INVALID, fn, "null pointer");
  const size_t esz = dtype == UAD_DTYPE_F32 ? 4 : 2;
  if (!aligned(a, esz) || !aligned(b, esz)) return kv_fail(kv, UAD_E_INVALID, fn, "data not aligned to its type");
  return UAD_OK;
}

}  // namespace

extern "C" {

const char *uad_kv_last_error(const uad_kv *kv) { return kv ? kv->err.c_str() : g_kv_create_err.c_str(); }

uad_status uad_kv_create(const uad_kv_config *cfg, int32_t device, void *hip_stream, uad_kv **out) {
  if (out) *out = nullptr;
  uad_kv *kv = nullptr;
  auto cerr = [&](uad_status st, const char *m, hipError_t e = hipSuccess) {
    if (e != hipSuccess) (void)hipGetLastError();
    uad_kv_destroy(kv);
    try {
      g_kv_create_err = std::string("uad_kv_create: ") + m;
      if (e != hipSuccess) g_kv_create_err += std::string(": ") + hipGetErrorString(e);
    } catch (...) {
      g_kv_create_err.clear();
    }
    return st;
  };
  if (!cfg || !out) return cerr(UAD_E_INVALID, "null cfg/out");
  const uad_kv_config &m = *cfg;
  if (m.n_layers < 1 || m.n_heads < 1 || m.n_kv_heads < 1 || m.head_dim < 1 || m.page_size < 1 || m.n_pages < 1 ||
      m.max_seqs < 1)
    return cerr(UAD_E_INVALID, "every dimension must be positive");
  if (m.dtype != UAD_DTYPE_BF16 && m.dtype != UAD_DTYPE_F8) return cerr(UAD_E_INVALID, "pools must be BF16 or F8");
  if (m.rope_dim < 0 || m.rope_dim > m.head_dim || m.rope_pairs < 0 || m.rope_pairs > 1)
    return cerr(UAD_E_INVALID, "rope_dim must be 0 .. head_dim, rope_pairs 0 or 1");
  if (m.rope_dim && !(m.rope_theta > 0.0 && std::isfinite(m.rope_theta)))
    return cerr(UAD_E_INVALID, "rope_theta must be finite and > 0");
  if (!(m.k_scale > 0.f && std::isfinite(m.k_scale) && m.v_scale > 0.f && std::isfinite(m.v_scale)))
    return cerr(UAD_E_INVALID, "scales must be finite and > 0");
  if (!std::isfinite(1.f / m.k_scale) || !std::isfinite(1.f / m.v_scale))
    return cerr(UAD_E_INVALID, "the reciprocal of a scale overflows");
  if (!std::isfinite(448.f * m.k_scale) || !std::isfinite(448.f * m.v_scale))
    return cerr(UAD_E_INVALID, "448 times a scale overflows");
  if (m.dtype == UAD_DTYPE_BF16 && (m.k_scale != 1.f || m.v_scale != 1.f))
    return cerr(UAD_E_INVALID, "bf16 pools take no scale (k_scale and v_scale 1)");
  if (m.head_dim != 64 && m.head_dim != 128 && m.head_dim != 256)
    return cerr(UAD_E_UNSUPPORTED, "head_dim must be 64, 128 or 256");
  if (m.page_size < 16 || m.page_size > 256 || (m.page_size & (m.page_size - 1)))
    return cerr(UAD_E_UNSUPPORTED, "page_size must be 16, 32, 64, 128 or 256");
  if (m.rope_dim % 16) return cerr(UAD_E_UNSUPPORTED, "rope_dim must be a multiple of 16");
  if (m.n_heads % m.n_kv_heads) return cerr(UAD_E_UNSUPPORTED, "n_kv_heads must divide n_heads");
  if ((int64_t)m.n_kv_heads * ((m.n_heads / m.n_kv_heads + 15) / 16) * m.max_seqs > (1 << 22))
    return cerr(UAD_E_UNSUPPORTED, "max_seqs * n_kv_heads * ceil(n_heads / n_kv_heads / 16) must be at most 2^22");
  if (!m.k || !m.v) return cerr(UAD_E_INVALID, "null pool");
  if (!aligned(m.k, 16) || !aligned(m.v, 16)) return cerr(UAD_E_INVALID, "the pools must be 16-byte aligned");

  OnDevice on(device);
  if (on.err() != hipSuccess) return cerr(UAD_E_HIP, "hipSetDevice", on.err());
  kv = new (std::nothrow) uad_kv();
  if (!kv) return cerr(UAD_E_OOM, "handle");
  kv->cfg = m;
  kv->device = device;
  kv->stream = (hipStream_t)hip_stream;
  kv->layer_elems = (size_t)m.n_pages * m.n_kv_heads * m.page_size * m.head_dim;
  // n_layers * n_pages * heads * page * dim stays below 2^31 * 2^31 * 2^16 * 2^16 only by luck: check
  if (kv->layer_elems / ((size_t)m.n_kv_heads * m.page_size * m.head_dim) != (size_t)m.n_pages ||
      kv->layer_elems > ((size_t)1 << 46) || (size_t)m.n_layers > ((size_t)1 << 46) / kv->layer_elems)
    return cerr(UAD_E_SHAPE, "a pool beyond any device's memory");
  const size_t bytes = kv->layer_elems * m.n_layers * pool_esz(kv);
  if (!device_range(device, m.k, bytes) || !device_range(device, m.v, bytes))
    return cerr(UAD_E_SHAPE, "a pool is not device memory of this device for its whole length");
  hipError_t e = hipDeviceGetAttribute(&kv->n_cu, hipDeviceAttributeMultiprocessorCount, device);
  if (e != hipSuccess) return cerr(UAD_E_HIP, "hipDeviceGetAttribute", e);
  const size_t o_turns = 256, n_turns = m.rope_dim / 2;
  const size_t rows = std::min(16, m.n_heads / m.n_kv_heads);
  kv->slots = max_slots(kv_attend_target(kv->n_cu, m.head_dim));
  const size_t o_arrived = o_turns + 128 * sizeof(double), o_ml = o_arrived + 2 * (size_t)kv->slots * sizeof(unsigned);
  const size_t o_part = o_ml + kv->slots * rows * sizeof(uint64_t);
  const size_t total = o_part + kv->slots * rows * m.head_dim * sizeof(float);
  e = hipMalloc(&kv->buf, total);
  if (e != hipSuccess) return cerr(UAD_E_OOM, "hipMalloc(workspace)", e);
  e = hipMemset(kv->buf, 0, o_ml);
  if (e == hipSuccess) e = hipEventCreateWithFlags(&kv->ev, hipEventDisableTiming);
  kv->status = (unsigned *)kv->buf;
  kv->turns = (double *)((char *)kv->buf + o_turns);
  kv->arrived = (unsigned *)((char *)kv->buf + o_arrived);
  kv->part_ml = (uint64_t *)((char *)kv->buf + o_ml);
  kv->part = (float *)((char *)kv->buf + o_part);
  if (e == hipSuccess) e = kv_attend_init(m.head_dim);
  if (n_turns) {
    // turns (angle / 2 pi) per position of pair i: theta^(-2i/rope_dim) / 2 pi
    double turns[128];
    for (size_t i = 0; i < n_turns; ++i)
      turns[i] = std::pow(m.rope_theta, -2.0 * (double)i / (double)m.rope_dim) / (2.0 * M_PI);
    if (e == hipSuccess) e = hipMemcpy(kv->turns, turns, n_turns * sizeof(double), hipMemcpyHostToDevice);
  }
  // the null-stream memset may still run when another stream's work begins
  if (e == hipSuccess) e = hipStreamSynchronize(nullptr);
  if (e != hipSuccess) return cerr(UAD_E_HIP, "workspace", e);
  *out = kv;
  g_kv_create_err.clear();
  return UAD_OK;
}

void uad_kv_destroy(uad_kv *kv) {
  if (!kv) return;
  OnDevice on(kv->device);
  if (kv->buf) (void)hipStreamSynchronize(kv->stream);
  if (kv->buf) (void)hipFree(kv->buf);
  if (kv->ev) (void)hipEventDestroy(kv->ev);
  delete kv;
}

uad_status uad_kv_set_stream(uad_kv *kv, void *hip_stream) {
  if (!kv) return UAD_E_INVALID;
  OnDevice on(kv->device);
  hipError_t e = on.err();
  if (e == hipSuccess) e = hipStreamSynchronize(kv->stream);
  if (e != hipSuccess) return kv_hip_fail(kv, e, "uad_kv_set_stream", "hipStreamSynchronize");
  kv->stream = (hipStream_t)hip_stream;
  return UAD_OK;
}

uad_status uad_kv_append(uad_kv *kv, int32_t layer, const void *k, const void *v, int32_t dtype, int64_t ldk,
                         int64_t ldv, int32_t n_rows, const int32_t *row_start, const int32_t *lens,
                         const int32_t *positions, const int32_t *page_table, int32_t pages_per_seq, int32_t n_seqs) {
  if (!kv) return UAD_E_INVALID;
  const char *fn = "uad_kv_append";
  const bool none = n_rows == 0;
  uad_status st = check_call(kv, fn, layer, dtype, none ? kv->cfg.k : k, none ? kv->cfg.v : v, lens, page_table,
                             pages_per_seq, n_seqs);
  if (st != UAD_OK) return st;
  if (n_rows < 0) return kv_fail(kv, UAD_E_INVALID, fn, "n_rows must be >= 0");
  const int64_t row = (int64_t)kv->cfg.n_kv_heads * kv->cfg.head_dim;
  if (ldk < row || ldv < row || ldk > kMaxLd || ldv > kMaxLd)
    return kv_fail(kv, UAD_E_INVALID, fn, "ldk / ldv below n_kv_heads * head_dim or above 2^30");
  if (!row_start && n_rows != n_seqs) return kv_fail(kv, UAD_E_SHAPE, fn, "n_rows != n_seqs without row_start");
  if (none || n_seqs == 0) return UAD_OK;
  OnDevice on(kv->device);
  if (on.err() != hipSuccess) return kv_hip_fail(kv, on.err(), fn, "hipSetDevice");
  KvAppendArgs a{};
  a.d = dims_of(kv);
  a.k = k; a.v = v; a.ldk = ldk; a.ldv = ldv;
  a.kp = layer_of(kv, kv->cfg.k, layer); a.vp = layer_of(kv, kv->cfg.v, layer);
  a.row_start = row_start; a.lens = lens; a.positions = positions; a.table = page_table;
  a.n_rows = n_rows; a.n_seqs = n_seqs; a.pages_per_seq = pages_per_seq;
  a.turns = kv->turns; a.rope_dim = kv->cfg.rope_dim; a.rope_pairs = kv->cfg.rope_pairs;
  const int64_t per16 = dtype == UAD_DTYPE_F32 ? 4 : 8;
  a.in_vec = aligned(k, 16) && aligned(v, 16) && ldk % per16 == 0 && ldv % per16 == 0;
  a.k_scale = kv->cfg.k_scale; a.v_scale = kv->cfg.v_scale;
  a.k_inv = 1.f / a.k_scale; a.v_inv = 1.f / a.v_scale;
  a.status = kv->status;
  const hipError_t e = launch_kv_append(a, dtype == UAD_DTYPE_F32, kv->cfg.dtype == UAD_DTYPE_F8, kv->stream);
  return e == hipSuccess ? UAD_OK : kv_hip_fail(kv, e, fn, "launch");
}

uad_status uad_kv_attend(uad_kv *kv, int32_t layer, const void *q, void *out, int32_t dtype, int64_t ldq, int64_t ldo,
                         const int32_t *lens, const int32_t *positions, const int32_t *page_table,
                         int32_t pages_per_seq, int32_t n_seqs, float scale) {
  if (!kv) return UAD_E_INVALID;
  const char *fn = "uad_kv_attend";
  uad_status st = check_call(kv, fn, layer, dtype, q, out, lens, page_table, pages_per_seq, n_seqs);
  if (st != UAD_OK) return st;
  const int64_t row = (int64_t)kv->cfg.n_heads * kv->cfg.head_dim;
  if (ldq < row || ldo < row || ldq > kMaxLd || ldo > kMaxLd)
    return kv_fail(kv, UAD_E_INVALID, fn, "ldq / ldo below n_heads * head_dim or above 2^30");
  const float scale_log2 = (float)((double)scale * kv->cfg.k_scale * 1.4426950408889634);
  if (!std::isfinite(scale_log2)) return kv_fail(kv, UAD_E_INVALID, fn, "scale must be finite, times k_scale too");
  if (n_seqs == 0) return UAD_OK;
  OnDevice on(kv->device);
  if (on.err() != hipSuccess) return kv_hip_fail(kv, on.err(), fn, "hipSetDevice");
  KvAttendArgs a{};
  a.d = dims_of(kv);
  a.q = q; a.out = out; a.ldq = ldq; a.ldo = ldo;
  a.kp = layer_of(kv, kv->cfg.k, layer); a.vp = layer_of(kv, kv->cfg.v, layer);
  a.lens = lens; a.positions = positions; a.table = page_table;
  a.n_seqs = n_seqs; a.n_heads = kv->cfg.n_heads; a.group = kv->cfg.n_heads / kv->cfg.n_kv_heads;
  a.pages_per_seq = pages_per_seq;
  a.turns = kv->turns; a.rope_dim = kv->cfg.rope_dim; a.rope_pairs = kv->cfg.rope_pairs;
  a.scale_log2 = scale_log2;
  a.v_scale = kv->cfg.v_scale;
  a.status = kv->status;
  a.part = kv->part; a.part_ml = kv->part_ml; a.arrived = kv->arrived; a.slots = kv->slots;
  a.target = kv_attend_target(kv->n_cu, kv->cfg.head_dim);
  const size_t four = dtype == UAD_DTYPE_F32 ? 16 : 8;
  a.out_vec = aligned(out, four) && ldo % 4 == 0;
  const hipError_t e = launch_kv_attend(a, dtype == UAD_DTYPE_F32, kv->cfg.dtype == UAD_DTYPE_F8, kv->stream);
  return e == hipSuccess ? UAD_OK : kv_hip_fail(kv, e, fn, "launch");
}

uad_status uad_set_prefix_paged(uad_ctx *c, uad_kv *kv, const int32_t *lens, const int32_t *page_table,
                                int32_t pages_per_seq, int32_t batch, int32_t prefix_len) {
  if (!c) return UAD_E_INVALID;
  if (!kv || !lens || !page_table) return ctx_fail(c, UAD_E_INVALID, "null kv/lens/page_table");
  if (batch < 1 || prefix_len < 0 || pages_per_seq < 1)
    return ctx_fail(c, UAD_E_INVALID, "batch and pages_per_seq must be >= 1, prefix_len >= 0");
  if (batch > c->cfg.max_batch) return ctx_fail(c, UAD_E_SHAPE, "batch > max_batch");
  if (prefix_len > c->cfg.max_prefix) return ctx_fail(c, UAD_E_SHAPE, "prefix_len > max_prefix");
  if (prefix_len > (int64_t)pages_per_seq * kv->cfg.page_size || (int64_t)pages_per_seq * kv->cfg.page_size > kMaxTokens)
    return ctx_fail(c, UAD_E_SHAPE, "prefix_len beyond the page table, or a table of more than 2^30 tokens per sequence");
  if (kv->device != c->device) return ctx_fail(c, UAD_E_SHAPE, "the cache is on another device");
  if (kv->cfg.n_layers != c->L || kv->cfg.n_kv_heads != c->Hkv || kv->cfg.head_dim != c->hd)
    return ctx_fail(c, UAD_E_SHAPE, "the cache has another number of layers or KV heads, or another head_dim");
  OnDevice on(c->device);
  hipError_t e = on.err();
  KvPrefixArgs a{};
  a.d = dims_of(kv);
  a.kp = kv->cfg.k; a.vp = kv->cfg.v; a.src_layer = kv->layer_elems;
  a.lens = lens; a.table = page_table; a.pages_per_seq = pages_per_seq;
  a.n_keys = prefix_len; a.s_alloc = c->s_alloc; a.dst_layer = c->kv_layer_elems; a.kc = c->kcache; a.vtc = c->vtcache;
  a.k_scale = kv->cfg.k_scale; a.v_scale = kv->cfg.v_scale;
  a.status = kv->status; a.ctx_status = c->status;
  // The context's queued steps read the old prefix before this, the cache's queued
  // appends come before it and later ones after it.
  const bool cross = kv->stream != c->stream;
  if (e == hipSuccess && cross) e = hipEventRecord(kv->ev, kv->stream);
  if (e == hipSuccess && cross) e = hipStreamWaitEvent(c->stream, kv->ev, 0);
  if (e == hipSuccess) {
    c->prefix_set = false;
    e = launch_kv_prefix(a, batch, c->L, kv->cfg.dtype == UAD_DTYPE_F8, c->stream);
  }
  if (e == hipSuccess && cross) e = hipEventRecord(kv->ev, c->stream);
  if (e == hipSuccess && cross) e = hipStreamWaitEvent(kv->stream, kv->ev, 0);
  if (e != hipSuccess) {
    (void)hipGetLastError();
    try {
      c->err = std::string("uad_set_prefix_paged: ") + hipGetErrorString(e);
    } catch (...) {
      c->err.clear();
    }
    return UAD_E_HIP;
  }
  c->prefix_len = prefix_len;
  c->prefix_batch = batch;
  c->prefix_set = true;
  return UAD_OK;
}

uad_status uad_kv_synchronize(uad_kv *kv) {
  if (!kv) return UAD_E_INVALID;
  const char *fn = "uad_kv_synchronize";
  OnDevice on(kv->device);
  hipError_t e = on.err();
  if (e == hipSuccess) e = hipStreamSynchronize(kv->stream);
  if (e != hipSuccess) return kv_hip_fail(kv, e, fn, "hipStreamSynchronize");
  unsigned w = 0;
  e = hipMemcpy(&w, kv->status, sizeof(w), hipMemcpyDeviceToHost);
  // on the stream itself and waited for: work that is queued next, or a graph that is
  // replayed on another stream, must not have its status cleared
  if (e == hipSuccess && w) e = hipMemsetAsync(kv->status, 0, sizeof(w), kv->stream);
  if (e == hipSuccess && w) e = hipStreamSynchronize(kv->stream);
  if (e != hipSuccess) return kv_hip_fail(kv, e, fn, "status word");
  if (w)
    return kv_fail(kv, UAD_E_PAGE, fn, "a page id, a length or a row of the queued work could not be used (results of "
                                       "that work are invalid)");
  return UAD_OK;
}

}  // extern "C"
