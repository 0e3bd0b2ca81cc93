// What the entry points of the paged K/V cache share: the calling thread's device, errors,
// and argument checks.
#pragma once

#include <hip/hip_runtime.h>

#include <string>

#include "kv_internal.h"

namespace uad {

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

inline uad_status kv_fail(uad_kv *kv, uad_status st, const char *fn, const char *what) {
  try {
    kv->err = std::string(fn) + ": " + what;
  } catch (...) {
    kv->err.clear();
  }
  return st;
}

inline uad_status kv_hip_fail(uad_kv *kv, hipError_t e, const char *fn, const char *what) {
  (void)hipGetLastError();
  try {
    kv->err = std::string(fn) + ": " + what + ": " + hipGetErrorString(e);
  } catch (...) {
    kv->err.clear();
  }
  return UAD_E_HIP;
}

// Whether `bytes` from p on are device memory of `device`, in one allocation or in
// adjacent ones: a kernel would read and write past a shorter one.
inline bool device_range(int device, const void *p, size_t bytes) {
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

inline PagedDims dims_of(const uad_kv *kv) {
  PagedDims d{};
  d.n_pages = kv->cfg.n_pages;
  while ((1 << d.page_shift) < kv->cfg.page_size) ++d.page_shift;
  d.n_kv_heads = kv->cfg.n_kv_heads;
  d.head_dim = kv->cfg.head_dim;
  return d;
}

inline size_t pool_esz(const uad_kv *kv) { return kv->cfg.dtype == UAD_DTYPE_F8 ? 1 : 2; }
inline void *layer_of(const uad_kv *kv, void *pool, int layer) { return (char *)pool + layer * kv->layer_elems * pool_esz(kv); }
// A layer's scales of blocks, or null.
inline float *scales_of(const uad_kv *kv, float *scales, int layer) {
  return scales ? scales + layer * (kv->layer_elems / kv->cfg.head_dim / kScaleBlock) : nullptr;
}

// Row strides (elements) and tokens of a sequence: products with row numbers stay
// within 64 bits, positions and the tiles behind the last one within 32.
constexpr int64_t kMaxLd = (int64_t)1 << 30, kMaxTokens = (int64_t)1 << 30;

inline bool aligned(const void *p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

// What append and attend check alike.
inline uad_status check_call(uad_kv *kv, const char *fn, int layer, int dtype, const void *a, const void *b, const void *lens,
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

}  // namespace uad
