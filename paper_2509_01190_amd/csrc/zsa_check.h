// Argument checks that the C entry points share: each returns ZSA_OK, or the
// status with its text set (zsa_last_error).
#pragma once

#include "../../include/zsa.h"
#include "zsa_internal.h"

namespace zsa {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline size_t esize(int dtype) { return dtype == ZSA_BF16 ? 2 : 4; }
inline size_t round256(size_t b) { return (b + 255) & ~static_cast<size_t>(255); }

// validate packed sequence offsets; returns total rows and the longest length
inline int check_seqs(int32_t batch, const int32_t* cu_host, const int32_t* cu_dev, int32_t* total,
               int32_t* max_len) {
  if (batch < 0) return set_error(ZSA_EINVAL, "batch %d < 0", batch);
  if (cu_host == nullptr || cu_dev == nullptr) return set_error(ZSA_EINVAL, "cu_host / cu_dev is NULL");
  if (cu_host[0] != 0) return set_error(ZSA_ESHAPE, "cu[0] = %d, must be 0", cu_host[0]);
  int32_t ml = 0;
  for (int b = 0; b < batch; ++b) {
    // (before the difference: between offsets below 0 it may not fit)
    if (cu_host[b + 1] < cu_host[b]) return set_error(ZSA_ESHAPE, "cu not monotone at sequence %d", b);
    const int32_t len = cu_host[b + 1] - cu_host[b];
    if (len > ml) ml = len;
  }
  *total = cu_host[batch];
  *max_len = ml;
  return ZSA_OK;
}

inline int check_dtype(int32_t dtype) {
  if (dtype != ZSA_F32 && dtype != ZSA_BF16) return set_error(ZSA_EINVAL, "dtype %d unknown", dtype);
  return ZSA_OK;
}

inline int check_ptr16(const void* p, const char* name, bool may_be_null = false) {
  if (p == nullptr) {
    if (may_be_null) return ZSA_OK;
    return set_error(ZSA_EINVAL, "%s is NULL", name);
  }
  if (!aligned16(p)) return set_error(ZSA_EALIGN, "%s is not 16-byte aligned", name);
  return ZSA_OK;
}

inline int check_width(int32_t dtype, int64_t width, const char* name) {
  if (width <= 0) return set_error(ZSA_ESHAPE, "%s = %lld must be positive", name, (long long)width);
  if ((width * static_cast<int64_t>(esize(dtype))) % 16 != 0)
    return set_error(ZSA_EALIGN, "%s = %lld rows are not a multiple of 16 bytes", name, (long long)width);
  return ZSA_OK;
}

inline int check_head_dim(int32_t hd) {
  if (hd != 16 && hd != 32 && hd != 64 && hd != 128)
    return set_error(ZSA_EUNSUPPORTED, "head_dim %d (supported: 16, 32, 64, 128)", hd);
  return ZSA_OK;
}

inline int check_kv_heads(int32_t n_heads, int32_t n_kv_heads, int* group) {
  if (n_heads <= 0) return set_error(ZSA_EINVAL, "n_heads %d", n_heads);
  const int32_t hkv = n_kv_heads == 0 ? n_heads : n_kv_heads;
  if (hkv < 0 || n_heads % hkv != 0)
    return set_error(ZSA_ESHAPE, "n_kv_heads %d must divide n_heads %d", n_kv_heads, n_heads);
  *group = n_heads / hkv;
  return ZSA_OK;
}

}  // namespace zsa
