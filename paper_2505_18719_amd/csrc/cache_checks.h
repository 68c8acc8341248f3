// Argument checks that the C entries of the cache's and the prompt's operators share.
#pragma once

#include <hip/hip_runtime_api.h>

#include <cmath>
#include <cstdio>

#include "cache.h"
#include "kernels.h"
#include "vla_cache.h"

namespace vla {

inline int hip_status(const char* call, hipError_t e) {
  if (e == hipSuccess) return set_error(VLA_OK, "");
  char msg[256];
  std::snprintf(msg, sizeof msg, "%s: %s", call, hipGetErrorString(e));
  return set_error(VLA_EHIP, msg);
}

inline bool aligned(const void* p, size_t n = 16) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// A tensor of rows of `width` elements: NULL, alignment, row stride.
inline int check_rows(const char* name, const void* p, int64_t ld, int64_t width) {
  char msg[128];
  if (!p) {
    std::snprintf(msg, sizeof msg, "%s is NULL", name);
    return set_error(VLA_EINVAL, msg);
  }
  if (!aligned(p) || ld % 8 != 0 || ld < width || ld > (int64_t)1 << 40) {
    std::snprintf(msg, sizeof msg, "%s must start on 16 bytes, its row stride hold a row and be a multiple of 8", name);
    return set_error(VLA_EINVAL, msg);
  }
  return VLA_OK;
}

inline int check_heads(int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t dtype) {
  if (n_heads < 1 || n_kv_heads < 1) return set_error(VLA_EINVAL, "need at least one head");
  if (n_heads > 1024 || n_kv_heads > 1024) return set_error(VLA_EUNSUPPORTED, "at most 1024 heads");
  if (head_dim != 64 && head_dim != 128 && head_dim != 256)
    return set_error(VLA_EUNSUPPORTED, "head_dim must be 64, 128 or 256");
  if (dtype != VLA_DTYPE_BF16 && dtype != VLA_DTYPE_F16) return set_error(VLA_EUNSUPPORTED, "unknown dtype");
  return VLA_OK;
}

// Scores are scaled to base 2.
inline int check_scale(float scale) {
  if (!std::isfinite(scale * 1.44269504f)) return set_error(VLA_EINVAL, "scale must be finite, times log2(e) too");
  return VLA_OK;
}

inline HeadRows rows_of(const void* p, int64_t ld) { return {static_cast<bf16_t*>(const_cast<void*>(p)), ld}; }

}  // namespace vla
