// C ABI of the paged cache's operators (vla_cache.h): argument checks and the host-side rotation frequencies.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdio>

#include "cache.h"
#include "kernels.h"
#include "vla_cache.h"

using namespace vla;

namespace {

int hip_status(const char* call, hipError_t e) {
  if (e == hipSuccess) return set_error(VLA_OK, "");
  char msg[256];
  std::snprintf(msg, sizeof msg, "%s: %s", call, hipGetErrorString(e));
  return set_error(VLA_EHIP, msg);
}

bool aligned(const void* p, size_t n = 16) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// A tensor of rows of `width` elements: NULL, alignment, row stride.
int check_rows(const char* name, const void* p, int64_t ld, int64_t width) {
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

int check_heads(int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t dtype) {
  if (n_heads < 1 || n_kv_heads < 1) return set_error(VLA_EINVAL, "need at least one head");
  if (n_heads > 1024 || n_kv_heads > 1024) return set_error(VLA_EUNSUPPORTED, "at most 1024 heads");
  if (head_dim != 64 && head_dim != 128 && head_dim != 256)
    return set_error(VLA_EUNSUPPORTED, "head_dim must be 64, 128 or 256");
  if (dtype != VLA_DTYPE_BF16 && dtype != VLA_DTYPE_F16) return set_error(VLA_EUNSUPPORTED, "unknown dtype");
  return VLA_OK;
}

int check_rotation(int32_t rot_dim, int32_t head_dim, int32_t layout, float eps, float rope_scale,
                   const int32_t* row_pos, const double* freqs) {
  if (rot_dim < 0 || rot_dim > head_dim || rot_dim % 16 != 0)
    return set_error(VLA_EUNSUPPORTED, "rot_dim must be a multiple of 16, at most head_dim");
  if (layout != VLA_ROPE_HALF && layout != VLA_ROPE_INTERLEAVED) return set_error(VLA_EINVAL, "unknown rotation layout");
  if (!(eps >= 0.f) || !std::isfinite(eps)) return set_error(VLA_EINVAL, "eps must be finite and >= 0");
  if (!std::isfinite(rope_scale)) return set_error(VLA_EINVAL, "rope_scale must be finite");
  if (rot_dim > 0 && (!row_pos || !freqs)) return set_error(VLA_EINVAL, "a rotation needs row_pos and freqs");
  if (rot_dim > 0 && !aligned(freqs)) return set_error(VLA_EINVAL, "freqs must start on 16 bytes");
  return VLA_OK;
}

HeadRows rows_of(const void* p, int64_t ld) { return {static_cast<bf16_t*>(const_cast<void*>(p)), ld}; }

}  // namespace

extern "C" {

int vla_kv_plan(int32_t n_env, const int32_t* cached_lens, const int32_t* new_lens, int32_t* page_table,
                int64_t ld_table, int32_t max_pages, const int32_t* free_pages, int32_t n_free,
                const int32_t* free_head, int32_t n_pages, int32_t max_rows, int32_t* lens, int32_t* row_start,
                int32_t* row_pos, int32_t* row_env, int32_t* row_slot, int32_t* stats, void* stream) {
  if (n_env < 0 || max_pages < 0 || n_free < 0 || n_pages < 0 || max_rows < 0) return set_error(VLA_EINVAL, "negative size");
  if (n_pages >= 1 << 27 || max_pages >= 1 << 27) return set_error(VLA_EUNSUPPORTED, "n_pages and max_pages must be below 2^27");
  if (ld_table < max_pages || ld_table > (int64_t)1 << 40) return set_error(VLA_EINVAL, "ld_table must hold a row of the page table");
  if (!row_start || !stats || (n_env > 0 && (!cached_lens || !new_lens || !lens)) ||
      (n_env > 0 && max_pages > 0 && !page_table) || (n_free > 0 && !free_pages) ||
      (max_rows > 0 && (!row_pos || !row_env || !row_slot)))
    return set_error(VLA_EINVAL, "NULL argument");
  if (n_env > 0 && (lens == cached_lens || lens == new_lens)) return set_error(VLA_EINVAL, "lens may not be an input");
  if (stats == free_head) return set_error(VLA_EINVAL, "stats may not be free_head");
  KvPlanArgs a{n_env, cached_lens, new_lens, page_table, ld_table, max_pages, free_pages, n_free, free_head,
               n_pages, max_rows, lens, row_start, row_pos, row_env, row_slot, stats};
  return hip_status("vla_kv_plan", launch_kv_plan(a, static_cast<hipStream_t>(stream)));
}

int vla_rope_freqs(int32_t rot_dim, double base, int32_t scaling, double factor, double low, double high,
                   double context, double* freqs_host, float* scale_host) {
  if (rot_dim < 2 || rot_dim > 256 || rot_dim % 2 != 0) return set_error(VLA_EINVAL, "rot_dim must be even, 2 to 256");
  if (!(base > 1.0) || !std::isfinite(base)) return set_error(VLA_EINVAL, "base must be finite and > 1");
  if (scaling < VLA_ROPE_NONE || scaling > VLA_ROPE_RAMP) return set_error(VLA_EINVAL, "unknown scaling");
  if (scaling != VLA_ROPE_NONE && (!(factor >= 1.0) || !std::isfinite(factor)))
    return set_error(VLA_EINVAL, "factor must be finite and >= 1");
  if (scaling == VLA_ROPE_BASE && rot_dim < 4) return set_error(VLA_EINVAL, "a changed base needs rot_dim >= 4");
  if (scaling >= VLA_ROPE_BANDS && (!(low > 0.0) || !(high > low) || !std::isfinite(high) || !(context > 0.0) ||
                                    !std::isfinite(context)))
    return set_error(VLA_EINVAL, "need 0 < low < high and context > 0, all finite");
  if (!freqs_host) return set_error(VLA_EINVAL, "freqs_host is NULL");
  constexpr double kTwoPi = 6.283185307179586476925;
  const double d = rot_dim;
  if (scaling == VLA_ROPE_BASE) base *= std::pow(factor, d / (d - 2));
  if (!std::isfinite(base)) return set_error(VLA_EINVAL, "the changed base must be finite");
  double a = 0, b = 0;
  if (scaling == VLA_ROPE_RAMP) {
    auto index = [&](double turns) { return d / 2 * std::log(context / (kTwoPi * turns)) / std::log(base); };
    a = std::max(0.0, std::floor(index(high)));
    b = std::min(d - 1, std::ceil(index(low)));
    if (a == b) b = a + 0.001;
  }
  for (int i = 0; i < rot_dim / 2; ++i) {
    double f = std::pow(base, -2.0 * i / d);
    if (scaling == VLA_ROPE_LINEAR) f /= factor;
    if (scaling == VLA_ROPE_BANDS) {
      const double w = std::min(1.0, std::max(0.0, (context * f / kTwoPi - low) / (high - low)));
      f *= w + (1 - w) / factor;
    }
    if (scaling == VLA_ROPE_RAMP) {
      const double w = std::min(1.0, std::max(0.0, (i - a) / (b - a)));
      f *= 1 - w + w / factor;
    }
    freqs_host[i] = f;
  }
  if (scale_host) *scale_host = scaling == VLA_ROPE_RAMP ? (float)(0.1 * std::log(factor) + 1.0) : 1.f;
  return set_error(VLA_OK, "");
}

int vla_qk_norm_rope(int32_t rows, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t dtype,
                     const void* q, int64_t ld_q, const void* k, int64_t ld_k, const void* v, int64_t ld_v,
                     const void* q_gain, const void* k_gain, float eps, const int32_t* row_pos, const double* freqs,
                     int32_t rot_dim, int32_t layout, float rope_scale, void* q_out, int64_t ld_qo, void* k_out,
                     int64_t ld_ko, void* k_pages, void* v_pages, int32_t n_pages, const int32_t* row_slot,
                     void* stream) {
  if (rows < 0 || n_pages < 0) return set_error(VLA_EINVAL, "negative size");
  if (n_pages >= 1 << 27) return set_error(VLA_EUNSUPPORTED, "n_pages must be below 2^27");
  int rc = check_heads(n_heads, n_kv_heads, head_dim, dtype);
  if (rc == VLA_OK && rows == 0) return set_error(VLA_OK, "");
  if (rc == VLA_OK) rc = check_rotation(rot_dim, head_dim, layout, eps, rope_scale, row_pos, freqs);
  if (rc != VLA_OK) return rc;
  const int64_t wq = (int64_t)n_heads * head_dim, wk = (int64_t)n_kv_heads * head_dim;
  const bool cache = k_pages != nullptr;
  if ((v != nullptr) != cache || (v_pages != nullptr) != cache || (row_slot != nullptr) != cache)
    return set_error(VLA_EINVAL, "v, k_pages, v_pages and row_slot go together");
  if (!cache && !k_out) return set_error(VLA_EINVAL, "k has nowhere to go: no k_out and no cache");
  if (!qk_rope_fits(rows, n_heads, n_kv_heads, head_dim, cache)) return set_error(VLA_EUNSUPPORTED, "too many rows for one call");
  if ((rc = check_rows("q", q, ld_q, wq)) || (rc = check_rows("k", k, ld_k, wk)) ||
      (rc = check_rows("q_out", q_out, ld_qo, wq)) || (k_out && (rc = check_rows("k_out", k_out, ld_ko, wk))) ||
      (cache && (rc = check_rows("v", v, ld_v, wk))))
    return rc;
  if ((q_out == q && ld_qo != ld_q) || (k_out == k && ld_ko != ld_k))
    return set_error(VLA_EINVAL, "an output in place of its input needs the same row stride");
  if (!aligned(q_gain) || !aligned(k_gain) || !aligned(k_pages) || !aligned(v_pages))
    return set_error(VLA_EINVAL, "gains and pages must start on 16 bytes");
  QkRopeArgs a{rows, n_heads, n_kv_heads, head_dim, static_cast<CacheType>(dtype), rows_of(q, ld_q), rows_of(k, ld_k),
               rows_of(v, ld_v), static_cast<const bf16_t*>(q_gain), static_cast<const bf16_t*>(k_gain), eps, row_pos,
               freqs, rot_dim, layout, rope_scale, rows_of(q_out, ld_qo), rows_of(k_out, ld_ko),
               {static_cast<bf16_t*>(k_pages), static_cast<bf16_t*>(v_pages)}, n_pages, row_slot};
  return hip_status("vla_qk_norm_rope", launch_qk_rope(a, static_cast<hipStream_t>(stream)));
}

int vla_qk_norm_rope_workspace_size(int32_t head_dim, size_t* bytes_host) {
  if (!bytes_host) return set_error(VLA_EINVAL, "NULL argument");
  const int rc = check_heads(1, 1, head_dim, VLA_DTYPE_BF16);
  if (rc != VLA_OK) return rc;
  *bytes_host = qk_rope_bwd_floats(head_dim) * sizeof(float);
  return set_error(VLA_OK, "");
}

int vla_qk_norm_rope_backward(int32_t rows, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t dtype,
                              const void* q, int64_t ld_q, const void* k, int64_t ld_k, const void* dq_out,
                              int64_t ld_dqo, const void* dk_out, int64_t ld_dko, const void* q_gain,
                              const void* k_gain, float eps, const int32_t* row_pos, const double* freqs,
                              int32_t rot_dim, int32_t layout, float rope_scale, void* dq, int64_t ld_dq, void* dk,
                              int64_t ld_dk, float* dq_gain, float* dk_gain, void* workspace, size_t workspace_bytes,
                              void* stream) {
  if (rows < 0) return set_error(VLA_EINVAL, "negative size");
  int rc = check_heads(n_heads, n_kv_heads, head_dim, dtype);
  if (rc != VLA_OK) return rc;
  if ((q_gain && !dq_gain) || (k_gain && !dk_gain)) return set_error(VLA_EINVAL, "a gain's gradient is NULL");
  if (!aligned(q_gain) || !aligned(k_gain)) return set_error(VLA_EINVAL, "gains must start on 16 bytes");
  if (q_gain || k_gain) {
    if (!workspace || !aligned(workspace) || workspace_bytes < qk_rope_bwd_floats(head_dim) * sizeof(float))
      return set_error(VLA_EWORKSPACE, "workspace smaller than vla_qk_norm_rope_workspace_size() or misaligned");
  } else if (rows == 0) {
    return set_error(VLA_OK, "");
  }
  if (rows > 0) {
    const int64_t wq = (int64_t)n_heads * head_dim, wk = (int64_t)n_kv_heads * head_dim;
    if ((rc = check_rotation(rot_dim, head_dim, layout, eps, rope_scale, row_pos, freqs)) ||
        (q_gain && (rc = check_rows("q", q, ld_q, wq))) || (k_gain && (rc = check_rows("k", k, ld_k, wk))) ||
        (rc = check_rows("dq_out", dq_out, ld_dqo, wq)) || (rc = check_rows("dk_out", dk_out, ld_dko, wk)) ||
        (rc = check_rows("dq", dq, ld_dq, wq)) || (rc = check_rows("dk", dk, ld_dk, wk)))
      return rc;
    if ((dq == dq_out && ld_dq != ld_dqo) || (dk == dk_out && ld_dk != ld_dko))
      return set_error(VLA_EINVAL, "an output in place of its input needs the same row stride");
  }
  QkRopeBwdArgs a{rows, n_heads, n_kv_heads, head_dim, static_cast<CacheType>(dtype), rows_of(q, ld_q),
                  rows_of(k, ld_k), rows_of(dq_out, ld_dqo), rows_of(dk_out, ld_dko),
                  static_cast<const bf16_t*>(q_gain), static_cast<const bf16_t*>(k_gain), eps, row_pos, freqs, rot_dim,
                  layout, rope_scale, rows_of(dq, ld_dq), rows_of(dk, ld_dk), dq_gain, dk_gain,
                  static_cast<float*>(workspace)};
  return hip_status("vla_qk_norm_rope_backward", launch_qk_rope_bwd(a, static_cast<hipStream_t>(stream)));
}

static int check_attention(int32_t n_env, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t max_pages) {
  if (n_env < 0 || max_pages < 0) return set_error(VLA_EINVAL, "negative size");
  const int rc = check_heads(n_heads, n_kv_heads, head_dim, VLA_DTYPE_BF16);
  if (rc != VLA_OK) return rc;
  if (n_heads % n_kv_heads != 0) return set_error(VLA_EINVAL, "n_heads must be a multiple of n_kv_heads");
  if (n_env > 65535 || max_pages >= 1 << 26)
    return set_error(VLA_EUNSUPPORTED, "at most 65535 environments and 2^26 - 1 pages of one");
  if ((int64_t)max_pages * n_heads >= (int64_t)1 << 31 || (int64_t)max_pages * n_env >= (int64_t)1 << 31 ||
      (double)n_env * max_pages * n_heads >= 0x1p40)
    return set_error(VLA_EUNSUPPORTED, "max_pages * n_heads and max_pages * n_env must be below 2^31, all three below 2^40");
  return VLA_OK;
}

int vla_paged_attention_workspace_size(int32_t n_env, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                                       int32_t max_pages, size_t* bytes_host) {
  if (!bytes_host) return set_error(VLA_EINVAL, "NULL argument");
  const int rc = check_attention(n_env, n_heads, n_kv_heads, head_dim, max_pages);
  if (rc != VLA_OK) return rc;
  *bytes_host = paged_attn_bytes(n_env, n_heads, n_kv_heads, head_dim, max_pages);
  return set_error(VLA_OK, "");
}

int vla_paged_attention(int32_t n_env, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t dtype,
                        const void* q, int64_t ld_q, const void* k_pages, const void* v_pages, int32_t n_pages,
                        const int32_t* page_table, int64_t ld_table, int32_t max_pages, const int32_t* lens,
                        float scale, void* out, int64_t ld_o, float* lse, void* workspace, size_t workspace_bytes,
                        void* stream) {
  int rc = check_attention(n_env, n_heads, n_kv_heads, head_dim, max_pages);
  if (rc == VLA_OK) rc = check_heads(n_heads, n_kv_heads, head_dim, dtype);
  if (rc != VLA_OK) return rc;
  if (n_pages < 0) return set_error(VLA_EINVAL, "negative size");
  if (n_pages >= 1 << 27) return set_error(VLA_EUNSUPPORTED, "n_pages must be below 2^27");
  if (!std::isfinite(scale * 1.44269504f)) return set_error(VLA_EINVAL, "scale must be finite, times log2(e) too");
  if (n_env == 0) return set_error(VLA_OK, "");
  const int64_t width = (int64_t)n_heads * head_dim;
  if ((rc = check_rows("q", q, ld_q, width)) || (rc = check_rows("out", out, ld_o, width))) return rc;
  if (ld_table < max_pages || ld_table > (int64_t)1 << 40) return set_error(VLA_EINVAL, "ld_table must hold a row of the page table");
  if (!lens || (max_pages > 0 && !page_table) || (n_pages > 0 && (!k_pages || !v_pages)))
    return set_error(VLA_EINVAL, "NULL argument");
  if (!aligned(k_pages) || !aligned(v_pages)) return set_error(VLA_EINVAL, "pages must start on 16 bytes");
  const size_t need = paged_attn_bytes(n_env, n_heads, n_kv_heads, head_dim, max_pages);
  if (need > 0 && (!workspace || !aligned(workspace, 256) || workspace_bytes < need))
    return set_error(VLA_EWORKSPACE, "workspace smaller than vla_paged_attention_workspace_size() or misaligned");
  PagedAttnArgs a{n_env, n_heads, n_kv_heads, head_dim, static_cast<CacheType>(dtype), static_cast<const bf16_t*>(q),
                  ld_q, {static_cast<bf16_t*>(const_cast<void*>(k_pages)), static_cast<bf16_t*>(const_cast<void*>(v_pages))},
                  n_pages, page_table, ld_table, max_pages, lens, scale, static_cast<bf16_t*>(out), ld_o, lse, workspace};
  return hip_status("vla_paged_attention", launch_paged_attn(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
