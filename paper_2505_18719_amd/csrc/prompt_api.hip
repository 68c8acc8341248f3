// C ABI of attention over whole prompts (vla_prompt.h): argument checks.
#include <hip/hip_runtime.h>

#include "cache_checks.h"
#include "prompt.h"
#include "vla_prompt.h"

using namespace vla;

namespace {

int check_prompt(int32_t rows, int32_t n_seq, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t dtype) {
  if (rows < 0 || n_seq < 0) return set_error(VLA_EINVAL, "negative size");
  const int rc = check_heads(n_heads, n_kv_heads, head_dim, dtype);
  if (rc != VLA_OK) return rc;
  if (n_heads % n_kv_heads != 0) return set_error(VLA_EINVAL, "n_heads must be a multiple of n_kv_heads");
  if (!prompt_fits(rows, n_seq, n_heads)) return set_error(VLA_EUNSUPPORTED, "too many rows and sequences for one call");
  return VLA_OK;
}

// A tensor of rows whose tiles of 64 are addressed by 32-bit offsets.
int check_tile_rows(const char* name, const void* p, int64_t ld, int64_t width) {
  const int rc = check_rows(name, p, ld, width);
  if (rc == VLA_OK && ld > 1 << 23) return set_error(VLA_EUNSUPPORTED, "row strides must be at most 2^23");
  return rc;
}

// Whether [p, p + bytes of rows) and another tensor's bytes meet, by the spans of their addresses; views of one buffer whose rows lie
// between each other's do not if neither's row reaches into the other's.
bool overlap(const HeadRows& x, int64_t wx, const HeadRows& y, int64_t wy, int64_t rows) {
  const uintptr_t x0 = reinterpret_cast<uintptr_t>(x.p), y0 = reinterpret_cast<uintptr_t>(y.p);
  const uintptr_t x1 = x0 + 2 * ((rows - 1) * x.ld + wx), y1 = y0 + 2 * ((rows - 1) * y.ld + wy);
  if (x1 <= y0 || y1 <= x0) return false;
  if (x.ld != y.ld) return true;
  const int64_t ld = 2 * x.ld, d = ((int64_t)(y0 - x0) % ld + ld) % ld;  // y's rows begin d bytes behind x's
  return d < 2 * wx || d + 2 * wy > ld;
}

}  // namespace

extern "C" {

int vla_prompt_attention(int32_t rows, int32_t n_seq, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                         int32_t dtype, const void* q, int64_t ld_q, const void* k, int64_t ld_k, const void* v,
                         int64_t ld_v, const int32_t* row_start, float scale, void* out, int64_t ld_o, float* lse,
                         void* stream) {
  int rc = check_prompt(rows, n_seq, n_heads, n_kv_heads, head_dim, dtype);
  if (rc == VLA_OK) rc = check_scale(scale);
  if (rc != VLA_OK) return rc;
  if (rows == 0 || n_seq == 0) return set_error(VLA_OK, "");
  const int64_t wq = (int64_t)n_heads * head_dim, wk = (int64_t)n_kv_heads * head_dim;
  if ((rc = check_tile_rows("q", q, ld_q, wq)) || (rc = check_tile_rows("k", k, ld_k, wk)) ||
      (rc = check_tile_rows("v", v, ld_v, wk)) || (rc = check_tile_rows("out", out, ld_o, wq)))
    return rc;
  if (!row_start) return set_error(VLA_EINVAL, "row_start is NULL");
  PromptArgs a{rows, n_seq, n_heads, n_kv_heads, head_dim, static_cast<CacheType>(dtype), rows_of(q, ld_q),
               rows_of(k, ld_k), rows_of(v, ld_v), row_start, scale, rows_of(out, ld_o), lse};
  if (overlap(a.o, wq, a.q, wq, rows) || overlap(a.o, wq, a.k, wk, rows) || overlap(a.o, wq, a.v, wk, rows))
    return set_error(VLA_EINVAL, "out may not overlap an input");
  return hip_status("vla_prompt_attention", launch_prompt_attn(a, static_cast<hipStream_t>(stream)));
}

int vla_prompt_attention_backward_workspace_size(int32_t rows, int32_t n_seq, int32_t n_heads, int32_t n_kv_heads,
                                                 int32_t head_dim, size_t* bytes_host) {
  if (!bytes_host) return set_error(VLA_EINVAL, "NULL argument");
  const int rc = check_prompt(rows, n_seq, n_heads, n_kv_heads, head_dim, VLA_DTYPE_BF16);
  if (rc != VLA_OK) return rc;
  *bytes_host = prompt_bwd_bytes(rows, n_seq, n_heads, n_kv_heads, head_dim);
  return set_error(VLA_OK, "");
}

int vla_prompt_attention_backward(int32_t rows, int32_t n_seq, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                                  int32_t dtype, const void* q, int64_t ld_q, const void* k, int64_t ld_k,
                                  const void* v, int64_t ld_v, const void* out, int64_t ld_o, const float* lse,
                                  const void* dout, int64_t ld_do, const int32_t* row_start, float scale, void* dq,
                                  int64_t ld_dq, void* dk, int64_t ld_dk, void* dv, int64_t ld_dv, void* workspace,
                                  size_t workspace_bytes, void* stream) {
  int rc = check_prompt(rows, n_seq, n_heads, n_kv_heads, head_dim, dtype);
  if (rc == VLA_OK) rc = check_scale(scale);
  if (rc != VLA_OK) return rc;
  if (rows == 0 || n_seq == 0) return set_error(VLA_OK, "");
  const int64_t wq = (int64_t)n_heads * head_dim, wk = (int64_t)n_kv_heads * head_dim;
  if ((rc = check_tile_rows("q", q, ld_q, wq)) || (rc = check_tile_rows("k", k, ld_k, wk)) ||
      (rc = check_tile_rows("v", v, ld_v, wk)) || (rc = check_tile_rows("out", out, ld_o, wq)) ||
      (rc = check_tile_rows("dout", dout, ld_do, wq)) || (rc = check_tile_rows("dq", dq, ld_dq, wq)) ||
      (rc = check_tile_rows("dk", dk, ld_dk, wk)) || (rc = check_tile_rows("dv", dv, ld_dv, wk)))
    return rc;
  if (!row_start || !lse) return set_error(VLA_EINVAL, "NULL argument");
  PromptBwdArgs b{{rows, n_seq, n_heads, n_kv_heads, head_dim, static_cast<CacheType>(dtype), rows_of(q, ld_q),
                   rows_of(k, ld_k), rows_of(v, ld_v), row_start, scale, rows_of(out, ld_o), const_cast<float*>(lse)},
                  rows_of(dout, ld_do), rows_of(dq, ld_dq), rows_of(dk, ld_dk), rows_of(dv, ld_dv), workspace};
  const HeadRows in[] = {b.fwd.q, b.fwd.o, b.dout, b.fwd.k, b.fwd.v}, to[] = {b.dq, b.dk, b.dv};
  for (int i = 0; i < 3; ++i) {
    const int64_t w = i == 0 ? wq : wk;
    for (int j = 0; j < 5; ++j)
      if (overlap(to[i], w, in[j], j < 3 ? wq : wk, rows)) return set_error(VLA_EINVAL, "a gradient may not overlap an input");
    for (int j = 0; j < i; ++j)
      if (overlap(to[i], w, to[j], j == 0 ? wq : wk, rows)) return set_error(VLA_EINVAL, "gradients may not overlap");
  }
  if (!workspace || !aligned(workspace, 256) || workspace_bytes < prompt_bwd_bytes(rows, n_seq, n_heads, n_kv_heads, head_dim))
    return set_error(VLA_EWORKSPACE, "workspace smaller than vla_prompt_attention_backward_workspace_size() or misaligned");
  return hip_status("vla_prompt_attention_backward", launch_prompt_attn_bwd(b, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
