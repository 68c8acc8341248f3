// Launch interface of the paged cache's operators (vla_cache.h), as kernels.h for the rollout's kernels.
#pragma once

#include "kernels.h"

namespace vla {

// Types of q, k, v, pages and outputs (VLA_DTYPE_*).
enum CacheType { kBf16 = 0, kF16 = 1 };

// Pages, rows and slots of a step's new tokens (vla_kv_plan).
struct KvPlanArgs {
  int n_env;
  const int32_t* cached;      // [n_env]
  const int32_t* added;       // [n_env] new tokens
  int32_t* page_table;        // [n_env, max_pages], row stride ld_table
  int64_t ld_table;
  int max_pages;
  const int32_t* free_pages;  // [n_free]
  int n_free;
  const int32_t* free_head;   // [1], or null: 0
  int n_pages, max_rows;
  int32_t* lens;              // [n_env]
  int32_t* row_start;         // [n_env + 1]
  int32_t* row_pos;           // [max_rows]
  int32_t* row_env;
  int32_t* row_slot;
  int32_t* stats;             // [3]
};
hipError_t launch_kv_plan(const KvPlanArgs& a, hipStream_t s);

// Rows of head vectors: row r, head h at p + r * ld + h * head_dim.
struct HeadRows {
  bf16_t* p;
  int64_t ld;
};
struct QkRopeArgs {
  int rows, n_heads, n_kv_heads, head_dim;
  CacheType type;
  HeadRows q, k, v;            // inputs; v only with pages
  const bf16_t* q_gain;        // [head_dim], or null: no norm
  const bf16_t* k_gain;
  float eps;
  const int32_t* row_pos;      // [rows], or null with rot_dim == 0
  const double* freqs;         // [rot_dim / 2]
  int rot_dim, layout;         // layout: 0 half, 1 interleaved
  float rope_scale;
  HeadRows q_out, k_out;       // k_out.p may be null with pages
  KvCache pages;               // null: no cache
  int n_pages;
  const int32_t* row_slot;     // [rows] with pages
};
// Whether one launch takes that many rows: its threads have to stay below 2^32.
bool qk_rope_fits(int rows, int n_heads, int n_kv_heads, int head_dim, bool cache);
hipError_t launch_qk_rope(const QkRopeArgs& a, hipStream_t s);

struct QkRopeBwdArgs {
  int rows, n_heads, n_kv_heads, head_dim;
  CacheType type;
  HeadRows q, k;               // inputs of the forward
  HeadRows dq_out, dk_out;     // gradients of its outputs
  const bf16_t* q_gain;
  const bf16_t* k_gain;
  float eps;
  const int32_t* row_pos;
  const double* freqs;
  int rot_dim, layout;
  float rope_scale;
  HeadRows dq, dk;             // out
  float* dq_gain;              // [head_dim] out
  float* dk_gain;
  float* part;                 // qk_rope_bwd_floats(head_dim) floats
};
size_t qk_rope_bwd_floats(int head_dim);
hipError_t launch_qk_rope_bwd(const QkRopeBwdArgs& a, hipStream_t s);

// Attention of one token per environment over its cached tokens (vla_paged_attention).
struct PagedAttnArgs {
  int n_env, n_heads, n_kv_heads, head_dim;
  CacheType type;
  const bf16_t* q;             // [n_env, n_heads, head_dim], row stride ld_q
  int64_t ld_q;
  KvCache pages;
  int n_pages;
  const int32_t* page_table;   // [n_env, max_pages], row stride ld_table
  int64_t ld_table;
  int max_pages;
  const int32_t* lens;         // [n_env]
  float scale;
  bf16_t* o;                   // [n_env, n_heads, head_dim], row stride ld_o
  int64_t ld_o;
  float* lse;                  // [n_env, n_heads], or null
  void* ws;                    // paged_attn_bytes(...) bytes
};
size_t paged_attn_bytes(int n_env, int n_heads, int n_kv_heads, int head_dim, int max_pages);
hipError_t launch_paged_attn(const PagedAttnArgs& a, hipStream_t s);

}  // namespace vla
