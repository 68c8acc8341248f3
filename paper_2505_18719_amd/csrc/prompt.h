// Launch interface of attention over whole prompts and its gradient (vla_prompt.h).
#pragma once

#include "cache.h"

namespace vla {

// Causal attention of packed sequences.
struct PromptArgs {
  int rows, n_seq, n_heads, n_kv_heads, head_dim;
  CacheType type;
  HeadRows q, k, v;
  const int32_t* row_start;  // [n_seq + 1]
  float scale;
  HeadRows o;
  float* lse;                // [rows, n_heads], or null
};
// Whether the launch's workgroups can be counted.
bool prompt_fits(int rows, int n_seq, int n_heads);
hipError_t launch_prompt_attn(const PromptArgs& a, hipStream_t s);

struct PromptBwdArgs {
  PromptArgs fwd;            // o and lse as the forward left them
  HeadRows dout, dq, dk, dv;
  void* ws;                  // prompt_bwd_bytes(...) bytes
};
size_t prompt_bwd_bytes(int rows, int n_seq, int n_heads, int n_kv_heads, int head_dim);
hipError_t launch_prompt_attn_bwd(const PromptBwdArgs& a, hipStream_t s);

}  // namespace vla
