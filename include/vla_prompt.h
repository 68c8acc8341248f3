/*
 * vla_prompt.h -- C ABI of causal attention over whole prompts and its
 * gradient: packed sequences of any lengths, grouped key heads.  It takes
 * vla_qk_norm_rope's q and k as they come out (and v beside them) with
 * vla_kv_plan's row_start, and its gradients go on to
 * vla_qk_norm_rope_backward.
 *
 * Conventions are those of vla.h and vla_cache.h: device pointers,
 * `hipStream_t` passed as `void*`, asynchronous on that stream of the current
 * device, no device allocation, status codes VLA_* with vla_last_error();
 * `dtype` VLA_DTYPE_*, rows of heads with strides `ld_*` in elements that are
 * multiples of 8, here at most 2^23; tensors of `dtype` start on 16 bytes,
 * others on 4.  All launches are ordinary kernels: every call can be captured
 * into a graph, and calls on different streams may overlap if they share no
 * buffer that either writes.
 *
 * Scores, softmax statistics and sums are fp32.  Where they meet the other
 * factor of a product, softmax weights are rounded once to `dtype`, as are the
 * scores' gradients for dk; for dq they enter as pairs of numbers of `dtype`.
 * Each output is rounded once, to nearest even.  The same bits every run.
 *
 * Sequence s holds rows row_start[s] .. row_start[s + 1] - 1 of q, k and v.
 * Its row i attends rows 0 .. i of it:
 *     out_i = sum_j p_ij v_j,  p_ij = softmax_{j <= i}(scale q_i . k_j)
 * with head h reading key head h n_kv_heads / n_heads (rounded down).  Rows of
 * no sequence are neither read nor written: those before the first and behind
 * the last, and those of a sequence whose bounds descend or lie outside
 * [0, rows].  Of up to 512 sequences such bounds change nothing for the
 * others; more have to ascend within [0, rows].  What the rows of sequences
 * get where these do not, or where sequences share rows, is left open.
 * Infinite and NaN elements reach what the formulas say they reach and nothing
 * else: no earlier row's outputs and no later key's gradients; whether they
 * arrive as an infinity or as NaN is left open.  A row's head all of whose
 * scores are -inf gets zeros in out and dq and has no part in dk and dv,
 * whatever its elements of q and dout are.
 */
#ifndef VLA_PROMPT_H_
#define VLA_PROMPT_H_

#include "vla_cache.h"

#ifdef __cplusplus
extern "C" {
#endif

/*   rows         rows of the tensors; n_seq sequences lie among them
 *   q, out       [rows, n_heads, head_dim]; head_dim 64, 128 or 256; n_heads
 *                a multiple of n_kv_heads; out may not overlap an input
 *   k, v         [rows, n_kv_heads, head_dim]
 *   row_start    int32 [n_seq + 1]
 *   scale        finite, at most 2.3e38 in size (softmax is taken to base 2)
 *   lse          fp32 [rows, n_heads] out, or NULL: log sum_j exp(scale q_i . k_j)
 * rows == 0 or n_seq == 0 is a no-op. */
int vla_prompt_attention(int32_t rows, int32_t n_seq, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                         int32_t dtype, const void* q, int64_t ld_q, const void* k, int64_t ld_k, const void* v,
                         int64_t ld_v, const int32_t* row_start, float scale, void* out, int64_t ld_o, float* lse,
                         void* stream);

/* The gradient of vla_prompt_attention with respect to q, k and v, from its
 * inputs, its outputs out and lse, and the gradient dout of out: with D_i =
 * out_i . dout_i and dS_ij = p_ij (dout_i . v_j - D_i),
 *     dq_i = scale sum_j dS_ij k_j,  dk_j = scale sum_i dS_ij q_i,
 *     dv_j = sum_i p_ij dout_i,
 * the last two summed over the query heads that read the key head, too.
 *   dq, dk, dv   as q, k and v; none may overlap an input or another
 *   workspace    vla_prompt_attention_backward_workspace_size bytes, 256-byte
 *                aligned
 * rows == 0 or n_seq == 0 is a no-op. */
int vla_prompt_attention_backward_workspace_size(int32_t rows, int32_t n_seq, int32_t n_heads, int32_t n_kv_heads,
                                                 int32_t head_dim, size_t* bytes_host);
int vla_prompt_attention_backward(int32_t rows, int32_t n_seq, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                                  int32_t dtype, const void* q, int64_t ld_q, const void* k, int64_t ld_k,
                                  const void* v, int64_t ld_v, const void* out, int64_t ld_o, const float* lse,
                                  const void* dout, int64_t ld_do, const int32_t* row_start, float scale, void* dq,
                                  int64_t ld_dq, void* dk, int64_t ld_dk, void* dv, int64_t ld_dv, void* workspace,
                                  size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* VLA_PROMPT_H_ */
