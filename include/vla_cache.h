/*
 * vla_cache.h -- C ABI of the operators of a paged KV cache that grows on the
 * device: a policy step whose lengths, page tables and cache slots never
 * visit the host.  One step of a decoder layer is
 *     vla_kv_plan            once per step: pages and slots of the new tokens
 *     vla_qk_norm_rope       per layer: head norms and rotation of q and k,
 *                            k and v appended to the cache
 *     vla_paged_attention    per layer: every environment's new token over
 *                            all of its cached tokens
 * and vla_qk_norm_rope_backward is the gradient of the norms and rotation.
 * None of them needs a model handle.  Where vla_prefill and
 * vla_decode_actions run a fixed decoder over at most 320 tokens, these take
 * grouped key heads, normed heads, partial, interleaved and scaled rotations,
 * and histories of any length.
 *
 * Conventions are those of vla.h: device pointers unless a name ends in
 * `_host`, `hipStream_t` passed as `void*`, asynchronous on that stream of the
 * current device, no device allocation, status codes VLA_* with
 * vla_last_error().  All launches are ordinary kernels, so every call can be
 * captured into a graph.  Calls keep no state: calls on different streams may
 * overlap if they share no buffer that either writes (workspaces included).
 *
 * The cache of one layer is a pool of n_pages pages of 16 tokens, the layout
 * of the handle's own cache:
 *     k_pages  [n_pages, n_kv_heads, 16, head_dim]   a token's key contiguous
 *     v_pages  [n_pages, n_kv_heads, head_dim, 16]   a feature's 16 tokens contiguous
 * Token p of environment e lies in page page_table[e, p / 16], slot p % 16; its
 * number `slot` is 16 * page + p % 16.  n_pages < 2^27.
 *
 * `dtype` is the type of q, k, v, gains, pages and outputs.  Sums, softmax
 * statistics and rotation angles are held in 32 bits or more, and each output
 * is rounded once, to nearest even; softmax weights meet the values as pairs of
 * numbers of `dtype` (16 bits in bf16, 22 in fp16).  Tensors of `dtype` and fp64
 * start on 16 bytes, others on 4; a row holds its heads contiguously, and row
 * strides (`ld_*`, in elements) are multiples of 8 that hold a row, so q, k and
 * v may be parts of one projection's output.
 * At most 1024 heads and 1024 key heads.
 */
#ifndef VLA_CACHE_H_
#define VLA_CACHE_H_

#include "vla.h"

#ifdef __cplusplus
extern "C" {
#endif

#define VLA_DTYPE_BF16 0
#define VLA_DTYPE_F16 1

/* Pages, rows and slots of a step's new tokens.  Environment e holds c =
 * cached_lens[e] tokens and gets w = new_lens[e] more, whose rows follow those
 * of environment e - 1 in the packed batch.  It needs ceil((c + w) / 16) -
 * ceil(c / 16) new pages and takes the next ones of free_pages, in the order
 * of the environments, from index *free_head on.  An environment is refused
 * if c or w is negative, c + w > 16 * max_pages, its rows end past max_rows,
 * or it needs pages and free_pages does not hold them (nor then those of a
 * later environment); it gets no pages, and keeps its length.
 *   cached_lens, new_lens  int32 [n_env]
 *   page_table   int32 [n_env, max_pages] (row stride ld_table): the entries
 *                of new pages are written, all others are left as they are
 *   free_pages   int32 [n_free]
 *   free_head    int32 [1], or NULL for 0; outside [0, n_free] no page is left
 *   n_pages      pages of the pool: a row whose page lies outside has no slot
 *   lens         int32 [n_env] out: c + w; of a refused environment max(c, 0)
 *   row_start    int32 [n_env + 1] out: first packed row of each environment
 *                and the number of rows, none above max_rows
 *   row_pos, row_env, row_slot  int32 [max_rows] out: position, environment
 *                and slot of each row; slot -1 where the environment was
 *                refused; rows past the last one 0, -1 and -1
 *   stats        int32 [3] out: free_head after the step, rows of the step
 *                (as row_start's last), environments refused
 * Outputs may not overlap inputs (lens and cached_lens, stats and free_head
 * are checked). */
int vla_kv_plan(int32_t n_env, const int32_t* cached_lens, const int32_t* new_lens, int32_t* page_table,
                int64_t ld_table, int32_t max_pages, const int32_t* free_pages, int32_t n_free,
                const int32_t* free_head, int32_t n_pages, int32_t max_rows, int32_t* lens, int32_t* row_start,
                int32_t* row_pos, int32_t* row_env, int32_t* row_slot, int32_t* stats, void* stream);

/* Rotation frequencies, on the host.  freqs_host receives the rot_dim / 2
 * radians per position of a rotation over rot_dim features,
 *     f_i = base^(-2 i / rot_dim),
 * changed for contexts `factor` (>= 1) times as long as those trained on, and
 * *scale_host the factor on cos and sin that belongs to it (1 but for RAMP):
 *   VLA_ROPE_NONE    f_i as it is (factor, low, high and context unused)
 *   VLA_ROPE_LINEAR  f_i / factor: positions interpolated
 *   VLA_ROPE_BASE    base times factor^(rot_dim / (rot_dim - 2)), which
 *                    divides the lowest frequency by factor and leaves the
 *                    highest (rot_dim >= 4, the new base finite)
 *   VLA_ROPE_BANDS   by turns over the trained context, n_i = context f_i /
 *                    (2 pi): f_i from `high` turns on, f_i / factor up to
 *                    `low`, between them f_i (w + (1 - w) / factor) with w =
 *                    (n_i - low) / (high - low)
 *   VLA_ROPE_RAMP    by index: with i(n) = rot_dim / 2 log(context / (2 pi n))
 *                    / log(base) the index of n turns, a = max(0, floor
 *                    i(high)), b = min(rot_dim - 1, ceil i(low)), b = a + 0.001
 *                    where they are equal, and w = clamp((i - a) / (b - a), 0,
 *                    1): f_i (1 - w + w / factor); scale 0.1 ln(factor) + 1
 * rot_dim even, 2 .. 256; base > 1; for BANDS and RAMP 0 < low < high and
 * context > 0.  scale_host may be NULL. */
#define VLA_ROPE_NONE 0
#define VLA_ROPE_LINEAR 1
#define VLA_ROPE_BASE 2
#define VLA_ROPE_BANDS 3
#define VLA_ROPE_RAMP 4
int vla_rope_freqs(int32_t rot_dim, double base, int32_t scaling, double factor, double low, double high,
                   double context, double* freqs_host, float* scale_host);

/* Norms of q and k per head and their rotation, in one pass, with the append
 * to the cache.  For each row at position p = row_pos[row] and each head,
 *     y = x gain / sqrt(mean(x^2) + eps)      (y = x where the gain is NULL;
 * the sum of the squares is fp32's: past 3.4e38 the head becomes zeros)
 * then, with (a, b) the pair i of y's first rot_dim features, t = p freqs[i]
 * (taken in 64 bits) and s = rope_scale,
 *     (a, b) -> (s (a cos t - b sin t), s (b cos t + a sin t));
 * the other features stay.  layout VLA_ROPE_HALF pairs features i and i +
 * rot_dim / 2, VLA_ROPE_INTERLEAVED 2 i and 2 i + 1.
 *   head_dim     64, 128 or 256; rot_dim a multiple of 16, 0 .. head_dim
 *   q, k         [rows, n_heads, head_dim], [rows, n_kv_heads, head_dim]
 *   q_gain, k_gain  [head_dim], or NULL
 *   freqs        fp64 [rot_dim / 2] (vla_rope_freqs), or NULL if rot_dim is 0
 *   row_pos      int32 [rows], or NULL if rot_dim is 0
 *   q_out        [rows, n_heads, head_dim] out; may be q, with the same stride
 *   k_out        [rows, n_kv_heads, head_dim] out, or NULL if there is a
 *                cache; may be k, with the same stride
 * With a cache (v, k_pages, v_pages and row_slot all given, else all NULL) the
 * new key and v [rows, n_kv_heads, head_dim] go to slot row_slot[row]; a row
 * whose slot lies outside [0, 16 n_pages) is passed over: neither the cache
 * nor its rows of q_out and k_out are written.  Slots are distinct.
 * rows == 0 is a no-op.  At most 2^26 - 4 rows; with a cache ceil(rows / 4) +
 * ceil(rows / 16) ceil(n_kv_heads head_dim / 256) must be below 2^24. */
#define VLA_ROPE_HALF 0
#define VLA_ROPE_INTERLEAVED 1
int vla_qk_norm_rope(int32_t rows, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t dtype,
                     const void* q, int64_t ld_q, const void* k, int64_t ld_k, const void* v, int64_t ld_v,
                     const void* q_gain, const void* k_gain, float eps, const int32_t* row_pos, const double* freqs,
                     int32_t rot_dim, int32_t layout, float rope_scale, void* q_out, int64_t ld_qo, void* k_out,
                     int64_t ld_ko, void* k_pages, void* v_pages, int32_t n_pages, const int32_t* row_slot,
                     void* stream);

/* Gradient of vla_qk_norm_rope from q and k as they went in and the gradients
 * dq_out, dk_out of its outputs: with dy the gradient turned back by the
 * transposed rotation, r = 1 / sqrt(mean(x^2) + eps) and h = x r,
 *     dx = r (g dy - h mean(h g dy)),   dgain = sum over rows and heads of h dy
 * (dx = dy without a gain).
 *   q, k             read only where their gain is given, else may be NULL
 *   dq_out, dk_out, dq, dk  as q and k; dq may be dq_out (dk dk_out), with
 *                    the same stride
 *   dq_gain, dk_gain fp32 [head_dim] out, not NULL where the gain is given
 *   workspace        vla_qk_norm_rope_workspace_size bytes, 16-byte aligned
 *                    (may be NULL if no gain is given)
 * The gains' sums have a fixed order: the same bits every run.  rows == 0
 * leaves dq and dk alone and writes zeros to the gains' gradients. */
int vla_qk_norm_rope_workspace_size(int32_t head_dim, size_t* bytes_host);
int vla_qk_norm_rope_backward(int32_t rows, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t dtype,
                              const void* q, int64_t ld_q, const void* k, int64_t ld_k, const void* dq_out,
                              int64_t ld_dqo, const void* dk_out, int64_t ld_dko, const void* q_gain,
                              const void* k_gain, float eps, const int32_t* row_pos, const double* freqs,
                              int32_t rot_dim, int32_t layout, float rope_scale, void* dq, int64_t ld_dq, void* dk,
                              int64_t ld_dk, float* dq_gain, float* dk_gain, void* workspace, size_t workspace_bytes,
                              void* stream);

/* Attention of one token per environment over its cached tokens 0 .. lens[e] -
 * 1 (the new token's own key among them): for head h, reading key head h
 * n_kv_heads / n_heads (rounded down),
 *     out[e, h] = sum_j p_j v_j,  p = softmax_j(scale q[e, h] . k_j).
 * An environment of length 0 gets zeros, as does a head all of whose scores
 * are -inf, whatever its values; a NaN or +inf among them gives NaN.  An
 * infinite value makes its feature's sum infinite however small its weight,
 * and NaN beside one of the other sign or at a score of -inf.  What the last
 * page holds past the length does not matter, nor do the table's entries past
 * the last page.  A length below 0 or above 16 * max_pages, or a page outside [0, n_pages)
 * among those of the length, gives an environment of NaN (nothing outside the
 * pool is read).
 *   q, out       [n_env, n_heads, head_dim] (row strides ld_q, ld_o); head_dim
 *                64, 128 or 256; n_heads a multiple of n_kv_heads
 *   page_table   int32 [n_env, max_pages] (row stride ld_table); environments
 *                may share pages.  The work is laid out for lengths up to 16 *
 *                max_pages: columns that no length needs cost some time (where
 *                lengths are not known beforehand, as in a graph, they are the
 *                price) and change no result by more than its rounding
 *   lens         int32 [n_env] (vla_kv_plan's)
 *   scale        finite, at most 2.3e38 in size (softmax is taken to base 2)
 *   lse          fp32 [n_env, n_heads] out, or NULL: log sum_j exp(scale q . k_j)
 *                (-inf where the output is zeros for want of a key)
 *   workspace    vla_paged_attention_workspace_size bytes, 256-byte aligned
 * n_env == 0 is a no-op.  The same bits every run on the same device. */
int vla_paged_attention_workspace_size(int32_t n_env, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                                       int32_t max_pages, size_t* bytes_host);
int vla_paged_attention(int32_t n_env, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t dtype,
                        const void* q, int64_t ld_q, const void* k_pages, const void* v_pages, int32_t n_pages,
                        const int32_t* page_table, int64_t ld_table, int32_t max_pages, const int32_t* lens,
                        float scale, void* out, int64_t ld_o, float* lse, void* workspace, size_t workspace_bytes,
                        void* stream);

#ifdef __cplusplus
}
#endif
#endif /* VLA_CACHE_H_ */
