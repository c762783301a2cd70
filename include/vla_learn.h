/*
 * vla_learn.h — operators of a policy's learning pass over whole sequences: what carries the gradient of
 * the token log-probs (vla_lm.h, Eq. 2) on through a decoder layer beside its matrix products.  Same library and
 * conventions as vla_lm.h: device pointers, asynchronous on `cuda_stream`, host-checkable errors returned at once
 * (vla_last_error(NULL) has the message), errors found on the device OR-ed into the op status word
 * (vla_op_read_status).  No call allocates, waits for the GPU or keeps anything from one call to the next; all may be
 * captured into a CUDA graph.  Element types are vla_dtype.
 *
 * Sequences are packed: sequence s is the rows seq_start[s] .. seq_start[s + 1] - 1 of every tensor, seq_start int32
 * [n_seq + 1] on the device, not decreasing (a sequence may be empty); the row_start of vla_page_plan is one.  Rows
 * that belong to no sequence (before the first, behind the last: a batch of fixed size) give zeros.
 */
#ifndef VLA_LEARN_H_
#define VLA_LEARN_H_

#include "vla_lm.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Device status bit: sequence starts that decrease or lie outside the rows.  The call stays within its tensors;
 * its results are then undefined. */
#define VLA_STATUS_SEQUENCES 0x40u

/* Causal attention of packed sequences:
 *   out[i][h] = sum_j softmax_j(scale q[i][h] . k[j][g]) v[j][g] over the rows j <= i of i's sequence,
 *   g = h / (n_q_heads / n_kv_heads) (n_q_heads a multiple of n_kv_heads);
 *   q, out     [rows][n_q_heads][head_dim], row strides ldq, ldo;  k, v  [rows][n_kv_heads][head_dim], row strides ldk, ldv:
 *              of type `dtype` (VLA_F16 or VLA_BF16), 16-byte aligned, strides multiples of 8 elements (parts of one q|k|v
 *              buffer fit); head_dim 64 or 128;
 *   scale      1e-30 or more;
 *   lse        f32 [rows][n_q_heads] or NULL: log sum_j exp(scale q . k[j]); -infinity in rows of no sequence.
 * A key whose score is -infinity has no weight; a row with no other keys gives zeros and -infinity.
 * Scores, their maxima and sums are 32-bit; the weights of the values are rounded to `dtype`, relative to their maximum (so means of values
 * within 1 part in 512 of the type's largest number may come out infinite).  A row depends on nothing behind it and on no other sequence: NaN
 * and infinities there stay there.  In the rows that see one it shows, or not where its weight is 0 in 32 bits.  (Up to 127 rows before such a
 * value are computed again, one by one over all their keys: 0.15 s where it is the last of 16384.)  Equal calls give equal bits.  out
 * overlaps nothing that the call reads.  rows 0 or more; rows * n_q_heads at most 2^30. */
int vla_prompt_attn(const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv, int dtype, int rows,
                    int n_q_heads, int n_kv_heads, int head_dim, const int32_t* seq_start, int n_seq, float scale, void* out,
                    int64_t ldo, float* lse, void* cuda_stream);

/* Its gradient: d_q, d_k, d_v of sum(d_out * out), of type `dtype`, laid out and aligned like q, k, v (d_out like out; parts of one
 * d_q|d_k|d_v buffer fit).  out and lse are those of vla_prompt_attn; gradients of keys and values are summed over the query heads
 * that share them, in 32 bits.  With P the softmax weights, D[i] = d_out[i] . out[i]:
 *   d_v[j] = sum_i P[i][j] d_out[i],   dS[i][j] = P[i][j] (d_out[i] . v[j] - D[i]),
 *   d_q[i] = scale sum_j dS[i][j] k[j],   d_k[j] = scale sum_i dS[i][j] q[i].
 * P and dS are rounded to `dtype` in these sums, in fp16 dS relative to the largest that it can be in the row of d_q or d_k (what lies 2^38
 * below that may count as 0): rows, heads and sequences of very different sizes keep their own bits.  NaN and infinities stay in their sequence.
 * The gradients may overwrite nothing that the call reads.  Equal calls give equal bits (no atomics).  `workspace` of
 * vla_prompt_attn_grad_workspace_bytes, 16-byte aligned, any content; not shared by calls that may overlap. */
int vla_prompt_attn_grad(const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv, int dtype, int rows,
                         int n_q_heads, int n_kv_heads, int head_dim, const int32_t* seq_start, int n_seq, float scale,
                         const void* out, int64_t ldo, const float* lse, const void* d_out, int64_t lddo, void* d_q, int64_t lddq,
                         void* d_k, int64_t lddk, void* d_v, int64_t lddv, void* workspace, size_t workspace_bytes,
                         void* cuda_stream);
size_t vla_prompt_attn_grad_workspace_bytes(int rows, int n_q_heads, int n_kv_heads, int head_dim);

/* What lies between two blocks of a decoder, for each of `rows` rows of `dim` channels:
 *   u = y / sqrt(mean(y^2) + eps) * post_gain, or y where post_gain is NULL;
 *   h_out = h + residual_scale * gate * u;
 *   x = h_out / sqrt(mean(h_out^2) + eps) * pre_gain   (of h_out before it is rounded).
 *   y          the block's output, or NULL: x is then the norm of h alone (the first block's; post_gain, gate and h_out
 *              are NULL too);  gate  [rows][dim], row stride ldg, or [dim] for all rows (ldg 0), or NULL (1);
 *   h, h_out   the residual stream, of type h_dtype: VLA_F32 or `dtype`; h_out may be h (same stride);
 *   x          the next block's input;
 *   post_gain, pre_gain  bf16 [dim];  rstd  f32 [rows][2] or NULL: 1 / sqrt(..) of y (0 without post_gain) and of h_out, for
 *              the gradient.
 * y, gate and x are of type `dtype`.  Pointers are aligned to their elements, row strides at least dim; 32-bit arithmetic, one
 * rounding.  dim 1 to 16384; eps >= 0; rows 0 or more. */
int vla_block_norm(const void* y, int64_t ldy, int dtype, const void* h, int64_t ldh, int h_dtype, int rows, int dim,
                   const void* post_gain, const void* gate, int64_t ldg, float residual_scale, const void* pre_gain, float eps,
                   void* h_out, int64_t ldho, void* x, int64_t ldx, float* rstd, void* cuda_stream);

/* Its gradient, from d_x and d_h_out (type h_dtype, or NULL: zeros):
 *   d_h        [rows][dim], type h_dtype: d_h_out plus what comes through the norm behind it; may be d_h_out (same stride);
 *   d_y        [rows][dim], type `dtype` (NULL with y);
 *   d_gate     with a gate of each row: [rows][dim] of type `dtype`, row stride lddg; with one for all rows: f32 [dim]; NULL
 *              without a gate;
 *   d_post_gain (NULL without post_gain), d_pre_gain  f32 [dim];
 *   h_out, rstd  those of vla_block_norm (with y NULL: h).
 * Sums over rows are in 32 bits and in a fixed order.  `workspace` of vla_block_norm_grad_workspace_bytes, 16-byte aligned, any
 * content; not shared by calls that may overlap. */
int vla_block_norm_grad(const void* y, int64_t ldy, int dtype, const void* h_out, int64_t ldho, int h_dtype, int rows, int dim,
                        const void* post_gain, const void* gate, int64_t ldg, float residual_scale, const void* pre_gain,
                        const float* rstd, const void* d_x, int64_t lddx, const void* d_h_out, int64_t lddho, void* d_h,
                        int64_t lddh, void* d_y, int64_t lddy, void* d_gate, int64_t lddg, float* d_post_gain, float* d_pre_gain,
                        void* workspace, size_t workspace_bytes, void* cuda_stream);
size_t vla_block_norm_grad_workspace_bytes(int rows, int dim);

#ifdef __cplusplus
}
#endif
#endif /* VLA_LEARN_H_ */
