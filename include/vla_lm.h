/*
 * vla_lm.h — operators of a token policy over a paged key-value cache, and its token log-probs with
 * their gradient.  Same library and conventions as vla_ops.h: device pointers, asynchronous on
 * `cuda_stream`, host-checkable errors returned at once (vla_last_error(NULL) has the message), errors
 * found on the device OR-ed into the op status word (vla_op_read_status).  No call allocates, waits
 * for the GPU or keeps anything from one call to the next; all may be captured into a CUDA graph.
 *
 * A paged cache is one pool of pages of `page_size` positions each; an environment's positions
 * p = 0, 1, .. live in the pages table[env][p / page_size], slot p % page_size.  One step of a rollout over
 * it: vla_page_plan takes pages for the step's new tokens and maps each row to (env, position, slot);
 * then per layer vla_rope_append normalises and rotates queries and keys and files keys and values, and
 * vla_paged_attn lets every row attend to its environment's positions; vla_token_logprobs reads the
 * log-prob of each chosen token off the logits (Eq. 1), and vla_token_logprobs_grad carries the gradient of
 * the learning phase (Eq. 2) back to them.
 *
 * Rows of a fixed-size step (a captured graph) that hold no token carry env = pos = slot = -1: nothing
 * is cached for them and their outputs are zeros.
 */
#ifndef VLA_LM_H_
#define VLA_LM_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Element types. */
typedef enum { VLA_F32 = 0, VLA_F16 = 1, VLA_BF16 = 2 } vla_dtype;

/* Device status bit: a page plan that does not fit (too few free pages, table columns or rows, or a
 * negative length), or a row whose page, slot, position or environment is outside its range. */
#define VLA_STATUS_PAGES 0x20u

/* One layer of a paged cache.  Channel c of (page, head, slot) is at element
 * page * page_stride + head * head_stride + slot * slot_stride + c of k and of v, so both orders
 * [page][head][slot][c] and [page][slot][head][c] fit, and so do k and v interleaved in one buffer.
 * dtype VLA_F16 or VLA_BF16; head_dim 64 or 128; k, v 16-byte aligned, strides multiples of 8;
 * n_pages * page_size < 2^31 (element offsets are 64-bit). */
typedef struct {
  void* k;
  void* v;
  int dtype;
  int n_pages, page_size, n_heads, head_dim;
  int64_t page_stride, head_stride, slot_stride;
} vla_paged_kv;

/* Takes pages for `new_len` more tokens of each environment and maps the step's rows.
 *   ctx_in     int32 [n_env]: positions that each environment has cached;
 *   new_len    int32 [n_env]: tokens to append, 0 or more;
 *   release    int32 [n_env] or NULL: nonzero = the environment starts over: its pages go back to the
 *              pool first (in order of environment and column) and its context counts as empty;
 *   table      int32 [n_env][max_pages], updated: columns ceil(ctx / page_size) .. ceil((ctx + new) /
 *              page_size) - 1 of each row are filled, the others are left alone;
 *   pool       int32 [n_pages]: a stack of free pages, entries 0 .. n_free - 1, taken from its end
 *              (environments in order, each its columns in order); entries are written only by releases;
 *   ctx_out    int32 [n_env]: ctx + new (may be ctx_in);  n_free_out  int32 [1] (may be n_free_in);
 *   row_start  int32 [n_env + 1]: rows of environment e are row_start[e] .. row_start[e + 1] - 1;
 *   row_env / row_pos / row_slot  int32 [max_rows]: each row's environment, position and cache slot
 *              (page * page_size + position % page_size); -1 for the rows past the last.
 * Where the plan does not fit, VLA_STATUS_PAGES is set, nothing is taken or released, and all rows are -1.
 * A row whose page (from the table or the pool) is no page of the pool sets it too and gets slot -1.
 * row_env, row_pos and row_slot may be NULL when max_rows is 0.  n_env <= 4096 (else VLA_ERR_UNSUPPORTED). */
int vla_page_plan(const int32_t* ctx_in, const int32_t* new_len, const int32_t* release, int n_env, int page_size, int32_t* table,
                  int max_pages, int32_t* pool, int n_pages, const int32_t* n_free_in, int32_t* ctx_out, int32_t* n_free_out,
                  int32_t* row_start, int32_t* row_env, int32_t* row_pos, int32_t* row_slot, int max_rows, void* cuda_stream);

/* How rotary frequencies f_i = theta^(-2i / dim) are scaled for contexts longer than trained.  With
 * t_i = original_len * f_i / (2 pi), the turns that pair i makes over the trained length:
 *   VLA_ROPE_PLAIN    f_i;
 *   VLA_ROPE_LINEAR   f_i / factor;
 *   VLA_ROPE_TURNS    f_i (s + (1 - s) / factor), s = clamp((t_i - low) / (high - low), 0, 1): pairs of fewer
 *                     than `low` turns are stretched, those of more than `high` are left alone;
 *   VLA_ROPE_LOG_TURNS  the same with s = clamp((log t_i - log low) / (log high - log low), 0, 1).
 * `amplitude` multiplies every cosine and sine (1 = a rotation). */
typedef enum { VLA_ROPE_PLAIN = 0, VLA_ROPE_LINEAR = 1, VLA_ROPE_TURNS = 2, VLA_ROPE_LOG_TURNS = 3 } vla_rope_kind;

/* table f32 [n_pos][rope_dim / 2][2]: (cos, sin) of position x frequency, computed in 64 bits (a 32-bit
 * angle is off by 4e-3 at position 131072).  rope_dim even; theta > 0; factor >= 1, original_len > 0 and
 * 0 < low < high where the kind uses them; amplitude > 0. */
int vla_rope_table(float* table, int n_pos, int rope_dim, double theta, int kind, double factor, double original_len, double low,
                   double high, double amplitude, void* cuda_stream);

/* Queries and keys of `rows` rows, normalised per head and rotated, and keys and values filed:
 *   q [rows][n_q_heads][hd], k and v [rows][kv->n_heads][hd] of type `dtype` (row strides ldq, ldk, ldv in
 *              elements, multiples of 8; 16-byte aligned: parts of one q|k|v buffer fit);
 *   q_gain, k_gain  bf16 [hd] or NULL: x becomes x / sqrt(mean(x^2) + eps) * gain over each head;
 *   rope       f32 [n_pos][rope_dim / 2][2] (vla_rope_table) or NULL: rotates the first rope_dim channels of
 *              each head at the row's position; pairs are (i, i + rope_dim / 2), or (2i, 2i + 1) when
 *              `interleaved`; rope_dim a multiple of 16, at most hd;
 *   row_pos, row_slot  int32 [rows]: position and cache slot of each row (vla_page_plan);
 *   q_out      [rows][n_q_heads][hd] of type `dtype`, row stride ldqo; may be q itself (same stride).
 * A row of position -1 gets zero queries and caches nothing; a slot of -1 caches nothing.  Arithmetic in
 * 32 bits, rounded once.  Keys and values beyond the fp16 range go to an fp16 cache as +-65504 and raise
 * VLA_STATUS_SATURATED.  rows 0 or more.  hd = kv->head_dim. */
int vla_rope_append(const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv, int dtype, int rows,
                    int n_q_heads, const vla_paged_kv* kv, const void* q_gain, const void* k_gain, float eps, const float* rope,
                    int n_pos, int rope_dim, int interleaved, const int32_t* row_pos, const int32_t* row_slot, void* q_out,
                    int64_t ldqo, void* cuda_stream);

/* Attention of one new token per row over its environment's cached positions:
 *   out[r][h] = sum_p softmax_p(scale q[r][h] . K[p][g]) V[p][g], p = 0 .. row_pos[r], g = h / (n_q_heads /
 *   kv->n_heads) (n_q_heads a multiple of kv->n_heads);
 *   q, out     [rows][n_q_heads][hd] of type `dtype`, row strides ldq, ldo (multiples of 8 elements), 16-byte
 *              aligned; dtype is the cache's, or VLA_F32 over an fp16 cache (VLA_ERR_UNSUPPORTED otherwise);
 *   table      int32 [n_env][max_pages];  row_env, row_pos  int32 [rows];
 *   lse        f32 [rows][n_q_heads] or NULL: log sum_p exp(scale q . K[p]);
 *   workspace  vla_paged_attn_workspace_bytes(hd) bytes, 16-byte aligned, zeroed once before its first use;
 *              every call leaves it fit for the next, of any size.  Not shared by calls that may overlap.
 * f32 queries may be of any size: a head counts relative to its largest channel.
 * A row of position -1 gives zeros (lse -infinity).  Positions past row_pos[r] may hold anything (NaN
 * included): they are not read; a NaN or infinity at one that is read may give NaN.  Products and softmax weights
 * keep at least 16 significant bits (22 over an fp16 cache), sums are 32-bit; the split of long contexts and the
 * order of its sums depend on the lengths alone, so equal calls give equal bits.  rows 0 or more, rows * n_q_heads at most 2^30. */
int vla_paged_attn(const void* q, int64_t ldq, int dtype, int rows, int n_q_heads, const vla_paged_kv* kv, const int32_t* table,
                   int max_pages, int n_env, const int32_t* row_env, const int32_t* row_pos, float scale, void* out, int64_t ldo,
                   float* lse, void* workspace, size_t workspace_bytes, void* cuda_stream);
size_t vla_paged_attn_workspace_bytes(int head_dim);

/* Log-probs of given tokens, entropy and the best alternatives of `rows` rows of logits z (type `dtype`,
 * row stride ld elements), as log softmax(z / T) over `vocab` ids:
 *   tokens        int32 [rows] or NULL; -1 = no token in this row (log-prob 0); another id outside
 *                 [0, vocab) is read as -1 and raises VLA_STATUS_BAD_TOKEN;
 *   temperature   T > 0, and log2(e) / T a 32-bit number (T from 4.3e-39 on); 0 stands for 1, as in vla_decode_actions;
 *   logprob, entropy, lse  f32 [rows]: the token's log-prob, -sum p log p, and log sum exp(z / T); any of
 *                 them may be NULL;
 *   top_ids, top_logprobs  int32 / f32 [rows][top_k]: the top_k largest logits, largest first, the lower id
 *                 first among equals (0 <= top_k <= 32, at most vocab; both may be NULL when it is 0); vocab at most
 *                 2^30.
 * Logits of -infinity (masked ids) have probability 0; a row of nothing else has lse -infinity, entropy 0
 * and log-probs of -infinity.  A NaN or +infinity makes the row's numbers NaN and raises
 * VLA_STATUS_NONFINITE.  rows 0 or more. */
int vla_token_logprobs(const void* logits, int64_t ld, int dtype, int rows, int vocab, const int32_t* tokens, float temperature,
                       int top_k, float* logprob, float* entropy, float* lse, int32_t* top_ids, float* top_logprobs,
                       void* cuda_stream);

/* The gradient of sum_r g_logprob[r] logprob[r] + g_entropy[r] entropy[r] with respect to the logits:
 *   d_logits[r][j] = (g_logprob ([j = token] - p_j) - g_entropy p_j (log p_j + entropy)) / T,
 * of type `dtype`, row stride ldd; may be the logits themselves (same stride).  lse and entropy f32 [rows]
 * are those of vla_token_logprobs at the same T; g_logprob f32 [rows]; g_entropy f32 [rows] or NULL (zeros; entropy
 * may then be NULL).  Where |lse| is 128 or more, and its rounding to 32 bits would show in p_j, the row's maximum and the sum
 * relative to it are taken from the logits again.  Rows whose token is -1 (or out of range, as above) get zeros.
 * rows 0 or more. */
int vla_token_logprobs_grad(const void* logits, int64_t ld, int dtype, int rows, int vocab, const int32_t* tokens, float temperature,
                            const float* lse, const float* entropy, const float* g_logprob, const float* g_entropy,
                            void* d_logits, int64_t ldd, void* cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* VLA_LM_H_ */
