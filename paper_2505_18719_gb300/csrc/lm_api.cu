// C entry points of include/vla_lm.h: argument checks, then the launches of paged.cu, paged_attn.cu and
// token_logprobs.cu.  Nothing here throws.
#include <math.h>

#include "lm.h"

namespace vla {
namespace {

constexpr int kMostHeads = 65535;  // channels of a row fit 32 bits
constexpr int kMostIds = 1 << 30;  // a round past the last id fits 32 bits

bool misaligned(const void* p, uintptr_t bytes) { return reinterpret_cast<uintptr_t>(p) & (bytes - 1); }
bool is_dtype(int d) { return d == VLA_F32 || d == VLA_F16 || d == VLA_BF16; }
int elem_bytes(int d) { return d == VLA_F32 ? 4 : 2; }

// 0 stands for 1; the kernels take 1 / T times log2(e), which has to be a 32-bit number.
bool bad_temperature(float t) { return !(t >= 0.f) || !isfinite(t) || (t > 0.f && !isfinite(1.44269504f * (1.f / t))); }

// Rows of n elements at stride ld that 16-byte accesses can read: VLA_OK or an error code.
bool bad_rows(const void* p, int64_t ld, int64_t n) { return !p || misaligned(p, 16) || ld < n || (ld & 7); }

// The descriptor's own consistency; `name` heads the message.
int check_kv(const vla_paged_kv* kv, const char* null_msg, const char* bad_msg, const char* unsupported_msg) {
  if (!kv || !kv->k || !kv->v) return record_error(VLA_ERR_ARG, null_msg);
  if (kv->n_pages < 1 || kv->page_size < 1 || kv->n_heads < 1 || misaligned(kv->k, 16) || misaligned(kv->v, 16) ||
      kv->page_stride < 0 || kv->head_stride < 0 || kv->slot_stride < 0 ||
      ((kv->page_stride | kv->head_stride | kv->slot_stride) & 7) ||
      static_cast<int64_t>(kv->n_pages) * kv->page_size > 0x7fffffff)
    return record_error(VLA_ERR_ARG, bad_msg);
  if ((kv->dtype != VLA_F16 && kv->dtype != VLA_BF16) || (kv->head_dim != 64 && kv->head_dim != 128))
    return record_error(VLA_ERR_UNSUPPORTED, unsupported_msg);
  return VLA_OK;
}

}  // namespace
}  // namespace vla

using namespace vla;

extern "C" {

int vla_page_plan(const int32_t* ctx_in, const int32_t* new_len, const int32_t* release, int n_env, int page_size, int32_t* table,
                  int max_pages, int32_t* pool, int n_pages, const int32_t* n_free_in, int32_t* ctx_out, int32_t* n_free_out,
                  int32_t* row_start, int32_t* row_env, int32_t* row_pos, int32_t* row_slot, int max_rows, void* cuda_stream) {
  if (!ctx_in || !new_len || !table || !pool || !n_free_in || !ctx_out || !n_free_out || !row_start)
    return record_error(VLA_ERR_ARG, "vla_page_plan: NULL argument");
  if (max_rows < 0 || (max_rows > 0 && (!row_env || !row_pos || !row_slot)))
    return record_error(VLA_ERR_ARG, "vla_page_plan: max_rows < 0, or rows without their arrays");
  if (n_env < 1 || page_size < 1 || max_pages < 1 || n_pages < 1 || static_cast<int64_t>(n_pages) * page_size > 0x7fffffff)
    return record_error(VLA_ERR_ARG, "vla_page_plan: n_env, page_size, max_pages and n_pages are at least 1, n_pages * page_size "
                                     "below 2^31");
  if (n_env > kMaxPlanEnvs) return record_error(VLA_ERR_UNSUPPORTED, "vla_page_plan: more than 4096 environments");
  PagePlanArgs a{ctx_in, new_len, release, n_env, page_size, table, max_pages, pool, n_pages, n_free_in, ctx_out, n_free_out,
                 row_start, row_env, row_pos, row_slot, max_rows, nullptr};
  if (const int rs = op_status_word(&a.status)) return rs;
  return page_plan_launch(a, static_cast<cudaStream_t>(cuda_stream));
}

int vla_rope_table(float* table, int n_pos, int rope_dim, double theta, int kind, double factor, double original_len, double low,
                   double high, double amplitude, void* cuda_stream) {
  if (!table || misaligned(table, 8) || n_pos < 1 || rope_dim < 2 || (rope_dim & 1) || !(theta > 0.0) || !isfinite(theta) ||
      !(amplitude > 0.0) || !isfinite(amplitude))
    return record_error(VLA_ERR_ARG, "vla_rope_table: bad argument");
  if (kind < VLA_ROPE_PLAIN || kind > VLA_ROPE_LOG_TURNS) return record_error(VLA_ERR_UNSUPPORTED, "vla_rope_table: unknown kind");
  if (kind != VLA_ROPE_PLAIN && (!(factor >= 1.0) || !isfinite(factor)))
    return record_error(VLA_ERR_ARG, "vla_rope_table: factor is at least 1");
  if (kind >= VLA_ROPE_TURNS && (!(original_len > 0.0) || !isfinite(original_len) || !(low > 0.0) || !(high > low) || !isfinite(high)))
    return record_error(VLA_ERR_ARG, "vla_rope_table: original_len > 0 and 0 < low < high");
  const RopeTableArgs a{reinterpret_cast<float2*>(table), n_pos, rope_dim / 2, kind, theta, factor, original_len, low, high, amplitude};
  return rope_table_launch(a, static_cast<cudaStream_t>(cuda_stream));
}

int vla_rope_append(const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv, int dtype, int rows,
                    int n_q_heads, const vla_paged_kv* kv, const void* q_gain, const void* k_gain, float eps, const float* rope,
                    int n_pos, int rope_dim, int interleaved, const int32_t* row_pos, const int32_t* row_slot, void* q_out,
                    int64_t ldqo, void* cuda_stream) {
  if (const int rc = check_kv(kv, "vla_rope_append: NULL cache", "vla_rope_append: bad cache sizes, strides or alignment",
                              "vla_rope_append: cache of fp16 or bf16 with heads of 64 or 128"))
    return rc;
  if (!is_dtype(dtype)) return record_error(VLA_ERR_UNSUPPORTED, "vla_rope_append: unknown dtype");
  if (n_q_heads > kMostHeads || kv->n_heads > kMostHeads) return record_error(VLA_ERR_UNSUPPORTED, "vla_rope_append: more than 65535 heads");
  if (rows < 0 || n_q_heads < 1) return record_error(VLA_ERR_ARG, "vla_rope_append: rows < 0 or no query heads");
  if (rows == 0) return VLA_OK;
  const int64_t hd = kv->head_dim;
  if (bad_rows(q, ldq, n_q_heads * hd) || bad_rows(k, ldk, kv->n_heads * hd) || bad_rows(v, ldv, kv->n_heads * hd) ||
      bad_rows(q_out, ldqo, n_q_heads * hd))
    return record_error(VLA_ERR_ARG, "vla_rope_append: q, k, v, q_out: 16-byte aligned, row strides multiples of 8 that hold a row");
  if (q_out == q && ldqo != ldq) return record_error(VLA_ERR_ARG, "vla_rope_append: queries in place need one stride");
  if (!row_pos || !row_slot || misaligned(q_gain, 16) || misaligned(k_gain, 16) || !(eps >= 0.f) || !isfinite(eps))
    return record_error(VLA_ERR_ARG, "vla_rope_append: NULL rows, gains off 16 bytes, or eps < 0");
  if (rope && (misaligned(rope, 16) || n_pos < 1 || rope_dim < 16 || (rope_dim & 15) || rope_dim > hd))
    return record_error(VLA_ERR_ARG, "vla_rope_append: rope_dim a multiple of 16 up to the head, table 16-byte aligned");
  RopeAppendArgs a{q, k, v, ldq, ldk, ldv, dtype, rows, n_q_heads, *kv, static_cast<const bf16*>(q_gain),
                   static_cast<const bf16*>(k_gain), eps, reinterpret_cast<const float2*>(rope), n_pos, rope_dim, interleaved,
                   row_pos, row_slot, q_out, ldqo, nullptr};
  if (const int rs = op_status_word(&a.status)) return rs;
  return rope_append_launch(a, static_cast<cudaStream_t>(cuda_stream));
}

size_t vla_paged_attn_workspace_bytes(int head_dim) {
  return head_dim == 64 || head_dim == 128 ? paged_attn_workspace(head_dim) : 0;
}

int vla_paged_attn(const void* q, int64_t ldq, int dtype, int rows, int n_q_heads, const vla_paged_kv* kv, const int32_t* table,
                   int max_pages, int n_env, const int32_t* row_env, const int32_t* row_pos, float scale, void* out, int64_t ldo,
                   float* lse, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  if (const int rc = check_kv(kv, "vla_paged_attn: NULL cache", "vla_paged_attn: bad cache sizes, strides or alignment",
                              "vla_paged_attn: cache of fp16 or bf16 with heads of 64 or 128"))
    return rc;
  if (dtype != kv->dtype && !(dtype == VLA_F32 && kv->dtype == VLA_F16))
    return record_error(VLA_ERR_UNSUPPORTED, "vla_paged_attn: queries of the cache's type, or f32 over an fp16 cache");
  if (n_q_heads > kMostHeads) return record_error(VLA_ERR_UNSUPPORTED, "vla_paged_attn: more than 65535 heads");
  if (rows < 0 || n_q_heads < 1 || n_q_heads % kv->n_heads)
    return record_error(VLA_ERR_ARG, "vla_paged_attn: rows < 0, or query heads no multiple of the cache's");
  if (rows == 0) return VLA_OK;
  if (static_cast<int64_t>(rows) * n_q_heads > (1 << 30)) return record_error(VLA_ERR_UNSUPPORTED, "vla_paged_attn: more than 2^30 rows x query heads");
  const int64_t width = static_cast<int64_t>(n_q_heads) * kv->head_dim;
  if (bad_rows(q, ldq, width) || bad_rows(out, ldo, width))
    return record_error(VLA_ERR_ARG, "vla_paged_attn: q and out: 16-byte aligned, row strides multiples of 8 that hold a row");
  if (!table || max_pages < 1 || n_env < 1 || !row_env || !row_pos || !isfinite(scale))
    return record_error(VLA_ERR_ARG, "vla_paged_attn: bad argument");
  if (!workspace || misaligned(workspace, 16) || workspace_bytes < paged_attn_workspace(kv->head_dim))
    return record_error(VLA_ERR_ARG, "vla_paged_attn: workspace NULL, off 16 bytes or too small");
  PagedAttnArgs a{q, ldq, dtype, rows, n_q_heads, *kv, table, max_pages, n_env, row_env, row_pos, scale, out, ldo, lse, workspace,
                  nullptr};
  if (const int rs = op_status_word(&a.status)) return rs;
  return paged_attn_launch(a, static_cast<cudaStream_t>(cuda_stream));
}

int vla_token_logprobs(const void* logits, int64_t ld, int dtype, int rows, int vocab, const int32_t* tokens, float temperature,
                       int top_k, float* logprob, float* entropy, float* lse, int32_t* top_ids, float* top_logprobs,
                       void* cuda_stream) {
  if (!is_dtype(dtype)) return record_error(VLA_ERR_UNSUPPORTED, "vla_token_logprobs: unknown dtype");
  if (rows < 0 || vocab < 1 || bad_temperature(temperature) || top_k < 0 || top_k > vocab)
    return record_error(VLA_ERR_ARG, "vla_token_logprobs: bad argument");
  if (vocab > kMostIds) return record_error(VLA_ERR_UNSUPPORTED, "vla_token_logprobs: more than 2^30 ids");
  if (top_k > kMaxTopK) return record_error(VLA_ERR_UNSUPPORTED, "vla_token_logprobs: more than 32 alternatives");
  if (rows == 0) return VLA_OK;
  if (!logits || ld < vocab || misaligned(logits, elem_bytes(dtype)) || (top_k > 0 && (!top_ids || !top_logprobs)))
    return record_error(VLA_ERR_ARG, "vla_token_logprobs: logits NULL or ld < vocab, or alternatives without their arrays");
  if (logprob && !tokens) return record_error(VLA_ERR_ARG, "vla_token_logprobs: log-probs of no tokens");
  LogprobArgs a{logits, ld, dtype, rows, vocab, tokens, temperature > 0.f ? temperature : 1.f, top_k, logprob, entropy, lse, top_ids,
                top_logprobs, nullptr};
  if (const int rs = op_status_word(&a.status)) return rs;
  return token_logprobs_launch(a, static_cast<cudaStream_t>(cuda_stream));
}

int vla_token_logprobs_grad(const void* logits, int64_t ld, int dtype, int rows, int vocab, const int32_t* tokens, float temperature,
                            const float* lse, const float* entropy, const float* g_logprob, const float* g_entropy,
                            void* d_logits, int64_t ldd, void* cuda_stream) {
  if (!is_dtype(dtype)) return record_error(VLA_ERR_UNSUPPORTED, "vla_token_logprobs_grad: unknown dtype");
  if (rows < 0 || vocab < 1 || bad_temperature(temperature))
    return record_error(VLA_ERR_ARG, "vla_token_logprobs_grad: bad argument");
  if (vocab > kMostIds) return record_error(VLA_ERR_UNSUPPORTED, "vla_token_logprobs_grad: more than 2^30 ids");
  if (rows == 0) return VLA_OK;
  if (!logits || ld < vocab || !d_logits || ldd < vocab || misaligned(logits, elem_bytes(dtype)) ||
      misaligned(d_logits, elem_bytes(dtype)) || (d_logits == logits && ldd != ld))
    return record_error(VLA_ERR_ARG, "vla_token_logprobs_grad: logits or gradient NULL, off their type, or of a stride below vocab");
  if (!tokens || !lse || !g_logprob || (g_entropy && !entropy))
    return record_error(VLA_ERR_ARG, "vla_token_logprobs_grad: NULL argument");
  LogprobGradArgs a{logits, ld, dtype, rows, vocab, tokens, temperature > 0.f ? temperature : 1.f, lse, entropy, g_logprob, g_entropy,
                    d_logits, ldd, nullptr};
  if (const int rs = op_status_word(&a.status)) return rs;
  return token_logprobs_grad_launch(a, static_cast<cudaStream_t>(cuda_stream));
}

}  // extern "C"
