// C entry points of include/vla_learn.h: argument checks, then the launches of prompt_attn.cu, prompt_grad.cu and
// block_norm.cu.  Nothing here throws.
#include <math.h>

#include "learn.h"

namespace vla {
namespace {

constexpr int kMostHeads = 65535;
constexpr float kLeastScale = 1e-30f;  // the gradient takes lse / scale

bool misaligned(const void* p, uintptr_t bytes) { return reinterpret_cast<uintptr_t>(p) & (bytes - 1); }
int elem_bytes(int d) { return d == VLA_F32 ? 4 : 2; }
bool is_dtype(int d) { return d == VLA_F32 || d == VLA_F16 || d == VLA_BF16; }
// Rows of n elements at stride ld that 16-byte accesses can read.
bool bad_rows(const void* p, int64_t ld, int64_t n) { return !p || misaligned(p, 16) || ld < n || (ld & 7); }
// Rows of n elements at stride ld, aligned to their elements.
bool bad_plain_rows(const void* p, int64_t ld, int n, int dtype) { return !p || ld < n || misaligned(p, elem_bytes(dtype)); }

struct PromptNames {
  const char *dtype, *heads, *head_dim, *rows, *tensors, *sequences;
};
// What both directions check, in their own names.
int check_prompt(const PromptArgs& a, int dtype, const PromptNames& n) {
  if (dtype != VLA_F16 && dtype != VLA_BF16) return record_error(VLA_ERR_UNSUPPORTED, n.dtype);
  if (a.rows < 0 || a.n_q_heads < 1 || a.n_kv_heads < 1 || a.n_q_heads % a.n_kv_heads) return record_error(VLA_ERR_ARG, n.heads);
  if (a.head_dim != 64 && a.head_dim != 128) return record_error(VLA_ERR_UNSUPPORTED, n.head_dim);
  if (a.n_q_heads > kMostHeads || static_cast<int64_t>(a.rows) * a.n_q_heads > (1 << 30)) return record_error(VLA_ERR_UNSUPPORTED, n.rows);
  if (a.rows == 0) return VLA_OK;
  const int64_t hd = a.head_dim;
  if (bad_rows(a.q, a.ldq, a.n_q_heads * hd) || bad_rows(a.k, a.ldk, a.n_kv_heads * hd) || bad_rows(a.v, a.ldv, a.n_kv_heads * hd) ||
      bad_rows(a.out, a.ldo, a.n_q_heads * hd))
    return record_error(VLA_ERR_ARG, n.tensors);
  if (misaligned(a.lse, 4)) return record_error(VLA_ERR_ARG, n.tensors);
  if (!a.seq_start || misaligned(a.seq_start, 4) || a.n_seq < 1 || !(a.scale >= kLeastScale) || !isfinite(a.scale)) return record_error(VLA_ERR_ARG, n.sequences);
  return VLA_OK;
}

struct NormNames {
  const char *dtype, *dim, *rows, *forms, *missing;
};
int check_norm(const BlockNormArgs& a, const NormNames& n) {
  if (!is_dtype(a.dtype) || (a.h_dtype != VLA_F32 && a.h_dtype != a.dtype)) return record_error(VLA_ERR_UNSUPPORTED, n.dtype);
  if (a.rows < 0 || a.dim < 1 || !(a.eps >= 0.f) || !isfinite(a.eps) || !isfinite(a.residual_scale)) return record_error(VLA_ERR_ARG, n.dim);
  if (a.dim > kMostNormDim) return record_error(VLA_ERR_UNSUPPORTED, n.dim);
  if (!a.y && (a.post_gain || a.gate)) return record_error(VLA_ERR_ARG, n.forms);
  if (a.rows == 0) return VLA_OK;
  if ((a.y && bad_plain_rows(a.y, a.ldy, a.dim, a.dtype)) || bad_plain_rows(a.h, a.ldh, a.dim, a.h_dtype) ||
      (a.gate && (misaligned(a.gate, elem_bytes(a.dtype)) || (a.ldg != 0 && a.ldg < a.dim))))
    return record_error(VLA_ERR_ARG, n.rows);
  if (!a.pre_gain || misaligned(a.pre_gain, 2) || misaligned(a.post_gain, 2) || misaligned(a.rstd, 4)) return record_error(VLA_ERR_ARG, n.missing);
  return VLA_OK;
}

}  // namespace
}  // namespace vla

using namespace vla;

extern "C" {

int vla_prompt_attn(const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv, int dtype, int rows,
                    int n_q_heads, int n_kv_heads, int head_dim, const int32_t* seq_start, int n_seq, float scale, void* out,
                    int64_t ldo, float* lse, void* cuda_stream) {
  static constexpr PromptNames kNames{"vla_prompt_attn: fp16 or bf16", "vla_prompt_attn: rows < 0, or query heads no multiple of the key-value heads",
                                      "vla_prompt_attn: heads of 64 or 128", "vla_prompt_attn: more than 65535 heads or 2^30 rows x query heads",
                                      "vla_prompt_attn: q, k, v, out: 16-byte aligned, row strides multiples of 8 that hold a row",
                                      "vla_prompt_attn: no sequences, or a scale below 1e-30 or infinite"};
  PromptArgs a{q, k, v, ldq, ldk, ldv, dtype == VLA_F16, rows, n_q_heads, n_kv_heads, head_dim, seq_start, n_seq, scale, out, ldo, lse, nullptr};
  if (const int rc = check_prompt(a, dtype, kNames)) return rc;
  if (rows == 0) return VLA_OK;
  if (const int rs = op_status_word(&a.status)) return rs;
  return prompt_attn_launch(a, static_cast<cudaStream_t>(cuda_stream));
}

size_t vla_prompt_attn_grad_workspace_bytes(int rows, int n_q_heads, int n_kv_heads, int head_dim) {
  if (rows < 0 || n_q_heads < 1 || n_kv_heads < 1 || n_q_heads % n_kv_heads || n_q_heads > kMostHeads ||
      static_cast<int64_t>(rows) * n_q_heads > (1 << 30) || (head_dim != 64 && head_dim != 128))
    return 0;
  return prompt_attn_grad_workspace(rows, n_q_heads, n_kv_heads, head_dim);
}

int vla_prompt_attn_grad(const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv, int dtype, int rows,
                         int n_q_heads, int n_kv_heads, int head_dim, const int32_t* seq_start, int n_seq, float scale,
                         const void* out, int64_t ldo, const float* lse, const void* d_out, int64_t lddo, void* d_q, int64_t lddq,
                         void* d_k, int64_t lddk, void* d_v, int64_t lddv, void* workspace, size_t workspace_bytes,
                         void* cuda_stream) {
  static constexpr PromptNames kNames{
      "vla_prompt_attn_grad: fp16 or bf16", "vla_prompt_attn_grad: rows < 0, or query heads no multiple of the key-value heads",
      "vla_prompt_attn_grad: heads of 64 or 128", "vla_prompt_attn_grad: more than 65535 heads or 2^30 rows x query heads",
      "vla_prompt_attn_grad: q, k, v, out: 16-byte aligned, row strides multiples of 8 that hold a row",
      "vla_prompt_attn_grad: no sequences, or a scale below 1e-30 or infinite"};
  PromptGradArgs a{{q, k, v, ldq, ldk, ldv, dtype == VLA_F16, rows, n_q_heads, n_kv_heads, head_dim, seq_start, n_seq, scale,
                    const_cast<void*>(out), ldo, const_cast<float*>(lse), nullptr},
                   d_out, lddo, d_q, d_k, d_v, lddq, lddk, lddv, workspace};
  if (const int rc = check_prompt(a.f, dtype, kNames)) return rc;
  if (rows == 0) return VLA_OK;
  const int64_t q_row = static_cast<int64_t>(n_q_heads) * head_dim, kv_row = static_cast<int64_t>(n_kv_heads) * head_dim;
  if (bad_rows(d_out, lddo, q_row) || bad_rows(d_q, lddq, q_row) || bad_rows(d_k, lddk, kv_row) || bad_rows(d_v, lddv, kv_row))
    return record_error(VLA_ERR_ARG, "vla_prompt_attn_grad: gradients: 16-byte aligned, row strides multiples of 8 that hold a row");
  if (!lse || misaligned(lse, 4)) return record_error(VLA_ERR_ARG, "vla_prompt_attn_grad: no lse");
  if (!workspace || misaligned(workspace, 16) || workspace_bytes < prompt_attn_grad_workspace(rows, n_q_heads, n_kv_heads, head_dim))
    return record_error(VLA_ERR_ARG, "vla_prompt_attn_grad: workspace NULL, off 16 bytes or too small");
  if (const int rs = op_status_word(&a.f.status)) return rs;
  return prompt_attn_grad_launch(a, static_cast<cudaStream_t>(cuda_stream));
}

int vla_block_norm(const void* y, int64_t ldy, int dtype, const void* h, int64_t ldh, int h_dtype, int rows, int dim,
                   const void* post_gain, const void* gate, int64_t ldg, float residual_scale, const void* pre_gain, float eps,
                   void* h_out, int64_t ldho, void* x, int64_t ldx, float* rstd, void* cuda_stream) {
  static constexpr NormNames kNames{"vla_block_norm: unknown dtype, or a stream that is neither f32 nor of the block's type",
                                    "vla_block_norm: rows < 0, dim outside 1 to 16384, eps < 0 or no number",
                                    "vla_block_norm: y, h, gate: aligned to their type, strides of at least dim (a gate's may be 0)",
                                    "vla_block_norm: a gain, a gate or an output behind the sum without a block's output", "vla_block_norm: no pre_gain, or off its type"};
  const BlockNormArgs a{y, ldy, dtype, h, ldh, h_dtype, rows, dim, static_cast<const bf16*>(post_gain), gate, ldg, residual_scale,
                        static_cast<const bf16*>(pre_gain), eps, h_out, ldho, x, ldx, rstd};
  if (const int rc = check_norm(a, kNames)) return rc;
  if (!y && h_out) return record_error(VLA_ERR_ARG, kNames.forms);
  if (rows == 0) return VLA_OK;
  if ((y && bad_plain_rows(h_out, ldho, dim, h_dtype)) || bad_plain_rows(x, ldx, dim, dtype) || (h_out && h_out == h && ldho != ldh))
    return record_error(VLA_ERR_ARG, "vla_block_norm: h_out, x: aligned to their type, strides of at least dim; h in place needs one stride");
  return block_norm_launch(a, static_cast<cudaStream_t>(cuda_stream));
}

size_t vla_block_norm_grad_workspace_bytes(int rows, int dim) {
  return rows < 0 || dim < 1 || dim > kMostNormDim ? 0 : block_norm_grad_workspace(rows, dim);
}

int vla_block_norm_grad(const void* y, int64_t ldy, int dtype, const void* h_out, int64_t ldho, int h_dtype, int rows, int dim,
                        const void* post_gain, const void* gate, int64_t ldg, float residual_scale, const void* pre_gain,
                        const float* rstd, const void* d_x, int64_t lddx, const void* d_h_out, int64_t lddho, void* d_h,
                        int64_t lddh, void* d_y, int64_t lddy, void* d_gate, int64_t lddg, float* d_post_gain, float* d_pre_gain,
                        void* workspace, size_t workspace_bytes, void* cuda_stream) {
  static constexpr NormNames kNames{"vla_block_norm_grad: unknown dtype, or a stream that is neither f32 nor of the block's type",
                                    "vla_block_norm_grad: rows < 0, dim outside 1 to 16384 or no number",
                                    "vla_block_norm_grad: y, h_out, gate: aligned to their type, strides of at least dim (a gate's may be 0)",
                                    "vla_block_norm_grad: a gain or a gate without a block's output", "vla_block_norm_grad: no pre_gain, or off its type"};
  BlockNormGradArgs a{{y, ldy, dtype, h_out, ldho, h_dtype, rows, dim, static_cast<const bf16*>(post_gain), gate, ldg, residual_scale,
                       static_cast<const bf16*>(pre_gain), 0.f, nullptr, 0, nullptr, 0, const_cast<float*>(rstd)},
                      d_x, lddx, d_h_out, lddho, d_h, lddh, d_y, lddy, d_gate, lddg, d_post_gain, d_pre_gain,
                      static_cast<float*>(workspace), nullptr, g_wait_limit_ns.load(std::memory_order_relaxed)};
  if (const int rc = check_norm(a.f, kNames)) return rc;
  if (!d_pre_gain || misaligned(d_pre_gain, 4) || (post_gain && (!d_post_gain || misaligned(d_post_gain, 4))))
    return record_error(VLA_ERR_ARG, "vla_block_norm_grad: a gain without its gradient, or that off 4 bytes");
  if (gate && (!d_gate || misaligned(d_gate, ldg ? elem_bytes(dtype) : 4) || (ldg != 0 && rows > 0 && lddg < dim)))
    return record_error(VLA_ERR_ARG, "vla_block_norm_grad: a gate without its gradient, or that off its type or of a stride below dim");
  if (rows > 0) {
    if (!rstd || bad_plain_rows(d_x, lddx, dim, dtype) || (d_h_out && bad_plain_rows(d_h_out, lddho, dim, h_dtype)) ||
        bad_plain_rows(d_h, lddh, dim, h_dtype) || (y && bad_plain_rows(d_y, lddy, dim, dtype)) || (d_h_out == d_h && lddho != lddh))
      return record_error(VLA_ERR_ARG, "vla_block_norm_grad: rstd NULL, or d_x, d_h_out, d_h, d_y NULL, off their type or of a stride below dim");
    if (!workspace || misaligned(workspace, 16) || workspace_bytes < block_norm_grad_workspace(rows, dim))
      return record_error(VLA_ERR_ARG, "vla_block_norm_grad: workspace NULL, off 16 bytes or too small");
    if (const int rs = op_status_word(&a.status)) return rs;
  }
  return block_norm_grad_launch(a, static_cast<cudaStream_t>(cuda_stream));
}

}  // extern "C"
