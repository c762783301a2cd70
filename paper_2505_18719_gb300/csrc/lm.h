// Internal interface of the paged cache's kernels (paged.cu, paged_attn.cu) and of the token log-probs
// (token_logprobs.cu); the C entry points that check their arguments are in lm_api.cu.
#pragma once
#include "../../include/vla_lm.h"
#include "common.cuh"

namespace vla {

struct PagePlanArgs {
  const int* ctx_in;
  const int* new_len;
  const int* release;  // or null
  int n_env, page_size;
  int* table;
  int max_pages;
  int* pool;
  int n_pages;
  const int* n_free_in;
  int* ctx_out;
  int* n_free_out;
  int* row_start;
  int* row_env;
  int* row_pos;
  int* row_slot;
  int max_rows;
  uint32_t* status;
};
constexpr int kMaxPlanEnvs = 4096;
int page_plan_launch(const PagePlanArgs& a, cudaStream_t s);

struct RopeTableArgs {
  float2* table;
  int n_pos, pairs, kind;
  double theta, factor, original_len, low, high, amplitude;
};
int rope_table_launch(const RopeTableArgs& a, cudaStream_t s);

struct RopeAppendArgs {
  const void* q;
  const void* k;
  const void* v;
  int64_t ldq, ldk, ldv;
  int dtype, rows, n_q_heads;
  vla_paged_kv kv;
  const bf16* q_gain;
  const bf16* k_gain;
  float eps;
  const float2* rope;  // or null
  int n_pos, rope_dim, interleaved;
  const int* row_pos;
  const int* row_slot;
  void* q_out;
  int64_t ldqo;
  uint32_t* status;
};
int rope_append_launch(const RopeAppendArgs& a, cudaStream_t s);

struct PagedAttnArgs {
  const void* q;
  int64_t ldq;
  int dtype, rows, n_q_heads;
  vla_paged_kv kv;
  const int* table;
  int max_pages, n_env;
  const int* row_env;
  const int* row_pos;
  float scale;
  void* out;
  int64_t ldo;
  float* lse;  // or null
  void* workspace;
  uint32_t* status;
};
int paged_attn_launch(const PagedAttnArgs& a, cudaStream_t s);
size_t paged_attn_workspace(int head_dim);

struct LogprobArgs {
  const void* logits;
  int64_t ld;
  int dtype, rows, vocab;
  const int* tokens;  // or null
  float temperature;  // > 0
  int top_k;
  float* logprob;
  float* entropy;
  float* lse;
  int* top_ids;
  float* top_logprobs;
  uint32_t* status;
};
constexpr int kMaxTopK = 32;
int token_logprobs_launch(const LogprobArgs& a, cudaStream_t s);

struct LogprobGradArgs {
  const void* logits;
  int64_t ld;
  int dtype, rows, vocab;
  const int* tokens;
  float temperature;
  const float* lse;
  const float* entropy;
  const float* g_logprob;
  const float* g_entropy;  // or null
  void* d_logits;
  int64_t ldd;
  uint32_t* status;
};
int token_logprobs_grad_launch(const LogprobGradArgs& a, cudaStream_t s);

// An element of type `dtype` as fp32, and back (rounded to nearest).
__device__ __forceinline__ float load_as_float(const void* p, int64_t i, int dtype) {
  if (dtype == VLA_F32) return static_cast<const float*>(p)[i];
  return dtype == VLA_F16 ? __half2float(static_cast<const f16*>(p)[i]) : __bfloat162float(static_cast<const bf16*>(p)[i]);
}
__device__ __forceinline__ void store_from_float(void* p, int64_t i, float x, int dtype) {
  if (dtype == VLA_F32)
    static_cast<float*>(p)[i] = x;
  else if (dtype == VLA_F16)
    static_cast<f16*>(p)[i] = __float2half_rn(x);
  else
    static_cast<bf16*>(p)[i] = __float2bfloat16_rn(x);
}
__device__ __forceinline__ void raise_status(uint32_t* status, uint32_t bit) {
  if (status) atomicOr(status, bit);
}

}  // namespace vla
