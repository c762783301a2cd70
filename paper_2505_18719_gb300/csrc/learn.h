// Internal interface of the learning pass's kernels (prompt_attn.cu, prompt_grad.cu, block_norm.cu); the C entry points that check
// their arguments are in learn_api.cu.
#pragma once
#include "../../include/vla_learn.h"
#include "lm.h"

namespace vla {

// SMs of the current device.
inline int device_sms(int* sms) {
  int dev = 0;
  VLA_CUDA_TRY(cudaGetDevice(&dev));
  VLA_CUDA_TRY(cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev));
  return VLA_OK;
}

struct PromptArgs {
  const void* q;
  const void* k;
  const void* v;
  int64_t ldq, ldk, ldv;
  bool fp16;  // else bf16
  int rows, n_q_heads, n_kv_heads, head_dim;
  const int* seq_start;
  int n_seq;
  float scale;
  void* out;  // read by the gradient
  int64_t ldo;
  float* lse;
  uint32_t* status;
};
int prompt_attn_launch(const PromptArgs& a, cudaStream_t s);

struct PromptGradArgs {
  PromptArgs f;
  const void* d_out;
  int64_t lddo;
  void* d_q;
  void* d_k;
  void* d_v;
  int64_t lddq, lddk, lddv;
  void* workspace;
};
int prompt_attn_grad_launch(const PromptGradArgs& a, cudaStream_t s);
size_t prompt_attn_grad_workspace(int rows, int n_q_heads, int n_kv_heads, int head_dim);

struct BlockNormArgs {
  const void* y;  // or null
  int64_t ldy;
  int dtype;
  const void* h;  // the gradient's: the stream behind the sum
  int64_t ldh;
  int h_dtype, rows, dim;
  const bf16* post_gain;  // or null
  const void* gate;       // or null
  int64_t ldg;            // 0: one for all rows
  float residual_scale;
  const bf16* pre_gain;
  float eps;
  void* h_out;
  int64_t ldho;
  void* x;
  int64_t ldx;
  float* rstd;
};
int block_norm_launch(const BlockNormArgs& a, cudaStream_t s);

struct BlockNormGradArgs {
  BlockNormArgs f;  // without h_out and x
  const void* d_x;
  int64_t lddx;
  const void* d_h_out;  // or null
  int64_t lddho;
  void* d_h;
  int64_t lddh;
  void* d_y;
  int64_t lddy;
  void* d_gate;
  int64_t lddg;
  float* d_post_gain;
  float* d_pre_gain;
  float* workspace;
  uint32_t* status;
  uint64_t wait_limit;
};
int block_norm_grad_launch(const BlockNormGradArgs& a, cudaStream_t s);
size_t block_norm_grad_workspace(int rows, int dim);
constexpr int kMostNormDim = 16384;

}  // namespace vla
