// Gradient of the causal attention of packed sequences (include/vla_learn.h).
//
// One warp a row and query head for D and d_q, then one a row and key-value head for d_k and d_v, which sums over the
// query heads that share it: no sums meet between warps, so no atomics.
#include <algorithm>

#include "prompt_rows.cuh"

namespace vla {

namespace {

constexpr int kWarps = 8;

template <int HD, bool FP16>
__global__ void __launch_bounds__(32 * kWarps) prompt_grad_query_rows_kernel(const PromptGradArgs a) {
  const int64_t item = static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5);
  if (blockIdx.x == 0) check_starts(a.f.seq_start, a.f.n_seq, a.f.rows, threadIdx.x, 32 * kWarps, a.f.status);
  if (item >= static_cast<int64_t>(a.f.rows) * a.f.n_q_heads) return;
  const int row = static_cast<int>(item / a.f.n_q_heads), h = static_cast<int>(item % a.f.n_q_heads);
  const Span sp = span_of_row(a.f.seq_start, a.f.n_seq, a.f.rows, row);
  if (sp.begin == sp.end) return store_lane<HD, FP16>(elem(a.d_q, row * a.lddq + h * HD), Lane<HD>{}, 0.f);
  const float delta = row_delta<HD, FP16>(a, row, h);
  if ((threadIdx.x & 31) == 0) static_cast<float*>(a.workspace)[static_cast<int64_t>(h) * a.f.rows + row] = delta;
  grad_query_row<HD, FP16>(a, row, h, sp.begin, delta);
}

template <int HD, bool FP16>
__global__ void __launch_bounds__(32 * kWarps) prompt_grad_key_rows_kernel(const PromptGradArgs a) {
  const int64_t item = static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5);
  if (item >= static_cast<int64_t>(a.f.rows) * a.f.n_kv_heads) return;
  const int row = static_cast<int>(item / a.f.n_kv_heads), g = static_cast<int>(item % a.f.n_kv_heads);
  const Span sp = span_of_row(a.f.seq_start, a.f.n_seq, a.f.rows, row);
  if (sp.begin < sp.end) return grad_key_row<HD, FP16>(a, row, g, sp.end, static_cast<const float*>(a.workspace));
  store_lane<HD, FP16>(elem(a.d_k, row * a.lddk + g * HD), Lane<HD>{}, 0.f);
  store_lane<HD, FP16>(elem(a.d_v, row * a.lddv + g * HD), Lane<HD>{}, 0.f);
}

template <int HD, bool FP16>
int launch(const PromptGradArgs& a, cudaStream_t s) {
  const auto ctas = [&](int heads) { return dim3(static_cast<unsigned>((static_cast<int64_t>(a.f.rows) * heads + kWarps - 1) / kWarps)); };
  VLA_CUDA_TRY(launch_at(Start::kInOrder, prompt_grad_query_rows_kernel<HD, FP16>, ctas(a.f.n_q_heads), dim3(32 * kWarps), 0, s, a));
  note_launch();
  VLA_CUDA_TRY(launch_at(Start::kInOrder, prompt_grad_key_rows_kernel<HD, FP16>, ctas(a.f.n_kv_heads), dim3(32 * kWarps), 0, s, a));
  note_launch();
  return VLA_OK;
}

}  // namespace

size_t prompt_attn_grad_workspace(int rows, int n_q_heads, int, int) { return static_cast<size_t>(rows) * n_q_heads * 4; }

int prompt_attn_grad_launch(const PromptGradArgs& a, cudaStream_t s) {
  if (a.f.head_dim == 128) return a.f.fp16 ? launch<128, true>(a, s) : launch<128, false>(a, s);
  return a.f.fp16 ? launch<64, true>(a, s) : launch<64, false>(a, s);
}

}  // namespace vla
