// Causal attention of packed sequences (include/vla_learn.h).
//
// One warp a row and query head, sequences and positions as they stand: right for every case, and bound by the
// instructions of a key (its two rows read from L2, five shuffles for the score, the weight).
#include <algorithm>

#include "prompt_rows.cuh"

namespace vla {

namespace {

constexpr int kWarps = 8;

template <int HD, bool FP16>
__global__ void __launch_bounds__(32 * kWarps) prompt_attn_rows_kernel(const PromptArgs a) {
  const int64_t item = static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5);
  if (blockIdx.x == 0) check_starts(a.seq_start, a.n_seq, a.rows, threadIdx.x, 32 * kWarps, a.status);
  if (item >= static_cast<int64_t>(a.rows) * a.n_q_heads) return;
  const int row = static_cast<int>(item / a.n_q_heads), h = static_cast<int>(item % a.n_q_heads);
  const Span sp = span_of_row(a.seq_start, a.n_seq, a.rows, row);
  if (sp.begin < sp.end) return attend_row<HD, FP16>(a, row, h, sp.begin);
  store_lane<HD, FP16>(elem(a.out, row * a.ldo + h * HD), Lane<HD>{}, 0.f);
  if (a.lse && (threadIdx.x & 31) == 0) a.lse[item] = -INFINITY;
}

}  // namespace

int prompt_attn_launch(const PromptArgs& a, cudaStream_t s) {
  const int64_t ctas = (static_cast<int64_t>(a.rows) * a.n_q_heads + kWarps - 1) / kWarps;
  const auto kern = a.head_dim == 128 ? (a.fp16 ? prompt_attn_rows_kernel<128, true> : prompt_attn_rows_kernel<128, false>)
                                      : (a.fp16 ? prompt_attn_rows_kernel<64, true> : prompt_attn_rows_kernel<64, false>);
  VLA_CUDA_TRY(launch_at(Start::kInOrder, kern, dim3(static_cast<unsigned>(ctas)), dim3(32 * kWarps), 0, s, a));
  note_launch();
  return VLA_OK;
}

}  // namespace vla
