// Attention of one new token per row over its environment's paged positions.
#include "lm.h"

namespace vla {

namespace {

// One warp per (row, query head), lanes over the channels, one position after the other: the running
// maximum m, l = sum 2^(s - m) and o = sum 2^(s - m) v.
__global__ void __launch_bounds__(128) paged_attn_kernel(const PagedAttnArgs a) {
  pdl_launch_dependents();
  pdl_wait();
  const int lane = threadIdx.x & 31, hd = a.kv.head_dim, per = hd / 32;
  const int64_t item = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 5);
  if (item >= static_cast<int64_t>(a.rows) * a.n_q_heads) return;
  const int row = static_cast<int>(item / a.n_q_heads), head = static_cast<int>(item % a.n_q_heads);
  const int kv_head = head / (a.n_q_heads / a.kv.n_heads);
  const int env = a.row_env[row], pos = a.row_pos[row];
  bool empty = pos == -1;
  if (!empty && (pos < 0 || pos / a.kv.page_size >= a.max_pages || static_cast<unsigned>(env) >= static_cast<unsigned>(a.n_env))) {
    if (lane == 0) raise_status(a.status, VLA_STATUS_PAGES);
    empty = true;
  }
  const int64_t q_at = row * a.ldq + static_cast<int64_t>(head) * hd;
  float q[4], o[4] = {0.f, 0.f, 0.f, 0.f}, m = -INFINITY, l = 0.f;
  for (int i = 0; i < per; ++i) q[i] = load_as_float(a.q, q_at + lane + 32 * i, a.dtype) * a.scale * 1.44269504f;
  const int n = empty ? 0 : pos + 1;
  for (int p = 0; p < n; ++p) {
    const int page = a.table[static_cast<int64_t>(env) * a.max_pages + p / a.kv.page_size];
    if (static_cast<unsigned>(page) >= static_cast<unsigned>(a.kv.n_pages)) {
      if (lane == 0) raise_status(a.status, VLA_STATUS_PAGES);
      continue;
    }
    const int64_t at = page * a.kv.page_stride + kv_head * a.kv.head_stride + (p % a.kv.page_size) * a.kv.slot_stride + lane;
    float s = 0.f;
    for (int i = 0; i < per; ++i) s += q[i] * load_as_float(a.kv.k, at + 32 * i, a.kv.dtype);
    s = warp_sum(s);
    const float top = fmaxf(m, s);
    const float keep = top == -INFINITY ? 1.f : exp2f(m - top), w = top == -INFINITY ? 0.f : exp2f(s - top);
    m = top;
    l = l * keep + w;
    for (int i = 0; i < per; ++i) o[i] = o[i] * keep + w * load_as_float(a.kv.v, at + 32 * i, a.kv.dtype);
  }
  const float inv = l > 0.f ? 1.f / l : l == l ? 0.f : l;
  for (int i = 0; i < per; ++i)
    store_from_float(a.out, row * a.ldo + static_cast<int64_t>(head) * hd + lane + 32 * i, o[i] * inv, a.dtype);
  if (a.lse && lane == 0) a.lse[item] = (m + log2f(l)) * 0.693147181f;
}

}  // namespace

size_t paged_attn_workspace(int) { return 16; }

int paged_attn_launch(const PagedAttnArgs& a, cudaStream_t s) {
  const int64_t items = static_cast<int64_t>(a.rows) * a.n_q_heads;
  if ((items + 3) / 4 > 0x7fffffff) return record_error(VLA_ERR_UNSUPPORTED, "vla_paged_attn: too many rows");
  VLA_CUDA_TRY(launch_pdl(paged_attn_kernel, dim3(static_cast<unsigned>((items + 3) / 4)), dim3(128), 0, s, a));
  note_launch();
  VLA_CUDA_TRY(cudaGetLastError());
  return VLA_OK;
}

}  // namespace vla
