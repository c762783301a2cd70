// Log-probs of given tokens with entropy and the best alternatives, and their gradient.
#include "lm.h"

namespace vla {

namespace {

constexpr int kLpThreads = 512;

// Whole numbers in the order of the floats (negative zero as zero), so that (value, lower id first) is one
// 64-bit comparison.
__device__ __forceinline__ int ordered(float x) {
  const int b = __float_as_int(x + 0.f);
  return b ^ ((b >> 31) & 0x7fffffff);
}
__device__ __forceinline__ int64_t top_key(float x, int id) {
  return (static_cast<int64_t>(ordered(x)) << 32) | static_cast<uint32_t>(0x7fffffff - id);
}
__device__ __forceinline__ float key_value(int64_t key) {
  const int b = static_cast<int>(key >> 32);
  return __int_as_float(b ^ ((b >> 31) & 0x7fffffff));
}
__device__ __forceinline__ int key_id(int64_t key) { return 0x7fffffff - static_cast<int>(key & 0x7fffffff); }

// One CTA per row.  With m the largest z / T: s = sum e^(z/T - m), w = sum (z/T - m) e^(z/T - m), lse = m + log s,
// entropy = log s - w / s; then the best ids one by one, each the largest key below the one before.
__global__ void __launch_bounds__(kLpThreads) token_logprobs_kernel(const LogprobArgs a) {
  __shared__ float red[3][kLpThreads / 32];
  __shared__ int64_t red_key[kLpThreads / 32];
  pdl_launch_dependents();
  pdl_wait();
  const int row = blockIdx.x, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int64_t at = row * a.ld;
  const float inv_t = 1.f / a.temperature;
  float m = -INFINITY;
  bool odd = false;
  for (int j = tid; j < a.vocab; j += kLpThreads) {
    const float z = load_as_float(a.logits, at + j, a.dtype);
    odd |= !(z < INFINITY);
    m = fmaxf(m, z * inv_t);
  }
  m = warp_max(m);
  if (lane == 0) red[0][warp] = m;
  odd = __syncthreads_or(odd);
  for (int i = 0; i < kLpThreads / 32; ++i) m = fmaxf(m, red[0][i]);
  __syncthreads();
  float s = 0.f, w = 0.f;
  for (int j = tid; j < a.vocab; j += kLpThreads) {
    const float d = load_as_float(a.logits, at + j, a.dtype) * inv_t - m;
    const float e = m == -INFINITY ? 0.f : expf(d);
    s += e;
    if (e > 0.f) w += d * e;
  }
  s = warp_sum(s);
  w = warp_sum(w);
  if (lane == 0) {
    red[1][warp] = s;
    red[2][warp] = w;
  }
  __syncthreads();
  s = w = 0.f;
  for (int i = 0; i < kLpThreads / 32; ++i) {
    s += red[1][i];
    w += red[2][i];
  }
  float log_s = logf(s), lse = m + log_s, entropy = s > 0.f ? log_s - w / s : 0.f;
  if (odd) lse = entropy = NAN;
  if (tid == 0) {
    if (odd) raise_status(a.status, VLA_STATUS_NONFINITE);
    if (a.lse) a.lse[row] = lse;
    if (a.entropy) a.entropy[row] = entropy;
    if (a.tokens) {
      const int t = a.tokens[row];
      const bool ok = static_cast<unsigned>(t) < static_cast<unsigned>(a.vocab);
      if (!ok && t != -1) raise_status(a.status, VLA_STATUS_BAD_TOKEN);
      if (a.logprob) {
        const float z = ok ? load_as_float(a.logits, at + t, a.dtype) * inv_t : 0.f;
        a.logprob[row] = !ok ? 0.f : odd ? NAN : z == -INFINITY ? z : z - lse;
      }
    }
  }
  int64_t last = INT64_MAX;
  for (int i = 0; i < a.top_k; ++i) {
    int64_t best = INT64_MIN;
    for (int j = tid; j < a.vocab; j += kLpThreads) {
      const int64_t key = top_key(load_as_float(a.logits, at + j, a.dtype), j);
      if (key < last && key > best) best = key;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
    __syncthreads();
    if (lane == 0) red_key[warp] = best;
    __syncthreads();
    for (int k = 0; k < kLpThreads / 32; ++k) best = max(best, red_key[k]);
    last = best;
    if (tid == 0) {
      const float z = key_value(best) * inv_t;
      a.top_ids[static_cast<int64_t>(row) * a.top_k + i] = key_id(best);
      a.top_logprobs[static_cast<int64_t>(row) * a.top_k + i] = odd ? NAN : z == -INFINITY ? z : z - lse;
    }
  }
}

// One CTA per row, one element per thread and round.
__global__ void __launch_bounds__(kLpThreads) token_logprobs_grad_kernel(const LogprobGradArgs a) {
  pdl_launch_dependents();
  pdl_wait();
  const int row = blockIdx.x, t = a.tokens[row];
  const bool ok = static_cast<unsigned>(t) < static_cast<unsigned>(a.vocab);
  if (!ok && t != -1 && threadIdx.x == 0) raise_status(a.status, VLA_STATUS_BAD_TOKEN);
  const float inv_t = 1.f / a.temperature, lse = a.lse[row];
  const float g = ok ? a.g_logprob[row] * inv_t : 0.f, h = ok && a.g_entropy ? a.g_entropy[row] * inv_t : 0.f;
  const float entropy = a.entropy ? a.entropy[row] : 0.f;
  for (int j = threadIdx.x; j < a.vocab; j += kLpThreads) {
    float d = 0.f;
    if (ok) {
      const float z = load_as_float(a.logits, row * a.ld + j, a.dtype) * inv_t;
      const float lp = z - lse, p = z == -INFINITY ? 0.f : expf(lp);
      if (z != -INFINITY) d = -p * (g + h * (lp + entropy));
      if (j == t) d += g;
    }
    store_from_float(a.d_logits, row * a.ldd + j, d, a.dtype);
  }
}

}  // namespace

int token_logprobs_launch(const LogprobArgs& a, cudaStream_t s) {
  VLA_CUDA_TRY(launch_pdl(token_logprobs_kernel, dim3(a.rows), dim3(kLpThreads), 0, s, a));
  note_launch();
  VLA_CUDA_TRY(cudaGetLastError());
  return VLA_OK;
}

int token_logprobs_grad_launch(const LogprobGradArgs& a, cudaStream_t s) {
  VLA_CUDA_TRY(launch_pdl(token_logprobs_grad_kernel, dim3(a.rows), dim3(kLpThreads), 0, s, a));
  note_launch();
  VLA_CUDA_TRY(cudaGetLastError());
  return VLA_OK;
}

}  // namespace vla
