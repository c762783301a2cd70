// What lies between two blocks of a decoder, and its gradient (include/vla_learn.h).
//
// A row is read once and stays in the registers of one CTA.  Forward, with r = 1 / sqrt(mean(.^2) + eps): two sums over the row, one
// behind the other (the second needs the first).  Gradient, with n = h_out r_h, m = y r_y, g = d_x pre_gain:
//   d_h = d_h_out + r_h (g - n c1),  c1 = mean(g n);
//   d_u = residual_scale gate d_h,  d_y = r_y (d_u post_gain - m c2),  c2 = mean(d_u post_gain m).
// c2 is linear in d_h, so with q = residual_scale gate post_gain m both means come from three sums taken together:
//   c2 = mean(q (d_h_out + r_h g)) - c1 mean(q r_h n).
// Column sums (gains, a gate for all rows) stay in registers over a CTA's rows; the CTAs' sums go to the workspace and are added in
// the order of the CTAs by a second kernel.
#include <algorithm>
#include <type_traits>

#include "learn.h"

namespace vla {

namespace {

constexpr int kParts = 304;  // CTAs of the gradient: two an SM

template <class T>
__device__ __forceinline__ float to_f(T x) {
  if constexpr (std::is_same_v<T, float>) return x;
  if constexpr (std::is_same_v<T, f16>) return __half2float(x);
  if constexpr (std::is_same_v<T, bf16>) return __bfloat162float(x);
}
template <class T>
__device__ __forceinline__ T from_f(float x) {
  if constexpr (std::is_same_v<T, float>) return x;
  if constexpr (std::is_same_v<T, f16>) return __float2half_rn(x);
  if constexpr (std::is_same_v<T, bf16>) return __float2bfloat16_rn(x);
}
template <class T>
struct alignas(16) Eight {
  T x[8];
};

// Elements of a row that a thread holds: V consecutive ones at a time (8: 16-byte accesses, or 1).  Past the row: zeros, not stored.
template <int V, int E, class T>
__device__ __forceinline__ void load_row(const T* row, int dim, float (&y)[E]) {
#pragma unroll
  for (int c = 0; c < E / V; ++c) {
    const int i = (c * blockDim.x + threadIdx.x) * V;
    if constexpr (V == 8) {
      Eight<T> w{};
      if (i < dim) w = *reinterpret_cast<const Eight<T>*>(row + i);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[c * 8 + e] = to_f(w.x[e]);
    } else {
      y[c] = i < dim ? to_f(row[i]) : 0.f;
    }
  }
}
template <int V, int E, class T>
__device__ __forceinline__ void store_row(T* row, int dim, const float (&y)[E]) {
#pragma unroll
  for (int c = 0; c < E / V; ++c) {
    const int i = (c * blockDim.x + threadIdx.x) * V;
    if (i >= dim) continue;
    if constexpr (V == 8) {
      Eight<T> w;
#pragma unroll
      for (int e = 0; e < 8; ++e) w.x[e] = from_f<T>(y[c * 8 + e]);
      *reinterpret_cast<Eight<T>*>(row + i) = w;
    } else {
      row[i] = from_f<T>(y[c]);
    }
  }
}

// N sums over the CTA, the same in every thread; `red` is free again after the caller's next barrier.
template <int N>
__device__ __forceinline__ void cta_sums(float (&v)[N], float* red) {
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = warp_sum(v[k]);
  const int warps = blockDim.x >> 5;
  if (warps == 1) return;
  if ((threadIdx.x & 31) == 0) {
#pragma unroll
    for (int k = 0; k < N; ++k) red[k * 32 + (threadIdx.x >> 5)] = v[k];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = warp_sum((threadIdx.x & 31) < warps ? red[k * 32 + (threadIdx.x & 31)] : 0.f);
}

template <class T, class H, int V, int E>
__global__ void __launch_bounds__(E == 8 ? 256 : 512) block_norm_kernel(const BlockNormArgs a) {
  __shared__ float red[2][32];
  const int64_t r = blockIdx.x;
  const int dim = a.dim;
  float h[E], u[E], w[E];
  load_row<V, E>(static_cast<const H*>(a.h) + r * a.ldh, dim, h);
  float r_y = 0.f;
  if (a.y) {
    load_row<V, E>(static_cast<const T*>(a.y) + r * a.ldy, dim, u);
    if (a.post_gain) {
      load_row<V, E>(a.post_gain, dim, w);
      float ss[1] = {0.f};
#pragma unroll
      for (int e = 0; e < E; ++e) ss[0] = fmaf(u[e], u[e], ss[0]);
      cta_sums(ss, red[0]);
      r_y = rsqrtf(ss[0] / static_cast<float>(dim) + a.eps);
#pragma unroll
      for (int e = 0; e < E; ++e) u[e] = u[e] * r_y * w[e];
    }
    if (a.gate) {
      load_row<V, E>(static_cast<const T*>(a.gate) + r * a.ldg, dim, w);
#pragma unroll
      for (int e = 0; e < E; ++e) u[e] *= w[e];
    }
#pragma unroll
    for (int e = 0; e < E; ++e) h[e] = fmaf(a.residual_scale, u[e], h[e]);
    store_row<V, E>(static_cast<H*>(a.h_out) + r * a.ldho, dim, h);
  }
  load_row<V, E>(a.pre_gain, dim, w);
  float ss[1] = {0.f};
#pragma unroll
  for (int e = 0; e < E; ++e) ss[0] = fmaf(h[e], h[e], ss[0]);
  cta_sums(ss, red[1]);
  const float r_h = rsqrtf(ss[0] / static_cast<float>(dim) + a.eps);
#pragma unroll
  for (int e = 0; e < E; ++e) h[e] = h[e] * r_h * w[e];
  store_row<V, E>(static_cast<T*>(a.x) + r * a.ldx, dim, h);
  if (a.rstd && threadIdx.x == 0) {
    a.rstd[2 * r] = r_y;
    a.rstd[2 * r + 1] = r_h;
  }
}

template <class T, class H, int V, int E>
__global__ void __launch_bounds__(E == 8 ? 256 : 512) block_norm_grad_kernel(const BlockNormGradArgs a) {
  __shared__ float red[2][3 * 32];
  pdl_launch_dependents();
  const int dim = a.f.dim;
  const bool post = a.f.post_gain, gated = a.f.gate, own_gate = a.f.ldg != 0;
  float d_pre[E] = {}, d_post[E] = {}, d_gate[E] = {};
  int buf = 0;
  for (int64_t r = blockIdx.x; r < a.f.rows; r += gridDim.x, buf ^= 1) {
    const float r_y = post ? a.f.rstd[2 * r] : 1.f, r_h = a.f.rstd[2 * r + 1];
    float n[E], g[E], d[E], m[E], t[E];
    load_row<V, E>(static_cast<const H*>(a.f.h) + r * a.f.ldh, dim, n);
    load_row<V, E>(static_cast<const T*>(a.d_x) + r * a.lddx, dim, g);
    if (a.d_h_out) {
      load_row<V, E>(static_cast<const H*>(a.d_h_out) + r * a.lddho, dim, d);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) d[e] = 0.f;
    }
    if (a.f.y) load_row<V, E>(static_cast<const T*>(a.f.y) + r * a.f.ldy, dim, m);
    float sum[3] = {0.f, 0.f, 0.f};
    load_row<V, E>(a.f.pre_gain, dim, t);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      n[e] *= r_h;
      d_pre[e] = fmaf(g[e], n[e], d_pre[e]);
      g[e] *= t[e];
      sum[0] = fmaf(g[e], n[e], sum[0]);
      d[e] = fmaf(r_h, g[e], d[e]);
    }
    float q[E];  // residual_scale gate post_gain
    if (post) {
      load_row<V, E>(a.f.post_gain, dim, t);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        q[e] = a.f.residual_scale * t[e];
        m[e] *= r_y;
      }
      if (gated) {
        load_row<V, E>(static_cast<const T*>(a.f.gate) + r * a.f.ldg, dim, t);
#pragma unroll
        for (int e = 0; e < E; ++e) q[e] *= t[e];
      }
#pragma unroll
      for (int e = 0; e < E; ++e) {
        sum[1] = fmaf(q[e] * m[e], d[e], sum[1]);
        sum[2] = fmaf(q[e] * m[e], r_h * n[e], sum[2]);
      }
      cta_sums(sum, red[buf]);
    } else {
      if (a.f.y) {
#pragma unroll
        for (int e = 0; e < E; ++e) q[e] = a.f.residual_scale;
        if (gated) {
          load_row<V, E>(static_cast<const T*>(a.f.gate) + r * a.f.ldg, dim, t);
#pragma unroll
          for (int e = 0; e < E; ++e) q[e] *= t[e];
        }
      }
      float one[1] = {sum[0]};
      cta_sums(one, red[buf]);
      sum[0] = one[0];
    }
    const float inv = 1.f / static_cast<float>(dim), c1 = sum[0] * inv, c2 = (sum[1] - c1 * sum[2]) * inv;
#pragma unroll
    for (int e = 0; e < E; ++e) d[e] = fmaf(-r_h * c1, n[e], d[e]);
    store_row<V, E>(static_cast<H*>(a.d_h) + r * a.lddh, dim, d);
    if (!a.f.y) continue;
    if (gated) {  // d_gate = residual_scale u d_h
      if (post) {
        load_row<V, E>(a.f.post_gain, dim, t);
#pragma unroll
        for (int e = 0; e < E; ++e) t[e] *= m[e];
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) t[e] = m[e];
      }
#pragma unroll
      for (int e = 0; e < E; ++e) {
        t[e] *= a.f.residual_scale * d[e];
        d_gate[e] += t[e];
      }
      if (own_gate) store_row<V, E>(static_cast<T*>(a.d_gate) + r * a.lddg, dim, t);
    }
    if (post) {
      if (gated) {
        load_row<V, E>(static_cast<const T*>(a.f.gate) + r * a.f.ldg, dim, t);
#pragma unroll
        for (int e = 0; e < E; ++e) t[e] *= a.f.residual_scale;
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) t[e] = a.f.residual_scale;
      }
#pragma unroll
      for (int e = 0; e < E; ++e) {
        d_post[e] = fmaf(t[e] * d[e], m[e], d_post[e]);
        d[e] = r_y * fmaf(q[e], d[e], -m[e] * c2);
      }
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) d[e] *= q[e];
    }
    store_row<V, E>(static_cast<T*>(a.d_y) + r * a.lddy, dim, d);
  }
  float* part = a.workspace + static_cast<int64_t>(blockIdx.x) * 3 * dim;
  auto keep = [&](int k, const float(&v)[E]) {
#pragma unroll
    for (int c = 0; c < E / V; ++c) {
      const int i = (c * blockDim.x + threadIdx.x) * V;
      if (i >= dim) continue;
#pragma unroll
      for (int e = 0; e < V; ++e) part[k * static_cast<int64_t>(dim) + i + e] = v[c * V + e];
    }
  };
  keep(0, d_pre);
  if (post) keep(1, d_post);
  if (gated && !own_gate) keep(2, d_gate);
}

struct ColumnSums {
  const float* parts;  // [n][3][dim]
  int n, dim;
  float* out[3];       // or null
};
__global__ void __launch_bounds__(256) column_sums_kernel(const ColumnSums a) {
  __shared__ float red[8][33];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int i = blockIdx.x * 32 + lane, k = blockIdx.y;
  pdl_wait();
  if (!a.out[k]) return;
  float s = 0.f;
  if (i < a.dim) {
#pragma unroll 8
    for (int p = w; p < a.n; p += 8) s += __ldcg(a.parts + (static_cast<int64_t>(p) * 3 + k) * a.dim + i);
  }
  red[w][lane] = s;
  __syncthreads();
  if (w || i >= a.dim) return;
#pragma unroll
  for (int j = 1; j < 8; ++j) s += red[j][lane];
  a.out[k][i] = s;
}

// 16-byte accesses to every row?
bool wide(const void* p, int64_t ld) {
  return !p || (!(reinterpret_cast<uintptr_t>(p) & 15) && (ld & 7) == 0);
}

// Elements of a thread: 8 up to 2048 channels, 16 up to 8192 (three sums, four inputs: 108 registers), else 32; threads for one row.
int per_thread(int dim) { return dim <= 2048 ? 8 : dim <= 8192 ? 16 : 32; }
unsigned threads_for(int dim) { return static_cast<unsigned>(std::max(32, (dim + per_thread(dim) * 32 - 1) / (per_thread(dim) * 32) * 32)); }

// f(act type, stream type, vector, elements)
template <class F>
int dispatch(int dtype, int h_dtype, bool vec, int dim, const F& f) {
  auto shape = [&](auto t, auto h) {
    if (per_thread(dim) == 8)
      return vec ? f(t, h, std::integral_constant<int, 8>(), std::integral_constant<int, 8>())
                 : f(t, h, std::integral_constant<int, 1>(), std::integral_constant<int, 8>());
    if (per_thread(dim) == 16)
      return vec ? f(t, h, std::integral_constant<int, 8>(), std::integral_constant<int, 16>())
                 : f(t, h, std::integral_constant<int, 1>(), std::integral_constant<int, 16>());
    return vec ? f(t, h, std::integral_constant<int, 8>(), std::integral_constant<int, 32>())
               : f(t, h, std::integral_constant<int, 1>(), std::integral_constant<int, 32>());
  };
  if (dtype == VLA_F32) return shape(float(), float());
  if (dtype == VLA_F16) return h_dtype == VLA_F32 ? shape(f16(), float()) : shape(f16(), f16());
  return h_dtype == VLA_F32 ? shape(bf16(), float()) : shape(bf16(), bf16());
}

}  // namespace

int block_norm_launch(const BlockNormArgs& a, cudaStream_t s) {
  const bool vec = a.dim % 8 == 0 && wide(a.y, a.ldy) && wide(a.h, a.ldh) && wide(a.gate, a.ldg) && wide(a.post_gain, 0) &&
                   wide(a.pre_gain, 0) && wide(a.h_out, a.ldho) && wide(a.x, a.ldx);
  return dispatch(a.dtype, a.h_dtype, vec, a.dim, [&](auto t, auto h, auto v, auto e) -> int {
    VLA_CUDA_TRY(launch_at(Start::kInOrder, block_norm_kernel<decltype(t), decltype(h), v(), e()>, dim3(static_cast<unsigned>(a.rows)),
                           dim3(threads_for(a.dim)), 0, s, a));
    note_launch();
    return VLA_OK;
  });
}

size_t block_norm_grad_workspace(int rows, int dim) { return static_cast<size_t>(std::max(1, std::min(rows, kParts))) * 3 * dim * sizeof(float); }

int block_norm_grad_launch(const BlockNormGradArgs& a, cudaStream_t s) {
  const BlockNormArgs& f = a.f;
  const int parts = std::min(f.rows, kParts);
  if (parts > 0) {
    const bool vec = f.dim % 8 == 0 && wide(f.y, f.ldy) && wide(f.h, f.ldh) && wide(f.gate, f.ldg) &&
                     wide(f.post_gain, 0) && wide(f.pre_gain, 0) && wide(a.d_x, a.lddx) && wide(a.d_h_out, a.lddho) &&
                     wide(a.d_h, a.lddh) && wide(a.d_y, a.lddy) && (!f.ldg || wide(a.d_gate, a.lddg));
    const int rc = dispatch(f.dtype, f.h_dtype, vec, f.dim, [&](auto t, auto h, auto v, auto e) -> int {
      VLA_CUDA_TRY(launch_at(Start::kInOrder, block_norm_grad_kernel<decltype(t), decltype(h), v(), e()>, dim3(static_cast<unsigned>(parts)),
                             dim3(threads_for(f.dim)), 0, s, a));
      note_launch();
      return VLA_OK;
    });
    if (rc) return rc;
  }
  const ColumnSums c{a.workspace, parts, f.dim, {a.d_pre_gain, a.d_post_gain, f.gate && !f.ldg ? static_cast<float*>(a.d_gate) : nullptr}};
  VLA_CUDA_TRY(launch_pdl(column_sums_kernel, dim3(static_cast<unsigned>((f.dim + 31) / 32), 3), dim3(256), 0, s, c));
  note_launch();
  return VLA_OK;
}

}  // namespace vla
