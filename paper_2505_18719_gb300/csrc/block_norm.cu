// What lies between two blocks of a decoder, and its gradient (include/vla_learn.h).
//
// Forward, with r = 1 / sqrt(mean(.^2) + eps): two sums over the row, one behind the other (the second needs the first); a row is read
// once and stays in the registers of one CTA (of one warp up to 256 channels, 8 rows a CTA).  Gradient, with n = h_out r_h, m = y r_y,
// g = d_x pre_gain:
//   d_h = d_h_out + r_h (g - n c1),  c1 = mean(g n);
//   d_u = residual_scale gate d_h,  d_y = r_y (d_u post_gain - m c2),  c2 = mean(d_u post_gain m).
// c2 is linear in d_h, so with q = residual_scale gate post_gain m both means come from three sums taken together:
//   c2 = mean(q (d_h_out + r_h g)) - c1 mean(q r_h n).
// A CTA takes every n-th row; the next one comes to shared memory by bulk copies while it works at this one.  Short rows stay in registers between the
// sums and the outputs (8 elements a thread: a row of 1155 by single elements, 2311 of them, 24 us where reading shared memory again took 65),
// longer ones are read from shared memory twice.  Column sums (gains, a gate for all rows) stay in registers over a CTA's rows; the CTAs' sums
// go to the workspace and are added in the order of the CTAs by a second kernel, which waits for the first already started.
//
// Bound by HBM: 18385 rows of 4096, bf16 blocks and a fp32 stream, norm and gate behind the block: forward 141 us (6.4 TB/s, 0.95 of the copy
// rate), gradient 262 us (5.2 TB/s; 342 without the copies ahead); 448 rows: 17 us, of which the second kernel and the start are half.
#include <algorithm>
#include <type_traits>

#include "learn.h"
#include "ptx.cuh"
#include "row_copy.h"

namespace vla {

namespace {

// CTAs of the gradient, each a share of the rows: as many as the registers of 152 SMs hold at once (512 threads of 128 registers an SM, and 8 elements a
// thread up to 2048 channels, 16 up to 4096); a share more than that waits for a second round.  18385 rows of 1152, 1280 and 1400 channels: with 2 a
// SM 122, 126, 133 us, with 3 95, 99, 165 (192 threads do not fit three times), with 4 131, 135, 138.  The number is a GB300's whatever
// the device, for the workspace's size goes by it.
int parts_of(int rows, int dim) { return std::min(rows, 152 * (dim <= 256 ? 16 : dim <= 512 ? 8 : dim <= 1024 ? 4 : dim <= 1280 ? 3 : dim <= 4096 ? 2 : 1)); }
uint32_t staged_limit(int dim) { return dim <= 4096 ? 100 * 1024 : 200 * 1024; }  // of two rows of each of those CTAs

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
template <class T, int V>
struct alignas(V * sizeof(T) < 16 ? V * sizeof(T) : 16) Some {
  T x[V];
};

// Elements of a row that a thread holds: V consecutive ones at a time (8: 16-byte accesses, 2, or 1).  Past the row: zeros, not stored.
template <int V, int E, class T>
__device__ __forceinline__ void load_row(const T* row, int dim, float (&y)[E]) {
#pragma unroll
  for (int c = 0; c < E / V; ++c) {
    const int i = (c * blockDim.x + threadIdx.x) * V;
    Some<T, V> w{};
    if (i < dim) w = *reinterpret_cast<const Some<T, V>*>(row + i);
#pragma unroll
    for (int e = 0; e < V; ++e) y[c * V + e] = to_f(w.x[e]);
  }
}
template <int V, int E, class T>
__device__ __forceinline__ void store_row(T* row, int dim, const float (&y)[E]) {
#pragma unroll
  for (int c = 0; c < E / V; ++c) {
    const int i = (c * blockDim.x + threadIdx.x) * V;
    if (i >= dim) continue;
    Some<T, V> w;
#pragma unroll
    for (int e = 0; e < V; ++e) w.x[e] = from_f<T>(y[c * V + e]);
    *reinterpret_cast<Some<T, V>*>(row + i) = w;
  }
}

template <int V, class T>
__device__ __forceinline__ void load_some(const T* p, float (&y)[V]) {
  const Some<T, V> w = *reinterpret_cast<const Some<T, V>*>(p);
#pragma unroll
  for (int e = 0; e < V; ++e) y[e] = to_f(w.x[e]);
}
// An element from shared memory.
template <class T>
__device__ __forceinline__ float load_shared(uint32_t at) {
  if constexpr (sizeof(T) == 2) {
    uint16_t w;
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(w) : "r"(at));
    return std::is_same_v<T, f16> ? __half2float(__ushort_as_half(w)) : __bfloat162float(__ushort_as_bfloat16(w));
  } else {
    float y;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(y) : "r"(at));
    return y;
  }
}
template <int V, class T>
__device__ __forceinline__ void store_some(T* p, const float (&y)[V]) {
  Some<T, V> w;
#pragma unroll
  for (int e = 0; e < V; ++e) w.x[e] = from_f<T>(y[e]);
  *reinterpret_cast<Some<T, V>*>(p) = w;
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
__global__ void __launch_bounds__(E == 8 && V < 8 ? 1024 : 512) block_norm_kernel(const BlockNormArgs a) {
  __shared__ float red[2][32];
  pdl_launch_dependents();
  pdl_wait();
  const int64_t r = E == 8 ? static_cast<int64_t>(blockIdx.x) * blockDim.y + threadIdx.y : blockIdx.x;  // (rows of one warp: several a CTA)
  const int dim = a.dim;
  if (r >= a.rows) return;
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

// Rows on their way through shared memory: two, each its h_out, d_x, d_h_out, y and gate behind one another.  A row that does not begin or end on
// a 16-byte boundary comes with the bytes around it up to the next, as far as its tensor has them (row_copy).
struct Stage {
  uint32_t at[5], bytes;  // offsets of the five, of the next row
};
__host__ __device__ inline Stage stage_of(int dim, int act, int stream, bool d_h_out, bool y, bool gate) {
  Stage s{};
  const int size[5] = {stream, act, d_h_out ? stream : 0, y ? act : 0, gate ? act : 0};
  for (int k = 0; k < 5; ++k) {
    s.at[k] = s.bytes;
    s.bytes += size[k] ? (static_cast<uint32_t>(dim * size[k]) + 31u) & ~15u : 0u;
  }
  return s;
}

template <class T, class H, int V, int E, bool STAGED>
__global__ void __launch_bounds__(E == 8 && V == 8 ? 256 : 512, E == 8 && V == 8 ? 2 : 1) block_norm_grad_kernel(const BlockNormGradArgs a) {
  __shared__ float red[2][3 * 32];
  __shared__ uint64_t full[2];
  extern __shared__ uint8_t rows_raw[];
  pdl_launch_dependents();
  if constexpr (STAGED) pdl_wait_async(); else pdl_wait();
  const int dim = a.f.dim;
  const bool post = a.f.post_gain, gated = a.f.gate, own_gate = a.f.ldg != 0;
  const Stage st = stage_of(dim, sizeof(T), sizeof(H), a.d_h_out, a.f.y, gated && own_gate);
  uint8_t* stages = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(rows_raw) + 15) & ~static_cast<uintptr_t>(15));
  const void* const base[5] = {a.f.h, a.d_x, a.d_h_out, a.f.y, own_gate ? a.f.gate : nullptr};
  const int64_t ld[5] = {a.f.ldh * static_cast<int64_t>(sizeof(H)), a.lddx * static_cast<int64_t>(sizeof(T)),
                         a.lddho * static_cast<int64_t>(sizeof(H)), a.f.ldy * static_cast<int64_t>(sizeof(T)),
                         a.f.ldg * static_cast<int64_t>(sizeof(T))};
  // A tensor's first and last rows, of which bytes around them may lie outside it (rows for 16-byte accesses have none around them).
  const int ends = V < 8 ? (8 + dim - 1) / dim : 0;
  auto is_end = [&](int64_t r) { return V < 8 && (r < ends || r >= a.f.rows - ends); };
  auto copy_of = [&](int64_t r, int k) {
    const uint32_t n = static_cast<uint32_t>(dim) * (k == 0 || k == 2 ? sizeof(H) : sizeof(T));
    const uintptr_t lo = reinterpret_cast<uintptr_t>(base[k]);
    return row_copy(lo + static_cast<uintptr_t>(r * ld[k]), n, lo, lo + static_cast<uintptr_t>((a.f.rows - 1) * ld[k]) + n);
  };
  auto request = [&](int64_t r, int s) {  // one thread
    const uint32_t bar = smem_u32(full + s), to = smem_u32(stages + s * st.bytes);
    if (is_end(r)) {
      uint32_t total = 0;
#pragma unroll
      for (int k = 0; k < 5; ++k) total += base[k] ? copy_of(r, k).bytes : 0u;
      mbar_arrive_expect_tx(bar, total);
#pragma unroll
      for (int k = 0; k < 5; ++k) {
        if (!base[k]) continue;
        const RowCopy c = copy_of(r, k);
        const uintptr_t p = reinterpret_cast<uintptr_t>(base[k]) + static_cast<uintptr_t>(r * ld[k]);
        if (c.bytes) bulk_load(to + st.at[k] + static_cast<uint32_t>(c.from - (p & ~static_cast<uintptr_t>(15))), reinterpret_cast<const void*>(c.from), c.bytes, bar);
      }
      return;
    }
    uint32_t total = 0, bytes[5];
    uintptr_t from[5];
#pragma unroll
    for (int k = 0; k < 5; ++k) {
      const uintptr_t p = reinterpret_cast<uintptr_t>(base[k]) + static_cast<uintptr_t>(r * ld[k]);
      const uintptr_t end = (p + static_cast<uint32_t>(dim) * (k == 0 || k == 2 ? sizeof(H) : sizeof(T)) + 15) & ~static_cast<uintptr_t>(15);
      from[k] = p & ~static_cast<uintptr_t>(15);
      bytes[k] = base[k] ? static_cast<uint32_t>(end - from[k]) : 0u;
      total += bytes[k];
    }
    mbar_arrive_expect_tx(bar, total);
#pragma unroll
    for (int k = 0; k < 5; ++k)
      if (bytes[k]) bulk_load(to + st.at[k], reinterpret_cast<const void*>(from[k]), bytes[k], bar);
  };
  // What a request leaves out of such a row, 2 bytes a thread (8 threads its begin, 8 its end), by the whole CTA.
  auto add_ends = [&](int64_t r, int s) {
    uint16_t w[5] = {};
    uint32_t at[5];
    const uint32_t i = 2 * (threadIdx.x & 7);
#pragma unroll
    for (int k = 0; k < 5; ++k) {
      at[k] = ~0u;
      if (!base[k] || threadIdx.x >= 16) continue;
      const RowCopy c = copy_of(r, k);
      if (i >= (threadIdx.x < 8 ? c.head : c.tail)) continue;
      at[k] = threadIdx.x < 8 ? i : static_cast<uint32_t>(dim) * (k == 0 || k == 2 ? sizeof(H) : sizeof(T)) - c.tail + i;
      w[k] = *reinterpret_cast<const uint16_t*>(static_cast<const uint8_t*>(base[k]) + r * ld[k] + at[k]);
    }
#pragma unroll
    for (int k = 0; k < 5; ++k) {
      const uint32_t row = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(base[k]) + static_cast<uintptr_t>(r * ld[k])) & 15;
      if (at[k] != ~0u)
        asm volatile("st.shared.u16 [%0], %1;" ::"r"(smem_u32(stages + s * st.bytes + st.at[k]) + row + at[k]), "h"(w[k]) : "memory");
    }
    __syncthreads();
  };
  if constexpr (STAGED) {
    if (threadIdx.x == 0) {
      mbar_init(smem_u32(full), 1);
      mbar_init(smem_u32(full + 1), 1);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
      if (static_cast<int>(blockIdx.x) < a.f.rows) request(blockIdx.x, 0);
    }
    __syncthreads();
  }
  float d_pre[E] = {}, d_post[E] = {}, d_gate[E] = {};
  float w_pre[E == 8 ? E : 1], w_post[E == 8 ? E : 1];
  if constexpr (E == 8) {
#pragma unroll
    for (int c = 0; c < E / V; ++c) {
      const int i = min(static_cast<int>((c * blockDim.x + threadIdx.x) * V), dim - V);
      float x[V];
      load_some<V>(a.f.pre_gain + i, x);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        w_pre[c * V + e] = x[e];
        x[e] = 1.f;
      }
      if (post) load_some<V>(a.f.post_gain + i, x);
#pragma unroll
      for (int e = 0; e < V; ++e) w_post[c * V + e] = x[e];
    }
  }
  int n_rows = 0;
  for (int64_t r = blockIdx.x; r < a.f.rows; r += gridDim.x, ++n_rows) {
    const int buf = n_rows & 1;
    const float r_y = post ? a.f.rstd[2 * r] : 1.f, r_h = a.f.rstd[2 * r + 1];
    const uint8_t* row[5];
#pragma unroll
    for (int k = 0; k < 5; ++k) {
      row[k] = reinterpret_cast<const uint8_t*>(base[k]) + r * ld[k];
      if (STAGED) row[k] = stages + buf * st.bytes + st.at[k] + (reinterpret_cast<uintptr_t>(row[k]) & 15);
    }
    // element i of the row's h_out, d_x, d_h_out, y or gate of its own
    auto load = [&](auto type, int k, int i, float(&y)[V]) {
      using X = decltype(type);
      if constexpr (STAGED && V == 1)
        y[0] = load_shared<X>(smem_u32(row[k]) + static_cast<uint32_t>(i * sizeof(X)));
      else
        load_some<V>(reinterpret_cast<const X*>(row[k]) + i, y);
    };
    auto load_gate = [&](int i, float(&y)[V]) {
      if (own_gate)
        load(T(), 4, i, y);
      else
        load_some<V>(static_cast<const T*>(a.f.gate) + i, y);
    };
    if constexpr (STAGED) {
      if (!mbar_try_wait(smem_u32(full + buf), (n_rows >> 1) & 1) &&
          !wait_drain_reported(smem_u32(full + buf), (n_rows >> 1) & 1, a.status, a.wait_limit))
        break;
      if (is_end(r)) add_ends(r, buf);
    }
    if constexpr (E == 8) {  // values and gains of a short row stay in registers
      float n[E], g[E], d[E], m[E], q[E], sum[3] = {0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < E / V; ++c) {
        const int own = (c * blockDim.x + threadIdx.x) * V, i = min(own, dim - V);
        const bool on = own < dim;
        float x[V];
        load(H(), 0, i, x);
#pragma unroll
        for (int e = 0; e < V; ++e) n[c * V + e] = on ? x[e] * r_h : 0.f;
        load(T(), 1, i, x);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          d_pre[c * V + e] = fmaf(x[e], n[c * V + e], d_pre[c * V + e]);
          g[c * V + e] = on ? x[e] * w_pre[c * V + e] : 0.f;
          x[e] = 0.f;
        }
        if (a.d_h_out) load(H(), 2, i, x);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          sum[0] = fmaf(g[c * V + e], n[c * V + e], sum[0]);
          d[c * V + e] = on ? fmaf(r_h, g[c * V + e], x[e]) : 0.f;
          x[e] = 0.f;
        }
        if (a.f.y) load(T(), 3, i, x);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          m[c * V + e] = on ? x[e] * r_y : 0.f;
          x[e] = 1.f;
        }
        if (gated) load_gate(i, x);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          g[c * V + e] = x[e];
          q[c * V + e] = a.f.residual_scale * x[e] * w_post[c * V + e];
        }
        if (post) {
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const float z = on ? q[c * V + e] * m[c * V + e] : 0.f;
            sum[1] = fmaf(z, d[c * V + e], sum[1]);
            sum[2] = fmaf(z, r_h * n[c * V + e], sum[2]);
          }
        }
      }
      cta_sums(sum, red[buf]);
      if constexpr (STAGED) {
        __syncwarp();
        if (threadIdx.x == 0 && r + gridDim.x < a.f.rows) request(r + gridDim.x, buf ^ 1);
      }
      const float inv = 1.f / static_cast<float>(dim), c1 = sum[0] * inv, c2 = (sum[1] - c1 * sum[2]) * inv;
#pragma unroll
      for (int c = 0; c < E / V; ++c) {
        const int i = (c * blockDim.x + threadIdx.x) * V;
        if (i >= dim) continue;
        float x[V], z[V];
#pragma unroll
        for (int e = 0; e < V; ++e) x[e] = fmaf(-r_h * c1, n[c * V + e], d[c * V + e]);
        store_some<V>(static_cast<H*>(a.d_h) + r * a.lddh + i, x);
        if (!a.f.y) continue;
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float y = a.f.residual_scale * x[e] * m[c * V + e];  // times post_gain: d_gate
          z[e] = y * w_post[c * V + e];
          d_gate[c * V + e] += z[e];
          d_post[c * V + e] = fmaf(y, g[c * V + e], d_post[c * V + e]);
          x[e] = post ? r_y * fmaf(q[c * V + e], x[e], -m[c * V + e] * c2) : q[c * V + e] * x[e];
        }
        if (gated && own_gate) store_some<V>(static_cast<T*>(a.d_gate) + r * a.lddg + i, z);
        store_some<V>(static_cast<T*>(a.d_y) + r * a.lddy + i, x);
      }
      continue;
    }
    float sum[3] = {0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < E / V; ++c) {
      // (past the row: its last channels again, without effect)
      const int own = (c * blockDim.x + threadIdx.x) * V, i = min(own, dim - V);
      const bool on = own < dim;
      float n[V], g[V], w[V];
      load(H(), 0, i, n);
      load(T(), 1, i, g);
      load_some<V>(a.f.pre_gain + i, w);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        n[e] *= r_h;
        g[e] = on ? g[e] : 0.f;
        d_pre[c * V + e] = fmaf(g[e], n[e], d_pre[c * V + e]);
        g[e] *= w[e];
        sum[0] = fmaf(g[e], n[e], sum[0]);
      }
      if (!post) continue;
      float m[V], q[V];
      load(T(), 3, i, m);
      load_some<V>(a.f.post_gain + i, q);
#pragma unroll
      for (int e = 0; e < V; ++e) q[e] = on ? q[e] * (a.f.residual_scale * r_y * m[e]) : 0.f;
      if (gated) {
        load_gate(i, w);
#pragma unroll
        for (int e = 0; e < V; ++e) q[e] *= w[e];
      }
      if (a.d_h_out) {
        load(H(), 2, i, w);
#pragma unroll
        for (int e = 0; e < V; ++e) g[e] = fmaf(r_h, g[e], w[e]);
      } else {
#pragma unroll
        for (int e = 0; e < V; ++e) g[e] *= r_h;
      }
#pragma unroll
      for (int e = 0; e < V; ++e) {
        sum[1] = fmaf(q[e], g[e], sum[1]);
        sum[2] = fmaf(q[e], r_h * n[e], sum[2]);
      }
    }
    cta_sums(sum, red[buf]);
    if constexpr (STAGED) {
      __syncwarp();
      // (the row before, in the other stage, is done with: all threads have come to these sums)
      if (threadIdx.x == 0 && r + gridDim.x < a.f.rows) request(r + gridDim.x, buf ^ 1);
    }
    const float inv = 1.f / static_cast<float>(dim), c1 = sum[0] * inv, c2 = (sum[1] - c1 * sum[2]) * inv;
#pragma unroll
    for (int c = 0; c < E / V; ++c) {
      // (past the row: its last channels again, without effect)
      const int own = (c * blockDim.x + threadIdx.x) * V, i = min(own, dim - V);
      const bool on = own < dim;
      float d[V], n[V], w[V];
      load(T(), 1, i, d);
      load_some<V>(a.f.pre_gain + i, w);
      load(H(), 0, i, n);
#pragma unroll
      for (int e = 0; e < V; ++e) d[e] = r_h * fmaf(-r_h * n[e], c1, d[e] * w[e]);
      if (a.d_h_out) {
        load(H(), 2, i, w);
#pragma unroll
        for (int e = 0; e < V; ++e) d[e] += w[e];
      }
      if (on) store_some<V>(static_cast<H*>(a.d_h) + r * a.lddh + i, d);
      if (!a.f.y) continue;
      float m[V];
      load(T(), 3, i, m);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        d[e] *= a.f.residual_scale;
        m[e] *= r_y;  // (1 without post_gain)
        w[e] = 1.f;
      }
      if (post) load_some<V>(a.f.post_gain + i, w);
      if (gated) {  // d_gate = residual_scale d_h u
#pragma unroll
        for (int e = 0; e < V; ++e) {
          n[e] = d[e] * m[e] * w[e];
          d_gate[c * V + e] += n[e];
        }
        if (own_gate && on) store_some<V>(static_cast<T*>(a.d_gate) + r * a.lddg + i, n);
        load_gate(i, n);
#pragma unroll
        for (int e = 0; e < V; ++e) d[e] *= n[e];
      }
      if (post) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
          d_post[c * V + e] = fmaf(d[e], m[e], d_post[c * V + e]);
          d[e] = r_y * fmaf(w[e], d[e], -m[e] * c2);
        }
      }
      if (on) store_some<V>(static_cast<T*>(a.d_y) + r * a.lddy + i, d);
    }
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
// 32 columns a CTA, every 32nd part a warp, 10 to 30 loads in flight a thread.
__global__ void __launch_bounds__(1024) column_sums_kernel(const ColumnSums a) {
  __shared__ float red[32][33];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int i = blockIdx.x * 32 + lane, k = blockIdx.y;
  if (!a.out[k]) return;
  pdl_wait();
  float s = 0.f;
  if (i < a.dim) {
#pragma unroll 10
    for (int p = w; p < a.n; p += 32) s += __ldcg(a.parts + (static_cast<int64_t>(p) * 3 + k) * a.dim + i);
  }
  red[w][lane] = s;
  __syncthreads();
  s = warp_sum(red[lane][w]);
  const int j = blockIdx.x * 32 + w;
  if (lane == 0 && j < a.dim) a.out[k][j] = s;
}

// What accesses every row allows: 8 elements (16 bytes), 2 (one access of their 4 or 8 bytes), or 1.
struct Reach {
  int v;
  explicit Reach(int dim) : v(dim % 8 == 0 ? 8 : dim % 2 == 0 ? 2 : 1) {}
  void rows(const void* p, int64_t ld, int dtype) {
    const int size = dtype == VLA_F32 ? 4 : 2;
    if (!p) return;
    if (v == 8 && ((reinterpret_cast<uintptr_t>(p) & 15) || (ld & 7))) v = 2;
    if (v == 2 && ((reinterpret_cast<uintptr_t>(p) & static_cast<uintptr_t>(2 * size - 1)) || (ld & 1))) v = 1;
  }
};

// Elements of a thread and threads of a row.  With 16-byte accesses 8 elements up to 2048 channels, 16 up to 8192 (62 registers, 120 in the gradient
// with its three sums), else 32.  With smaller ones latency counts: 8 as long as the threads of a row fit a CTA (`most`); 9000 rows of 4100
// channels, accesses of 2 elements, take 85 us so, 225 with 16 elements and accesses of one.
struct Split {
  int e;
  unsigned threads;
};
Split split_of(int dim, int v, int most) {
  const int e = dim <= (v == 8 ? 2048 : most * 8) ? 8 : dim <= 8192 ? 16 : 32;
  return {e, static_cast<unsigned>((dim + e * 32 - 1) / (e * 32) * 32)};
}

// f(act type, stream type, vector, elements)
template <class F>
int dispatch(int dtype, int h_dtype, int vec, int e, const F& f) {
  auto elements = [&](auto t, auto h, auto v) {
    if (e == 8) return f(t, h, v, std::integral_constant<int, 8>());
    return e == 16 ? f(t, h, v, std::integral_constant<int, 16>()) : f(t, h, v, std::integral_constant<int, 32>());
  };
  auto shape = [&](auto t, auto h) {
    if (vec == 8) return elements(t, h, std::integral_constant<int, 8>());
    return vec == 2 ? elements(t, h, std::integral_constant<int, 2>()) : elements(t, h, std::integral_constant<int, 1>());
  };
  if (dtype == VLA_F32) return shape(float(), float());
  if (dtype == VLA_F16) return h_dtype == VLA_F32 ? shape(f16(), float()) : shape(f16(), f16());
  return h_dtype == VLA_F32 ? shape(bf16(), float()) : shape(bf16(), bf16());
}

}  // namespace

int block_norm_launch(const BlockNormArgs& a, cudaStream_t s) {
  Reach reach(a.dim);
  reach.rows(a.y, a.ldy, a.dtype);
  reach.rows(a.h, a.ldh, a.h_dtype);
  reach.rows(a.gate, a.ldg, a.dtype);
  reach.rows(a.post_gain, 0, VLA_BF16);
  reach.rows(a.pre_gain, 0, VLA_BF16);
  reach.rows(a.h_out, a.ldho, a.h_dtype);
  reach.rows(a.x, a.ldx, a.dtype);
  const Split split = split_of(a.dim, reach.v, 1024);
  const unsigned rows = split.threads == 32 ? 8 : 1;  // of a CTA
  return dispatch(a.dtype, a.h_dtype, reach.v, split.e, [&](auto t, auto h, auto v, auto e) -> int {
    VLA_CUDA_TRY(launch_pdl(block_norm_kernel<decltype(t), decltype(h), v(), e()>, dim3((static_cast<unsigned>(a.rows) + rows - 1) / rows),
                            dim3(split.threads, rows), 0, s, a));
    note_launch();
    return VLA_OK;
  });
}

size_t block_norm_grad_workspace(int rows, int dim) { return static_cast<size_t>(std::max(1, parts_of(rows, dim))) * 3 * dim * sizeof(float); }

int block_norm_grad_launch(const BlockNormGradArgs& a, cudaStream_t s) {
  const BlockNormArgs& f = a.f;
  const int parts = parts_of(f.rows, f.dim);
  if (parts > 0) {
    Reach reach(f.dim);
    reach.rows(f.y, f.ldy, f.dtype);
    reach.rows(f.h, f.ldh, f.h_dtype);
    reach.rows(f.gate, f.ldg, f.dtype);
    reach.rows(f.post_gain, 0, VLA_BF16);
    reach.rows(f.pre_gain, 0, VLA_BF16);
    reach.rows(a.d_x, a.lddx, f.dtype);
    reach.rows(a.d_h_out, a.lddho, f.h_dtype);
    reach.rows(a.d_h, a.lddh, f.h_dtype);
    reach.rows(a.d_y, a.lddy, f.dtype);
    if (f.ldg) reach.rows(a.d_gate, a.lddg, f.dtype);
    const Split split = split_of(f.dim, reach.v, 512);
    const int rc = dispatch(f.dtype, f.h_dtype, reach.v, split.e, [&](auto t, auto h, auto v, auto e) -> int {
      const uint32_t staged = 2 * stage_of(f.dim, sizeof(t), sizeof(h), a.d_h_out, f.y, f.gate && f.ldg).bytes + 16;
      if (staged <= staged_limit(f.dim)) {
        const auto kern = block_norm_grad_kernel<decltype(t), decltype(h), v(), e(), true>;
        static std::atomic<uint64_t> done{0};
        VLA_CUDA_TRY(set_smem_limit(kern, 200 * 1024, done));
        VLA_CUDA_TRY(launch_pdl(kern, dim3(static_cast<unsigned>(parts)), dim3(split.threads), staged, s, a));
      } else {
        VLA_CUDA_TRY(launch_pdl(block_norm_grad_kernel<decltype(t), decltype(h), v(), e(), false>, dim3(static_cast<unsigned>(parts)),
                               dim3(split.threads), 0, s, a));
      }
      note_launch();
      return VLA_OK;
    });
    if (rc) return rc;
  }
  const ColumnSums c{a.workspace, parts, f.dim, {a.d_pre_gain, a.d_post_gain, f.gate && !f.ldg ? static_cast<float*>(a.d_gate) : nullptr}};
  VLA_CUDA_TRY(launch_pdl(column_sums_kernel, dim3(static_cast<unsigned>((f.dim + 31) / 32), 3), dim3(1024), 0, s, c));
  note_launch();
  return VLA_OK;
}

}  // namespace vla
