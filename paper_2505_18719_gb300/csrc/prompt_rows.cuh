// Sequences by their starts, and what one warp does for one row of packed causal attention, in 32 bits and without matrix instructions: the
// sums of include/vla_learn.h as they stand, over the rows that take part and no others.
#pragma once
#include "learn.h"

namespace vla {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct Span {
  int begin, end;  // rows of a sequence
};
// Starts outside the rows and sequences that end before they begin are clamped (and reported by check_starts).
__device__ __forceinline__ Span span_of(const int* seq_start, int s, int rows) {
  const int b = min(max(seq_start[s], 0), rows);
  return Span{b, min(max(seq_start[s + 1], b), rows)};
}
__device__ __forceinline__ void check_starts(const int* seq_start, int n_seq, int rows, int first, int step, uint32_t* status) {
  bool bad = false;
  for (int s = first; s < n_seq; s += step) bad |= seq_start[s] < 0 || seq_start[s + 1] < seq_start[s] || seq_start[s + 1] > rows;
  if (bad) raise_status(status, VLA_STATUS_SEQUENCES);
}

// HD / 32 channels of a head, lane after lane.
template <int HD>
struct Lane {
  static constexpr int N = HD / 32;
  float x[N];
};
template <int HD, bool FP16>
__device__ __forceinline__ Lane<HD> load_lane(const void* row) {
  Lane<HD> y;
  const uint32_t* p = static_cast<const uint32_t*>(row) + (threadIdx.x & 31) * (HD / 64);
#pragma unroll
  for (int i = 0; i < HD / 64; ++i) {
    const uint32_t w = p[i];
    const float2 f = FP16 ? unpack_f16x2(w) : unpack_bf16x2(w);
    y.x[2 * i] = f.x;
    y.x[2 * i + 1] = f.y;
  }
  return y;
}
template <int HD, bool FP16>
__device__ __forceinline__ void store_lane(void* row, const Lane<HD>& v, float scale) {
  uint32_t* p = static_cast<uint32_t*>(row) + (threadIdx.x & 31) * (HD / 64);
#pragma unroll
  for (int i = 0; i < HD / 64; ++i) {
    const float a = v.x[2 * i] * scale, b = v.x[2 * i + 1] * scale;
    p[i] = FP16 ? pack_f16x2(a, b) : pack_bf16x2(a, b);
  }
}
template <int HD>
__device__ __forceinline__ float lane_dot(const Lane<HD>& a, const Lane<HD>& b) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < Lane<HD>::N; ++i) s = fmaf(a.x[i], b.x[i], s);
  return s;
}
template <int HD>
__device__ __forceinline__ void lane_add(Lane<HD>& y, float p, const Lane<HD>& v) {
#pragma unroll
  for (int i = 0; i < Lane<HD>::N; ++i) y.x[i] = fmaf(p, v.x[i], y.x[i]);
}
__device__ __forceinline__ const void* elem(const void* p, int64_t i) { return static_cast<const uint16_t*>(p) + i; }
__device__ __forceinline__ void* elem(void* p, int64_t i) { return static_cast<uint16_t*>(p) + i; }

// out[row][h] and its lse.  `work` (shared memory) grows every 64 keys.
template <int HD, bool FP16>
__device__ __noinline__ void attend_row(const PromptArgs& a, int row, int h, int first, int* work) {
  constexpr int U = 4;
  const int g = h / (a.n_q_heads / a.n_kv_heads);
  const float c = a.scale * kLog2e;
  const Lane<HD> q = load_lane<HD, FP16>(elem(a.q, row * a.ldq + h * HD));
  Lane<HD> o = {};
  float m = -INFINITY, l = 0.f;
  for (int j0 = first; j0 <= row; j0 += U) {
    if (((j0 - first) & 63) == 0 && (threadIdx.x & 31) == 0) atomicAdd(work, 1);
    Lane<HD> v[U];
    float s[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = min(j0 + u, row);
      s[u] = lane_dot<HD>(q, load_lane<HD, FP16>(elem(a.k, j * a.ldk + g * HD)));
      v[u] = load_lane<HD, FP16>(elem(a.v, j * a.ldv + g * HD));
    }
    float top = m;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      s[u] = warp_sum(s[u]) * c;
      if (j0 + u <= row) top = fmaxf(top, s[u]);
    }
    const float ref = top == -INFINITY ? 0.f : top, alpha = exp2f(m - ref);
    m = top;
    l *= alpha;
#pragma unroll
    for (int i = 0; i < Lane<HD>::N; ++i) o.x[i] *= alpha;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (j0 + u > row) continue;
      const float p = exp2f(s[u] - ref);
      l += p;
      if (p != 0.f) lane_add<HD>(o, p, v[u]);
    }
  }
  store_lane<HD, FP16>(elem(a.out, row * a.ldo + h * HD), o, l > 0.f || l != l ? 1.f / l : 0.f);
  if (a.lse && (threadIdx.x & 31) == 0) a.lse[static_cast<int64_t>(row) * a.n_q_heads + h] = (m + log2f(l)) * kLn2;
}

// Which of `rows` (bits, of the 32 rows from `row` on) that have a channel without a number have it from values behind them, which do not
// count for them: no value that the row sees is without a number in that channel.  The others show what they see, and computing them again would
// take longer for every row the longer the sequence is.  Looks from the sequence's begin on, until all such channels have been seen.
template <int HD, bool FP16>
__device__ __noinline__ uint32_t spoilt_rows(const PromptArgs& a, int row, int h, int first, uint32_t rows, int* work) {
  constexpr int N = Lane<HD>::N, U = 8;
  const int g = h / (a.n_q_heads / a.n_kv_heads), last = row + 31 - __clz(static_cast<int>(rows));
  auto no_number = [](const Lane<HD>& y) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) m |= static_cast<uint32_t>(!(fabsf(y.x[i]) < INFINITY)) << i;
    return m;
  };
  auto of_row = [&](int r) { return no_number(load_lane<HD, FP16>(elem(a.out, (row + r) * a.ldo + h * HD))); };
  uint32_t open = 0;  // channels of this lane that none of the values so far explains
  for (uint32_t rest = rows; rest; rest &= rest - 1) open |= of_row(__ffs(static_cast<int>(rest)) - 1);
  int seen[N];
#pragma unroll
  for (int i = 0; i < N; ++i) seen[i] = 0x7fffffff;
  for (int j0 = first; j0 <= last && __any_sync(0xffffffffu, open != 0); j0 += U) {
    if (((j0 - first) & 63) == 0 && (threadIdx.x & 31) == 0) atomicAdd(work, 1);
    Lane<HD> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = load_lane<HD, FP16>(elem(a.v, min(j0 + u, last) * a.ldv + g * HD));
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t found = no_number(v[u]) & open;
#pragma unroll
      for (int i = 0; i < N; ++i) seen[i] = (found >> i) & 1 ? min(j0 + u, last) : seen[i];
      open &= ~found;
    }
  }
  uint32_t spoilt = 0;
  for (uint32_t rest = rows; rest; rest &= rest - 1) {
    const int r = __ffs(static_cast<int>(rest)) - 1;
    const uint32_t m = of_row(r);
    bool behind = false;
#pragma unroll
    for (int i = 0; i < N; ++i) behind |= (m >> i) & 1 && seen[i] > row + r;
    if (__any_sync(0xffffffffu, behind)) spoilt |= 1u << r;
  }
  return spoilt;
}

}  // namespace vla
