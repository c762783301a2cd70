// Log-probs of given tokens with entropy and the best alternatives, and their gradient.
//
// Forward, one row of logits z, in powers of two: with c = log2(e) / T, any reference r near the largest z c,
// s = sum 2^(z c - r) and w = sum (z c - r) 2^(z c - r), log p_j = ln 2 (z_j c - r - log2 s), lse = ln 2 (r + log2 s) and the entropy is
// ln 2 (log2 s - w / s).  One pass with a running reference per thread (a sum relative to r goes over to r' by s' = f s,
// w' = f (w + (r - r') s), f = 2^(r - r')).  The reference is the rounded product of the maximum and c and every z c - r
// one fma, exact up to its own size: logits far from zero lose nothing while |r| is below 2^24.  (Rows beyond, such as one of
// nothing but a type's lowest values, are read again with the difference to the maximum taken first.)  Bound by reading the
// logits, for 16-bit types nearly as much by issuing 5 instructions an element (two elements share an fma, an addition and an
// fma): 3584 x 32064 bf16 take 38 us (6.0 TB/s, 0.88 of the copy rate), 45 with 4 alternatives.
//
// The best alternatives come from the same pass: each thread's maximum is known, and the k-th largest maximum over
// disjoint groups of threads is a bound that at least k logits reach.  Only threads whose maximum reaches it read
// logits again (from L2), and only those rounds of the pass whose maximum, kept in shared memory, reaches it too; what
// lies above the bound is ranked by counting.  That is a chain of some 3 us a row, which the rows on an SM do at about the same
// time; 64 x 32064 fp32 take 6.5 us with 8 alternatives and 3.8 without.
#include <algorithm>
#include <type_traits>

#include "lm.h"
#include "ptx.cuh"

namespace vla {

namespace {

constexpr int kLongRow = 160 << 10;  // bytes from which a row of logits may be cut: rows of 128 KB lose by it, of 200 KB gain; between them not measured
constexpr int kGradShort = 8192;     // ids up to which a row's gradient has 64 threads

constexpr float kLog2e = 1.44269504f, kLn2 = 0.693147181f;

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float max_nan(float a, float b) {  // NaN if either is
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}

// 16 bytes of logits.
template <int DT>
struct Vec {
  static constexpr int kN = DT == VLA_F32 ? 4 : 8;
  static constexpr int kBytes = 16 / kN;
  static constexpr uint32_t kLowest = DT == VLA_F32 ? 0xFF800000u : DT == VLA_F16 ? 0xFC00FC00u : 0xFF80FF80u;  // -infinity
  static __device__ __forceinline__ void unpack(const uint4& v, float (&z)[kN]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (DT == VLA_F32) {
        z[i] = __uint_as_float(w[i]);
      } else {
        const float2 f = DT == VLA_F16 ? unpack_f16x2(w[i]) : make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
        z[2 * i] = f.x;
        z[2 * i + 1] = f.y;
      }
    }
  }
  static __device__ __forceinline__ uint32_t word_max(uint32_t a, uint32_t b) {
    if constexpr (DT == VLA_F32) {
      return __float_as_uint(max_nan(__uint_as_float(a), __uint_as_float(b)));
    } else if constexpr (DT == VLA_F16) {
      const __half2 y = __hmax2_nan(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
      return *reinterpret_cast<const uint32_t*>(&y);
    } else {
      const __nv_bfloat162 y = __hmax2_nan(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
      return *reinterpret_cast<const uint32_t*>(&y);
    }
  }
  static __device__ __forceinline__ float word_float_max(uint32_t a) {
    if constexpr (DT == VLA_F32) return __uint_as_float(a);
    const float2 f = DT == VLA_F16 ? unpack_f16x2(a) : make_float2(__uint_as_float(a << 16), __uint_as_float(a & 0xFFFF0000u));
    return max_nan(f.x, f.y);
  }
  static __device__ __forceinline__ float load(const void* p, int64_t i) { return load_as_float(p, i, DT); }
};

// Elements before the first 16-byte boundary of a row at `p`, at most n.
template <int DT>
__device__ __forceinline__ int head_of(const void* p, int n) {
  return min(n, static_cast<int>((-reinterpret_cast<uintptr_t>(p) & 15u) / Vec<DT>::kBytes));
}

// Whole numbers in the order of the floats (negative zero as zero); with the id they make one 64-bit key, larger
// for a larger value and, among equals, for a lower id.
__device__ __forceinline__ int ordered(float x) {
  const int b = __float_as_int(x + 0.f);
  return b ^ ((b >> 31) & 0x7fffffff);
}
__device__ __forceinline__ int64_t make_key(int order, int id) {
  return (static_cast<int64_t>(order) << 32) | static_cast<uint32_t>(0x7fffffff - id);
}
__device__ __forceinline__ float float_of(int order) { return __int_as_float(order ^ ((order >> 31) & 0x7fffffff)); }
__device__ __forceinline__ float key_value(int64_t key) { return float_of(static_cast<int>(key >> 32)); }
__device__ __forceinline__ int key_id(int64_t key) { return 0x7fffffff - static_cast<int>(key & 0x7fffffff); }

// m c rounded, as a reference has to be before anything is taken from it: a compiler that makes one fma of the product and the
// subtraction has another reference there, off by up to half an ulp (3e-4 in each log-prob at logits of 1e4).
__device__ __forceinline__ float rounded_product(float m, float c) { return __fmul_rn(m, c); }
// Whether the rounding of m c may be more than a fraction of a power of two.
constexpr float kFar = 16777216.f;
__device__ __forceinline__ bool is_far(float m, float c) { return m != -INFINITY && !(fabsf(rounded_product(m, c)) < kFar); }
// Below 2^-200 a weight is 0, and 0 * -infinity no number.
constexpr float kFloor = -200.f;
// The reference that goes with a maximum of some of a row's logits: none for one so low that its logits weigh nothing
// beside any row that is not far, that is, more than the floor below the lowest of those.
__device__ __forceinline__ float reference_of(float m, float c) {
  const float r = rounded_product(m, c);
  return r > -kFar - 256.f ? r : -INFINITY;
}
static_assert(-kFloor < 256.f, "what has no reference weighs nothing");
// The reference of a set of maximum m (m c itself where that is far, else rounded) less that of one of maximum top.
__device__ __forceinline__ float reference_difference(float m, float top, float c) {
  const float low = rounded_product(m, c), high = rounded_product(top, c);
  if (is_far(m, c)) return is_far(top, c) ? (m - top) * c : fmaf(m, c, -high);
  return is_far(top, c) ? -fmaf(top, c, -low) : low - high;
}

// Running sums of a set of logits relative to 2^r; r = -infinity: nothing but zeros so far.
struct Sums {
  float r = -INFINITY, s = 0.f, w = 0.f;
  __device__ __forceinline__ void rise(float to) {
    const float d = r == -INFINITY ? 0.f : fmaxf(r - to, kFloor), f = exp2_fast(d);
    w = f * fmaf(d, s, w);
    s *= f;
    r = to;
  }
  __device__ __forceinline__ void add(float d) {
    d = fmaxf(d, kFloor);
    const float e = exp2_fast(d);
    s += e;
    w = fmaf(d, e, w);
  }
  // two at a time into pairs of sums
  static __device__ __forceinline__ void add_pair(uint64_t d, uint64_t& s, uint64_t& w) {
    float2 x = halves_of(d);
    x.x = fmaxf(x.x, kFloor);
    x.y = fmaxf(x.y, kFloor);
    const uint64_t e = pair_of(exp2_fast(x.x), exp2_fast(x.y));
    s = add2(s, e);
    w = fma2(pair_of(x.x, x.y), e, w);
  }
};

// CUT: one cluster of `parts` CTAs per row, each a slice of the ids; else one CTA per row.  TOP: with alternatives.  (Both known when
// compiled: 2500 x 32064 fp32 without alternatives 50 us, 57 with one kernel for all; 3584 x 32064 bf16 with 4 of them 45.4 and 46.7.)
template <int DT, int THREADS, bool TOP, bool CUT>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) token_logprobs_kernel(const LogprobArgs a, const int parts) {
  using V = Vec<DT>;
  constexpr int kWarps = THREADS / 32, kUnroll = 4;
  constexpr int kGroups = THREADS == 32 ? 32 : 64, kGroupLanes = kGroups / kWarps;  // lanes of a warp that are equal modulo kGroupLanes
  constexpr int kList = THREADS == 32 ? 128 : 512;
  constexpr int kMostParts = 8;
  constexpr int kRounds = 16;                      // rounds of the pass are kept modulo 16
  __shared__ float round_max[kRounds][THREADS];
  __shared__ __align__(16) int group_max[kGroups];
  __shared__ float red[3][kWarps];
  __shared__ int64_t above[kList];
  __shared__ int level_ids[kList];
  __shared__ int n_above, n_level, bound;
  __shared__ __align__(16) int64_t all_best[CUT ? kMostParts * kMaxTopK : 2];  // the slices' best keys, each in order
  __shared__ float all_slices[kMostParts][3];      // (m, s, w) of the slices
  __shared__ int64_t round_key[kWarps];
  pdl_launch_dependents();
  pdl_wait();
  if constexpr (CUT) cluster_arrive();  // the first CTA has begun once all have passed the wait
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int row = CUT ? blockIdx.x / parts : blockIdx.x, part = CUT ? blockIdx.x % parts : 0;
  const int first = CUT ? static_cast<int>(static_cast<int64_t>(a.vocab) * part / parts) : 0;
  const int n = CUT ? static_cast<int>(static_cast<int64_t>(a.vocab) * (part + 1) / parts) - first : a.vocab;
  const char* base = static_cast<const char*>(a.logits) + (row * a.ld + first) * V::kBytes;
  const int head = head_of<DT>(base, n), vecs = (n - head) / V::kN, tail = n - head - vecs * V::kN;
  const uint4* body = reinterpret_cast<const uint4*>(base + head * V::kBytes);
  const float inv_t = 1.f / a.temperature, c = kLog2e * inv_t;
  const int k = TOP ? min(a.top_k, n) : 0;  // of this slice

  // the token's logit is read beside the pass
  int token = -1;
  float chosen = 0.f;
  if (part == 0 && tid == 0 && a.tokens) {
    token = a.tokens[row];
    if (static_cast<unsigned>(token) < static_cast<unsigned>(a.vocab)) {
      chosen = V::load(a.logits, row * a.ld + token);
    } else {
      if (token != -1) raise_status(a.status, VLA_STATUS_BAD_TOKEN);
      token = -1;
    }
  }
  if (tid == 0) n_above = n_level = 0;

  Sums x;
  float most = -INFINITY;  // this thread's maximum
  const uint64_t c2 = pair_of(c, c);
  for (int i = tid, round = 0; i < vecs; i += THREADS * kUnroll, ++round) {
    uint4 v[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      v[u] = make_uint4(V::kLowest, V::kLowest, V::kLowest, V::kLowest);
      if (i + u * THREADS < vecs) v[u] = body[i + u * THREADS];
    }
    uint32_t up = v[0].x;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) up = V::word_max(up, V::word_max(V::word_max(v[u].x, v[u].y), V::word_max(v[u].z, v[u].w)));
    const float peak = V::word_float_max(up);
    if constexpr (TOP) {
      float& kept = round_max[round % kRounds][tid];
      kept = round < kRounds ? peak : fmaxf(kept, peak);
    }
    most = max_nan(most, peak);
    x.rise(reference_of(most, c));
    const float ref = x.r == -INFINITY ? 0.f : x.r;
    const uint64_t r2 = pair_of(-ref, -ref);
    uint64_t s2 = 0, w2 = 0;  // zeros
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      float z[V::kN];
      V::unpack(v[u], z);
#pragma unroll
      for (int j = 0; j < V::kN; j += 2) Sums::add_pair(fma2(pair_of(z[j], z[j + 1]), c2, r2), s2, w2);
    }
    const float2 s = halves_of(s2), w = halves_of(w2);
    x.s += s.x + s.y;
    x.w += w.x + w.y;
  }
  // up to 7 elements before and after the vectors: one a thread
  const int edge = tid < head ? tid : tid < head + tail ? n - tail + tid - head : -1;
  if (edge >= 0) {
    const float z = V::load(base, edge);
    most = max_nan(most, z);
    x.rise(reference_of(most, c));
    if (x.r != -INFINITY) x.add(fmaf(z, c, -x.r));
  }
  const int mine = ordered(most);

  // the CTA's maximum and its groups'
  float top = most;
  if (kGroupLanes == 32) group_max[warp * 32 + lane] = mine;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (o == kGroupLanes && lane < kGroupLanes) group_max[warp * kGroupLanes + lane] = ordered(top);
  }
  if (lane == 0) red[0][warp] = top;
  __syncthreads();
  top = red[0][0];
#pragma unroll
  for (int i = 1; i < kWarps; ++i) top = max_nan(top, red[0][i]);
  const bool odd = !(top < INFINITY);  // a NaN or +infinity in the slice
  const bool far = !odd && is_far(top, c);
  if (far) {
    x = Sums();
    x.r = 0.f;
    for (int j = tid; j < n; j += THREADS) x.add((V::load(base, j) - top) * c);
  } else if (x.r != -INFINITY) {
    x.rise(rounded_product(top, c));
  }
  x.s = warp_sum(x.s);
  x.w = warp_sum(x.w);
  if (lane == 0) {
    red[1][warp] = x.s;
    red[2][warp] = x.w;
  }
  if (TOP && warp == kWarps - 1) {
    // the largest maximum that k groups reach: the largest ones go in turn, two a lane
    int hi = group_max[lane], lo = INT32_MIN, reach = 0, v;
    if (kGroups == 64) {
      const int other = group_max[lane + 32];
      lo = min(hi, other);
      hi = max(hi, other);
    }
    do {
      v = __reduce_max_sync(0xffffffffu, hi);
      const bool goes = hi == v;
      reach += __popc(__ballot_sync(0xffffffffu, goes));
      hi = goes ? lo : hi;
      lo = goes ? INT32_MIN : lo;
    } while (reach < k);
    if (lane == 0) bound = v;
  }
  __syncthreads();
  Sums total;  // relative to the reference of the maximum `top`, or (far) to the maximum
#pragma unroll
  for (int i = 0; i < kWarps; ++i) {
    total.s += red[1][i];
    total.w += red[2][i];
  }

  // The row's numbers, of all slices once they have met; the difference to the maximum in natural units (a log-prob may be
  // as low as a type's lowest value), and what the reference is off the maximum.
  float log2_s, rest;
  bool bad, none, apart;
  auto settle = [&]() {
    bad = !(top < INFINITY);
    none = top == -INFINITY;
    apart = !bad && is_far(top, c);
    log2_s = log2f(total.s);
    rest = (apart ? 0.f : fmaf(top, c, -rounded_product(top, c))) - log2_s;
  };
  auto logprob = [&](float z) { return bad ? NAN : none ? -INFINITY : fmaf(rest, kLn2, (z - top) * inv_t); };
  auto put = [&](int rank, int64_t key) {
    const int64_t at = static_cast<int64_t>(row) * a.top_k + rank;
    a.top_ids[at] = key_id(key);
    a.top_logprobs[at] = logprob(key_value(key));
  };
  settle();
  if constexpr (CUT) cluster_wait();

  // ---- the slice's best keys
  auto place = [&](int rank, int64_t key) {
    if constexpr (CUT)
      asm volatile("st.shared::cluster.s64 [%0], %1;" ::"r"(mapa_shared(smem_u32(&all_best[part * a.top_k + rank]), 0)), "l"(key) : "memory");
    else
      put(rank, key);
  };
  if constexpr (TOP) {
    const int at_least = bound;
    const float limit = float_of(at_least);
    const bool lowest = limit == -INFINITY;  // then all that is not above it is equal to it
    bool fits = !odd;
    if (!odd) {
      auto take = [&](int j) {
        const int o = ordered(V::load(base, j));
        int* const count = o > at_least ? &n_above : &n_level;
        const int at = atomicAdd(count, 1);
        if (at >= kList) return;
        if (o > at_least)
          above[at] = make_key(o, first + j);
        else
          level_ids[at] = first + j;
      };
      if (lowest ? mine > at_least : mine >= at_least) {
        uint32_t rounds = 0;
#pragma unroll 4
        for (int i = 0; i < min(kRounds, (vecs - tid + THREADS * kUnroll - 1) / (THREADS * kUnroll)); ++i) {
          const float there = round_max[i][tid];
          rounds |= (lowest ? there > limit : there >= limit) ? 1u << i : 0u;
        }
        // each lane its own rounds, so that a warp's loads go together
        for (; rounds; rounds &= rounds - 1) {
          for (int i = tid + (__ffs(rounds) - 1) * (THREADS * kUnroll); i < vecs; i += kRounds * THREADS * kUnroll) {
            uint4 v[kUnroll];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) v[u] = body[min(i + u * THREADS, vecs - 1)];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
              if (i + u * THREADS >= vecs) break;
              const float peak = V::word_float_max(V::word_max(V::word_max(v[u].x, v[u].y), V::word_max(v[u].z, v[u].w)));
              if (lowest ? !(peak > limit) : !(peak >= limit)) continue;
              float z[V::kN];
              V::unpack(v[u], z);
              uint32_t found = 0;
#pragma unroll
              for (int j = 0; j < V::kN; ++j) found |= (lowest ? z[j] > limit : z[j] >= limit) ? 1u << j : 0u;
              for (; found; found &= found - 1) take(head + (i + u * THREADS) * V::kN + __ffs(found) - 1);
            }
          }
        }
        if (edge >= 0) {
          const float z = V::load(base, edge);
          if (lowest ? z > limit : z >= limit) take(edge);
        }
      }
      __syncthreads();
      const bool ties = n_above < k;  // equals of the bound are among the best
      if (lowest && ties) {  // the first k + n_above ids hold k of them
        for (int j = tid; j < min(n, k + n_above); j += THREADS)
          if (V::load(base, j) == limit) {
            const int at = atomicAdd(&n_level, 1);
            if (at < kList) level_ids[at] = first + j;
          }
        __syncthreads();
      }
      fits = n_above <= kList && (!ties || n_level <= kList);
      if (fits) {
        const int more = ties ? n_level : 0, count = n_above + more;
        for (int i = tid; i < count; i += THREADS) {
          const int64_t key = i < n_above ? above[i] : make_key(at_least, level_ids[i - n_above]);
          int rank = 0;
          for (int j = 0; j < n_above; ++j) rank += above[j] > key;
          if (i >= n_above)  // equals follow in the order of their ids
            for (int j = 0; j < more; ++j) rank += level_ids[j] < level_ids[i - n_above];
          if (rank < k) place(rank, key);
        }
      }
    }
    if (!fits) {  // more equal logits than the list holds: the largest key below the one before, k times over
      int64_t last = INT64_MAX;
      for (int i = 0; i < k; ++i) {
        int64_t key = INT64_MIN;
        for (int j = tid; j < n; j += THREADS) {
          const int64_t q = make_key(ordered(V::load(base, j)), first + j);
          if (q < last && q > key) key = q;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) key = max(key, __shfl_xor_sync(0xffffffffu, key, o));
        __syncthreads();
        if (lane == 0) round_key[warp] = key;
        __syncthreads();
        for (int w = 0; w < kWarps; ++w) key = max(key, round_key[w]);
        last = key;
        if (tid == 0) place(i, key);
      }
    }
  }

  // ---- the slices' results meet in the first CTA
  if constexpr (CUT) {
    if (tid < 3) {
      const float mine = tid == 0 ? top : tid == 1 ? total.s : total.w;
      asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(mapa_shared(smem_u32(&all_slices[part][tid]), 0)), "f"(mine) : "memory");
    }
    cluster_sync();
    if (part != 0) return;
    top = -INFINITY;
    for (int i = 0; i < parts; ++i) top = max_nan(top, all_slices[i][0]);
    total.s = total.w = 0.f;
    for (int i = 0; i < parts; ++i) {
      const float m = all_slices[i][0];
      if (m == -INFINITY) continue;
      const float d = fmaxf(reference_difference(m, top, c), kFloor), f = exp2_fast(d);
      total.s = fmaf(f, all_slices[i][1], total.s);
      total.w = fmaf(f, fmaf(d, all_slices[i][1], all_slices[i][2]), total.w);
    }
    settle();
    // disjoint sets of keys: a key's place is the number of larger ones
    if (tid < parts * a.top_k) {
      const int64_t key = all_best[tid];
      int rank = 0;
#pragma unroll 4
      for (int j = 0; j < parts * a.top_k; j += 2) {
        const longlong2 two = *reinterpret_cast<const longlong2*>(all_best + j);
        rank += (two.x > key) + (two.y > key);
      }
      if (rank < a.top_k) put(rank, key);
    }
  }

  if (tid == 0) {
    if (bad) raise_status(a.status, VLA_STATUS_NONFINITE);
    // (the maximum in natural units, rounded once with the sum: the gradient's weights are as far off as this is)
    if (a.lse) a.lse[row] = bad ? NAN : none ? -INFINITY : fmaf(top, inv_t, -rest * kLn2);
    if (a.entropy) a.entropy[row] = bad ? NAN : none ? 0.f : fmaf(log2_s, total.s, -total.w) / total.s * kLn2;
    if (a.logprob) a.logprob[row] = token < 0 ? 0.f : logprob(chosen);
  }
}

// A log-sum of this size and more is off by over 2^-18 in 32 bits (or is no number of theirs), and each weight e^(z / T - lse) by
// as much.
constexpr float kLargeLse = 128.f;

// The largest of n logits and log sum exp((z - largest) / T), by all threads of a cluster of CTAs, each of which gets both.  No CTA
// returns before all have read their share of the logits.
template <int DT, int THREADS>
__device__ __forceinline__ void log_sum_below_top(const char* row, int n, float c, int cluster, float& top, float& log_sum) {
  using V = Vec<DT>;
  constexpr int kWarps = THREADS / 32, kUnroll = 4;
  __shared__ float2 shares[kWarps];  // (largest, sum relative to it) of each warp
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int64_t rank = cluster > 1 ? cluster_ctarank() : 0;
  const int first = static_cast<int>(n * rank / cluster), mine = static_cast<int>(n * (rank + 1) / cluster) - first;
  row += static_cast<int64_t>(first) * V::kBytes;
  const int head = head_of<DT>(row, mine), vecs = (mine - head) / V::kN, tail = mine - head - vecs * V::kN;
  const uint4* body = reinterpret_cast<const uint4*>(row + head * V::kBytes);
  float m = -INFINITY, s = 0.f;
  auto reach = [&](float to) {  // whether there is anything to add
    if (to > m) {
      s *= exp2_fast((m - to) * c);
      m = to;
    }
    return m != -INFINITY;
  };
  for (int i = tid; i < vecs; i += THREADS * kUnroll) {
    uint4 v[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      v[u] = make_uint4(V::kLowest, V::kLowest, V::kLowest, V::kLowest);
      if (i + u * THREADS < vecs) v[u] = body[i + u * THREADS];
    }
    uint32_t up = v[0].x;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) up = V::word_max(up, V::word_max(V::word_max(v[u].x, v[u].y), V::word_max(v[u].z, v[u].w)));
    if (!reach(V::word_float_max(up))) continue;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      float z[V::kN];
      V::unpack(v[u], z);
#pragma unroll
      for (int j = 0; j < V::kN; ++j) s += exp2_fast((z[j] - m) * c);
    }
  }
  const int edge = tid < head ? tid : tid < head + tail ? mine - tail + tid - head : -1;
  if (edge >= 0) {
    const float z = V::load(row, edge);
    if (reach(z)) s += exp2_fast((z - m) * c);
  }
  auto join = [&]() {  // over a warp
    const float high = warp_max(m);
    s = warp_sum(m == -INFINITY ? 0.f : s * exp2_fast((m - high) * c));
    m = high;
  };
  join();
  if (lane == 0) shares[warp] = make_float2(m, s);
  cluster_sync();
  m = -INFINITY;
  s = 0.f;
  for (int i = lane; i < cluster * kWarps; i += 32) {
    float2 x;
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(x.x), "=f"(x.y) : "r"(mapa_shared(smem_u32(&shares[i % kWarps]), i / kWarps)) : "memory");
    if (reach(x.x)) s = fmaf(x.y, exp2_fast((x.x - m) * c), s);
  }
  join();
  cluster_sync();  // (until then the others' shared memory is there)
  top = m;
  log_sum = log2f(s) * kLn2;
}

// The gradient, element by element: with d = z / T - lse, -e^d (g + h (d + entropy)) / T, and g / T more at the token.
// Rows far from zero (kLargeLse) are read once more first, for d as a difference to the maximum less a log-sum relative to it,
// by clusters of their CTAs, in place by all of them.  Bound by HBM.  One CTA per row and slice, in 16-byte
// pieces of the gradient; where the logits lie differently towards 16 bytes, a piece of theirs is cut out of the two aligned ones
// that it lies in (the row's ends, whose neighbours are not the row's, element by element).  3584 x 32064 bf16 take 68.6 us (6.7 TB/s,
// the copy rate), 85 where all rows are far from zero; a row waits for its log-sum before its first loads, which is 0.5 us of it.
// 4000 x 8000 bf16 with logits 5 elements further apart than the gradient's took 25.0 us, 46 element by element.  ALIKE: all rows of
// both lie alike (known when compiled: 1500 x 20000 bf16 21.4 us, 24.1 with the check; 3000 x 10000 24.1 and 27.2).
template <int DT, int THREADS, bool ALIKE>
__global__ void __launch_bounds__(THREADS) token_logprobs_grad_kernel(const LogprobGradArgs a, const int parts, const int cluster) {
  using V = Vec<DT>;
  constexpr int kUnroll = 4;
  pdl_launch_dependents();
  pdl_wait();
  const int tid = threadIdx.x, row = blockIdx.x / parts, part = blockIdx.x % parts;
  // slices begin at multiples of 64 elements, so that none cuts a 16-byte piece of an aligned row
  const int units = (a.vocab + 63) / 64;
  const int first = static_cast<int>(static_cast<int64_t>(units) * part / parts) * 64;
  const int n = min(a.vocab, static_cast<int>(static_cast<int64_t>(units) * (part + 1) / parts) * 64) - first;
  const char* src = static_cast<const char*>(a.logits) + (row * a.ld + first) * V::kBytes;
  char* dst = static_cast<char*>(a.d_logits) + (row * a.ldd + first) * V::kBytes;
  const int head = head_of<DT>(dst, n);
  const int off = ALIKE ? 0 : static_cast<int>(reinterpret_cast<uintptr_t>(src + head * V::kBytes) & 15u);
  // pieces [v0, v1) whose logits, or both aligned pieces around them, are the row's
  const int inside = (n - head) * V::kBytes;
  const int v0 = off > head * V::kBytes ? 1 : 0, v1 = max(v0, off ? (inside + off - 16) / 16 : inside / 16);
  const uint4* from = reinterpret_cast<const uint4*>(src + head * V::kBytes - off);
  uint4* to = reinterpret_cast<uint4*>(dst + head * V::kBytes);
  const int words = off >> 2, bits = (off & 3) * 8;
  int token = a.tokens[row];
  // x = z scale - base, d = x ratio - rest
  const float inv_t = 1.f / a.temperature;
  float scale = inv_t, base = a.lse[row], ratio = 1.f, rest = 0.f;
  const bool kept = static_cast<unsigned>(token) < static_cast<unsigned>(a.vocab);
  if (!kept && token != -1 && part == 0 && tid == 0) raise_status(a.status, VLA_STATUS_BAD_TOKEN);
  float g = kept ? a.g_logprob[row] * inv_t : 0.f;
  float h = kept && a.g_entropy ? a.g_entropy[row] * inv_t : 0.f;
  if (kept && base != base) g = base;  // a row whose numbers are none
  token = kept ? token - first : -1;
  if (kept && fabsf(base) >= kLargeLse) {
    float top, log_sum;
    log_sum_below_top<DT, THREADS>(static_cast<const char*>(a.logits) + row * a.ld * V::kBytes, a.vocab, kLog2e * inv_t, cluster, top, log_sum);
    if (fabsf(top) < INFINITY) {
      // differences to the top, at the power of two next below 1 / T: no product is rounded.  Where that takes the top past 32 bits,
      // what is not equal to the top weighs nothing, and does so at a scale that takes the top to 2^100.
      const uint32_t exponent = (__float_as_uint(top) >> 23) & 255u;
      scale = __uint_as_float(max(__float_as_uint(inv_t) & 0x7f800000u, 0x00800000u));
      ratio = inv_t / scale;
      if (!(fabsf(top * scale) < INFINITY)) {
        scale = __uint_as_float((354u - exponent) << 23);
        ratio = 1.f;
      }
      base = top * scale;
      rest = log_sum;
    }
  }
  const float gh = h != 0.f ? fmaf(h, a.entropy[row] - rest, g) : g, to_log2 = ratio * kLog2e, rest2 = rest * kLog2e;
  h *= ratio;
  auto slope = [&](float z) {
    // below e^-1000 a weight is 0, and 0 * -infinity no number
    const float x = fmaxf(fmaf(z, scale, -base), -1000.f);
    return -exp2_fast(fmaf(x, to_log2, -rest2)) * fmaf(h, x, gh);
  };
  for (int i = v0 + tid; i < v1; i += THREADS * kUnroll) {
    uint4 v[kUnroll], w[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
      if (kept && i + u * THREADS < v1) {
        v[u] = from[i + u * THREADS];
        if (off) w[u] = from[i + u * THREADS + 1];
      }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      if (i + u * THREADS >= v1) break;
      uint4 y = make_uint4(0u, 0u, 0u, 0u);
      if (kept) {
        if (off) {
          uint32_t c[8] = {v[u].x, v[u].y, v[u].z, v[u].w, w[u].x, w[u].y, w[u].z, w[u].w};
#pragma unroll
          for (int j = 0; j < 6; ++j) c[j] = words & 2 ? c[j + 2] : c[j];
#pragma unroll
          for (int j = 0; j < 5; ++j) c[j] = words & 1 ? c[j + 1] : c[j];
          v[u] = make_uint4(__funnelshift_r(c[0], c[1], bits), __funnelshift_r(c[1], c[2], bits), __funnelshift_r(c[2], c[3], bits),
                            __funnelshift_r(c[3], c[4], bits));
        }
        float z[V::kN];
        V::unpack(v[u], z);
#pragma unroll
        for (int j = 0; j < V::kN; ++j) z[j] = slope(z[j]);
        const int at = token - (head + (i + u * THREADS) * V::kN);
        if (static_cast<unsigned>(at) < static_cast<unsigned>(V::kN)) {
#pragma unroll
          for (int j = 0; j < V::kN; ++j)
            if (j == at) z[j] += g;
        }
        uint32_t* p = reinterpret_cast<uint32_t*>(&y);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          p[j] = DT == VLA_F32 ? __float_as_uint(z[j]) : DT == VLA_F16 ? pack_f16x2(z[2 * j % V::kN], z[(2 * j + 1) % V::kN]) : pack_bf16x2(z[2 * j % V::kN], z[(2 * j + 1) % V::kN]);
      }
      to[i + u * THREADS] = y;
    }
  }
  // the ends: before piece v0 and from piece v1 on
  const int before = min(n, head + v0 * V::kN), after = min(n, head + v1 * V::kN), ends = before + n - after;
  for (int e = tid; e < ends; e += THREADS) {
    const int j = e < before ? e : after + e - before;
    float d = kept ? slope(V::load(src, j)) : 0.f;
    if (j == token) d += g;
    store_from_float(dst, j, d, DT);
  }
}

template <int DT>
int logprobs_of(const LogprobArgs& a, cudaStream_t s, int sms) {
  // Threads a row: the SMs hold 1024 each, so rows go in waves of 1024 sms / threads, and a wave takes about as long as
  // 44 ids a thread for the row's own steps and one for each id that a thread has (bf16 with 4 alternatives on 32, 64, 128,
  // 256 threads: 3584 x 32064 49, 48, 45, 53 us; 4000 x 1200 8.5, 10, 15, 24; 500 x 32064 27, 17, 15, 10).
  int threads = 32;
  int64_t least = INT64_MAX;
  for (int t = 32; t <= 256; t *= 2) {
    const int64_t waves = (static_cast<int64_t>(a.rows) * t - 1) / (1024LL * sms) + 1, cost = waves * (44 + a.vocab / t);
    if (cost < least) {
      least = cost;
      threads = t;
    }
  }
  // Few long rows are cut over a cluster, which costs 2 to 4 us: from kLongRow on, while two of its CTAs an SM are not reached, or
  // four with slices of 36 KB (with 8 alternatives on 1, 2, 4, 8 CTAs a row: 64 x 32064 f32 6.6, 7.5, 7.8, 7.7 us, one row
  // of it 6.0, 6.2, 5.7, 5.8; 130 x 50000 f32 12.1, 11.5, 10.0, 15.7, one row 7.6, 7.1, 6.5, 6.2; 64 x 151000 bf16 13.6, 12.9, 12.3, 11.2).
  int parts = 1;
  const int64_t bytes = static_cast<int64_t>(a.vocab) * Vec<DT>::kBytes;
  while (threads == 256 && bytes >= kLongRow && parts < 8) {
    const int64_t ctas = static_cast<int64_t>(a.rows) * parts * 2, slice = bytes / (parts * 2);
    if (ctas > 2 * sms && !(ctas <= 4 * sms && slice >= 36864)) break;
    parts *= 2;
  }
  if (static_cast<int64_t>(a.rows) * parts > 0x7fffffff) return record_error(VLA_ERR_UNSUPPORTED, "vla_token_logprobs: too many rows");
  auto pick = [&](auto top) {
    constexpr bool TOP = decltype(top)::value;
    return parts > 1        ? token_logprobs_kernel<DT, 256, TOP, true>
           : threads == 256 ? token_logprobs_kernel<DT, 256, TOP, false>
           : threads == 128 ? token_logprobs_kernel<DT, 128, TOP, false>
           : threads == 64  ? token_logprobs_kernel<DT, 64, TOP, false>
                            : token_logprobs_kernel<DT, 32, TOP, false>;
  };
  auto kern = a.top_k > 0 ? pick(std::true_type()) : pick(std::false_type());
  VLA_CUDA_TRY(launch_pdl_cluster(kern, dim3(a.rows * parts), dim3(threads), 0, s, parts, a, parts));
  note_launch();
  VLA_CUDA_TRY(cudaGetLastError());
  return VLA_OK;
}

int num_sms(int* sms) {
  int dev = 0;
  VLA_CUDA_TRY(cudaGetDevice(&dev));
  VLA_CUDA_TRY(cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev));
  return VLA_OK;
}

}  // namespace

int token_logprobs_launch(const LogprobArgs& a, cudaStream_t s) {
  int sms = 0;
  if (const int rc = num_sms(&sms)) return rc;
  return a.dtype == VLA_F32 ? logprobs_of<VLA_F32>(a, s, sms) : a.dtype == VLA_F16 ? logprobs_of<VLA_F16>(a, s, sms) : logprobs_of<VLA_BF16>(a, s, sms);
}

int token_logprobs_grad_launch(const LogprobGradArgs& a, cudaStream_t s) {
  int sms = 0;
  if (const int rc = num_sms(&sms)) return rc;
  // few rows: slices of at least 2048 elements while the rows alone do not fill the SMs four times; short rows: fewer threads
  // (f16, 64 against 256 threads: 7607 x 1438 13.1 and 26.2 us, 4785 x 5319 19.9 and 24.3, 4000 x 8000 23.6 and 23.8)
  const int threads = a.vocab <= kGradShort ? 64 : 256;
  // a row's slices are clusters of up to 8, which read a row far from zero together, in place one such cluster (16 x 151936 bf16 4.7 us,
  // 15.8 with all rows far, 40 where each slice's CTA reads the whole row; clusters cost 0.1 to 0.4 us; in place one row of 151936 3.6
  // us, 2.2 as 64 slices)
  const int most = a.d_logits == a.logits ? 8 : 64;
  int parts = 1;
  while (parts < most && static_cast<int64_t>(a.rows) * parts < 4 * sms && a.vocab / (parts * 2) >= 2048) parts *= 2;
  if (static_cast<int64_t>(a.rows) * parts > 0x7fffffff) return record_error(VLA_ERR_UNSUPPORTED, "vla_token_logprobs_grad: too many rows");
  auto pick = [&](auto type) {
    constexpr int DT = decltype(type)::value;
    const bool alike = !(((reinterpret_cast<uintptr_t>(a.logits) ^ reinterpret_cast<uintptr_t>(a.d_logits)) | ((a.ld - a.ldd) * Vec<DT>::kBytes)) & 15);
    return threads == 64 ? (alike ? token_logprobs_grad_kernel<DT, 64, true> : token_logprobs_grad_kernel<DT, 64, false>)
                         : (alike ? token_logprobs_grad_kernel<DT, 256, true> : token_logprobs_grad_kernel<DT, 256, false>);
  };
  auto kern = a.dtype == VLA_F32   ? pick(std::integral_constant<int, VLA_F32>())
              : a.dtype == VLA_F16 ? pick(std::integral_constant<int, VLA_F16>())
                                   : pick(std::integral_constant<int, VLA_BF16>());
  const int cluster = std::min(parts, 8);
  VLA_CUDA_TRY(launch_pdl_cluster(kern, dim3(a.rows * parts), dim3(threads), 0, s, cluster, a, parts, cluster));
  note_launch();
  VLA_CUDA_TRY(cudaGetLastError());
  return VLA_OK;
}

}  // namespace vla
