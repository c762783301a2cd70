// The paged cache's bookkeeping and its writes: the page plan of a step (pages taken from a pool,
// rows mapped to slots), the rotary table, and the step that normalises, rotates and files queries,
// keys and values.
#include <algorithm>

#include "lm.h"
#include "ptx.cuh"

namespace vla {

namespace {

// ------------------------------------------------------------------------------------ page plan
// With ctx_e the positions cached (0 for an environment that starts over), have_e = ceil(ctx_e / ps) and
// want_e = ceil((ctx_e + new_e) / ps), environment e takes want_e - have_e pages; exclusive sums over the
// environments give its first row, its first page off the pool's end and, for releases, the place of its old
// pages.  Bound by latency for a decode step; a prefill writes 12 bytes a row.  One cluster: every CTA makes the sums
// for itself (a block scan into shared memory), then the CTAs share the pages and the rows, four rows a thread,
// which finds the first one's environment by bisection.  The cluster's barriers stand between reading
// the state and writing it, and between pages given back and pages taken.  16 environments of a row each take 3.6 us of
// device time, 256 of about 296 rows 8.3 (84 as one CTA with a thread a row).
__device__ __forceinline__ int64_t warp_inclusive(int64_t v) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t u = __shfl_up_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) >= o) v += u;
  }
  return v;
}

// The last e with start[e] <= i (start[0] = 0 <= i).
__device__ __forceinline__ int env_of(const int* start, int n, int i) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (start[mid] <= i)
      lo = mid;
    else
      hi = mid - 1;
  }
  return lo;
}

// POW2: pages of 1 << page_shift positions (known when compiled 0.3 to 0.7 us a call).
template <int kPlanThreads, bool POW2>
__global__ void __launch_bounds__(kPlanThreads) page_plan_kernel(const PagePlanArgs a, const int parts, const int page_shift) {
  extern __shared__ int plan_sm[];
  int* row_first = plan_sm;                   // [n_env + 1]
  int* page_first = row_first + a.n_env + 1;  // [n_env]
  int* ctx0 = page_first + a.n_env;           // [n_env] positions that stay
  int* old_first = ctx0 + a.n_env;            // [n_env] released pages before this environment's
  __shared__ int64_t sums[3][kPlanThreads / 32];
  __shared__ int64_t carry[3];
  __shared__ int bad;
  pdl_launch_dependents();
  pdl_wait();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int part = static_cast<int>(blockIdx.x), all = parts * kPlanThreads, me = part * kPlanThreads + tid;
  if (tid < 3) carry[tid] = 0;
  if (tid == 0) bad = 0;
  const int n_free = *a.n_free_in;
  const int64_t room = static_cast<int64_t>(a.max_pages) * a.page_size;
  auto page_of = [&](int position) { return POW2 ? position >> page_shift : position / a.page_size; };
  auto pages_of = [&](int64_t n) { return n > 0 ? page_of(static_cast<int>(n - 1)) + 1 : 0; };
  __syncthreads();
  for (int base = 0; base < a.n_env; base += kPlanThreads) {
    const int e = base + tid;
    int64_t v[3] = {0, 0, 0};  // rows, pages taken, pages released
    if (e < a.n_env) {
      const int64_t ctx = a.ctx_in[e], add = a.new_len[e];
      const bool out = a.release && a.release[e] != 0;
      const int64_t kept = out ? 0 : ctx;
      if (ctx < 0 || add < 0 || ctx > room || kept + add > room || kept + add > 0x7fffffff) {
        bad = 1;
        ctx0[e] = 0;
      } else {
        v[0] = add;
        v[1] = pages_of(kept + add) - pages_of(kept);
        v[2] = out ? pages_of(ctx) : 0;
        ctx0[e] = static_cast<int>(kept);
      }
    }
    int64_t inc[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      inc[i] = warp_inclusive(v[i]);
      if (lane == 31) sums[i][warp] = inc[i];
    }
    __syncthreads();
    int64_t before[3], total[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      before[i] = total[i] = carry[i];
#pragma unroll
      for (int w = 0; w < kPlanThreads / 32; ++w) {
        if (w < warp) before[i] += sums[i][w];
        total[i] += sums[i][w];
      }
    }
    if (e < a.n_env) {
      // totals beyond 32 bits do not fit the rows or the pool and are refused below
      row_first[e] = static_cast<int>(before[0] + inc[0] - v[0]);
      page_first[e] = static_cast<int>(before[1] + inc[1] - v[1]);
      old_first[e] = static_cast<int>(before[2] + inc[2] - v[2]);
    }
    __syncthreads();
    if (tid < 3) carry[tid] = tid == 0 ? total[0] : tid == 1 ? total[1] : total[2];
    __syncthreads();
  }
  const int64_t rows64 = carry[0], taken64 = carry[1], old64 = carry[2];
  const bool fits = !bad && n_free >= 0 && n_free + old64 <= a.n_pages && taken64 <= n_free + old64 && rows64 <= a.max_rows;
  const int rows = fits ? static_cast<int>(rows64) : 0, taken = fits ? static_cast<int>(taken64) : 0;
  const int old = fits ? static_cast<int>(old64) : 0;
  const int top = n_free + old;
  if (!fits && me == 0) raise_status(a.status, VLA_STATUS_PAGES);
  if (tid == 0) row_first[a.n_env] = static_cast<int>(rows64);
  for (int i = me; i < old; i += all) {
    const int e = env_of(old_first, a.n_env, i);
    a.pool[n_free + i] = a.table[static_cast<int64_t>(e) * a.max_pages + (i - old_first[e])];
  }
  if (parts > 1)
    cluster_sync();
  else
    __syncthreads();
  for (int i = me; i < taken; i += all) {
    const int e = env_of(page_first, a.n_env, i);
    const int col = pages_of(ctx0[e]) + i - page_first[e];
    a.table[static_cast<int64_t>(e) * a.max_pages + col] = __ldcg(a.pool + top - 1 - i);
  }
  const bool wide = !((reinterpret_cast<uintptr_t>(a.row_env) | reinterpret_cast<uintptr_t>(a.row_pos) | reinterpret_cast<uintptr_t>(a.row_slot)) & 15u);
  for (unsigned next = me * 4u; next < static_cast<unsigned>(a.max_rows); next += all * 4u) {
    const int r0 = static_cast<int>(next);
    int env[4], pos[4], slot[4];
    int e = r0 < rows ? env_of(row_first, a.n_env, r0) : 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      env[i] = pos[i] = slot[i] = -1;
      if (r0 + i < rows) {
        while (r0 + i >= row_first[e + 1]) ++e;
        env[i] = e;
        pos[i] = ctx0[e] + r0 + i - row_first[e];
        const int have = pages_of(ctx0[e]), col = page_of(pos[i]);
        // a page of this call comes from the pool, where its table entry comes from too
        slot[i] = col < have ? a.table[static_cast<int64_t>(e) * a.max_pages + col] : __ldcg(a.pool + top - 1 - (page_first[e] + col - have));
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (r0 + i >= rows) continue;
      if (static_cast<unsigned>(slot[i]) < static_cast<unsigned>(a.n_pages)) {
        slot[i] = slot[i] * a.page_size + pos[i] - page_of(pos[i]) * a.page_size;
      } else {
        slot[i] = -1;
        raise_status(a.status, VLA_STATUS_PAGES);
      }
    }
    if (wide && r0 <= a.max_rows - 4) {
      *reinterpret_cast<int4*>(a.row_env + r0) = make_int4(env[0], env[1], env[2], env[3]);
      *reinterpret_cast<int4*>(a.row_pos + r0) = make_int4(pos[0], pos[1], pos[2], pos[3]);
      *reinterpret_cast<int4*>(a.row_slot + r0) = make_int4(slot[0], slot[1], slot[2], slot[3]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (i >= a.max_rows - r0) break;
        a.row_env[r0 + i] = env[i];
        a.row_pos[r0 + i] = pos[i];
        a.row_slot[r0 + i] = slot[i];
      }
    }
  }
  for (int e = me; e < a.n_env; e += all) {
    a.row_start[e] = fits ? row_first[e] : 0;
    a.ctx_out[e] = fits ? ctx0[e] + row_first[e + 1] - row_first[e] : a.ctx_in[e];
  }
  if (me == 0) {
    a.row_start[a.n_env] = rows;
    *a.n_free_out = fits ? top - taken : n_free;
  }
}

// ----------------------------------------------------------------------------------- rotary table
// In 64 bits: the angle of position 131071 and frequency 1 needs 17 bits before its point, which leaves a 32-bit angle
// 4e-3 off.  Bound by the 64-bit units: a thread has one pair and every `apart`-th position, takes two cosines and sines of
// angles and goes from position to position by a rotation of 4 operations, each of which adds about 2^-52.  131072
// positions of 64 pairs take 205 us, 2218 with a power, a cosine and a sine for each element.
__global__ void __launch_bounds__(256) rope_table_kernel(const RopeTableArgs a, const int apart) {
  pdl_launch_dependents();
  pdl_wait();
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i >= static_cast<int64_t>(apart) * a.pairs) return;
  const int pos = static_cast<int>(i / a.pairs), pair = static_cast<int>(i % a.pairs);
  double f = pow(a.theta, -static_cast<double>(pair) / a.pairs);
  if (a.kind == VLA_ROPE_LINEAR) f /= a.factor;
  if (a.kind >= VLA_ROPE_TURNS) {
    const double turns = a.original_len * f / 6.283185307179586476925;
    const double s = a.kind == VLA_ROPE_TURNS ? (turns - a.low) / (a.high - a.low) : (log(turns) - log(a.low)) / (log(a.high) - log(a.low));
    const double keep = fmin(fmax(s, 0.0), 1.0);
    f *= keep + (1.0 - keep) / a.factor;
  }
  double sn, cs, step_sn = 0.0, step_cs = 1.0;
  sincos(static_cast<double>(pos) * f, &sn, &cs);
  if (apart < a.n_pos) sincos(static_cast<double>(apart) * f, &step_sn, &step_cs);
  cs *= a.amplitude;
  sn *= a.amplitude;
  for (int64_t p = pos; p < a.n_pos; p += apart) {
    a.table[p * a.pairs + pair] = make_float2(static_cast<float>(cs), static_cast<float>(sn));
    const double c = cs * step_cs - sn * step_sn;
    sn = sn * step_cs + cs * step_sn;
    cs = c;
  }
}

// ------------------------------------------------------------------------------------ rope append
// x <- x / sqrt(mean x^2 + eps) gain, then per pair (a, b) of channels (a cos - b sin, b cos + a sin).  Each element is
// read and written once; bound by HBM for a prefill, for 16-bit types as much by issuing instructions, by latency for a
// decode step.  hd / 8 lanes hold a head, 8 channels each, so that an access of a warp is 256 channels that follow each
// other in the row.  Where pairs lie half a rotation apart, the partner of a 16-bit channel is a shuffle away; in fp32 a
// lane has 4 channels of each half instead (fp32 rows of 32 / 32 heads: 226 us for 18432 against 232; 16-bit ones in pieces
// of 8 bytes: 131 against 95).  A warp walks over the queries, keys and values of one row, some accesses ahead (the
// first ones before the row's position is known), and the row's cosines and sines stay in registers; a row of few
// is cut over several warps so that a decode step fills the GPU.  18432 bf16 rows of 32 / 8 heads of 128 with norms take 73 us
// (6.2 TB/s of each byte once, 0.91 of the copy rate; three of four issue slots are used), 64 fp32 rows of 32 / 32 heads 2.8 us.
enum RopeLayout : int { kNoRope = 0, kHalves = 1, kPairs = 2 };

__device__ __forceinline__ float clamp_f16(float x, uint32_t& sat) {
  if (fabsf(x) > 65504.f && fabsf(x) != INFINITY) {
    x = copysignf(65504.f, x);
    sat = 1u;
  }
  return x;
}

template <int DT>
struct Eight {  // 8 channels of type DT, in two pieces of 4 that follow each other in memory or (SPLIT) do not
  uint4 v[DT == VLA_F32 ? 2 : 1];
  template <bool SPLIT>
  __device__ __forceinline__ void load(const char* p, int gap) {  // the second piece `gap` bytes after the first
    if constexpr (DT == VLA_F32) {
      v[0] = *reinterpret_cast<const uint4*>(p);
      v[1] = *reinterpret_cast<const uint4*>(p + gap);
    } else if constexpr (SPLIT) {
      const uint2 a = *reinterpret_cast<const uint2*>(p), b = *reinterpret_cast<const uint2*>(p + gap);
      v[0] = make_uint4(a.x, a.y, b.x, b.y);
    } else {
      v[0] = *reinterpret_cast<const uint4*>(p);
    }
  }
  template <bool SPLIT>
  __device__ __forceinline__ void store(char* p, int gap) const {
    if constexpr (DT == VLA_F32) {
      *reinterpret_cast<uint4*>(p) = v[0];
      *reinterpret_cast<uint4*>(p + gap) = v[1];
    } else if constexpr (SPLIT) {
      *reinterpret_cast<uint2*>(p) = make_uint2(v[0].x, v[0].y);
      *reinterpret_cast<uint2*>(p + gap) = make_uint2(v[0].z, v[0].w);
    } else {
      *reinterpret_cast<uint4*>(p) = v[0];
    }
  }
  __device__ __forceinline__ void unpack(float (&x)[8]) const {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(v);
#pragma unroll
    for (int i = 0; i < (DT == VLA_F32 ? 8 : 4); ++i) {
      if constexpr (DT == VLA_F32) {
        x[i] = __uint_as_float(w[i]);
      } else {
        const float2 f = DT == VLA_F16 ? unpack_f16x2(w[i]) : unpack_bf16x2(w[i]);
        x[2 * i] = f.x;
        x[2 * i + 1] = f.y;
      }
    }
  }
};
__device__ __forceinline__ uint4 pack8(const float (&x)[8], bool f16_type) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = f16_type ? pack_f16x2(x[2 * i], x[2 * i + 1]) : pack_bf16x2(x[2 * i], x[2 * i + 1]);
  return make_uint4(w[0], w[1], w[2], w[3]);
}

constexpr int kAppendThreads = 128;

// `slices` warps share a row's heads (CUT: more than one).  Accesses ahead and warps an SM as measured on 18432 bf16 rows of
// 32 / 8 heads with norms, in pairs and in halves: 3 ahead and 32 warps 73 and 79 us, 4 and 28 76 and 80, 4 and 32 74 and 102 (too
// few registers), 2 and 32 79 and 80, 3 and 36 92 and 105; 15600 rows of 32 / 32 heads in halves without norms 120 with 3 and 32, 116
// with 4 and 28; f32 of 32 / 32 heads 225 with 2 ahead, 276 with 4.  (Kernels with norms spill 2 to 28 bytes at these settings; the
// times have that in them.)  CUT and HD known when
// compiled: 65536 rows of 64 / 8 heads 437 us, 482 without.
template <int DT, int LAYOUT, bool NORM>
struct Ahead {
  static constexpr bool kPlainHalves = LAYOUT == kHalves && !NORM;
  static constexpr int kAccesses = DT == VLA_F32 ? 2 : kPlainHalves ? 4 : 3;
  static constexpr int kCtas = DT == VLA_F32 ? (LAYOUT == kHalves && NORM ? 6 : 7) : kPlainHalves ? 7 : 8;
};

template <int DT, int LAYOUT, bool NORM, bool CUT, int HD>
__global__ void __launch_bounds__(kAppendThreads, Ahead<DT, LAYOUT, NORM>::kCtas) rope_append_kernel(const RopeAppendArgs a, const int slices, const int page_shift) {
  constexpr int kAhead = Ahead<DT, LAYOUT, NORM>::kAccesses, kSize = DT == VLA_F32 ? 4 : 2, kSpan = 256;  // channels of an access
  constexpr bool kSplit = LAYOUT == kHalves && DT == VLA_F32, kShuffle = LAYOUT == kHalves && !kSplit;
  pdl_launch_dependents();
  pdl_wait();
  constexpr int hd = HD, span = HD / 8, span_shift = HD == 64 ? 3 : 4;  // lanes of a head
  const int lane = threadIdx.x & 31;
  const int64_t unit = static_cast<int64_t>(blockIdx.x) * (kAppendThreads / 32) + (threadIdx.x >> 5);
  if (unit >= static_cast<int64_t>(a.rows) * slices) return;
  int row = static_cast<int>(unit), slice = 0;
  if constexpr (CUT) {  // (then rows * slices fits 32 bits)
    slice = row % slices;
    row /= slices;
  }
  const int half = a.rope_dim / 2, part = lane & (span - 1), head_of_span = lane >> span_shift;
  const bool in_turn = LAYOUT != kNoRope && part * 8 < a.rope_dim;
  // this lane's channels of a head: 4 from c0, 4 more `gap` on
  const int c0 = kSplit && in_turn ? part * 4 : part * 8, gap = kSplit && in_turn ? half : 4, mine = head_of_span * hd + c0;
  // accesses: queries, keys, values; this warp's
  const int q_channels = a.n_q_heads * hd, kv_channels = a.kv.n_heads * hd;
  const int keys = (q_channels + kSpan - 1) / kSpan, kv_steps = (kv_channels + kSpan - 1) / kSpan, values = keys + kv_steps;
  const int steps = values + kv_steps, from = CUT ? steps * slice / slices : 0, to = CUT ? steps * (slice + 1) / slices : steps;
  // the rows' first elements, as if each began at access 0
  const char* const q_row = static_cast<const char*>(a.q) + (row * a.ldq + mine) * kSize;
  const char* const k_row = static_cast<const char*>(a.k) + (row * a.ldk + mine - keys * kSpan) * kSize;
  const char* const v_row = static_cast<const char*>(a.v) + (row * a.ldv + mine - values * kSpan) * kSize;
  // whether this lane's head of access j is there
  auto there = [&](int j) {
    const int first = j < keys ? 0 : j < values ? keys : values;
    return (j - first) * kSpan + head_of_span * hd < (j < keys ? q_channels : kv_channels);
  };
  Eight<DT> raw[kAhead];
  auto fetch = [&](int j, Eight<DT>& r) {
    if (j < to && there(j)) r.template load<kSplit>((j < keys ? q_row : j < values ? k_row : v_row) + j * (kSpan * kSize), gap * kSize);
  };
#pragma unroll
  for (int u = 0; u < kAhead; ++u) fetch(from + u, raw[u]);

  const int pos = a.row_pos[row], slot = a.row_slot[row];
  const bool lost = pos < -1 || (LAYOUT != kNoRope && pos >= a.n_pos), empty = pos == -1 || lost;
  const bool stray = slot < -1 || slot >= a.kv.n_pages * a.kv.page_size;
  if ((lost || (stray && !empty)) && lane == 0 && slice == 0) raise_status(a.status, VLA_STATUS_PAGES);
  const bool file = !empty && !stray && slot != -1;

  // the rotations of this lane's pairs (one for each channel where the partner is elsewhere); none: (1, 0)
  constexpr int kTurns = kShuffle ? 8 : 4;
  const bool second = kShuffle && in_turn && c0 >= half;
  const int partner = (second ? lane - half / 8 : lane + half / 8) & 31;
  float cs[kTurns], sn[kTurns];
  if (LAYOUT != kNoRope && from < values) {
    const float4* t = reinterpret_cast<const float4*>(a.rope + static_cast<int64_t>(pos) * half + (kShuffle ? (second ? c0 - half : c0) : part * 4));
#pragma unroll
    for (int i = 0; i < kTurns / 2; ++i) {
      float4 x = make_float4(1.f, 0.f, 1.f, 0.f);
      if (in_turn && !empty) x = t[i];
      cs[2 * i] = x.x;
      sn[2 * i] = kShuffle && !second ? -x.y : x.y;  // a cos - b sin, b cos + a sin: the partner's sign turns
      cs[2 * i + 1] = x.z;
      sn[2 * i + 1] = kShuffle && !second ? -x.w : x.w;
    }
  }
  const bool f16_cache = a.kv.dtype == VLA_F16;
  char* const out = static_cast<char*>(a.q_out) + (row * a.ldqo + mine) * kSize;
  int64_t cell = 0, hop = 0;  // this lane's channels in the cache's slot, and from access to access
  if (file) {
    const int page = page_shift >= 0 ? slot >> page_shift : slot / a.kv.page_size;
    cell = page * a.kv.page_stride + (slot - page * a.kv.page_size) * a.kv.slot_stride + head_of_span * a.kv.head_stride + c0;
    hop = a.kv.head_stride << (5 - span_shift);
  }
  float gain[8];
  bool normed = false;
  uint32_t sat = 0;
  for (int base = from; base < to; base += kAhead) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int j = base + u;
      if (j >= to) break;
      const bool is_q = j < keys, is_v = j >= values;
      float x[8];
      raw[u].unpack(x);
      fetch(j + kAhead, raw[u]);
      if constexpr (NORM) {
        if (j == from || j == keys || j == values) {
          const bf16* g = is_q ? a.q_gain : is_v ? nullptr : a.k_gain;
          normed = g != nullptr;
          if (normed) {
            Eight<VLA_BF16> e;
            e.load<kSplit>(reinterpret_cast<const char*>(g + c0), gap * 2);
            e.unpack(gain);
          }
        }
        if (normed) {
          float ss = 0.f;
#pragma unroll
          for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], ss);
          ss += __shfl_xor_sync(0xffffffffu, ss, 4);
          ss += __shfl_xor_sync(0xffffffffu, ss, 2);
          ss += __shfl_xor_sync(0xffffffffu, ss, 1);
          if (span == 16) ss += __shfl_xor_sync(0xffffffffu, ss, 8);
          const float r = rsqrtf(ss * (span == 16 ? 1.f / 128.f : 1.f / 64.f) + a.eps);
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] *= r * gain[i];
        }
      }
      if (kShuffle && !is_v) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float y = __shfl_sync(0xffffffffu, x[i], partner);
          if (in_turn) x[i] = x[i] * cs[i % kTurns] + y * sn[i % kTurns];
        }
      } else if (LAYOUT != kNoRope && !is_v) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float &p = x[kSplit ? i : 2 * i], &q = x[kSplit ? i + 4 : 2 * i + 1];
          const float turned = p * cs[i] - q * sn[i];
          q = q * cs[i] + p * sn[i];
          p = turned;
        }
      }
      if (!there(j)) continue;
      if (is_q) {
        if (empty) {
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = 0.f;
        }
        Eight<DT> y;
        if constexpr (DT == VLA_F32) {
          y.v[0] = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
          y.v[1] = make_uint4(__float_as_uint(x[4]), __float_as_uint(x[5]), __float_as_uint(x[6]), __float_as_uint(x[7]));
        } else {
          y.v[0] = pack8(x, DT == VLA_F16);
        }
        y.template store<kSplit>(out + j * (kSpan * kSize), gap * kSize);
      } else if (file) {
        if (f16_cache) {
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = clamp_f16(x[i], sat);
        }
        Eight<VLA_F16> y;  // (16 bits of either type)
        y.v[0] = pack8(x, f16_cache);
        y.store<kSplit>(reinterpret_cast<char*>(static_cast<uint16_t*>(is_v ? a.kv.v : a.kv.k) + cell + (j - (is_v ? values : keys)) * hop), gap * 2);
      }
    }
  }
  report_saturation(a.status, sat);
}

}  // namespace

namespace {
template <int THREADS, bool POW2>
int plan_of(const PagePlanArgs& a, cudaStream_t s) {
  static std::atomic<uint64_t> smem_done{0}, cluster_done{0};
  static std::atomic<int> cluster_size[64] = {};
  constexpr int kMost = (4 * kMaxPlanEnvs + 1) * static_cast<int>(sizeof(int));
  VLA_CUDA_TRY(set_smem_limit(page_plan_kernel<THREADS, POW2>, kMost, smem_done));
  VLA_CUDA_TRY(allow_wide_clusters(page_plan_kernel<THREADS, POW2>, cluster_done));
  // a thread has four rows and takes them twice before another CTA joins
  int parts = 1, most = 1;
  while (parts < 16 && a.max_rows > parts * THREADS * 8) parts *= 2;
  VLA_CUDA_TRY(max_cluster_size(page_plan_kernel<THREADS, POW2>, dim3(THREADS), kMost, 16, cluster_size, &most));
  parts = std::min(parts, most);
  const int shift = __builtin_ctz(a.page_size);
  VLA_CUDA_TRY(launch_pdl_cluster(page_plan_kernel<THREADS, POW2>, dim3(parts), dim3(THREADS), (4 * a.n_env + 1) * sizeof(int), s, parts, a, parts, shift));
  note_launch();
  VLA_CUDA_TRY(cudaGetLastError());
  return VLA_OK;
}
}  // namespace

int page_plan_launch(const PagePlanArgs& a, cudaStream_t s) {
  // the sums' barriers are shorter with fewer warps: 16 environments of a row each take 3.8 us with 256 threads and 4.5 with 512,
  // 186 of 106 rows 6.2 and 6.9, 256 of 296 rows 11.1 and 8.7, 438 of 5 rows 7.1 and 6.8
  const bool few = a.n_env <= 256 && a.max_rows <= 32768;
  if (a.page_size & (a.page_size - 1)) return few ? plan_of<256, false>(a, s) : plan_of<512, false>(a, s);
  return few ? plan_of<256, true>(a, s) : plan_of<512, true>(a, s);
}

int rope_table_launch(const RopeTableArgs& a, cudaStream_t s) {
  int dev = 0, sms = 0;
  VLA_CUDA_TRY(cudaGetDevice(&dev));
  VLA_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  // up to 64 positions a thread while every SM has 1024 threads (512: 311 us)
  const int64_t each = std::max<int64_t>(1, std::min<int64_t>(64, static_cast<int64_t>(a.n_pos) * a.pairs / (1024LL * sms)));
  const int apart = static_cast<int>((a.n_pos + each - 1) / each);
  const int64_t grid = (static_cast<int64_t>(apart) * a.pairs + 255) / 256;
  if (grid > 0x7fffffff) return record_error(VLA_ERR_UNSUPPORTED, "vla_rope_table: too many positions");
  VLA_CUDA_TRY(launch_pdl(rope_table_kernel, dim3(static_cast<unsigned>(grid)), dim3(256), 0, s, a, apart));
  note_launch();
  VLA_CUDA_TRY(cudaGetLastError());
  return VLA_OK;
}

namespace {
template <int DT, bool CUT, int HD>
auto append_kernel(int layout, bool norm) {
  return layout == kNoRope  ? (norm ? rope_append_kernel<DT, kNoRope, true, CUT, HD> : rope_append_kernel<DT, kNoRope, false, CUT, HD>)
         : layout == kPairs ? (norm ? rope_append_kernel<DT, kPairs, true, CUT, HD> : rope_append_kernel<DT, kPairs, false, CUT, HD>)
                            : (norm ? rope_append_kernel<DT, kHalves, true, CUT, HD> : rope_append_kernel<DT, kHalves, false, CUT, HD>);
}

template <int DT>
int append_of(const RopeAppendArgs& a, cudaStream_t s) {
  const int hd = a.kv.head_dim, steps = (a.n_q_heads * hd + 255) / 256 + 2 * ((a.kv.n_heads * hd + 255) / 256);
  int dev = 0, sms = 0;
  VLA_CUDA_TRY(cudaGetDevice(&dev));
  VLA_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  // fewer rows than give every SM 32 warps are cut into as many slices as stay below that, down to one access a warp (300 bf16 rows of
  // 28 / 4 heads 4.2 us, 4.8 rounded up; 4500 18.3 and 22.1; 3000 fp16 rows of 32 / 8 heads 20.4 and 18.3)
  const int64_t want = 32LL * sms / a.rows;
  const int slices = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(want, steps)));
  const int64_t units = static_cast<int64_t>(a.rows) * slices, grid = (units + kAppendThreads / 32 - 1) / (kAppendThreads / 32);
  if (grid > 0x7fffffff) return record_error(VLA_ERR_UNSUPPORTED, "vla_rope_append: too many rows");
  const int layout = !a.rope ? kNoRope : a.interleaved ? kPairs : kHalves;
  const bool norm = a.q_gain || a.k_gain;
  auto kern = slices > 1 ? (hd == 64 ? append_kernel<DT, true, 64>(layout, norm) : append_kernel<DT, true, 128>(layout, norm))
                         : (hd == 64 ? append_kernel<DT, false, 64>(layout, norm) : append_kernel<DT, false, 128>(layout, norm));
  const int ps = a.kv.page_size, shift = (ps & (ps - 1)) ? -1 : __builtin_ctz(ps);
  VLA_CUDA_TRY(launch_pdl(kern, dim3(static_cast<unsigned>(grid)), dim3(kAppendThreads), 0, s, a, slices, shift));
  note_launch();
  VLA_CUDA_TRY(cudaGetLastError());
  return VLA_OK;
}
}  // namespace

int rope_append_launch(const RopeAppendArgs& a, cudaStream_t s) {
  return a.dtype == VLA_F32 ? append_of<VLA_F32>(a, s) : a.dtype == VLA_F16 ? append_of<VLA_F16>(a, s) : append_of<VLA_BF16>(a, s);
}

}  // namespace vla
