// The paged cache's bookkeeping and its writes: the page plan of a step (pages taken from a pool,
// rows mapped to slots), the rotary table, and the step that normalises, rotates and files queries,
// keys and values.
#include "lm.h"

namespace vla {

namespace {

// ------------------------------------------------------------------------------------ page plan
// With ctx_e the positions cached (0 for an environment that starts over), have_e = ceil(ctx_e / ps) and
// want_e = ceil((ctx_e + new_e) / ps), environment e takes want_e - have_e pages; exclusive sums over the
// environments give its first row, its first page off the pool's end and, for releases, the place of its old
// pages.  One CTA: the sums by a block scan in shared memory, then one thread per page and per row, which
// finds its environment by bisection.
constexpr int kPlanThreads = 1024;

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

__device__ __forceinline__ int pages_of(int64_t positions, int page_size) {
  return static_cast<int>((positions + page_size - 1) / page_size);
}

__global__ void __launch_bounds__(kPlanThreads) page_plan_kernel(const PagePlanArgs a) {
  extern __shared__ int plan_sm[];
  int* row_first = plan_sm;                 // [n_env]
  int* page_first = row_first + a.n_env;    // [n_env]
  int* old_first = page_first + a.n_env;    // [n_env] released pages before this environment's
  int* ctx0 = old_first + a.n_env;          // [n_env] positions that stay
  __shared__ int64_t sums[3][33];
  __shared__ int64_t carry[3];
  __shared__ int bad;
  pdl_launch_dependents();
  pdl_wait();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid < 3) carry[tid] = 0;
  if (tid == 0) bad = 0;
  const int n_free = *a.n_free_in;
  const int64_t room = static_cast<int64_t>(a.max_pages) * a.page_size;
  __syncthreads();
  for (int base = 0; base < a.n_env; base += kPlanThreads) {
    const int e = base + tid;
    int64_t v[3] = {0, 0, 0};  // rows, pages taken, pages released
    if (e < a.n_env) {
      const int64_t ctx = a.ctx_in[e], add = a.new_len[e];
      const bool out = a.release && a.release[e] != 0;
      const int64_t kept = out ? 0 : ctx;
      if (ctx < 0 || add < 0 || ctx > room || kept + add > room) {
        bad = 1;
        ctx0[e] = 0;
      } else {
        v[0] = add;
        v[1] = pages_of(kept + add, a.page_size) - pages_of(kept, a.page_size);
        v[2] = out ? pages_of(ctx, a.page_size) : 0;
        ctx0[e] = static_cast<int>(kept);
      }
    }
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      const int64_t inc = warp_inclusive(v[i]);
      if (lane == 31) sums[i][warp] = inc;
      v[i] = inc - v[i];
    }
    __syncthreads();
    if (warp < 3) {
      const int64_t s = sums[warp][lane], inc = warp_inclusive(s);
      sums[warp][lane] = carry[warp] + inc - s;
      if (lane == 31) sums[warp][32] = carry[warp] + inc;
    }
    __syncthreads();
    if (e < a.n_env) {
      // totals beyond 32 bits do not fit the rows or the pool and are refused below
      row_first[e] = static_cast<int>(v[0] + sums[0][warp]);
      page_first[e] = static_cast<int>(v[1] + sums[1][warp]);
      old_first[e] = static_cast<int>(v[2] + sums[2][warp]);
    }
    if (tid < 3) carry[tid] = sums[tid][32];
    __syncthreads();
  }
  const int64_t rows64 = carry[0], taken64 = carry[1], old64 = carry[2];
  const bool fits = !bad && n_free >= 0 && n_free + old64 <= a.n_pages && taken64 <= n_free + old64 && rows64 <= a.max_rows;
  const int rows = fits ? static_cast<int>(rows64) : 0, taken = fits ? static_cast<int>(taken64) : 0;
  const int old = fits ? static_cast<int>(old64) : 0;
  const int top = n_free + old;
  if (!fits && tid == 0) raise_status(a.status, VLA_STATUS_PAGES);
  for (int i = tid; i < old; i += kPlanThreads) {
    const int e = env_of(old_first, a.n_env, i);
    a.pool[n_free + i] = a.table[static_cast<int64_t>(e) * a.max_pages + (i - old_first[e])];
  }
  __syncthreads();
  for (int i = tid; i < taken; i += kPlanThreads) {
    const int e = env_of(page_first, a.n_env, i);
    const int col = pages_of(ctx0[e], a.page_size) + i - page_first[e];
    a.table[static_cast<int64_t>(e) * a.max_pages + col] = a.pool[top - 1 - i];
  }
  for (int r = tid; r < a.max_rows; r += kPlanThreads) {
    int e = -1, pos = -1, slot = -1;
    if (r < rows) {
      e = env_of(row_first, a.n_env, r);
      pos = ctx0[e] + r - row_first[e];
      const int have = pages_of(ctx0[e], a.page_size), col = pos / a.page_size;
      const int page = col < have ? a.table[static_cast<int64_t>(e) * a.max_pages + col] : a.pool[top - 1 - (page_first[e] + col - have)];
      if (static_cast<unsigned>(page) < static_cast<unsigned>(a.n_pages))
        slot = page * a.page_size + pos % a.page_size;
      else
        raise_status(a.status, VLA_STATUS_PAGES);
    }
    a.row_env[r] = e;
    a.row_pos[r] = pos;
    a.row_slot[r] = slot;
  }
  for (int e = tid; e < a.n_env; e += kPlanThreads) {
    a.row_start[e] = fits ? row_first[e] : 0;
    a.ctx_out[e] = fits ? ctx0[e] + (e + 1 < a.n_env ? row_first[e + 1] : rows) - row_first[e] : a.ctx_in[e];
  }
  if (tid == 0) {
    a.row_start[a.n_env] = rows;
    *a.n_free_out = fits ? top - taken : n_free;
  }
}

// ----------------------------------------------------------------------------------- rotary table
// One thread per (position, pair), in 64 bits: the angle of position 131071 and frequency 1 needs 17 bits
// before its point, which leaves a 32-bit angle 4e-3 off.
__global__ void __launch_bounds__(256) rope_table_kernel(const RopeTableArgs a) {
  pdl_launch_dependents();
  pdl_wait();
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i >= static_cast<int64_t>(a.n_pos) * a.pairs) return;
  const int pos = static_cast<int>(i / a.pairs), pair = static_cast<int>(i % a.pairs);
  double f = pow(a.theta, -static_cast<double>(pair) / a.pairs);
  if (a.kind == VLA_ROPE_LINEAR) f /= a.factor;
  if (a.kind >= VLA_ROPE_TURNS) {
    const double turns = a.original_len * f / 6.283185307179586476925;
    const double s = a.kind == VLA_ROPE_TURNS ? (turns - a.low) / (a.high - a.low) : (log(turns) - log(a.low)) / (log(a.high) - log(a.low));
    const double keep = fmin(fmax(s, 0.0), 1.0);
    f *= keep + (1.0 - keep) / a.factor;
  }
  double sn, cs;
  sincos(static_cast<double>(pos) * f, &sn, &cs);
  a.table[i] = make_float2(static_cast<float>(cs * a.amplitude), static_cast<float>(sn * a.amplitude));
}

// ------------------------------------------------------------------------------------ rope append
// One warp per (row, head), the head's channels in shared memory between the norm and the rotation.
__device__ __forceinline__ float clamp_f16(float x, uint32_t& sat) {
  if (fabsf(x) > 65504.f && fabsf(x) != INFINITY) {
    x = copysignf(65504.f, x);
    sat = 1u;
  }
  return x;
}

__global__ void __launch_bounds__(256) rope_append_kernel(const RopeAppendArgs a) {
  __shared__ float head_sm[8][128];
  pdl_launch_dependents();
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int heads = a.n_q_heads + 2 * a.kv.n_heads, hd = a.kv.head_dim;
  const int64_t item = static_cast<int64_t>(blockIdx.x) * 8 + warp;
  if (item >= static_cast<int64_t>(a.rows) * heads) return;
  const int row = static_cast<int>(item / heads);
  int head = static_cast<int>(item % heads);
  const bool is_q = head < a.n_q_heads, is_v = head >= a.n_q_heads + a.kv.n_heads;
  if (!is_q) head -= is_v ? a.n_q_heads + a.kv.n_heads : a.n_q_heads;
  int pos = a.row_pos[row];
  const int slot = a.row_slot[row];
  bool bad = pos < -1 || (a.rope && pos >= a.n_pos);
  const bool empty = pos == -1 || bad;
  if (!is_q && !empty && slot != -1 && static_cast<unsigned>(slot) >= static_cast<unsigned>(a.kv.n_pages * a.kv.page_size)) bad = true;
  if (bad && lane == 0) raise_status(a.status, VLA_STATUS_PAGES);
  if (!is_q && (empty || bad || slot < 0)) return;
  const void* src = is_q ? a.q : is_v ? a.v : a.k;
  const int64_t at = row * (is_q ? a.ldq : is_v ? a.ldv : a.ldk) + static_cast<int64_t>(head) * hd;
  float* x = head_sm[warp];
  float ss = 0.f;
  for (int c = lane; c < hd; c += 32) {
    x[c] = load_as_float(src, at + c, a.dtype);
    ss += x[c] * x[c];
  }
  const bf16* gain = is_q ? a.q_gain : is_v ? nullptr : a.k_gain;
  if (gain) {
    const float r = rsqrtf(warp_sum(ss) / static_cast<float>(hd) + a.eps);
    for (int c = lane; c < hd; c += 32) x[c] = x[c] * r * bf2f(gain[c]);
  }
  __syncwarp();
  const int half = a.rope && !is_v ? a.rope_dim / 2 : 0;
  uint32_t sat = 0;
  for (int c = lane; c < hd; c += 32) {
    float y = x[c];
    if (c < 2 * half) {
      const int pair = a.interleaved ? c >> 1 : c < half ? c : c - half;
      const int other = a.interleaved ? c ^ 1 : c < half ? c + half : c - half;
      const bool second = a.interleaved ? c & 1 : c >= half;
      if (!empty) {
        const float2 t = a.rope[static_cast<int64_t>(pos) * half + pair];
        y = second ? x[c] * t.x + x[other] * t.y : x[c] * t.x - x[other] * t.y;
      }
    }
    if (is_q) {
      store_from_float(a.q_out, row * a.ldqo + static_cast<int64_t>(head) * hd + c, empty ? 0.f : y, a.dtype);
    } else {
      if (a.kv.dtype == VLA_F16) y = clamp_f16(y, sat);
      const int64_t to = (slot / a.kv.page_size) * a.kv.page_stride + head * a.kv.head_stride + (slot % a.kv.page_size) * a.kv.slot_stride + c;
      store_from_float(is_v ? a.kv.v : a.kv.k, to, y, a.kv.dtype);
    }
  }
  report_saturation(a.status, sat);
}

}  // namespace

int page_plan_launch(const PagePlanArgs& a, cudaStream_t s) {
  static std::atomic<uint64_t> smem_done{0};
  VLA_CUDA_TRY(set_smem_limit(page_plan_kernel, 4 * kMaxPlanEnvs * static_cast<int>(sizeof(int)), smem_done));
  VLA_CUDA_TRY(launch_pdl(page_plan_kernel, dim3(1), dim3(kPlanThreads), 4 * sizeof(int) * a.n_env, s, a));
  note_launch();
  VLA_CUDA_TRY(cudaGetLastError());
  return VLA_OK;
}

int rope_table_launch(const RopeTableArgs& a, cudaStream_t s) {
  const int64_t n = static_cast<int64_t>(a.n_pos) * a.pairs;
  if ((n + 255) / 256 > 0x7fffffff) return record_error(VLA_ERR_UNSUPPORTED, "vla_rope_table: too many positions");
  VLA_CUDA_TRY(launch_pdl(rope_table_kernel, dim3(static_cast<unsigned>((n + 255) / 256)), dim3(256), 0, s, a));
  note_launch();
  VLA_CUDA_TRY(cudaGetLastError());
  return VLA_OK;
}

int rope_append_launch(const RopeAppendArgs& a, cudaStream_t s) {
  const int64_t items = static_cast<int64_t>(a.rows) * (a.n_q_heads + 2 * a.kv.n_heads);
  if ((items + 7) / 8 > 0x7fffffff) return record_error(VLA_ERR_UNSUPPORTED, "vla_rope_append: too many rows");
  VLA_CUDA_TRY(launch_pdl(rope_append_kernel, dim3(static_cast<unsigned>((items + 7) / 8)), dim3(256), 0, s, a));
  note_launch();
  VLA_CUDA_TRY(cudaGetLastError());
  return VLA_OK;
}

}  // namespace vla
