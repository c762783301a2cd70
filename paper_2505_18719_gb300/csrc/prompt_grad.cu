// Gradient of the causal attention of packed sequences on the tcgen05 tensor cores (include/vla_learn.h).
//
// With c = scale log2(e), P[i][j] = 2^(c s[i][j] - lse[i] log2(e)), D[i] = d_out[i] . out[i], dP = d_out v^T, dS = P (dP - D):
//   d_v[j] = sum_i P[i][j] d_out[i],  d_k[j] = scale sum_i dS[i][j] q[i],  d_q[i] = scale sum_j dS[i][j] k[j].
// Three kernels: D (a row's dot products, bound by bytes); d_k and d_v, a CTA for 128 keys of a key-value head over all queries that
// see them and all query heads that share them; d_q, a CTA for 128 queries over their keys.  The scores and dP are computed in both
// (seven products where one pass would need five), for which every sum has one owner and one order: no atomics, no 32-bit copy
// of d_q in memory, nothing zeroed before.
//
// d_k, d_v: S^T = K Q^T and dP^T = V dO^T have keys as rows, so that P^T and dS^T, written over them, are the
// left operands of d_v += P^T dO and d_k += dS^T Q in tensor memory; Q and dO tiles serve as K-major and as MN-major operands.  While
// the threads compute P of a block the tensor cores work at d_k of the one before and at dP; during dS at d_v and
// the next scores.  Tensor memory: S / P [0, 128), dP / dS [128, 256), d_v [256, 256 + HD), d_k [384, 384 + HD).
// d_q: S [0, 128), dP and dS over it in two buffers [128, 256) [256, 384), d_q [384, 384 + HD).
//
// Weights of bf16 are rounded as they are.  fp16 has 5 bits of exponent: P counts 2^14-fold, and dS 2^e-fold with the e that brings
// 2 max |d_out[i]| max |v[j]| of the sequence, which no |dS| passes, below 2^15; so gradients of any size keep their bits.
// Rows of Q, dO and K behind a sequence's last one become zeros in shared memory (their weights are zeros, but
// a NaN would spoil the sums over rows), up to the next multiple of 16, where the products stop.
//
// Roles of both (384 threads): warp 0 TMA, warp 1 MMAs (and tensor memory), warp 2 tiles that end behind a sequence's last row, and the rows' lse and D, warp 3
// items, warps 4-11 the element-wise part, two warps a lane quarter with half of the columns each, and the output.
#include <algorithm>

#include "gemm.h"
#include "prompt_items.cuh"

namespace vla {

namespace {

constexpr int kThreads = 384;
constexpr int kRows = 4;         // blocks of rows' lse and D in flight
constexpr int kNormRows = 32;    // rows of one entry of the largest norms
constexpr float kPShift = 14.f;  // log2 of the fp16 weights' factor

struct Params {
  PromptGradArgs g;
  int group, items_bound;
  float c;               // scale log2(e)
  const float* delta;    // [rows][n_q_heads]
  const float* norms;    // [2][blocks of kNormRows rows]: largest |d_out| and |v| (fp16)
  int norm_blocks;
  uint64_t wait_limit;
};

// ------------------------------------------------------------------------------------------- D
template <int HD, bool FP16>
__global__ void __launch_bounds__(256) prompt_delta_kernel(const PromptGradArgs a, float* delta, float* norms, int norm_blocks) {
  constexpr int L = HD / 8, HEADS = 32 / L;  // lanes of a head, heads of a step
  __shared__ float red[2][8];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  float most[2] = {0.f, 0.f};
  if (blockIdx.x == 0) check_starts(a.f.seq_start, a.f.n_seq, a.f.rows, threadIdx.x, 256, a.f.status);
  auto eight = [](uint4 w, float (&y)[8]) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = FP16 ? unpack_f16x2(u[i]) : unpack_bf16x2(u[i]);
      y[2 * i] = f.x;
      y[2 * i + 1] = f.y;
    }
  };
  auto over_head = [](float v) {
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
  };
  // a sequence of finite numbers keeps its factor, whatever lies around it
  auto finite = [](float v) { return v <= 3e38f ? v : 0.f; };
  const Outside out(a.f.seq_start, a.f.n_seq, a.f.rows);
  for (int i = warp; i < kNormRows; i += 8) {
    const int row = blockIdx.x * kNormRows + i;
    if (row >= out.last) break;
    if (row < out.first) continue;
    const uint4* o = static_cast<const uint4*>(elem(a.f.out, row * a.f.ldo));
    const uint4* d = static_cast<const uint4*>(elem(a.d_out, row * a.lddo));
#pragma unroll 4
    for (int h = 0; h < a.f.n_q_heads; h += HEADS) {
      const bool on = h + lane / L < a.f.n_q_heads;
      float x[8], y[8], s = 0.f, n = 0.f;
      eight(on ? o[h * L + lane] : make_uint4(0u, 0u, 0u, 0u), x);
      eight(on ? d[h * L + lane] : make_uint4(0u, 0u, 0u, 0u), y);
#pragma unroll
      for (int e = 0; e < 8; ++e) s = fmaf(x[e], y[e], s);
      s = over_head(s);
      if (on && lane % L == 0) delta[static_cast<int64_t>(row) * a.f.n_q_heads + h + lane / L] = s;
      if (FP16) {
#pragma unroll
        for (int e = 0; e < 8; ++e) n = fmaf(y[e], y[e], n);
        most[0] = fmaxf(most[0], finite(over_head(n)));
      }
    }
    if (FP16) {
      const uint4* v = static_cast<const uint4*>(elem(a.f.v, row * a.f.ldv));
      for (int h = 0; h < a.f.n_kv_heads; h += HEADS) {
        float y[8], n = 0.f;
        eight(h + lane / L < a.f.n_kv_heads ? v[h * L + lane] : make_uint4(0u, 0u, 0u, 0u), y);
#pragma unroll
        for (int e = 0; e < 8; ++e) n = fmaf(y[e], y[e], n);
        most[1] = fmaxf(most[1], finite(over_head(n)));
      }
    }
  }
  if constexpr (FP16) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      most[k] = warp_max(most[k]);
      if (lane == 0) red[k][warp] = most[k];
    }
    __syncthreads();
    if (threadIdx.x >= 2) return;
    float m = 0.f;
    for (int w = 0; w < 8; ++w) m = fmaxf(m, red[threadIdx.x][w]);
    norms[threadIdx.x * norm_blocks + blockIdx.x] = sqrtf(m);
  }
}

// ------------------------------------------------------------------------------------- both kernels
// The exponent e of a sequence's factor 2^e of dS (fp16): 2 |d_out| |v| 2^e <= 2^15 (whole warp).
__device__ __forceinline__ int ds_exponent(const Params& p, const Item& it) {
  float n[2] = {0.f, 0.f};
  const int b0 = it.begin / kNormRows, b1 = (it.begin + it.len - 1) / kNormRows;
  for (int b = b0 + (threadIdx.x & 31); b <= b1; b += 32) {
    n[0] = fmaxf(n[0], p.norms[b]);
    n[1] = fmaxf(n[1], p.norms[p.norm_blocks + b]);
  }
  const float most = warp_max(n[0]) * warp_max(n[1]);
  if (!(most > 0.f) || most > 1e37f) return 0;
  int e;
  frexpf(most, &e);  // most <= 2^e
  return min(max(14 - e, -100), 100);
}
__device__ __forceinline__ float exp2_int(int e) { return __int_as_float((e + 127) << 23); }

template <int HD>
struct Smem {
  static constexpr int kStages = HD == 128 ? 2 : 4;
  static constexpr uint32_t kTileBytes = kTile * HD * 2;
  // two tiles of the item, two rings, a warp's rows on their way out, rows' lse and D, barriers
  static constexpr uint32_t kRingA = 2 * kTileBytes, kRingB = kRingA + kStages * kTileBytes, kStage = kRingB + kStages * kTileBytes;
  static constexpr uint32_t kRowData = kStage + 8 * 2048, kBars = kRowData + kRows * 1024, kTotal = 1024 + kBars + 1024;
  static_assert(kTotal <= 232448, "shared memory per CTA");
};

// Barriers: the item's two tiles, the rings A and B (up to 4 stages each), loads into them that go through warp 2, rows' data, the steps
// of a block, the item's end, descriptors.
enum : int {
  AFULL = 0, AFREE = 1, BFULL = 2, BFREE = 3, RAFULL = 4, RAFREE = 8, RBFULL = 12, RBFREE = 16, TAILA = 20, TAILB = 24, RFULL = 28, RFREE = 32,
  SFULL = 36, SREAD = 37, PFULL = 38, DPFULL = 39, DSFULL = 41, DONE = 42, DRAIN = 43, IFULL = 44, IFREE = 52, kBarCount = 60
};

struct Shared {
  uint8_t* smem;
  uint32_t s0, b0;
  Item* items;
  uint32_t* tmem_slot;
  volatile int* abort_flag;
  float* rows;
  __device__ __forceinline__ uint32_t bar(int i) const { return b0 + 8u * static_cast<uint32_t>(i); }
};
template <int HD>
__device__ __forceinline__ Shared shared_of(uint8_t* raw, int readers) {
  using Sm = Smem<HD>;
  Shared sh;
  sh.smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~static_cast<uintptr_t>(1023));
  uint64_t* bars = reinterpret_cast<uint64_t*>(sh.smem + Sm::kBars);
  sh.s0 = smem_u32(sh.smem);
  sh.b0 = smem_u32(bars);
  sh.items = reinterpret_cast<Item*>(bars + kBarCount);
  sh.tmem_slot = reinterpret_cast<uint32_t*>(sh.items + kItems);
  sh.abort_flag = reinterpret_cast<volatile int*>(sh.tmem_slot + 1);
  sh.rows = reinterpret_cast<float*>(sh.smem + Sm::kRowData);
  static_assert(kBarCount * 8 + kItems * 16 + 8 <= 1024 && kBarCount % 2 == 0, "barrier area");
  if (threadIdx.x == 0) {
    for (int i = 0; i < kBarCount; ++i) {
      const bool eight = i == SREAD || i == PFULL || i == DSFULL || (i >= RFREE && i < RFREE + kRows);
      mbar_init(sh.bar(i), i >= IFREE ? readers : eight ? 8 : 1);
    }
    *sh.abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if ((threadIdx.x >> 5) == 1) tmem_take(smem_u32(sh.tmem_slot));
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  return sh;
}
__device__ __forceinline__ void end_of_kernel(uint32_t tmem) {
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if ((threadIdx.x >> 5) == 1) {
    tc_fence_after();
    tmem_give(tmem);
  }
}
// Next descriptor, for one thread or a whole warp of which lane 0 answers; false at a timeout.
__device__ __forceinline__ bool next_item(const Shared& sh, int k, Item& it, uint32_t* status, uint64_t limit, bool whole_warp) {
  if (whole_warp ? !warp_waits(sh.bar(IFULL + (k & 7)), (k >> 3) & 1, sh.abort_flag, status, limit)
                 : !quick_wait(sh.bar(IFULL + (k & 7)), (k >> 3) & 1, sh.abort_flag, status, limit))
    return false;
  it = sh.items[k & 7];
  if (whole_warp) __syncwarp();
  if (!whole_warp || (threadIdx.x & 31) == 0) mbar_arrive(sh.bar(IFREE + (k & 7)));
  return it.len >= 0;
}
// The warp that finds the items; count(len) and what(len, number) as a pair.
template <class Count, class What>
__device__ __forceinline__ void put_items(const Params& p, const Shared& sh, const Count& count, const What& what) {
  const PromptArgs& f = p.g.f;
  const int lane = threadIdx.x & 31;
  int k = 0;
  auto put = [&](const Item& it) {
    if (k >= kItems && !warp_waits(sh.bar(IFREE + (k & 7)), ((k >> 3) - 1) & 1, sh.abort_flag, f.status, p.wait_limit)) return false;
    if (lane == 0) {
      sh.items[k & 7] = it;
      mbar_arrive(sh.bar(IFULL + (k & 7)));
    }
    ++k;
    return true;
  };
  if (find_items(f.seq_start, f.n_seq, f.rows, blockIdx.x, gridDim.x, p.items_bound, count, [&](int begin, int len, int u) {
        const int2 w = what(len, u);
        return put(Item{begin, len, w.x, w.y});
      }))
    put(Item{0, -1, 0, 0});
}
template <int HD>
__device__ __forceinline__ void load_tile(const Shared& sh, uint32_t dst, const CUtensorMap* map, int bar, int head, int row) {
  mbar_arrive_expect_tx(sh.bar(bar), Smem<HD>::kTileBytes);
#pragma unroll
  for (int kb = 0; kb < HD / 64; ++kb) tma_load_2d(dst + kb * kBlockBytes, map, sh.bar(bar), head * HD + kb * 64, row);
}
// Loads into a ring: of a sequence's last rows to the barrier of warp 2, which makes those behind the last zeros and hands the tile on.
template <int HD>
struct RingLoads {
  static constexpr int NS = Smem<HD>::kStages;
  const Shared& sh;
  int full, tail, n = 0;
  uint32_t base, on_tail = 0, tail_phase = 0;  // of each slot: its last load went to warp 2; how many did, modulo 2
  __device__ __forceinline__ void load(const CUtensorMap* map, int head, int row, bool is_tail) {
    const int s = n % NS;
    load_tile<HD>(sh, base + s * Smem<HD>::kTileBytes, map, (is_tail ? tail : full) + s, head, row);
    on_tail = (on_tail & ~(1u << s)) | (static_cast<uint32_t>(is_tail) << s);
    tail_phase ^= static_cast<uint32_t>(is_tail) << s;
    ++n;
  }
  // nothing may land after the CTA has gone
  __device__ __forceinline__ void drain(uint64_t limit) const {
    for (int i = max(0, n - NS); i < n; ++i) {
      const int s = i % NS;
      if ((on_tail >> s) & 1)
        wait_drain(sh.bar(tail + s), ((tail_phase >> s) & 1) ^ 1, limit);
      else
        wait_drain(sh.bar(full + s), (i / NS) & 1, limit);
    }
  }
};
// ------------------------------------------------------------------------------------------- d_k, d_v
// Item: key tile a, key-value head b.  Its blocks: query heads of the group, for each the query tiles from the last down to a (so that
// CTAs of one head read the same tiles at about the same time).
template <int HD, bool FP16>
__global__ void __launch_bounds__(kThreads, 1)
    prompt_grad_keys_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                            const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_g, const Params p) {
  using Sm = Smem<HD>;
  constexpr int NS = Sm::kStages;
  extern __shared__ uint8_t smem_raw[];
  const Shared sh = shared_of<HD>(smem_raw, 1 + 1 + 1 + 8);
  const uint32_t tmem = *sh.tmem_slot;
  const PromptArgs& f = p.g.f;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint32_t* status = f.status;
  const uint64_t limit = p.wait_limit;
  auto wait1 = [&](int bar, int phase) { return quick_wait(sh.bar(bar), static_cast<uint32_t>(phase) & 1u, sh.abort_flag, status, limit); };
  auto waitw = [&](int bar, int phase) { return warp_waits(sh.bar(bar), static_cast<uint32_t>(phase) & 1u, sh.abort_flag, status, limit); };
  auto tiles = [](const Item& it) { return (it.len + kTile - 1) / kTile; };
  auto rows_of = [](const Item& it, int t) { return min(kTile, it.len - t * kTile); };
  auto slot_a = [&](int w) { return sh.s0 + Sm::kRingA + (w % NS) * Sm::kTileBytes; };  // Q
  auto slot_b = [&](int w) { return sh.s0 + Sm::kRingB + (w % NS) * Sm::kTileBytes; };  // dO

  if (warp == 0) {
    if (lane == 0) {
      RingLoads<HD> q{sh, RAFULL, TAILA, 0, sh.s0 + Sm::kRingA}, g{sh, RBFULL, TAILB, 0, sh.s0 + Sm::kRingB};
      int w = 0, k = 0, n_k = 0, n_v = 0;  // blocks, items, K and V tiles loaded
      Item it;
      bool ok = true;
      for (; ok && next_item(sh, k, it, status, limit, false); ++k) {
        const int nt = tiles(it), row = it.begin + it.a * kTile;
        bool first = true;
        for (int h = it.b * p.group; h < (it.b + 1) * p.group && ok; ++h) {
          for (int t = nt - 1; t >= it.a && ok; --t, ++w, first = false) {
            const bool tail = rows_of(it, t) < kTile;
            if (first) {
              if (!(ok = k == 0 || wait1(AFREE, k - 1))) break;
              load_tile<HD>(sh, sh.s0, &tm_k, AFULL, it.b, row);
              ++n_k;
            }
            if (!(ok = w < NS || wait1(RAFREE + w % NS, w / NS - 1))) break;
            q.load(&tm_q, h, it.begin + t * kTile, tail);
            if (first) {
              if (!(ok = k == 0 || wait1(BFREE, k - 1))) break;
              load_tile<HD>(sh, sh.s0 + Sm::kTileBytes, &tm_v, BFULL, it.b, row);
              ++n_v;
            }
            if (!(ok = w < NS || wait1(RBFREE + w % NS, w / NS - 1))) break;
            g.load(&tm_g, h, it.begin + t * kTile, tail);
          }
        }
      }
      q.drain(limit);
      g.drain(limit);
      if (n_k) wait_drain(sh.bar(AFULL), (n_k - 1) & 1, limit);
      if (n_v) wait_drain(sh.bar(BFULL), (n_v - 1) & 1, limit);
    }
  } else if (warp == 1) {
    const uint32_t tS = tmem, tP = tmem + 128, tV = tmem + 256, tK = tmem + 384;
    const uint32_t dk = tile_desc(sh.s0), dv = tile_desc(sh.s0 + Sm::kTileBytes), io = tile_idesc(HD, FP16, true);
    int w = 0, k = 0;
    Item it;
    bool ok = true;
    for (; ok && next_item(sh, k, it, status, limit, true); ++k) {
      it = Item{0, uniform(it.len), uniform(it.a), uniform(it.b)};
      const int nt = tiles(it), per_head = nt - it.a, units = per_head * p.group;
      int ahead = 0;  // the next scores' block within its head
      auto steps_at = [&](int at) { return (rows_of(it, nt - 1 - at) + 15) / 16; };
      // S of block u; dP
      auto scores = [&](int u) {
        const int s = (w + u) % NS;
        if (!waitw(RAFULL + s, (w + u) / NS)) return false;
        tc_fence_after();
        const uint32_t dq = tile_desc(slot_a(w + u)), id = tile_idesc(16 * steps_at(ahead), FP16, false);
        if (elected()) {
#pragma unroll
          for (int i = 0; i < HD / 16; ++i) tile_mma(tS, dk + k_major_step(i), dq + k_major_step(i), id, i > 0);
          tc_commit(sh.bar(SFULL));
          if (u == units - 1) tc_commit(sh.bar(AFREE));
        }
        __syncwarp();
        return true;
      };
      auto products = [&](int u) {
        const int s = (w + u) % NS;
        if (!waitw(RBFULL + s, (w + u) / NS)) return false;
        tc_fence_after();
        const uint32_t dg = tile_desc(slot_b(w + u)), id = tile_idesc(16 * steps_at(ahead), FP16, false);
        if (elected()) {
#pragma unroll
          for (int i = 0; i < HD / 16; ++i) tile_mma(tP, dv + k_major_step(i), dg + k_major_step(i), id, i > 0);
          tc_commit(sh.bar(DPFULL));
          if (u == units - 1) tc_commit(sh.bar(BFREE));
        }
        __syncwarp();
        return true;
      };
      if (!(ok = waitw(AFULL, k) && (w == 0 || waitw(RBFREE + (w - 1) % NS, (w - 1) / NS)) && scores(0) && waitw(BFULL, k) &&
                 (w == 0 || waitw(RAFREE + (w - 1) % NS, (w - 1) / NS)) && products(0)))
        break;
      for (int u = 0; u < units && ok; ++u) {
        const int s = (w + u) % NS, steps = steps_at(ahead);
        ahead = ahead + 1 == per_head ? 0 : ahead + 1;
        if (!(ok = waitw(PFULL, w + u))) break;
        tc_fence_after();
        const uint32_t dg = tile_desc(slot_b(w + u)), dq = tile_desc(slot_a(w + u)), more = u > 0;
        if (elected()) {
#pragma unroll
          for (int i = 0; i < kTile / 16; ++i)
            if (i < steps) tile_mma_ts(tV, tS + halves_step(i), dg + mn_major_step(i), io, i > 0 ? 1u : more);
          tc_commit(sh.bar(RBFREE + s));
        }
        __syncwarp();
        // the next scores go over P once d_v has read it, the next dP over dS once d_k has; the first two in the order in which they get ready
        bool next_s = u + 1 < units, this_k = true;
        uint64_t since = 0;
        uint32_t spins = 0;
        while (ok && (next_s || this_k)) {
          if (this_k && warp_ready(sh.bar(DSFULL), (w + u) & 1)) {
            tc_fence_after();
            if (elected()) {
#pragma unroll
              for (int i = 0; i < kTile / 16; ++i)
                if (i < steps) tile_mma_ts(tK, tP + halves_step(i), dq + mn_major_step(i), io, i > 0 ? 1u : more);
              tc_commit(sh.bar(RAFREE + s));
            }
            __syncwarp();
            this_k = false;
          } else if (next_s && warp_ready(sh.bar(RBFREE + s), ((w + u) / NS) & 1)) {
            if (!(ok = scores(u + 1))) break;
            next_s = false;
          } else if ((++spins & 1023u) == 0) {  // (the clock is slow to read)
            if (spins == 1024) since = globaltimer();
            if (__any_sync(0xffffffffu, *sh.abort_flag != 0)) {
              ok = false;
            } else if (__any_sync(0xffffffffu, globaltimer() - since > limit)) {
              if (lane == 0) {
                *sh.abort_flag = 1;
                if (status) atomicOr(status, VLA_STATUS_TIMEOUT);
              }
              ok = false;
            }
          }
        }
        if (ok && u + 1 < units) ok = waitw(RAFREE + s, (w + u) / NS) && products(u + 1);
      }
      if (elected()) tc_commit(sh.bar(DONE));
      __syncwarp();
      w += units;
    }
    if (elected()) tc_commit(sh.bar(DRAIN));
    wait_drain(sh.bar(DRAIN), 0, limit);
  } else if (warp == 2) {
    int w = 0, k = 0, phase = 0;  // phase: of each slot, its tiles so far that came here first, modulo 2
    Item it;
    bool ok = true;
    for (; ok && next_item(sh, k, it, status, limit, true); ++k) {
      const int nt = tiles(it);
      for (int h = it.b * p.group; h < (it.b + 1) * p.group && ok; ++h) {
        for (int t = nt - 1; t >= it.a; --t, ++w) {
          const int live = rows_of(it, t), s = w % NS;
          float l[4], d[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int r = i * 32 + lane;
            const int64_t at = static_cast<int64_t>(it.begin + t * kTile + min(r, live - 1)) * f.n_q_heads + h;
            l[i] = r < live ? fmaf(f.lse[at], -kLog2e, FP16 ? kPShift : 0.f) : -INFINITY;  // weights of 0 behind the last row
            d[i] = r < live ? p.delta[at] : 0.f;
          }
          if (!(ok = w < kRows || waitw(RFREE + w % kRows, w / kRows - 1))) break;
          float* dst = sh.rows + (w % kRows) * 256;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            dst[i * 32 + lane] = l[i];
            dst[128 + i * 32 + lane] = d[i];
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(sh.bar(RFULL + w % kRows));
          if (live < kTile) {
            if (!(ok = waitw(TAILA + s, phase >> s))) break;
            zero_tile_rows<HD>(sh.smem + (slot_a(w) - sh.s0), live, (live + 15) & ~15);
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(sh.bar(RAFULL + s));
            if (!(ok = waitw(TAILB + s, phase >> s))) break;
            zero_tile_rows<HD>(sh.smem + (slot_b(w) - sh.s0), live, (live + 15) & ~15);
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(sh.bar(RBFULL + s));
            phase ^= 1 << s;
          }
        }
      }
    }
  } else if (warp == 3) {
    const int Hk = f.n_kv_heads;
    put_items(
        p, sh, [&](int len) { return static_cast<int64_t>((len + kTile - 1) / kTile) * Hk; }, [&](int, int u) { return make_int2(u / Hk, u % Hk); });
    const Outside out(f.seq_start, f.n_seq, f.rows);
    for (int i = blockIdx.x; i < out.count(); i += gridDim.x) {
      zero_row(elem(p.g.d_k, out.row(i) * p.g.lddk), Hk * HD);
      zero_row(elem(p.g.d_v, out.row(i) * p.g.lddv), Hk * HD);
    }
  } else {
    const int half = (warp - 4) >> 2, q4 = warp & 3, r = q4 * 32 + lane;  // columns 64 half .. 64 half + 63 of row (key) r
    const uint32_t quarter = static_cast<uint32_t>(q4 * 32) << 16;
    const uint32_t tS = tmem + quarter + 64 * half, tP = tS + 128;
    uint8_t* staging = sh.smem + Sm::kStage + (warp - 4) * 2048;
    int w = 0, k = 0;
    Item it;
    bool ok = true;
    for (; ok && next_item(sh, k, it, status, limit, true); ++k) {
      const int nt = tiles(it), e = FP16 ? ds_exponent(p, it) : 0;
      const float up = FP16 ? exp2_int(e - static_cast<int>(kPShift)) : 1.f;
      for (int h = 0; h < p.group && ok; ++h) {
        for (int t = nt - 1; t >= it.a; --t, ++w) {
          const bool work = 64 * half < rows_of(it, t);  // else no product reads these columns
          const float4* rl = reinterpret_cast<const float4*>(sh.rows + (w % kRows) * 256 + 64 * half);
          uint32_t s[64], x[64];
          if (!(ok = waitw(RFULL + w % kRows, w / kRows) && waitw(SFULL, w))) break;
          tc_fence_after();
          if (work) {
            tmem_ld32(tS, s);
            tmem_ld32(tS + 32, s + 32);
            tmem_wait_ld();
            const uint64_t c2 = pair_of(p.c, p.c);
#pragma unroll
            for (int i = 0; i < 64; i += 32) {
              uint32_t y[16];
#pragma unroll
              for (int j = 0; j < 32; j += 4) {
                const float4 l = rl[(i + j) / 4];
                const float2 a = halves_of(fma2(pair_of(__uint_as_float(s[i + j]), __uint_as_float(s[i + j + 1])), c2, pair_of(l.x, l.y)));
                const float2 b = halves_of(fma2(pair_of(__uint_as_float(s[i + j + 2]), __uint_as_float(s[i + j + 3])), c2, pair_of(l.z, l.w)));
                float v[4] = {ex2(a.x), ex2(a.y), ex2(b.x), ex2(b.y)};
                if (t == it.a) {  // queries before the key do not see it
#pragma unroll
                  for (int q = 0; q < 4; ++q) v[q] = 64 * half + i + j + q >= r ? v[q] : 0.f;
                }
#pragma unroll
                for (int q = 0; q < 4; ++q) s[i + j + q] = __float_as_uint(v[q]);
                y[j / 2] = pack2<FP16>(v[0], v[1]);
                y[j / 2 + 1] = pack2<FP16>(v[2], v[3]);
              }
              tmem_st16(tS + i / 2, y);
            }
            tmem_wait_st();
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(sh.bar(PFULL));
          if (!(ok = waitw(DPFULL, w))) break;
          tc_fence_after();
          if (work) {
            tmem_ld32(tP, x);
            tmem_ld32(tP + 32, x + 32);
            tmem_wait_ld();
            const uint64_t up2 = pair_of(up, up), minus = pair_of(-1.f, -1.f);
#pragma unroll
            for (int i = 0; i < 64; i += 32) {
              uint32_t y[16];
#pragma unroll
              for (int j = 0; j < 32; j += 4) {
                const float4 d = rl[32 + (i + j) / 4];
                uint64_t a = fma2(pair_of(d.x, d.y), minus, pair_of(__uint_as_float(x[i + j]), __uint_as_float(x[i + j + 1])));
                uint64_t b = fma2(pair_of(d.z, d.w), minus, pair_of(__uint_as_float(x[i + j + 2]), __uint_as_float(x[i + j + 3])));
                if (FP16) {
                  a = mul2(a, up2);
                  b = mul2(b, up2);
                }
                const float2 ya = halves_of(mul2(a, pair_of(__uint_as_float(s[i + j]), __uint_as_float(s[i + j + 1]))));
                const float2 yb = halves_of(mul2(b, pair_of(__uint_as_float(s[i + j + 2]), __uint_as_float(s[i + j + 3]))));
                y[j / 2] = pack2<FP16>(ya.x, ya.y);
                y[j / 2 + 1] = pack2<FP16>(yb.x, yb.y);
              }
              tmem_st16(tP + i / 2, y);
            }
            tmem_wait_st();
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(sh.bar(DSFULL));
            mbar_arrive(sh.bar(RFREE + w % kRows));
          }
        }
      }
      if (!ok || !(ok = waitw(DONE, k))) break;
      tc_fence_after();
      const int row0 = it.a * kTile + q4 * 32;
      if (half == 0)
        store_tile<FP16, HD / 32>(tmem + quarter + 256, staging, FP16 ? exp2_int(-static_cast<int>(kPShift)) : 1.f,
                                  elem(p.g.d_v, (it.begin + row0) * p.g.lddv + it.b * HD), p.g.lddv, it.len - row0);
      else
        store_tile<FP16, HD / 32>(tmem + quarter + 384, staging, FP16 ? f.scale * exp2_int(-e) : f.scale,
                                  elem(p.g.d_k, (it.begin + row0) * p.g.lddk + it.b * HD), p.g.lddk, it.len - row0);
      tc_fence_before();
    }
  }
  end_of_kernel(tmem);
}

// ------------------------------------------------------------------------------------------- d_q
// Item: query tile a, query head b; key tiles 0 .. a.
template <int HD, bool FP16>
__global__ void __launch_bounds__(kThreads, 1)
    prompt_grad_queries_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                               const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_g, const Params p) {
  using Sm = Smem<HD>;
  constexpr int NS = Sm::kStages;
  extern __shared__ uint8_t smem_raw[];
  const Shared sh = shared_of<HD>(smem_raw, 1 + 1 + 1 + 8);
  const uint32_t tmem = *sh.tmem_slot;
  const PromptArgs& f = p.g.f;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint32_t* status = f.status;
  const uint64_t limit = p.wait_limit;
  auto wait1 = [&](int bar, int phase) { return quick_wait(sh.bar(bar), static_cast<uint32_t>(phase) & 1u, sh.abort_flag, status, limit); };
  auto waitw = [&](int bar, int phase) { return warp_waits(sh.bar(bar), static_cast<uint32_t>(phase) & 1u, sh.abort_flag, status, limit); };
  auto slot_a = [&](int w) { return sh.s0 + Sm::kRingA + (w % NS) * Sm::kTileBytes; };  // K
  auto slot_b = [&](int w) { return sh.s0 + Sm::kRingB + (w % NS) * Sm::kTileBytes; };  // V

  if (warp == 0) {
    if (lane == 0) {
      RingLoads<HD> kr{sh, RAFULL, TAILA, 0, sh.s0 + Sm::kRingA}, vr{sh, RBFULL, TAILB, 0, sh.s0 + Sm::kRingB};
      int w = 0, k = 0, n_q = 0, n_g = 0;  // blocks, items, Q and dO tiles loaded
      Item it;
      bool ok = true;
      for (; ok && next_item(sh, k, it, status, limit, false); ++k) {
        const int g = it.b / p.group, row = it.begin + it.a * kTile;
        for (int j = 0; j <= it.a && ok; ++j, ++w) {
          if (j == 0) {
            if (!(ok = k == 0 || wait1(AFREE, k - 1))) break;
            load_tile<HD>(sh, sh.s0, &tm_q, AFULL, it.b, row);
            ++n_q;
          }
          if (!(ok = w < NS || wait1(RAFREE + w % NS, w / NS - 1))) break;
          kr.load(&tm_k, g, it.begin + j * kTile, it.len - j * kTile < kTile);
          if (j == 0) {
            if (!(ok = k == 0 || wait1(BFREE, k - 1))) break;
            load_tile<HD>(sh, sh.s0 + Sm::kTileBytes, &tm_g, BFULL, it.b, row);
            ++n_g;
          }
          if (!(ok = w < NS || wait1(RBFREE + w % NS, w / NS - 1))) break;
          vr.load(&tm_v, g, it.begin + j * kTile, false);
        }
      }
      kr.drain(limit);
      vr.drain(limit);
      if (n_q) wait_drain(sh.bar(AFULL), (n_q - 1) & 1, limit);
      if (n_g) wait_drain(sh.bar(BFULL), (n_g - 1) & 1, limit);
    }
  } else if (warp == 1) {
    const uint32_t tS = tmem, tQ = tmem + 384;
    const uint32_t dq = tile_desc(sh.s0), dg = tile_desc(sh.s0 + Sm::kTileBytes), io = tile_idesc(HD, FP16, true);
    int w = 0, k = 0;
    Item it;
    bool ok = true;
    for (; ok && next_item(sh, k, it, status, limit, true); ++k) {
      it = Item{0, uniform(it.len), uniform(it.a), uniform(it.b)};
      auto steps_of = [&](int j) { return (min(kTile, it.len - j * kTile) + 15) / 16; };
      auto scores = [&](int j) {
        const int s = (w + j) % NS;
        if (!waitw(RAFULL + s, (w + j) / NS)) return false;
        tc_fence_after();
        const uint32_t dk = tile_desc(slot_a(w + j)), id = tile_idesc(16 * steps_of(j), FP16, false);
        if (elected()) {
#pragma unroll
          for (int i = 0; i < HD / 16; ++i) tile_mma(tS, dq + k_major_step(i), dk + k_major_step(i), id, i > 0);
          tc_commit(sh.bar(SFULL));
          if (j == it.a) tc_commit(sh.bar(AFREE));
        }
        __syncwarp();
        return true;
      };
      auto products = [&](int j) {
        const int s = (w + j) % NS;
        if (!waitw(RBFULL + s, (w + j) / NS)) return false;
        tc_fence_after();
        const uint32_t dv = tile_desc(slot_b(w + j)), id = tile_idesc(16 * steps_of(j), FP16, false), tP = tmem + 128 + ((w + j) & 1) * 128;
        if (elected()) {
#pragma unroll
          for (int i = 0; i < HD / 16; ++i) tile_mma(tP, dg + k_major_step(i), dv + k_major_step(i), id, i > 0);
          tc_commit(sh.bar(DPFULL + ((w + j) & 1)));
          tc_commit(sh.bar(RBFREE + s));
          if (j == it.a) tc_commit(sh.bar(BFREE));
        }
        __syncwarp();
        return true;
      };
      // (an item's first dP: the item before has ended, or the threads would not have read its last scores)
      if (!(ok = waitw(AFULL, k) && (w == 0 || waitw(SREAD, w - 1)) && scores(0) && waitw(BFULL, k) &&
                 (w < 2 || waitw(RAFREE + (w - 2) % NS, (w - 2) / NS)) && products(0)))
        break;
      for (int j = 0; j <= it.a && ok; ++j) {
        // the next scores once the threads have read these, the next dP over the dS of the block before once d_q has read it
        if (j < it.a && !(ok = waitw(SREAD, w + j) && scores(j + 1) && (w + j == 0 || waitw(RAFREE + (w + j - 1) % NS, (w + j - 1) / NS)) &&
                               products(j + 1)))
          break;
        if (!(ok = waitw(DSFULL, w + j))) break;
        tc_fence_after();
        const uint32_t dk = tile_desc(slot_a(w + j)), tD = tmem + 128 + ((w + j) & 1) * 128, more = j > 0;
        const int steps = steps_of(j);
        if (elected()) {
#pragma unroll
          for (int i = 0; i < kTile / 16; ++i)
            if (i < steps) tile_mma_ts(tQ, tD + halves_step(i), dk + mn_major_step(i), io, i > 0 ? 1u : more);
          tc_commit(sh.bar(RAFREE + (w + j) % NS));
        }
        __syncwarp();
      }
      if (elected()) tc_commit(sh.bar(DONE));
      __syncwarp();
      w += it.a + 1;
    }
    if (elected()) tc_commit(sh.bar(DRAIN));
    wait_drain(sh.bar(DRAIN), 0, limit);
  } else if (warp == 2) {
    int w = 0, k = 0, phase = 0;
    Item it;
    for (; next_item(sh, k, it, status, limit, true); ++k) {
      w += it.a + 1;
      const int live = it.len - it.a * kTile, s = (w - 1) % NS;
      if (live >= kTile) continue;
      if (!waitw(TAILA + s, phase >> s)) break;
      phase ^= 1 << s;
      zero_tile_rows<HD>(sh.smem + (slot_a(w - 1) - sh.s0), live, (live + 15) & ~15);
      fence_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(sh.bar(RAFULL + s));
    }
  } else if (warp == 3) {
    const int H = f.n_q_heads;
    put_items(
        p, sh, [&](int len) { return static_cast<int64_t>((len + kTile - 1) / kTile) * H; },
        [&](int len, int u) { return make_int2((len + kTile - 1) / kTile - 1 - u / H, u % H); });
    const Outside out(f.seq_start, f.n_seq, f.rows);
    for (int i = blockIdx.x; i < out.count(); i += gridDim.x) zero_row(elem(p.g.d_q, out.row(i) * p.g.lddq), H * HD);
  } else {
    const int half = (warp - 4) >> 2, q4 = warp & 3, r = q4 * 32 + lane;
    const uint32_t quarter = static_cast<uint32_t>(q4 * 32) << 16;
    const uint32_t tS = tmem + quarter + 64 * half;
    uint8_t* staging = sh.smem + Sm::kStage + (warp - 4) * 2048;
    int w = 0, k = 0;
    Item it;
    bool ok = true;
    for (; ok && next_item(sh, k, it, status, limit, true); ++k) {
      const int e = FP16 ? ds_exponent(p, it) : 0;
      const int row = it.a * kTile + r;
      const int64_t at = static_cast<int64_t>(it.begin + min(row, it.len - 1)) * f.n_q_heads + it.b;
      // 2^e goes into the weights
      const float l = fmaf(f.lse[at], -kLog2e, static_cast<float>(e)), d = -p.delta[at];
      const uint64_t c2 = pair_of(p.c, p.c), l2 = pair_of(l, l), d2 = pair_of(d, d);
      for (int j = 0; j <= it.a; ++j, ++w) {
        const uint32_t tP = tS + 128 + (w & 1) * 128;
        const bool work = 64 * half < it.len - j * kTile;
        uint32_t s[64], x[64];
        if (!(ok = waitw(SFULL, w))) break;
        tc_fence_after();
        if (work) {
          tmem_ld32(tS, s);
          tmem_ld32(tS + 32, s + 32);
          tmem_wait_ld();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(sh.bar(SREAD));
        if (work) {
#pragma unroll
          for (int i = 0; i < 64; i += 2) {
            const float2 a = halves_of(fma2(pair_of(__uint_as_float(s[i]), __uint_as_float(s[i + 1])), c2, l2));
            s[i] = __float_as_uint(ex2(a.x));
            s[i + 1] = __float_as_uint(ex2(a.y));
          }
        }
        if (!(ok = waitw(DPFULL + (w & 1), w >> 1))) break;
        tc_fence_after();
        if (work) {
          tmem_ld32(tP, x);
          tmem_ld32(tP + 32, x + 32);
          tmem_wait_ld();
#pragma unroll
          for (int i = 0; i < 64; i += 32) {
            uint32_t y[16];
#pragma unroll
            for (int q = 0; q < 32; q += 2) {
              float2 a = halves_of(mul2(add2(pair_of(__uint_as_float(x[i + q]), __uint_as_float(x[i + q + 1])), d2),
                                        pair_of(__uint_as_float(s[i + q]), __uint_as_float(s[i + q + 1]))));
              if (j == it.a) {  // keys behind the query
                a.x = 64 * half + i + q <= r ? a.x : 0.f;
                a.y = 64 * half + i + q + 1 <= r ? a.y : 0.f;
              }
              y[q / 2] = pack2<FP16>(a.x, a.y);
            }
            tmem_st16(tP + i / 2, y);
          }
          tmem_wait_st();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(sh.bar(DSFULL));
      }
      if (!ok || !(ok = waitw(DONE, k))) break;
      tc_fence_after();
      const int row0 = it.a * kTile + q4 * 32;
      store_tile<FP16, HD / 64>(tmem + quarter + 384 + half * (HD / 2), staging, FP16 ? f.scale * exp2_int(-e) : f.scale,
                                elem(p.g.d_q, (it.begin + row0) * p.g.lddq + it.b * HD + half * (HD / 2)), p.g.lddq, it.len - row0);
      tc_fence_before();
    }
  }
  end_of_kernel(tmem);
}

int norm_blocks_of(int rows) { return (rows + kNormRows - 1) / kNormRows; }

template <int HD, bool FP16>
int launch(const PromptGradArgs& a, cudaStream_t s) {
  const PromptArgs& f = a.f;
  Params p{};
  p.g = a;
  p.group = f.n_q_heads / f.n_kv_heads;
  p.c = f.scale * kLog2e;
  float* delta = static_cast<float*>(a.workspace);
  float* norms = delta + static_cast<int64_t>(f.rows) * f.n_q_heads;
  p.delta = delta;
  p.norms = norms;
  p.norm_blocks = norm_blocks_of(f.rows);
  p.wait_limit = g_wait_limit_ns.load(std::memory_order_relaxed);
  CUtensorMap q, k, v, g;
  if (!make_tensor_map_2d(&q, f.q, f.rows, static_cast<int64_t>(f.n_q_heads) * HD, f.ldq, kTile, FP16) ||
      !make_tensor_map_2d(&k, f.k, f.rows, static_cast<int64_t>(f.n_kv_heads) * HD, f.ldk, kTile, FP16) ||
      !make_tensor_map_2d(&v, f.v, f.rows, static_cast<int64_t>(f.n_kv_heads) * HD, f.ldv, kTile, FP16) ||
      !make_tensor_map_2d(&g, a.d_out, f.rows, static_cast<int64_t>(f.n_q_heads) * HD, a.lddo, kTile, FP16))
    return cuda_fail(cudaErrorInvalidValue, "vla_prompt_attn_grad: tensor maps");
  int sms = 0;
  if (const int rc = device_sms(&sms)) return rc;
  VLA_CUDA_TRY(launch_at(Start::kInOrder, prompt_delta_kernel<HD, FP16>, dim3(static_cast<unsigned>(p.norm_blocks)), dim3(256), 0, s, a, delta,
                         norms, p.norm_blocks));
  note_launch();
  const int64_t most = f.rows / kTile + std::min(f.n_seq, f.rows);  // tiles that well-formed sequences can have
  static std::atomic<uint64_t> done_k{0}, done_q{0};
  VLA_CUDA_TRY(set_smem_limit(prompt_grad_keys_kernel<HD, FP16>, Smem<HD>::kTotal, done_k));
  VLA_CUDA_TRY(set_smem_limit(prompt_grad_queries_kernel<HD, FP16>, Smem<HD>::kTotal, done_q));
  p.items_bound = static_cast<int>(std::min<int64_t>(most * f.n_kv_heads, 0x7fffffff));
  VLA_CUDA_TRY(launch_at(Start::kInOrder, prompt_grad_keys_kernel<HD, FP16>, dim3(static_cast<unsigned>(std::min(p.items_bound, sms))), dim3(kThreads),
                         Smem<HD>::kTotal, s, q, k, v, g, p));
  note_launch();
  p.items_bound = static_cast<int>(std::min<int64_t>(most * f.n_q_heads, 0x7fffffff));
  VLA_CUDA_TRY(launch_at(Start::kInOrder, prompt_grad_queries_kernel<HD, FP16>, dim3(static_cast<unsigned>(std::min(p.items_bound, sms))), dim3(kThreads),
                         Smem<HD>::kTotal, s, q, k, v, g, p));
  note_launch();
  return VLA_OK;
}

}  // namespace

size_t prompt_attn_grad_workspace(int rows, int n_q_heads, int, int) {
  return (static_cast<size_t>(rows) * n_q_heads + 2 * static_cast<size_t>(norm_blocks_of(rows))) * sizeof(float);
}

int prompt_attn_grad_launch(const PromptGradArgs& a, cudaStream_t s) {
  if (a.f.head_dim == 128) return a.f.fp16 ? launch<128, true>(a, s) : launch<128, false>(a, s);
  return a.f.fp16 ? launch<64, true>(a, s) : launch<64, false>(a, s);
}

}  // namespace vla
