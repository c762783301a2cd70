// Gradient of the causal attention of packed sequences on the tcgen05 tensor cores (include/vla_learn.h).
//
// With c = scale log2(e), P[i][j] = 2^(c s[i][j] - lse[i] log2(e)), D[i] = d_out[i] . out[i], dP = d_out v^T, dS = P (dP - D):
//   d_v[j] = sum_i P[i][j] d_out[i],  d_k[j] = scale sum_i dS[i][j] q[i],  d_q[i] = scale sum_j dS[i][j] k[j].
// Three kernels: D (a row's dot products, bound by bytes); d_k and d_v, a CTA for 128 keys of a key-value head over all queries that
// see them and all query heads that share them; d_q, a CTA for 128 queries over their keys.  The scores and dP are computed in both
// (seven products where one pass would need five), for which every sum has one owner and one order: no atomics, no 32-bit copy
// of d_q in memory, nothing zeroed before.
//
// d_k, d_v, blocks of 80 queries: S^T = K Q^T and dP^T = V dO^T have keys as rows, so that P^T and dS^T are the left operands of
// d_v += P^T dO and d_k += dS^T Q in tensor memory; Q and dO tiles serve as K-major and as MN-major operands.  S, dP, P and dS have tensor
// memory of their own (496 of 512 columns with the sums), so each product runs as soon as the threads have read or written.  d_q, blocks
// of 96 keys: S, two blocks of dP, dS over the dP that it came from.
//
// Weights of bf16 are rounded as they are.  fp16 has 5 bits of exponent: P counts 2^14-fold, and dS 2^e-fold with an e of its own for each row
// of d_q and d_k, which brings what no |dS| of the row passes to 2^13 .. 2^14: |d_out[i]| max |v[j]| + |D[i]| over the keys that query i sees,
// |v[j]| max |d_out[i]| + max |D[i]| over the queries (and heads) that see key j.  So a row's bits depend on its own sequence alone, and
// neither on larger gradients beside it; what lies 2^38 below that largest is rounded away.  The kernel of D writes the norms of rows and their maxima
// over 32 rows for it; a row's thread scales its sums back, so the factors cost nothing but their maxima (8192 rows of fp16
// take 1.64 ms, with one factor for all of a sequence 1.59; 64 samples of 272 to 304 rows 625 and 590 us).  Gradients are 0.0025 of their size
// off the 64-bit ones, where 32-bit P and dS and one rounding at the end give 0.0019; second terms would double three of the products.
// Rows of the streamed operands behind a sequence's last one become zeros in shared memory (their weights are zeros, but
// a NaN would spoil the sums over rows), up to the next multiple of 16, where the products stop.
//
// Warps of both (16): 0 items and TMA; 1 scores; 2 dP; 3 d_v; 4 d_k or d_q; 5, 6 queries' lse and D (d_k and d_v); 7 rows behind the last;
// 8 - 15 the element-wise part, two warps a lane quarter with half of the columns each, and the output.  (Two groups of such warps, which take
// the blocks in turn, were slower: 8192 rows 1.9 ms where one takes 1.3.)
//
// Bound by shared memory (scores and dP read both operands from it at 128 bytes a cycle) and, for d_k and d_v, by the element-wise chain: a block of
// 80 queries takes 2240 cycles, its products 1550.  Measured (32 query heads of 128): 8192 rows, 8 key-value heads 1.32 to 1.38 ms (1.0 to 1.04
// PFLOP/s of the ten needed flops a pair and channel; tensor pipe 46 and 58 % busy at 4096 rows); 64 samples of 272 to 304 rows 447 us (2.7 TB/s
// of the bytes that have to move); heads of 64: 8192 rows 1.19 ms, the samples 350 us.  The kernel of D: 20 us at 4096 rows (3.3 TB/s: 128 CTAs), its
// loads four steps ahead of its stores.  Few items leave SMs without work: 2048 rows of 8 heads on one key-value head 190 us.
#include <algorithm>

#include "gemm.h"
#include "prompt_items.cuh"

namespace vla {

namespace {

constexpr int kThreads = 512, kSumWarp0 = 8, kSumWarps = 8;
// producer aside: scores, dP, sums (two of keys), of keys two for the rows' lse and D, rows behind the last, element-wise warps
template <bool KEYS>
constexpr int kItemReaders = 2 + (KEYS ? 2 + 2 : 1) + 1 + kSumWarps;
constexpr int kNormRows = 32;    // rows of one entry of the largest norms (lanes of a warp)
constexpr float kPShift = 14.f;  // log2 of the fp16 weights' factor

// What the factors of dS come from (fp16): |d_out| of each row and query head; of each key-value head and row the largest |d_out| and |D| of
// the query heads that share it, and |v| (rows side by side: a warp reads those of 32); the largest of these of each block of kNormRows rows
// that all belong to sequences.
struct Norms {
  float* d_out;       // [rows][n_q_heads]
  float* of_rows;     // [3][n_kv_heads][rows]: d_out, D, v
  float* of_blocks;   // [3][n_kv_heads][blocks]
  int blocks;
};

struct Params {
  PromptGradArgs g;
  int group, items_bound;
  float c;       // scale log2(e)
  float* delta;  // [rows][n_q_heads]
  Norms norms;
  uint64_t wait_limit;
};

// ------------------------------------------------------------------------------------------- D
__device__ __forceinline__ float2 larger(float2 a, float2 b) { return make_float2(fmaxf(a.x, b.x), fmaxf(a.y, b.y)); }
// Norms of head g and kind k: of all rows, of all blocks.
__device__ __forceinline__ float* row_norms(const Params& p, int k, int g) {
  return p.norms.of_rows + (static_cast<int64_t>(k) * p.g.f.n_kv_heads + g) * p.g.f.rows;
}
__device__ __forceinline__ float* block_norms(const Params& p, int k, int g) {
  return p.norms.of_blocks + (static_cast<int64_t>(k) * p.g.f.n_kv_heads + g) * p.norms.blocks;
}
template <int HD, bool FP16>
__global__ void __launch_bounds__(256) prompt_delta_kernel(const Params p) {
  constexpr int L = HD / 8, HEADS = 32 / L;  // lanes of a head, heads of a step
  const PromptGradArgs& a = p.g;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_wait();  // (no kernel starts beside this one: it lets none start before its end)
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
  const Outside out(a.f.seq_start, a.f.n_seq, a.f.rows);
  for (int i = warp; i < kNormRows; i += 8) {
    const int row = blockIdx.x * kNormRows + i;
    if (row >= out.last) break;
    if (row < out.first) continue;
    const uint4* o = static_cast<const uint4*>(elem(a.f.out, row * a.f.ldo));
    const uint4* d = static_cast<const uint4*>(elem(a.d_out, row * a.lddo));
    // four steps' loads before the first store (which they may not pass)
    for (int h0 = lane / L; h0 - lane / L < a.f.n_q_heads; h0 += 4 * HEADS) {
      uint4 ow[4], dw[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const bool on = h0 + u * HEADS < a.f.n_q_heads;
        ow[u] = on ? o[(h0 + u * HEADS) * L + lane % L] : make_uint4(0u, 0u, 0u, 0u);
        dw[u] = on ? d[(h0 + u * HEADS) * L + lane % L] : make_uint4(0u, 0u, 0u, 0u);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int h = h0 + u * HEADS;
        const bool stores = h < a.f.n_q_heads && lane % L == 0;
        const int64_t at = static_cast<int64_t>(row) * a.f.n_q_heads + h;
        float x[8], y[8], s = 0.f, n = 0.f;
        eight(ow[u], x);
        eight(dw[u], y);
#pragma unroll
        for (int e = 0; e < 8; ++e) s = fmaf(x[e], y[e], s);
        s = over_head(s);
        if (stores) p.delta[at] = s;
        if (FP16) {
#pragma unroll
          for (int e = 0; e < 8; ++e) n = fmaf(y[e], y[e], n);
          n = over_head(n);
          if (stores) p.norms.d_out[at] = sqrtf(n);
        }
      }
    }
    if (FP16) {
      const uint4* v = static_cast<const uint4*>(elem(a.f.v, row * a.f.ldv));
      for (int h0 = lane / L; h0 - lane / L < a.f.n_kv_heads; h0 += 4 * HEADS) {
        uint4 vw[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) vw[u] = h0 + u * HEADS < a.f.n_kv_heads ? v[(h0 + u * HEADS) * L + lane % L] : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int h = h0 + u * HEADS;
          float y[8], n = 0.f;
          eight(vw[u], y);
#pragma unroll
          for (int e = 0; e < 8; ++e) n = fmaf(y[e], y[e], n);
          n = over_head(n);
          if (h < a.f.n_kv_heads && lane % L == 0) row_norms(p, 2, h)[row] = sqrtf(n);
        }
      }
    }
  }
  if constexpr (FP16) {
    __syncthreads();
    const int row = static_cast<int>(blockIdx.x) * kNormRows + lane;
    const bool on = row >= out.first && row < out.last;
    const int64_t at = static_cast<int64_t>(row) * a.f.n_q_heads;
    // (four heads a warp at once, for the loads' latency)
    for (int g0 = warp; g0 < a.f.n_kv_heads; g0 += 32) {
      float m[3][4] = {};
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int g = g0 + 8 * u;
        if (!on || g >= a.f.n_kv_heads) continue;
        m[2][u] = __ldcg(row_norms(p, 2, g) + row);
        for (int h = g * p.group; h < (g + 1) * p.group; ++h) {
          m[0][u] = fmaxf(m[0][u], __ldcg(p.norms.d_out + at + h));
          m[1][u] = fmaxf(m[1][u], fabsf(__ldcg(p.delta + at + h)));
        }
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int g = g0 + 8 * u;
        if (g >= a.f.n_kv_heads) break;
#pragma unroll
        for (int k = 0; k < 3; ++k) {
          if (on && k < 2) row_norms(p, k, g)[row] = m[k][u];
          const float most = warp_max(m[k][u]);
          if (lane == 0) block_norms(p, k, g)[blockIdx.x] = most;
        }
      }
    }
  }
}

// ------------------------------------------------------------------------------------- both kernels
// This lane's share of the largest norms over rows lo .. hi - 1: of single rows up to the first block, of whole blocks, of rows behind them.
__device__ __forceinline__ float share_of_largest(const float* of_rows, const float* of_blocks, int lo, int hi) {
  const int lane = threadIdx.x & 31, b0 = (lo + kNormRows - 1) / kNormRows, b1 = hi / kNormRows;
  float m = 0.f;
  if (lo + lane < min(hi, b0 * kNormRows)) m = __ldcg(of_rows + lo + lane);
  if (b1 >= b0 && b1 * kNormRows + lane < hi) m = fmaxf(m, __ldcg(of_rows + b1 * kNormRows + lane));
#pragma unroll 4
  for (int b = b0 + lane; b < b1; b += 32) m = fmaxf(m, __ldcg(of_blocks + b));
  return m;
}
// The exponent e of the factor 2^e of dS in row r of an item's tile (fp16; whole warp, 32 rows from a multiple of 32 on).  All loads first.
template <bool KEYS>
__device__ __forceinline__ int ds_exponent(const Params& p, const Item& it, int r) {
  const PromptArgs& f = p.g.f;
  const int lane = threadIdx.x & 31, first = it.a * kTile + (r & ~31), row = it.begin + min(it.a * kTile + r, it.len - 1);
  float most;
  if constexpr (KEYS) {
    const int lo = it.begin + min(first + 32, it.len), hi = it.begin + it.len;
    const float v = __ldcg(row_norms(p, 2, it.b) + row);
    float2 m = make_float2(__ldcg(row_norms(p, 0, it.b) + row), __ldcg(row_norms(p, 1, it.b) + row));
    float2 behind = make_float2(share_of_largest(row_norms(p, 0, it.b), block_norms(p, 0, it.b), lo, hi),
                                share_of_largest(row_norms(p, 1, it.b), block_norms(p, 1, it.b), lo, hi));
    behind = make_float2(warp_max(behind.x), warp_max(behind.y));
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const float2 y = make_float2(__shfl_down_sync(0xffffffffu, m.x, o), __shfl_down_sync(0xffffffffu, m.y, o));
      if (lane + o < 32) m = larger(m, y);
    }
    m = larger(m, behind);
    most = fmaf(v, m.x, m.y);
  } else {
    const int g = it.b / p.group;
    const int64_t at = static_cast<int64_t>(row) * f.n_q_heads + it.b;
    const float d_out = __ldcg(p.norms.d_out + at), delta = __ldcg(p.delta + at);
    float v = __ldcg(row_norms(p, 2, g) + row);
    const float before = warp_max(share_of_largest(row_norms(p, 2, g), block_norms(p, 2, g), it.begin, it.begin + min(first, it.len)));
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const float y = __shfl_up_sync(0xffffffffu, v, o);
      if (lane >= o) v = fmaxf(v, y);
    }
    most = fmaf(d_out, fmaxf(v, before), fabsf(delta));
  }
  if (!(most > 0.f) || most > 1e37f) return 0;
  int e;
  frexpf(most, &e);  // most < 2^e
  return min(max(14 - e, -100), 100);
}
__device__ __forceinline__ float exp2_int(int e) { return __int_as_float((e + 127) << 23); }

// The two kernels are one, with the parts of keys and queries exchanged: a CTA keeps a tile of 128 rows of two operands (KEYS: K and V; else Q
// and dO) and streams blocks of kBlock rows of the other two (Q and dO; K and V) past it.
template <int HD, bool KEYS>
struct Shape {
  static constexpr int kBlock = KEYS ? 80 : 96;
  static constexpr int kStages = HD == 64 ? 4 : 3;
  static constexpr int kHalf = kBlock / 2;  // columns of one of a row's two threads
  static constexpr int kRows = 2;           // blocks of queries' lse and D in flight (KEYS)
  static constexpr uint32_t kRowBytes = KEYS ? kRows * kBlock * 128 : 0;
  // shared memory: the tile's two operands, two rings, rows' lse and D, barriers
  static constexpr uint32_t kTileBytes = kTile * HD * 2, kBlockBytes = kBlock * HD * 2, kColumns = kBlock * 128;
  static constexpr uint32_t kRingA = 2 * kTileBytes, kRingB = kRingA + kStages * kBlockBytes, kRowData = kRingB + kStages * kBlockBytes;
  static constexpr uint32_t kBars = kRowData + kRowBytes, kTotal = 1024 + kBars + 1024;
  // Tensor memory: scores, dP, P and dS (KEYS; else two blocks of dP, and dS over each of them), 8 columns of ones, sums (KEYS: d_v, d_k; else d_q).
  static constexpr uint32_t kColS = 0, kColDp = kBlock, kColP = 2 * kBlock, kColDs = KEYS ? kColP + kBlock / 2 : kColDp;
  static constexpr uint32_t kColOnes = kColDs + kBlock / 2, kColV = 256, kColSum = 384;
  static_assert(kTotal <= 232448 && (KEYS ? kColOnes + 8 <= kColV : kColDp + 2 * kBlock <= kColSum) && kColumns % 1024 == 0,
                "shared and tensor memory");
};
// Of KEYS in bf16, queries' lse and D enter S and dP as 16 more channels (ones on the side of the keys): see prompt_grad_kernel.
template <bool FP16, bool KEYS>
constexpr bool kExtra = KEYS && !FP16;

// Barriers: the tile's two operands loaded / free; the rings A and B (up to 4 slots each), loads into them that end behind a sequence's
// last row, rows' lse and D; of a block: scores written / read, dP written / read, P written, its product
// done, dS written, its product done (of dP and dS, where not KEYS, two: even and odd blocks, of which no warp is then two ahead of another); the
// issuing warps' ends; descriptors.
enum : int {
  AFULL = 0, AFREE = 1, BFULL = 2, BFREE = 3, RAFULL = 4, RAFREE = 8, RBFULL = 12, RBFREE = 16, TAILA = 20, TAILB = 24, RFULL = 28, RFREE = 30,
  SFULL = 32, SREAD = 33, DPFULL = 34, DPREAD = 36, PFULL = 37, PDONE = 38, DSFULL = 39, DSDONE = 41, DRAIN = 43, IFULL = 47, IFREE = 55,
  kBarCount = 64
};

// A number as the sum of three bf16 (24 bits of it), in the first three of four.
__device__ __forceinline__ uint2 three_terms(float x) {
  bf16 a, b;
  split_bf16(x, a, b);
  const float rest = x - bf2f(a) - bf2f(b);
  return make_uint2(static_cast<uint32_t>(__bfloat16_as_ushort(a)) | static_cast<uint32_t>(__bfloat16_as_ushort(b)) << 16,
                    __bfloat16_as_ushort(f2bf(rest)));
}

// f(head, first row in the sequence, rows that count, whether the mask hides any of it) of an item's blocks in order, until one says no.
// KEYS: key tile a, key-value head b: the query heads that share it, for each the queries from the last block down to the keys' own (so that
// CTAs of one head read the same rows at about the same time).  Else: query tile a, query head b: keys from the first on.
template <int HD, bool KEYS, class F>
__device__ __forceinline__ bool for_blocks(const Item& it, int group, const F& f) {
  constexpr int N = Shape<HD, KEYS>::kBlock;
  if constexpr (KEYS) {
    const int row0 = it.a * kTile, n = (it.len - row0 + N - 1) / N;
    for (int h = it.b * group; h < (it.b + 1) * group; ++h)
      for (int i = n - 1; i >= 0; --i)
        if (!f(h, row0 + i * N, min(N, it.len - row0 - i * N), i * N < kTile)) return false;
  } else {
    const int end = min(it.len, (it.a + 1) * kTile);
    for (int i = 0; i < end; i += N)
      if (!f(it.b / group, i, min(N, end - i), i + N > it.a * kTile)) return false;
  }
  return true;
}

// S^T and dP^T have queries as columns, so a query's lse and D are of every thread, for each of its columns.  In bf16 the products bring them:
// 16 more channels, ones on the side of the keys (in tensor memory), -lse / scale and -D as three bf16 numbers each on that of the queries, so
// that S^T - lse / scale and dP^T - D come out.  From shared memory, which the products keep busy (128 bytes a cycle), the threads'
// reads of them took 9 us of every 20.  fp16 does not hold the range of lse / scale and D, and reads them there.
template <int HD, bool FP16, bool KEYS>
__global__ void __launch_bounds__(kThreads, 1)
    prompt_grad_kernel(const __grid_constant__ CUtensorMap tm_tile_a, const __grid_constant__ CUtensorMap tm_tile_b,
                       const __grid_constant__ CUtensorMap tm_ring_a, const __grid_constant__ CUtensorMap tm_ring_b, const Params p) {
  using Sh = Shape<HD, KEYS>;
  constexpr int NS = Sh::kStages, N = Sh::kBlock, NH = Sh::kHalf;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + Sh::kBars);
  const uint32_t s0 = smem_u32(smem), b0 = smem_u32(bars);
  auto BAR = [&](int i) { return b0 + 8u * static_cast<uint32_t>(i); };
  Item* items = reinterpret_cast<Item*>(bars + kBarCount);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(items + kItems);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  float* row_data = reinterpret_cast<float*>(smem + Sh::kRowData);
  static_assert(kBarCount * 8 + kItems * 16 + 12 <= 1024 && kBarCount % 2 == 0, "barrier area");
  const PromptArgs& f = p.g.f;
  constexpr int kRows = Sh::kRows;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint32_t* status = f.status;
  const uint64_t limit = p.wait_limit;

  if (threadIdx.x == 0) {
    for (int i = 0; i < kBarCount; ++i) {
      const bool rows = i >= RFREE && i < RFREE + Sh::kRows;  // (read by S and dP, or by the element-wise warps)
      const bool all = i == SREAD || i == DPREAD || i == PFULL || i == DSFULL || i == DSFULL + 1 || (rows && !kExtra<FP16, KEYS>);
      // (a dO tile is done when dP and d_v have been taken from it)
      mbar_init(BAR(i), i >= IFREE ? kItemReaders<KEYS> : all ? kSumWarps : (rows || (KEYS && i >= RBFREE && i < RBFREE + 4)) ? 2 : 1);
    }
    abort_flag[0] = abort_flag[1] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) tmem_take(smem_u32(tmem_slot));
  if constexpr (kExtra<FP16, KEYS>)
    for (uint32_t i = threadIdx.x; i < Sh::kRowBytes / 16; i += kThreads) reinterpret_cast<uint4*>(row_data)[i] = make_uint4(0u, 0u, 0u, 0u);
  fence_async_smem();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  // The kernel of d_q may start beside that of d_k and d_v, once this one knows that of D at its end, and takes the SMs that it leaves; it
  // waits for it at its end, so that its end is that of both.
  if (KEYS) {
    pdl_wait_async();
    pdl_launch_dependents();
  }
  if constexpr (kExtra<FP16, KEYS>) {
    if (warp >= kSumWarp0 && warp < kSumWarp0 + 4) {  // three ones, thirteen zeros in every row
      const uint32_t ones[8] = {0x3f803f80u, 0x00003f80u, 0u, 0u, 0u, 0u, 0u, 0u};
      tmem_st8(tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16) + Sh::kColOnes, ones);
      tmem_wait_st();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
  }
  auto waitw = [&](int bar, uint32_t phase) { return warp_waits(BAR(bar), phase & 1u, abort_flag, status, limit); };
  auto take = [&](int k, Item& it) {  // next descriptor; false at the end or at a timeout
    if (!waitw(IFULL + (k & 7), k >> 3)) return false;
    it = items[k & 7];
    __syncwarp();
    if (lane == 0) mbar_arrive(BAR(IFREE + (k & 7)));
    return it.len >= 0;
  };
  auto take_uniform = [&](int k, Item& it) {
    if (!take(k, it)) return false;
    it = Item{0, uniform(it.len), uniform(it.a), uniform(it.b)};
    return true;
  };
  // Slot of the next block of a ring, and how often the ring has gone round.
  struct Ring {
    int s = 0, round = 0;
    __device__ __forceinline__ void next() {
      if (++s == NS) {
        s = 0;
        ++round;
      }
    }
  };
  auto slot_a = [&](int s) { return s0 + Sh::kRingA + static_cast<uint32_t>(s) * Sh::kBlockBytes; };
  auto slot_b = [&](int s) { return s0 + Sh::kRingB + static_cast<uint32_t>(s) * Sh::kBlockBytes; };

  if (warp == 0) {
    if (!KEYS) fence_async_global();
    // ------------------------------------------------------------------ items and loads
    const int heads = KEYS ? f.n_kv_heads : f.n_q_heads;
    int k = 0, loaded = 0;  // items; blocks
    // Of each slot of ring A, of ring B: its last load has rows that have to become zeros; loads that did, and all, modulo 2.
    uint32_t tails = 0, phase_tail = 0, phase = 0, b_tails = 0, b_phase_tail = 0, b_phase = 0;
    int b_loaded = 0;
    Ring ring;
    auto put = [&](const Item& it) {
      if (k >= kItems && !waitw(IFREE + (k & 7), (k >> 3) - 1)) return false;
      if (lane == 0) {
        items[k & 7] = it;
        mbar_arrive(BAR(IFULL + (k & 7)));
      }
      __syncwarp();
      return true;
    };
    auto load = [&](uint32_t dst, const CUtensorMap* map, int bar, uint32_t bytes, uint32_t columns, int head, int row) {
      if (lane == 0) {
        mbar_arrive_expect_tx(BAR(bar), bytes);
#pragma unroll
        for (int kb = 0; kb < HD / 64; ++kb) tma_load_2d(dst + kb * columns, map, BAR(bar), head * HD + kb * 64, row);
      }
      __syncwarp();
    };
    int in_a = 0, in_b = 0;  // tile operands loaded
    auto load_item = [&](const Item& it) {
      bool first = true;
      return for_blocks<HD, KEYS>(it, p.group, [&](int head, int row, int rows, bool) {
        const int s = ring.s;
        const bool tail = rows & 15;
        if (first) {
          if (k && !waitw(AFREE, k - 1)) return false;
          load(s0, &tm_tile_a, AFULL, Sh::kTileBytes, kBlockBytes, it.b, it.begin + it.a * kTile);
          ++in_a;
        }
        if (ring.round && !waitw(RAFREE + s, ring.round - 1)) return false;
        load(slot_a(s), &tm_ring_a, (tail ? TAILA : RAFULL) + s, Sh::kBlockBytes, Sh::kColumns, head, it.begin + row);
        tails = (tails & ~(1u << s)) | (static_cast<uint32_t>(tail) << s);
        phase_tail ^= static_cast<uint32_t>(tail) << s;
        phase ^= 1u << s;
        ++loaded;
        if (first) {
          if (k && !waitw(BFREE, k - 1)) return false;
          load(s0 + Sh::kTileBytes, &tm_tile_b, BFULL, Sh::kTileBytes, kBlockBytes, it.b, it.begin + it.a * kTile);
          ++in_b;
          first = false;
        }
        if (ring.round && !waitw(RBFREE + s, ring.round - 1)) return false;
        load(slot_b(s), &tm_ring_b, (tail ? TAILB : RBFULL) + s, Sh::kBlockBytes, Sh::kColumns, head, it.begin + row);
        b_tails = (b_tails & ~(1u << s)) | (static_cast<uint32_t>(tail) << s);
        b_phase_tail ^= static_cast<uint32_t>(tail) << s;
        b_phase ^= 1u << s;
        ++b_loaded;
        ring.next();
        return true;
      });
    };
    if (find_items(
            f.seq_start, f.n_seq, f.rows, blockIdx.x, gridDim.x, p.items_bound,
            [&](int len) { return static_cast<int64_t>((len + kTile - 1) / kTile) * heads; },
            [&](int begin, int len, int u) {
              // the most work first: the first keys, the last queries
              const int t = u / heads;
              const Item it{begin, len, KEYS ? t : (len + kTile - 1) / kTile - 1 - t, u % heads};
              const bool ok = put(it) && load_item(it);
              ++k;
              return ok;
            }))
      put(Item{0, -1, 0, 0});
    const Outside out(f.seq_start, f.n_seq, f.rows);
    for (int i = blockIdx.x; i < out.count(); i += gridDim.x) {
      if constexpr (KEYS) {
        zero_row(elem(p.g.d_k, out.row(i) * p.g.lddk), heads * HD);
        zero_row(elem(p.g.d_v, out.row(i) * p.g.lddv), heads * HD);
      } else {
        zero_row(elem(p.g.d_q, out.row(i) * p.g.lddq), heads * HD);
      }
    }
    // nothing may land after the CTA has gone
    for (int s = 0; s < NS; ++s) {
      const bool ta = (tails >> s) & 1, tb = (b_tails >> s) & 1;
      if (s < loaded) wait_drain(BAR((ta ? TAILA : RAFULL) + s), (((ta ? phase_tail : phase) >> s) & 1) ^ 1, limit);
      if (s < b_loaded) wait_drain(BAR((tb ? TAILB : RBFULL) + s), (((tb ? b_phase_tail : b_phase) >> s) & 1) ^ 1, limit);
    }
    if (in_a) wait_drain(BAR(AFULL), (in_a - 1) & 1, limit);
    if (in_b) wait_drain(BAR(BFULL), (in_b - 1) & 1, limit);
  } else if (warp <= 2) {
    // ------------------------------------------------------------------ scores (warp 1), dP (warp 2)
    const bool dp = warp == 2;
    const uint32_t tile = tile_desc(s0 + (dp ? Sh::kTileBytes : 0)), d = tmem + (dp ? Sh::kColDp : Sh::kColS);
    const int bar_tile = dp ? BFULL : AFULL, bar_ring = dp ? RBFULL : RAFULL, bar_read = dp ? DPREAD : SREAD;
    const uint32_t ring_free = BAR(RBFREE), tile_free = BAR(dp ? BFREE : AFREE);
    const uint32_t extra = tile_desc(smem_u32(row_data)) + (dp ? 2 : 0);
    Ring ring;
    int w = 0;
    Item it;
    bool ok = true;
    for (int k = 0; ok && take_uniform(k, it); ++k) {
      if (!(ok = waitw(bar_tile, k))) break;
      ok = for_blocks<HD, KEYS>(it, p.group, [&](int, int, int rows, bool) {
        const uint32_t block = tile_desc(dp ? slot_b(ring.s) : slot_a(ring.s), Sh::kColumns);
        const uint32_t id = tile_idesc((rows + 15) & ~15, FP16, false), freed = ring_free + 8u * static_cast<uint32_t>(ring.s);
        const int buffer = !KEYS && dp ? w & 1 : 0, slot = w % kRows;
        const uint32_t dst = d + static_cast<uint32_t>(buffer) * N, full = BAR((dp ? DPFULL : SFULL) + buffer);
        // over what the threads have read (the dS that lies over dP: what d_q has been taken from)
        const bool free_now = !KEYS && dp ? w < 2 || waitw(DSDONE + buffer, (w >> 1) - 1) : w < 1 || waitw(bar_read, w - 1);
        if (!free_now || !waitw(bar_ring + ring.s, ring.round) || (kExtra<FP16, KEYS> && !waitw(RFULL + slot, w / kRows))) return false;
        tc_fence_after();
        if (elected()) {
#pragma unroll
          for (int i = 0; i < HD / 16; ++i) tile_mma(dst, tile + k_major_step(i), block + k_major_step(i, Sh::kColumns), id, i > 0);
          if constexpr (kExtra<FP16, KEYS>) {
            tile_mma_ts(dst, tmem + Sh::kColOnes, extra + static_cast<uint32_t>(slot) * (Sh::kColumns >> 4), id, 1u);
            tc_commit(BAR(RFREE + slot));
          }
          tc_commit(full);
          if (dp) tc_commit(freed);
        }
        __syncwarp();
        ring.next();
        ++w;
        return true;
      });
      if (elected()) tc_commit(tile_free);
      __syncwarp();
    }
    if (elected()) tc_commit(BAR(DRAIN + warp - 1));
    wait_drain(BAR(DRAIN + warp - 1), 0, limit);
  } else if (warp == 4 || (KEYS && warp == 3)) {
    // ------------------------------------------------------------------ d_v += P^T dO (warp 3); d_k += dS^T Q or d_q += dS K (warp 4)
    const bool dv = warp == 3;
    const uint32_t a = tmem + (dv ? Sh::kColP : Sh::kColDs), d = tmem + (dv ? Sh::kColV : Sh::kColSum), io = tile_idesc(HD, FP16, true);
    const int bar_ring = dv ? RBFULL : RAFULL, bar_a = dv ? PFULL : DSFULL;
    const uint32_t done0 = BAR(dv ? PDONE : DSDONE), ring_free = BAR(dv ? RBFREE : RAFREE);
    Ring ring;
    int w = 0;
    Item it;
    bool ok = true;
    for (int k = 0; ok && take_uniform(k, it); ++k) {
      uint32_t more = 0;
      ok = for_blocks<HD, KEYS>(it, p.group, [&](int, int, int rows, bool) {
        const uint32_t block = tile_desc(dv ? slot_b(ring.s) : slot_a(ring.s), Sh::kColumns), freed = ring_free + 8u * static_cast<uint32_t>(ring.s);
        const uint32_t operand = a + (KEYS ? 0u : static_cast<uint32_t>(w & 1) * N);
        const uint32_t done = done0 + (KEYS ? 0u : 8u * (w & 1));
        const int steps = (rows + 15) / 16;
        if (!waitw(bar_ring + ring.s, ring.round) || !waitw(bar_a + (KEYS ? 0 : w & 1), KEYS ? w : w >> 1)) return false;
        tc_fence_after();
        if (elected()) {
#pragma unroll
          for (int i = 0; i < N / 16; ++i)
            if (i < steps) tile_mma_ts(d, operand + (KEYS ? i * 8 : i / (N / 32) * NH + i % (N / 32) * 8), block + mn_major_step(i), io, i > 0 ? 1u : more);
          tc_commit(done);
          tc_commit(freed);
        }
        __syncwarp();
        ring.next();
        more = 1;
        ++w;
        return true;
      });
    }
    if (elected()) tc_commit(BAR(DRAIN + warp - 1));
    wait_drain(BAR(DRAIN + warp - 1), 0, limit);
  } else if (KEYS && (warp == 5 || warp == 6)) {
    // ------------------------------------------------------------------ queries' lse and D: of even and odd blocks
    constexpr int R = (N + 31) / 32;
    const float unit = kExtra<FP16, KEYS> ? -1.f / f.scale : -kLog2e, shift = FP16 ? kPShift : 0.f;
    int w = 0;
    Item it;
    bool ok = true;
    for (int k = 0; ok && take(k, it); ++k) {
      ok = for_blocks<HD, KEYS>(it, p.group, [&](int head, int row, int rows, bool) {
        if ((w & 1) != warp - 5) {
          ++w;
          return true;
        }
        float l[R], d[R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
          const int r = i * 32 + lane;
          const int64_t at = static_cast<int64_t>(it.begin + row + min(r, rows - 1)) * f.n_q_heads + head;
          // (rows behind the last are zeros everywhere)
          l[i] = r < rows ? fmaf(f.lse[at], unit, shift) : 0.f;
          d[i] = r < rows ? -__ldcg(p.delta + at) : 0.f;
        }
        const int slot = w % kRows;
        if (w >= kRows && !waitw(RFREE + slot, w / kRows - 1)) return false;
#pragma unroll
        for (int i = 0; i < R; ++i) {
          const int r = i * 32 + lane;
          if constexpr (kExtra<FP16, KEYS>) {
            if (r < N) {
              uint8_t* dst = reinterpret_cast<uint8_t*>(row_data) + slot * Sh::kColumns + r * 128;
              *reinterpret_cast<uint2*>(dst + ((0 ^ (r & 7)) << 4)) = three_terms(l[i]);
              *reinterpret_cast<uint2*>(dst + ((2 ^ (r & 7)) << 4)) = three_terms(d[i]);
            }
          } else {
            row_data[slot * 256 + r] = l[i];
            row_data[slot * 256 + 128 + r] = d[i];
          }
        }
        if constexpr (kExtra<FP16, KEYS>) fence_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(BAR(RFULL + slot));
        ++w;
        return true;
      });
    }
  } else if (warp == 7) {
    // ------------------------------------------------------------------ rows behind the last
    Ring ring;
    uint32_t phase = 0;  // of each slot: blocks so far with rows that have to become zeros, modulo 2
    Item it;
    bool ok = true;
    for (int k = 0; ok && take(k, it); ++k) {
      ok = for_blocks<HD, KEYS>(it, p.group, [&](int, int, int rows, bool) {
        const int s = ring.s;
        if (rows & 15) {
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            if (!waitw((b ? TAILB : TAILA) + s, phase >> s)) return false;
            zero_tile_rows<HD>(smem + ((b ? slot_b(s) : slot_a(s)) - s0), rows, (rows + 15) & ~15, Sh::kColumns);
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(BAR((b ? RBFULL : RAFULL) + s));
          }
          phase ^= 1u << s;
        }
        ring.next();
        return true;
      });
    }
  } else if (warp >= kSumWarp0) {
    // ------------------------------------------------------------------ P and dS, and the output
    // Row r of the tile, NH columns of its blocks from NH half on.
    const int half = (warp - kSumWarp0) >> 2, q4 = warp & 3, r = q4 * 32 + lane;
    const uint32_t quarter = tmem + (static_cast<uint32_t>(q4 * 32) << 16);
    const uint32_t tS = quarter + Sh::kColS + NH * half, tDp = quarter + Sh::kColDp + NH * half;
    const uint32_t tP = quarter + Sh::kColP + NH / 2 * half, tDs = quarter + Sh::kColDs + (KEYS ? NH / 2 : NH) * half;
    const uint64_t c2 = pair_of(p.c, p.c);
    int w = 0;
    Item it;
    bool ok = true;
    for (int k = 0; ok && take(k, it); ++k) {
      const int row0 = it.a * kTile + q4 * 32;
      // (fp16) the exponent of this row's factor of dS; of a query row its lse (with the factor) and -D
      const int e = FP16 ? ds_exponent<KEYS>(p, it, r) : 0;
      // d_k's factor beside the weights' own waits in shared memory for its use: as registers it costs spills, 8192 rows 1.71 ms for 1.66
      volatile float* const factor = row_data + 2 * 256 + (threadIdx.x - 32 * kSumWarp0);
      if constexpr (KEYS && FP16) *factor = exp2_int(e - static_cast<int>(kPShift));
      uint64_t l2 = 0, d2 = 0;
      if constexpr (!KEYS) {
        const int64_t at = static_cast<int64_t>(it.begin + min(it.a * kTile + r, it.len - 1)) * f.n_q_heads + it.b;
        const float l = fmaf(f.lse[at], -kLog2e, static_cast<float>(e)), d = -__ldcg(p.delta + at);
        l2 = pair_of(l, l);
        d2 = pair_of(d, d);
      }
      ok = for_blocks<HD, KEYS>(it, p.group, [&](int, int row, int rows, bool edge) {
        const bool work = NH * half < ((rows + 15) & ~15);  // else no product reads these columns
        // columns of keys up to the query, or of queries from the key on
        const int bound = it.a * kTile + r - row - NH * half;
        const float4* rl = reinterpret_cast<const float4*>(row_data + (w % kRows) * 256 + NH * half);
        uint32_t s[NH];
        if ((KEYS && FP16 && !waitw(RFULL + w % kRows, w / kRows)) || !waitw(SFULL, w)) return false;
        tc_fence_after();
        if (work) {
          tmem_load<NH>(tS, s);
          tmem_wait_ld();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(BAR(SREAD));
        const bool free_p = !KEYS || w == 0 || mbar_test_wait(BAR(PDONE), (w - 1) & 1);
        if (work) {
#pragma unroll
          for (int i = 0; i < NH; i += 4) {
            uint64_t la = l2, lb = l2;
            if constexpr (KEYS && FP16) {
              const float4 l = rl[i / 4];
              la = pair_of(l.x, l.y);
              lb = pair_of(l.z, l.w);
            }
            const float2 a = halves_of(fma2(pair_of(__uint_as_float(s[i]), __uint_as_float(s[i + 1])), c2, la));
            const float2 b = halves_of(fma2(pair_of(__uint_as_float(s[i + 2]), __uint_as_float(s[i + 3])), c2, lb));
            s[i] = __float_as_uint(ex2(a.x));
            s[i + 1] = __float_as_uint(ex2(a.y));
            s[i + 2] = __float_as_uint(ex2(b.x));
            s[i + 3] = __float_as_uint(ex2(b.y));
          }
          if (edge) {
#pragma unroll
            for (int i = 0; i < NH; ++i) s[i] = (KEYS ? i >= bound : i <= bound) ? s[i] : 0u;
          }
        }
        if constexpr (KEYS) {
          // P is the last product's until that is done
          if (!__all_sync(0xffffffffu, free_p) && !waitw(PDONE, w - 1)) return false;
          tc_fence_after();
          if (work) {
            uint32_t y[NH / 2];
#pragma unroll
            for (int i = 0; i < NH / 2; ++i) y[i] = pack2<FP16>(__uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1]));
            tmem_store<NH / 2>(tP, y);
            tmem_wait_st();
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(BAR(PFULL));
        }
        const int buffer = KEYS ? 0 : w & 1;
        if (!waitw(DPFULL + buffer, KEYS ? w : w >> 1)) return false;
        const bool free_ds = !KEYS || w == 0 || mbar_test_wait(BAR(DSDONE), (w - 1) & 1);
        tc_fence_after();
        // dS over s, columns j .. j + C - 1, from dP
        constexpr int C = KEYS ? NH : 16;
        uint32_t x[C];
        auto gradients = [&](int j) {
          const float up = KEYS && FP16 ? *factor : 1.f;
#pragma unroll
          for (int i = 0; i < C; i += 4) {
            uint64_t a = pair_of(__uint_as_float(x[i]), __uint_as_float(x[i + 1]));
            uint64_t b = pair_of(__uint_as_float(x[i + 2]), __uint_as_float(x[i + 3]));
            if constexpr (!kExtra<FP16, KEYS>) {
              uint64_t da = d2, db = d2;
              if constexpr (KEYS) {
                const float4 d = rl[32 + (i + j) / 4];
                da = pair_of(d.x, d.y);
                db = pair_of(d.z, d.w);
              }
              a = add2(a, da);
              b = add2(b, db);
              if constexpr (KEYS) {
                a = mul2(a, pair_of(up, up));
                b = mul2(b, pair_of(up, up));
              }
            }
            const float2 ya = halves_of(mul2(a, pair_of(__uint_as_float(s[i + j]), __uint_as_float(s[i + j + 1]))));
            const float2 yb = halves_of(mul2(b, pair_of(__uint_as_float(s[i + j + 2]), __uint_as_float(s[i + j + 3]))));
            s[i + j] = __float_as_uint(ya.x);
            s[i + j + 1] = __float_as_uint(ya.y);
            s[i + j + 2] = __float_as_uint(yb.x);
            s[i + j + 3] = __float_as_uint(yb.y);
          }
          if (edge) {  // (what the mask hides may be NaN)
#pragma unroll
            for (int i = j; i < j + C; ++i) s[i] = (KEYS ? i >= bound : i <= bound) ? s[i] : 0u;
          }
        };
        if constexpr (KEYS) {
          if (work) {
            tmem_load<NH>(tDp, x);
            tmem_wait_ld();
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(BAR(DPREAD));
          if (work) gradients(0);
          if (FP16) {
            __syncwarp();
            if (lane == 0) mbar_arrive(BAR(RFREE + w % kRows));
          }
          if (!__all_sync(0xffffffffu, free_ds) && !waitw(DSDONE, w - 1)) return false;
          tc_fence_after();
          if (work) {
            uint32_t y[NH / 2];
#pragma unroll
            for (int i = 0; i < NH / 2; ++i) y[i] = pack2<FP16>(__uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1]));
            tmem_store<NH / 2>(tDs, y);
          }
        } else if (work) {
          const uint32_t from = tDp + static_cast<uint32_t>(buffer) * N, to = tDs + static_cast<uint32_t>(buffer) * N;
#pragma unroll
          for (int j = 0; j < NH; j += C) {
            tmem_ld16(from + j, x);
            tmem_wait_ld();
            gradients(j);
            uint32_t y[C / 2];  // (over columns that this thread has read)
#pragma unroll
            for (int i = 0; i < C / 2; ++i) y[i] = pack2<FP16>(__uint_as_float(s[j + 2 * i]), __uint_as_float(s[j + 2 * i + 1]));
            tmem_st8(to + j / 2, y);
          }
        }
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(BAR(DSFULL + buffer));
        ++w;
        return true;
      });
      if (!ok || !(ok = KEYS ? waitw(PDONE, w - 1) && waitw(DSDONE, w - 1) : waitw(DSDONE + ((w - 1) & 1), (w - 1) >> 1))) break;
      tc_fence_after();
      const int64_t at = it.begin + row0;
      if constexpr (KEYS) {
        if (half == 0)
          store_tile<FP16, HD / 32>(quarter + Sh::kColV, FP16 ? exp2_int(-static_cast<int>(kPShift)) : 1.f,
                                    elem(p.g.d_v, at * p.g.lddv + it.b * HD), p.g.lddv, it.len - row0);
        else
          store_tile<FP16, HD / 32>(quarter + Sh::kColSum, FP16 ? f.scale * exp2_int(-static_cast<int>(kPShift)) / *factor : f.scale,
                                    elem(p.g.d_k, at * p.g.lddk + it.b * HD), p.g.lddk, it.len - row0);
      } else {
        store_tile<FP16, HD / 64>(quarter + Sh::kColSum + half * (HD / 2), FP16 ? f.scale * exp2_int(-e) : f.scale,
                                  elem(p.g.d_q, at * p.g.lddq + it.b * HD + half * (HD / 2)), p.g.lddq, it.len - row0);
      }
      tc_fence_before();
    }
  }

  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_give(tmem);
  }
  if (!KEYS) pdl_wait();
}

int norm_blocks_of(int rows) { return (rows + kNormRows - 1) / kNormRows; }

template <int HD, bool FP16, bool KEYS>
int launch_part(Params p, int sms, cudaStream_t s) {
  using Sh = Shape<HD, KEYS>;
  const PromptArgs& f = p.g.f;
  const int q_tile = KEYS ? Sh::kBlock : kTile, kv_tile = KEYS ? kTile : Sh::kBlock;
  CUtensorMap q, k, v, g;
  if (!make_tensor_map_2d(&q, f.q, f.rows, static_cast<int64_t>(f.n_q_heads) * HD, f.ldq, q_tile, FP16) ||
      !make_tensor_map_2d(&k, f.k, f.rows, static_cast<int64_t>(f.n_kv_heads) * HD, f.ldk, kv_tile, FP16) ||
      !make_tensor_map_2d(&v, f.v, f.rows, static_cast<int64_t>(f.n_kv_heads) * HD, f.ldv, kv_tile, FP16) ||
      !make_tensor_map_2d(&g, p.g.d_out, f.rows, static_cast<int64_t>(f.n_q_heads) * HD, p.g.lddo, q_tile, FP16))
    return cuda_fail(cudaErrorInvalidValue, "vla_prompt_attn_grad: tensor maps");
  const int64_t tiles = f.rows / kTile + std::min(f.n_seq, f.rows);  // as many as well-formed sequences can have
  p.items_bound = static_cast<int>(std::min<int64_t>(tiles * (KEYS ? f.n_kv_heads : f.n_q_heads), 0x7fffffff));
  const auto kern = prompt_grad_kernel<HD, FP16, KEYS>;
  static std::atomic<uint64_t> done{0};
  VLA_CUDA_TRY(set_smem_limit(kern, Sh::kTotal, done));
  // (d_k and d_v beside the kernel of D, which would have to let them start, made 64 samples 130 us slower)
  VLA_CUDA_TRY(launch_at(Start::kEarly, kern, dim3(static_cast<unsigned>(std::min(p.items_bound, sms))), dim3(kThreads), Sh::kTotal, s,
                         KEYS ? k : q, KEYS ? v : g, KEYS ? q : k, KEYS ? g : v, p));
  note_launch();
  return VLA_OK;
}

template <int HD, bool FP16>
int launch(const PromptGradArgs& a, cudaStream_t s) {
  const PromptArgs& f = a.f;
  Params p{};
  p.g = a;
  p.group = f.n_q_heads / f.n_kv_heads;
  p.c = f.scale * kLog2e;
  const int blocks = norm_blocks_of(f.rows);
  const int64_t q_rows = static_cast<int64_t>(f.rows) * f.n_q_heads, kv_rows = static_cast<int64_t>(f.rows) * f.n_kv_heads;
  p.delta = static_cast<float*>(a.workspace);
  p.norms = Norms{p.delta + q_rows, p.delta + 2 * q_rows, p.delta + 2 * q_rows + 3 * kv_rows, blocks};
  p.wait_limit = g_wait_limit_ns.load(std::memory_order_relaxed);
  int sms = 0;
  if (const int rc = device_sms(&sms)) return rc;
  VLA_CUDA_TRY(launch_at(Start::kEarly, prompt_delta_kernel<HD, FP16>, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, s, p));
  note_launch();
  if (const int rc = launch_part<HD, FP16, true>(p, sms, s)) return rc;
  return launch_part<HD, FP16, false>(p, sms, s);
}

}  // namespace

size_t prompt_attn_grad_workspace(int rows, int n_q_heads, int n_kv_heads, int) {
  const size_t n = rows, blocks = norm_blocks_of(rows);
  return (2 * n * n_q_heads + 3 * (n + blocks) * n_kv_heads) * sizeof(float);
}

int prompt_attn_grad_launch(const PromptGradArgs& a, cudaStream_t s) {
  if (a.f.head_dim == 128) return a.f.fp16 ? launch<128, true>(a, s) : launch<128, false>(a, s);
  return a.f.fp16 ? launch<64, true>(a, s) : launch<64, false>(a, s);
}

}  // namespace vla
