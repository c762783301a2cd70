// Causal attention of packed sequences on the tcgen05 tensor cores (include/vla_learn.h).
//
// With c = scale log2(e), for a query i over blocks of 128 keys: s = q K^T, m = max s, weights 2^(c (s - m)), l their sum,
// O = 2^(c (m' - m)) O + P V; out = O / l, lse = ln 2 (c m + log2 l).  The reference m moves only when a maximum passes it by more than
// 2^8, so O is scaled again in few blocks.  Weights go to the values' type; fp16 ones are 2^7 times as large, so that one of
// 2^-21 of the row's largest still keeps all its bits (at most 2^15 with the reference 2^8 behind).
//
// A tile is 128 rows of one sequence and query head.  The tiles of a sequence and key-value head are numbered row tile after row tile, query
// head after query head, and an item is two neighbours: two query heads over the same rows where heads are shared, else two row tiles.
// Both go over the same keys, so a block of keys in shared memory serves 256 queries, and while one tile's weights
// are computed the tensor cores work for the other.  Items go sequence by sequence, the longest rows of a
// sequence first (its keys are read from HBM once, and the last items are short); persistent CTAs, one an SM.
//
// Roles (384 threads):
//   warp 0      TMA: Q tiles when the item before is done with them, key and value blocks into a ring;
//   warp 1      owns the tensor memory; issues S = Q K^T and O += P V (P in tensor memory over the S it came from, V as the
//               MN-major operand), a tile's next scores behind its product, so that one tile's softmax runs beside the other's products;
//   warp 2      a sequence's last values land with it: those behind the last row become zeros (their weights are zeros, but a NaN
//               would spoil the product), then the block counts as loaded;
//   warp 3      finds the items: a scan over the sequences' lengths, 32 sequences a step, into a ring of descriptors;
//               then the rows of no sequence;
//   warps 4-11  one query row a thread: softmax, output (through shared memory, so that rows are stored in whole lines).
// A row whose result is not finite is computed again from its own keys alone (attend_row): a NaN behind a row in its
// block of keys does not count for it.
// Tensor memory: S / P of the tiles [0, 128) [128, 256), O [256, 256 + HD) [384, 384 + HD).
#include <algorithm>

#include "gemm.h"
#include "prompt_items.cuh"

namespace vla {

namespace {

constexpr int kThreads = 384;
constexpr uint32_t kColS = 0, kColO = 256;

template <int HD>
struct Smem {
  static constexpr int kStages = HD == 128 ? 4 : 8;
  static constexpr uint32_t kTileBytes = kTile * HD * 2;
  static constexpr uint32_t kStaging = 8 * 4096;  // 32 rows x 128 bytes a softmax warp
  static constexpr uint32_t kRing = 2 * kTileBytes, kStage = kRing + kStages * kTileBytes, kBars = kStage + kStaging;
  static constexpr uint32_t kTotal = 1024 + kBars + 1024;
  static_assert(kTotal <= 232448, "shared memory per CTA");
};

// Barriers.
enum : int { QFULL = 0, QFREE = 2, SFULL = 4, PFULL = 6, PVDONE = 8, DRAIN = 10, IFULL = 11, IFREE = 19, KVFULL = 27, KVFREE = 35, TAIL = 43, kBarCount = 51 };
constexpr int kItemReaders = 1 + 1 + 1 + 8;  // producer, MMA, warp 2, softmax warps

struct Params {
  PromptArgs a;
  int group, items_bound;
  float c, offset;  // scale log2(e); log2 of the weights' common factor
  uint64_t wait_limit;
};

// An item is tiles 2 a and 2 a + 1 of key-value head b.  Blocks of keys of each (0: no such tile).
struct Tiles {
  int row_tile[2], head[2], nb[2];
};
__device__ __forceinline__ Tiles tiles_of(const Item& it, int group) {
  Tiles t;
  const int n = (it.len + kTile - 1) / kTile;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int x = 2 * it.a + k;
    t.row_tile[k] = x / group;
    t.head[k] = it.b * group + x % group;
    t.nb[k] = t.row_tile[k] < n ? t.row_tile[k] + 1 : 0;
  }
  return t;
}

template <int HD, bool FP16>
__global__ void __launch_bounds__(kThreads, 1)
    prompt_attn_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                       const __grid_constant__ CUtensorMap tm_v, const Params p) {
  using Sm = Smem<HD>;
  constexpr int KB = HD / 64, NS = Sm::kStages;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + Sm::kBars);
  const uint32_t s0 = smem_u32(smem), b0 = smem_u32(bars);
  auto BAR = [&](int i) { return b0 + 8u * static_cast<uint32_t>(i); };
  Item* items = reinterpret_cast<Item*>(bars + kBarCount + 1);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(items + kItems);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  static_assert((kBarCount + 1) * 8 + kItems * 16 + 8 <= 1024 && (kBarCount + 1) % 2 == 0, "barrier area");
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint32_t* status = p.a.status;
  const uint64_t limit = p.wait_limit;

  if (threadIdx.x == 0) {
    for (int t = 0; t < 2; ++t) {
      mbar_init(BAR(QFULL + t), 1);
      mbar_init(BAR(QFREE + t), 1);
      mbar_init(BAR(SFULL + t), 1);
      mbar_init(BAR(PFULL + t), 4);
      mbar_init(BAR(PVDONE + t), 1);
    }
    mbar_init(BAR(DRAIN), 1);
    for (int i = 0; i < kItems; ++i) {
      mbar_init(BAR(IFULL + i), 1);
      mbar_init(BAR(IFREE + i), kItemReaders);
    }
    for (int s = 0; s < NS; ++s) {
      mbar_init(BAR(KVFULL + s), 1);
      mbar_init(BAR(KVFREE + s), 2);
      mbar_init(BAR(TAIL + s), 1);
    }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) tmem_take(smem_u32(tmem_slot));
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  auto stage = [&](int f) { return s0 + Sm::kRing + (f % NS) * Sm::kTileBytes; };
  auto wait1 = [&](int bar, uint32_t parity) { return quick_wait(BAR(bar), parity & 1u, abort_flag, status, limit); };

  if (warp == 0) {
    if (lane == 0) {
      // ------------------------------------------------------------------ loads
      int f = 0, used[2] = {0, 0};          // ring slots filled; Q tiles loaded
      uint32_t on_tail = 0, tail_phase = 0;  // of each slot: its last load went to warp 2 first; how many did, modulo 2
      bool ok = true;
      for (int k = 0; ok; ++k) {
        if (!(ok = wait1(IFULL + (k & 7), k >> 3))) break;
        const Item it = items[k & 7];
        mbar_arrive(BAR(IFREE + (k & 7)));
        if (it.len < 0) break;
        const Tiles t = tiles_of(it, p.group);
        auto load_q = [&](int x) {
          if (used[x] && !wait1(QFREE + x, used[x] - 1)) return false;
          mbar_arrive_expect_tx(BAR(QFULL + x), Sm::kTileBytes);
#pragma unroll
          for (int kb = 0; kb < KB; ++kb)
            tma_load_2d(s0 + x * Sm::kTileBytes + kb * kBlockBytes, &tm_q, BAR(QFULL + x), t.head[x] * HD + kb * 64,
                        it.begin + t.row_tile[x] * kTile);
          ++used[x];
          return true;
        };
        auto load_kv = [&](const CUtensorMap* map, int j, bool tail) {
          const int s = f % NS, bar = (tail ? TAIL : KVFULL) + s;
          if (f >= NS && !wait1(KVFREE + s, f / NS - 1)) return false;
          mbar_arrive_expect_tx(BAR(bar), Sm::kTileBytes);
#pragma unroll
          for (int kb = 0; kb < KB; ++kb) tma_load_2d(stage(f) + kb * kBlockBytes, map, BAR(bar), it.b * HD + kb * 64, it.begin + j * kTile);
          on_tail = (on_tail & ~(1u << s)) | (static_cast<uint32_t>(tail) << s);
          tail_phase ^= static_cast<uint32_t>(tail) << s;
          ++f;
          return true;
        };
        auto load_k = [&](int j) { return load_kv(&tm_k, j, false); };
        auto load_v = [&](int j) { return load_kv(&tm_v, j, it.len - j * kTile < kTile); };
        const int nb = max(t.nb[0], t.nb[1]);
        ok = load_k(0) && (!t.nb[0] || load_q(0)) && (!t.nb[1] || load_q(1)) && load_v(0);
        for (int j = 1; j < nb && ok; ++j) ok = load_k(j) && load_v(j);
      }
      // nothing may land after the CTA has gone
      for (int i = max(0, f - NS); i < f; ++i) {
        const int s = i % NS;
        if ((on_tail >> s) & 1)
          wait_drain(BAR(TAIL + s), ((tail_phase >> s) & 1) ^ 1, limit);
        else
          wait_drain(BAR(KVFULL + s), (i / NS) & 1, limit);
      }
      for (int x = 0; x < 2; ++x)
        if (used[x]) wait_drain(BAR(QFULL + x), (used[x] - 1) & 1, limit);
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ MMAs
    const uint32_t is = tile_idesc(128, FP16, false), io = tile_idesc(HD, FP16, true);
    auto waits = [&](int bar, int phase) { return warp_waits(BAR(bar), static_cast<uint32_t>(phase) & 1u, abort_flag, status, limit); };
    int base = 0, q[2] = {0, 0}, block[2] = {0, 0};  // blocks of the items before; Q tiles and blocks of each tile so far
    auto free_kv = [&](int s, bool shared) {
      tc_commit(BAR(KVFREE + s));
      if (!shared) tc_commit(BAR(KVFREE + s));
    };
    // S of block j of tile x, over the weights of the block before (which its product has read)
    auto scores = [&](const Tiles& t, int base, const int x, int j) {
      const int f = 2 * (base + j), s = f % NS;
      const bool first = j == 0, last = j == t.nb[x] - 1;
      if (!waits(KVFULL + s, f / NS) || (first && !waits(QFULL + x, q[x])) || (block[x] > 0 && !waits(PVDONE + x, block[x] - 1))) return false;
      tc_fence_after();
      const uint32_t dq = tile_desc(s0 + x * Sm::kTileBytes), dk = tile_desc(stage(f)), tS = tmem + kColS + x * 128;
      if (elected()) {
#pragma unroll
        for (int k = 0; k < HD / 16; ++k) tile_mma(tS, dq + k_major_step(k), dk + k_major_step(k), is, k > 0);
        tc_commit(BAR(SFULL + x));
        if (last) tc_commit(BAR(QFREE + x));
        free_kv(s, j < t.nb[x ^ 1]);
      }
      __syncwarp();
      q[x] += last;
      return true;
    };
    auto product = [&](const Tiles& t, int len, const int x, int j) {
      const int f = 2 * (base + j) + 1, s = f % NS, steps = (min(kTile, len - j * kTile) + 15) / 16;
      if (!waits(KVFULL + s, f / NS) || !waits(PFULL + x, block[x])) return false;
      tc_fence_after();
      const uint32_t dv = tile_desc(stage(f)), tP = tmem + kColS + x * 128, tO = tmem + kColO + x * 128, more = j > 0;
      if (elected()) {
#pragma unroll
        for (int k = 0; k < kTile / 16; ++k)
          if (k < steps) tile_mma_ts(tO, tP + k * 8, dv + mn_major_step(k), io, k > 0 ? 1u : more);
        tc_commit(BAR(PVDONE + x));
        free_kv(s, j < t.nb[x ^ 1]);
      }
      __syncwarp();
      ++block[x];
      return true;
    };
    // An item's blocks: each tile's product, then its next scores; at the end the next item's first scores.
    Item it;
    auto take = [&](int k, Item& it, Tiles& t) {
      if (!waits(IFULL + (k & 7), k >> 3)) return false;
      const Item* src = items + (k & 7);
      it = Item{0, uniform(src->len), uniform(src->a), uniform(src->b)};
      if (lane == 0) mbar_arrive(BAR(IFREE + (k & 7)));
      if (it.len >= 0) t = tiles_of(it, p.group);
      return true;
    };
    Tiles t{};
    bool ok = take(0, it, t);
    if (ok && it.len >= 0) ok = scores(t, 0, 0, 0) && (!t.nb[1] || scores(t, 0, 1, 0));
    for (int k = 1; ok && it.len >= 0; ++k) {
      const int nb = max(t.nb[0], t.nb[1]);
      for (int j = 0; j < nb && ok; ++j) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          if (j < t.nb[x]) ok = ok && product(t, it.len, x, j);
          if (j + 1 < t.nb[x]) ok = ok && scores(t, base, x, j + 1);
        }
      }
      base += nb;
      ok = ok && take(k, it, t);
      if (ok && it.len >= 0) ok = scores(t, base, 0, 0) && (!t.nb[1] || scores(t, base, 1, 0));
    }
    if (elected()) tc_commit(BAR(DRAIN));
    wait_drain(BAR(DRAIN), 0, limit);
  } else if (warp == 2) {
    // ------------------------------------------------------------------ values behind the last row
    int base = 0;
    uint32_t phase = 0;
    for (int k = 0;; ++k) {
      if (!warp_waits(BAR(IFULL + (k & 7)), (k >> 3) & 1, abort_flag, status, limit)) break;
      const Item it = items[k & 7];
      __syncwarp();
      if (lane == 0) mbar_arrive(BAR(IFREE + (k & 7)));
      if (it.len < 0) break;
      const Tiles t = tiles_of(it, p.group);
      const int nb = max(t.nb[0], t.nb[1]), keys = it.len - (nb - 1) * kTile;
      if (keys < kTile) {
        const int f = 2 * (base + nb - 1) + 1, s = f % NS;
        if (!warp_waits(BAR(TAIL + s), (phase >> s) & 1, abort_flag, status, limit)) break;
        phase ^= 1u << s;
        zero_tile_rows<HD>(smem + Sm::kRing + s * Sm::kTileBytes, keys, (keys + 15) & ~15);
        fence_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(BAR(KVFULL + s));
      }
      base += nb;
    }
  } else if (warp == 3) {
    // ------------------------------------------------------------------ items
    const int n_seq = p.a.n_seq, group = p.group, Hk = p.a.n_kv_heads;
    if (blockIdx.x == 0) check_starts(p.a.seq_start, n_seq, p.a.rows, lane, 32, status);
    auto pairs_of = [&](int len) { return ((len + kTile - 1) / kTile * group + 1) / 2; };
    int k = 0;
    auto put = [&](const Item& it) {
      if (k >= kItems && !warp_waits(BAR(IFREE + (k & 7)), ((k >> 3) - 1) & 1, abort_flag, status, limit)) return false;
      if (lane == 0) {
        items[k & 7] = it;
        mbar_arrive(BAR(IFULL + (k & 7)));
      }
      ++k;
      return true;
    };
    if (find_items(
            p.a.seq_start, n_seq, p.a.rows, blockIdx.x, gridDim.x, p.items_bound,
            [&](int len) { return static_cast<int64_t>(pairs_of(len)) * Hk; },
            [&](int begin, int len, int u) { return put(Item{begin, len, pairs_of(len) - 1 - u / Hk, u % Hk}); }))
      put(Item{0, -1, 0, 0});
    const Outside out(p.a.seq_start, n_seq, p.a.rows);
    for (int i = blockIdx.x; i < out.count(); i += gridDim.x) {
      const int row = out.row(i);
      zero_row(elem(p.a.out, row * p.a.ldo), p.a.n_q_heads * HD);
      if (p.a.lse)
        for (int e = lane; e < p.a.n_q_heads; e += 32) p.a.lse[static_cast<int64_t>(row) * p.a.n_q_heads + e] = -INFINITY;
    }
  } else {
    // ------------------------------------------------------------------ softmax and output
    const int x = (warp - 4) >> 2, q4 = warp & 3, r = q4 * 32 + lane;  // tile, lane quarter, row in the tile
    const uint32_t tS = tmem + (static_cast<uint32_t>(q4 * 32) << 16) + kColS + x * 128;
    const uint32_t tO = tmem + (static_cast<uint32_t>(q4 * 32) << 16) + kColO + x * 128;
    uint8_t* staging = smem + Sm::kStage + (warp - 4) * 4096;
    const float c = p.c;
    int block = 0;
    bool ok = true;
    for (int k = 0; ok; ++k) {
      if (!warp_waits(BAR(IFULL + (k & 7)), (k >> 3) & 1, abort_flag, status, limit)) break;
      const Item it = items[k & 7];
      __syncwarp();
      if (lane == 0) mbar_arrive(BAR(IFREE + (k & 7)));
      if (it.len < 0) break;
      const Tiles t = tiles_of(it, p.group);
      const int nb = t.nb[x];
      if (!nb) continue;
      const int row0 = t.row_tile[x] * kTile + q4 * 32;  // the warp's first row in the sequence
      const int live = min(32, it.len - row0);           // its rows, at most 0: none
      float m = -INFINITY, l = 0.f;
      for (int j = 0; j < nb; ++j, ++block) {
        if (!warp_waits(BAR(SFULL + x), block & 1, abort_flag, status, limit)) {
          ok = false;
          break;
        }
        tc_fence_after();
        if (live > 0) {
          uint32_t s[128];
#pragma unroll
          for (int i = 0; i < 4; ++i) tmem_ld32(tS + 32 * i, s + 32 * i);
          tmem_wait_ld();
          if (j == nb - 1) {
#pragma unroll
            for (int i = 0; i < 128; ++i) s[i] = i <= r ? s[i] : 0xff800000u;
          }
          float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int i = 0; i < 128; ++i) top[i & 3] = fmaxf(top[i & 3], __uint_as_float(s[i]));
          const float mb = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
          float alpha = 1.f;
          if ((mb - m) * c > 8.f || j == 0) {
            alpha = j == 0 ? 0.f : ex2((m - mb) * c);
            m = mb == -INFINITY ? 0.f : mb;
            l *= alpha;
          }
          if (j > 0 && __any_sync(0xffffffffu, alpha != 1.f)) {
            if (!warp_waits(BAR(PVDONE + x), (block - 1) & 1, abort_flag, status, limit)) {
              ok = false;
              break;
            }
            tc_fence_after();
#pragma unroll 1
            for (int i = 0; i < HD; i += 16) {
              uint32_t v[16];
              tmem_ld16(tO + i, v);
              tmem_wait_ld();
#pragma unroll
              for (int e = 0; e < 16; ++e) v[e] = __float_as_uint(__uint_as_float(v[e]) * alpha);
              tmem_st16(tO + i, v);
            }
          }
          const float shift = fmaf(-m, c, p.offset);
          const uint64_t c2 = pair_of(c, c), shift2 = pair_of(shift, shift);
          uint64_t sum = 0;
#pragma unroll
          for (int i = 0; i < 128; i += 32) {
            uint32_t w[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const float2 y = halves_of(fma2(pair_of(__uint_as_float(s[i + 2 * e]), __uint_as_float(s[i + 2 * e + 1])), c2, shift2));
              const float a = ex2(y.x), b = ex2(y.y);
              sum = add2(sum, pair_of(a, b));
              w[e] = pack2<FP16>(a, b);
            }
            tmem_st16(tS + i / 2, w);
          }
          const float2 both = halves_of(sum);
          l += both.x + both.y;
          tmem_wait_st();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(BAR(PFULL + x));
      }
      if (!ok || !warp_waits(BAR(PVDONE + x), (block - 1) & 1, abort_flag, status, limit)) break;
      tc_fence_after();
      if (live <= 0) continue;
      // out = O / l: 64 channels at a time through shared memory, 4 rows of 128 bytes a store
      const float inv = 1.f / l;
      const int64_t row = it.begin + row0;
      float bad = 0.f;
#pragma unroll
      for (int b = 0; b < KB; ++b) {
        uint32_t v[64];
        tmem_ld32(tO + 64 * b, v);
        tmem_ld32(tO + 64 * b + 32, v + 32);
        tmem_wait_ld();
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          uint32_t w[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float y0 = __uint_as_float(v[8 * e + 2 * i]) * inv, y1 = __uint_as_float(v[8 * e + 2 * i + 1]) * inv;
            bad = fmaf(y0, 0.f, fmaf(y1, 0.f, bad));
            w[i] = pack2<FP16>(y0, y1);
          }
          *reinterpret_cast<uint4*>(staging + lane * 128 + ((e ^ (lane & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int rr = 4 * i + (lane >> 3), e = lane & 7;
          if (rr < live)
            *reinterpret_cast<uint4*>(elem(p.a.out, (row + rr) * p.a.ldo + t.head[x] * HD + b * 64 + e * 8)) =
                *reinterpret_cast<const uint4*>(staging + rr * 128 + ((e ^ (rr & 7)) << 4));
        }
        __syncwarp();
      }
      if (p.a.lse && lane < live) p.a.lse[(row + lane) * p.a.n_q_heads + t.head[x]] = (log2f(l) - fmaf(-m, c, p.offset)) * kLn2;
      uint32_t again = __ballot_sync(0xffffffffu, bad != 0.f && lane < live);
      while (again) {
        const int rr = __ffs(static_cast<int>(again)) - 1;
        again &= again - 1;
        attend_row<HD, FP16>(p.a, static_cast<int>(row) + rr, t.head[x], it.begin);
      }
    }
  }

  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_give(tmem);
  }
}

template <int HD, bool FP16>
int launch(const PromptArgs& a, cudaStream_t s) {
  Params p{};
  p.a = a;
  p.group = a.n_q_heads / a.n_kv_heads;
  p.c = a.scale * kLog2e;
  p.offset = FP16 ? 7.f : 0.f;
  p.wait_limit = g_wait_limit_ns.load(std::memory_order_relaxed);
  // as many items as well-formed sequences can have: a last row tile and a lone last tile each
  const int64_t seqs = std::min(a.n_seq, a.rows), tiles = (a.rows / kTile + seqs) * p.group;
  p.items_bound = static_cast<int>(std::min<int64_t>((tiles + seqs + 1) / 2 * a.n_kv_heads, 0x7fffffff));
  CUtensorMap q, k, v;
  if (!make_tensor_map_2d(&q, a.q, a.rows, static_cast<int64_t>(a.n_q_heads) * HD, a.ldq, kTile, FP16) ||
      !make_tensor_map_2d(&k, a.k, a.rows, static_cast<int64_t>(a.n_kv_heads) * HD, a.ldk, kTile, FP16) ||
      !make_tensor_map_2d(&v, a.v, a.rows, static_cast<int64_t>(a.n_kv_heads) * HD, a.ldv, kTile, FP16))
    return cuda_fail(cudaErrorInvalidValue, "vla_prompt_attn: tensor maps");
  int sms = 0;
  if (const int rc = device_sms(&sms)) return rc;
  static std::atomic<uint64_t> done{0};
  VLA_CUDA_TRY(set_smem_limit(prompt_attn_kernel<HD, FP16>, Smem<HD>::kTotal, done));
  VLA_CUDA_TRY(launch_at(Start::kInOrder, prompt_attn_kernel<HD, FP16>, dim3(static_cast<unsigned>(std::min(p.items_bound, sms))), dim3(kThreads),
                         Smem<HD>::kTotal, s, q, k, v, p));
  note_launch();
  return VLA_OK;
}

}  // namespace

int prompt_attn_launch(const PromptArgs& a, cudaStream_t s) {
  if (a.head_dim == 128) return a.fp16 ? launch<128, true>(a, s) : launch<128, false>(a, s);
  return a.fp16 ? launch<64, true>(a, s) : launch<64, false>(a, s);
}

}  // namespace vla
