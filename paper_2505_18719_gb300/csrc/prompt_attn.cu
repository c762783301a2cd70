// Causal attention of packed sequences on the tcgen05 tensor cores (include/vla_learn.h).
//
// With c = scale log2(e), for a query i over blocks of keys: s = q K^T, m = max s, weights 2^(c (s - m)), l their sum,
// O = 2^(c (m' - m)) O + P V; out = O / l, lse = ln 2 (c m + log2 l).  The reference m moves only when a maximum passes it by more than
// 2^8, so O is scaled again in few blocks; it is -infinity until a row has met a score above that.  Weights go to the values' type; fp16 ones are 2^7 times as large, so that one of
// 2^-21 of the row's largest still keeps all its bits (at most 2^15 with the reference 2^8 behind).  One 16-bit term a weight: outputs of bf16 are
// 0.0020 of their size off the 64-bit ones, where 32-bit weights and one rounding at the end give 0.0016; a second term would be a second product.
//
// A tile is 128 rows of one sequence and query head.  The tiles of a sequence and key-value head are numbered row tile after row tile, query
// head after query head, and an item is two neighbours: two query heads over the same rows where heads are shared, else two row tiles.
// Both go over the same keys, so a block of keys in shared memory serves 256 queries.  Items go sequence by sequence, the longest rows
// of a sequence first (its keys are read from HBM once, and the last items are short); persistent CTAs, one an SM.
//
// Where sequences are short (kShort rows on average), an item is one tile and each half of the CTA takes items of its own, with a ring of its own: a chain of 3 to 5
// blocks, loads and output does not fill an SM, two do (64 prefixes of about 290 rows, 32 heads: 173 us in pairs, 151 so).
//
// Blocks are 80 keys (64 there): so O, S and P of both tiles have tensor memory of their own (a tile's 256 columns: O [0, HD), S behind it, P
// behind that), and the next scores are under way as soon as the threads have read these.  With blocks of 128 keys for heads of 128 P
// has to lie over S, the chain scores - weights - product - next scores has no slack, and 16384 rows took 1.63 ms.  Products of 80 keys are
// bound by shared memory (4 KB of Q and 2.5 KB of K a step, 51 cycles where 128 keys take 65).
//
// Warps of 12 (16 in halves; there each half has the first, its own S and its own product warp):
//   warp 0       finds the items (a scan over the sequences' lengths, 32 sequences a step), hands their descriptors round and loads their tiles by
//                TMA: Q when the item before is done with it, key and value blocks into a ring; at the end the rows of no sequence;
//   warps 1, 2   issue S = Q K^T of a tile each;
//   warp 3       issues O += P V of both (V as the MN-major operand), after making values behind a sequence's last row zeros (their weights are
//                zeros, but a NaN would spoil the product).  One warp for all products cannot keep up, at 250 to 800 cycles from one group of
//                products to the next beside the softmax;
//   the last 8   one query row a thread: softmax, and the output.  (Two threads a row: the exchange of their maxima costs what the shorter rows
//                save.)
// A row that a value behind it spoilt (a weight of 0 times a NaN in the row's last blocks of keys) is computed again from its own keys alone
// (attend_row).  Rows that see such a value stay as they are (spoilt_rows): 16384 rows of 32 heads that all see a NaN take 1.5 ms, and
// took 880 when each of them was computed again; the 127 rows before a NaN in the last one take 150.
//
// Measured (32 query heads of 128): one sequence of 16384 rows, 8 key-value heads 1.41 to 1.45 ms warm (1.52 to 1.56 PFLOP/s; the tensor pipe 63 % busy at 8192 rows by
// its counter); 16 sequences of 1 to 2048 rows 198 us (0.95 PFLOP/s); 64 prefixes of 272 to 304 rows 140 us (4.3 TB/s); heads of 64: 8192 rows of 32 and
// 8 heads 342 us (0.80 PFLOP/s), the 64 prefixes 105 us.
#include <algorithm>
#include <type_traits>

#include "gemm.h"
#include "prompt_items.cuh"

namespace vla {

namespace {

constexpr int kSoftWarps = 8;

template <int HD, bool PAIRED>
struct Smem {
  static constexpr int kSoftWarp0 = PAIRED ? 4 : 8, kThreads = 32 * (kSoftWarp0 + kSoftWarps);
  static constexpr int kKeys = PAIRED ? 80 : 64;                    // keys of a block
  static constexpr int kStages = PAIRED ? 8 : 4;  // of a ring
  static constexpr int kRings = PAIRED ? 1 : 2;                     // for both tiles, or one each
  static constexpr int kItemReaders = PAIRED ? 3 + kSoftWarps : 2 + kSoftWarps / 2;
  static constexpr uint32_t kQBytes = kTile * HD * 2, kKvBytes = kKeys * HD * 2, kKvBlock = kKeys * 128;
  static constexpr uint32_t kRing = 2 * kQBytes, kBars = kRing + kRings * kStages * kKvBytes;
  static constexpr uint32_t kTotal = 1024 + kBars + 1024;
  static constexpr uint32_t kColS = HD, kColP = HD + kKeys;  // of a tile's 256 columns
  static_assert(kTotal <= 232448 && kColP + kKeys / 2 <= 256 && kKvBlock % 1024 == 0, "shared and tensor memory");
};

// Barriers.  Of each tile: Q loaded / free, S written / read, P written, its product done; end of the issuing warps' products; item
// descriptors (of each tile, where not PAIRED); ring slots (likewise), and loads into them that end behind a sequence's last row.
enum : int {
  QFULL = 0, QFREE = 2, SFULL = 4, SREAD = 6, PFULL = 8, PVDONE = 10, DRAIN = 12, IFULL = 16, IFREE = 32, KVFULL = 48, KVFREE = 56, TAIL = 64,
  kBarCount = 72
};

struct Params {
  PromptArgs a;
  int group, items_bound;
  float c, offset;  // scale log2(e); log2 of the weights' common factor
  uint64_t wait_limit;
};

// An item of PAIRED is tiles 2 a and 2 a + 1 of key-value head b, else tile a.  Of a tile: the row tile, the query head, how many keys its
// rows see, and its blocks (0: no such tile).
struct Tile {
  int row_tile, head, keys, nb;
};
template <int KN>
__device__ __forceinline__ Tile tile_of(const Item& it, int number, int group) {
  Tile t;
  t.row_tile = number / group;
  t.head = it.b * group + number % group;
  t.keys = t.row_tile * kTile < it.len ? min(it.len, (t.row_tile + 1) * kTile) : 0;
  t.nb = (t.keys + KN - 1) / KN;
  return t;
}

template <int HD, bool FP16, bool PAIRED>
__global__ void __launch_bounds__((Smem<HD, PAIRED>::kThreads), 1)
    prompt_attn_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                       const __grid_constant__ CUtensorMap tm_v, const Params p) {
  using Sm = Smem<HD, PAIRED>;
  constexpr int KB = HD / 64, NS = Sm::kStages, KN = Sm::kKeys;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + Sm::kBars);
  const uint32_t s0 = smem_u32(smem), b0 = smem_u32(bars);
  auto BAR = [&](int i) { return b0 + 8u * static_cast<uint32_t>(i); };
  Item* items = reinterpret_cast<Item*>(bars + kBarCount);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(items + 2 * kItems);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  static_assert(kBarCount * 8 + 2 * kItems * 16 + 12 <= 1024 && kBarCount % 2 == 0, "barrier area");
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint32_t* status = p.a.status;
  const uint64_t limit = p.wait_limit;

  if (threadIdx.x == 0) {
    for (int t = 0; t < 2; ++t) {
      mbar_init(BAR(QFULL + t), 1);
      mbar_init(BAR(QFREE + t), 1);
      mbar_init(BAR(SFULL + t), 1);
      mbar_init(BAR(SREAD + t), kSoftWarps / 2);
      mbar_init(BAR(PFULL + t), kSoftWarps / 2);
      mbar_init(BAR(PVDONE + t), 1);
    }
    for (int i = 0; i < 4; ++i) mbar_init(BAR(DRAIN + i), 1);
    for (int i = 0; i < 2 * kItems; ++i) {
      mbar_init(BAR(IFULL + i), 1);
      mbar_init(BAR(IFREE + i), Sm::kItemReaders);
    }
    for (int s = 0; s < 8; ++s) {
      mbar_init(BAR(KVFULL + s), 1);
      mbar_init(BAR(KVFREE + s), PAIRED && !(s & 1) ? 2 : 1);  // (keys of both tiles: read by a warp for each)
      mbar_init(BAR(TAIL + s), 1);
    }
    abort_flag[0] = abort_flag[1] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) tmem_take(smem_u32(tmem_slot));
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  // The tile that this warp works for (its S, its softmax; where not PAIRED also its loads and its product with the values), and its ring.
  const int x = warp >= Sm::kSoftWarp0 ? (warp - Sm::kSoftWarp0) >> 2 : PAIRED ? warp - 1 : warp & 1;
  const int lane0 = PAIRED ? 0 : x, ring0 = lane0 * NS;
  auto slot = [&](int s) { return s0 + Sm::kRing + static_cast<uint32_t>(ring0 + s) * Sm::kKvBytes; };
  auto waitw = [&](int bar, uint32_t phase) { return warp_waits(BAR(bar), phase & 1u, abort_flag, status, limit); };
  // Next descriptor; false at the end or at a timeout.
  auto take = [&](int k, Item& it) {
    const int i = 8 * lane0 + (k & 7);
    if (!waitw(IFULL + i, k >> 3)) return false;
    it = items[i];
    __syncwarp();
    if (lane == 0) mbar_arrive(BAR(IFREE + i));
    return it.len >= 0;
  };
  auto number = [&](const Item& it, int tile) { return PAIRED ? 2 * it.a + tile : it.a; };

  if (PAIRED ? warp == 0 : warp <= 1) {
    // ------------------------------------------------------------------ items and loads (a whole warp that waits, one thread that loads)
    const int n_seq = p.a.n_seq, group = p.group, Hk = p.a.n_kv_heads;
    if (blockIdx.x == 0 && warp == 0) check_starts(p.a.seq_start, n_seq, p.a.rows, lane, 32, status);
    auto items_of = [&](int len) {  // of a key-value head
      const int tiles = (len + kTile - 1) / kTile * group;
      return PAIRED ? (tiles + 1) / 2 : tiles;
    };
    int k = 0;
    auto put = [&](const Item& it) {
      const int i = 8 * lane0 + (k & 7);
      if (k >= kItems && !waitw(IFREE + i, (k >> 3) - 1)) return false;
      if (lane == 0) {
        items[i] = it;
        mbar_arrive(BAR(IFULL + i));
      }
      __syncwarp();
      ++k;
      return true;
    };
    int n = 0, used[2] = {0, 0};  // ring slots filled; Q tiles loaded
    // of each slot: its last load ends behind a sequence's last row; loads that did, and that did not, modulo 2
    uint32_t on_tail = 0, tail_phase = 0, full_phase = 0;
    auto load = [&](const Item& it) {
      const Tile t0 = tile_of<KN>(it, number(it, 0), group), t1 = tile_of<KN>(it, number(it, 1), group);
      auto load_q = [&](const Tile& t, int x) {
        if (!t.nb) return true;
        int& loaded = used[PAIRED ? x : 0];
        if (loaded && !waitw(QFREE + x, loaded - 1)) return false;
        if (lane == 0) {
          mbar_arrive_expect_tx(BAR(QFULL + x), Sm::kQBytes);
#pragma unroll
          for (int kb = 0; kb < KB; ++kb)
            tma_load_2d(s0 + x * Sm::kQBytes + kb * kBlockBytes, &tm_q, BAR(QFULL + x), t.head * HD + kb * 64, it.begin + t.row_tile * kTile);
        }
        __syncwarp();
        ++loaded;
        return true;
      };
      auto load_kv = [&](const CUtensorMap* map, int j, bool tail) {
        const int s = n % NS, bar = (tail ? TAIL : KVFULL) + ring0 + s;
        if (n >= NS && !waitw(KVFREE + ring0 + s, n / NS - 1)) return false;
        if (lane == 0) {
          mbar_arrive_expect_tx(BAR(bar), Sm::kKvBytes);
#pragma unroll
          for (int kb = 0; kb < KB; ++kb) tma_load_2d(slot(s) + kb * Sm::kKvBlock, map, BAR(bar), it.b * HD + kb * 64, it.begin + j * KN);
        }
        __syncwarp();
        on_tail = (on_tail & ~(1u << s)) | (static_cast<uint32_t>(tail) << s);
        tail_phase ^= static_cast<uint32_t>(tail) << s;
        full_phase ^= static_cast<uint32_t>(!tail) << s;
        ++n;
        return true;
      };
      auto load_k = [&](int j) { return load_kv(&tm_k, j, false); };
      auto load_v = [&](int j) { return load_kv(&tm_v, j, it.len - j * KN < KN); };
      const int nb = max(t0.nb, t1.nb);
      bool ok = load_k(0) && (PAIRED ? load_q(t0, 0) && load_q(t1, 1) : load_q(t0, lane0)) && load_v(0);
      for (int j = 1; j < nb && ok; ++j) ok = load_k(j) && load_v(j);
      return ok;
    };
    if (find_items(
            p.a.seq_start, n_seq, p.a.rows, blockIdx.x + lane0 * gridDim.x, Sm::kRings * gridDim.x, p.items_bound,
            [&](int len) { return static_cast<int64_t>(items_of(len)) * Hk; },
            [&](int begin, int len, int u) {
              const Item it{begin, len, items_of(len) - 1 - u / Hk, u % Hk};
              return put(it) && load(it);
            }))
      put(Item{0, -1, 0, 0});
    const Outside out(p.a.seq_start, p.a.n_seq, p.a.rows);
    for (int i = blockIdx.x + lane0 * gridDim.x; i < out.count(); i += Sm::kRings * gridDim.x) {
      const int row = out.row(i);
      zero_row(elem(p.a.out, row * p.a.ldo), p.a.n_q_heads * HD);
      if (p.a.lse)
        for (int e = lane; e < p.a.n_q_heads; e += 32) p.a.lse[static_cast<int64_t>(row) * p.a.n_q_heads + e] = -INFINITY;
    }
    // nothing may land after the CTA has gone
    for (int i = max(0, n - NS); i < n; ++i) {
      const int s = i % NS;
      const bool tail = (on_tail >> s) & 1;
      wait_drain(BAR((tail ? TAIL : KVFULL) + ring0 + s), (((tail ? tail_phase : full_phase) >> s) & 1) ^ 1, limit);
    }
    for (int i = 0; i < (PAIRED ? 2 : 1); ++i)
      if (used[i]) wait_drain(BAR(QFULL + (PAIRED ? i : lane0)), (used[i] - 1) & 1, limit);
  } else if (PAIRED ? warp <= 2 : warp <= 3) {
    // ------------------------------------------------------------------ S of tile x
    const uint32_t tS = tmem + static_cast<uint32_t>(x) * 256 + Sm::kColS, dq = tile_desc(s0 + x * Sm::kQBytes);
    int block = 0, q = 0;  // blocks and Q tiles of this tile so far
    int s = 0, round = 0;  // ring slot of the next block of keys, and how often the ring has gone round
    auto next_slot = [&]() {
      s += 2;
      if (s >= NS) {
        s = 0;
        ++round;
      }
    };
    Item it;
    bool ok = true;
    for (int k = 0; ok && take(k, it); ++k) {
      it = Item{0, uniform(it.len), uniform(it.a), uniform(it.b)};
      const Tile t = tile_of<KN>(it, number(it, x), p.group);
      const int nb = t.nb, other = PAIRED ? tile_of<KN>(it, number(it, x ^ 1), p.group).nb : 0, keys = t.keys;
      for (int j = 0; j < nb; ++j, ++block) {
        const uint32_t kv = tile_desc(slot(s), Sm::kKvBlock), is = tile_idesc((min(KN, keys - j * KN) + 15) & ~15, FP16, false);
        const uint32_t freed = BAR(KVFREE + ring0 + s);
        const bool last = j == nb - 1, lone = PAIRED && j >= other;
        // the scores go over those of the block before once the threads have read them
        if (!(ok = waitw(KVFULL + ring0 + s, round) && (j > 0 || waitw(QFULL + x, q)) && (block == 0 || waitw(SREAD + x, block - 1)))) break;
        tc_fence_after();
        if (elected()) {
#pragma unroll
          for (int i = 0; i < HD / 16; ++i) tile_mma(tS, dq + k_major_step(i), kv + k_major_step(i, Sm::kKvBlock), is, i > 0);
          tc_commit(BAR(SFULL + x));
          tc_commit(freed);
          if (lone) tc_commit(freed);
          if (last) tc_commit(BAR(QFREE + x));
        }
        __syncwarp();
        next_slot();
      }
      q += nb > 0;
      for (int j = nb; j < other; ++j) next_slot();
    }
    if (elected()) tc_commit(BAR(DRAIN + x));
    wait_drain(BAR(DRAIN + x), 0, limit);
  } else if (PAIRED ? warp == 3 : warp <= 5) {
    // ------------------------------------------------------------------ O += P V, of both tiles in turn (not PAIRED: of tile x)
    const uint32_t io = tile_idesc(HD, FP16, true);
    int block[2] = {0, 0};
    int s = 1;
    uint32_t tails = 0, fulls = 0;  // of each ring slot: its loads so far that end behind a sequence's last row, and the others, modulo 2
    Item it;
    bool ok = true;
    for (int k = 0; ok && take(k, it); ++k) {
      it = Item{0, uniform(it.len), uniform(it.a), uniform(it.b)};
      const Tile t[2] = {tile_of<KN>(it, number(it, 0), p.group), tile_of<KN>(it, number(it, 1), p.group)};
      const int nb = max(t[0].nb, t[1].nb);
      for (int j = 0; j < nb && ok; ++j) {
        const uint32_t kv = tile_desc(slot(s), Sm::kKvBlock), freed = BAR(KVFREE + ring0 + s);
        const int rows = it.len - j * KN;
        if (rows < KN) {
          // values behind a sequence's last row become zeros: their weights are zeros, but a NaN would spoil the product
          if (!(ok = waitw(TAIL + ring0 + s, tails >> s))) break;
          tails ^= 1u << s;
          zero_tile_rows<HD>(smem + Sm::kRing + (ring0 + s) * Sm::kKvBytes, rows, (rows + 15) & ~15, Sm::kKvBlock);
          fence_async_smem();
          __syncwarp();
        } else if (!(ok = waitw(KVFULL + ring0 + s, fulls >> s))) {
          break;
        } else {
          fulls ^= 1u << s;
        }
#pragma unroll
        for (int i2 = 0; i2 < (PAIRED ? 2 : 1); ++i2) {
          if (j >= t[i2].nb) continue;
          const int y = PAIRED ? i2 : x;
          const uint32_t tO = tmem + static_cast<uint32_t>(y) * 256, tP = tO + Sm::kColP, more = j > 0;
          const int steps = (min(KN, t[i2].keys - j * KN) + 15) / 16;
          const bool frees = !PAIRED || i2 == 1 || j >= t[1].nb;  // the block's last reader (a commit covers what was issued before)
          if (!(ok = ok && waitw(PFULL + y, block[i2]))) break;
          tc_fence_after();
          if (elected()) {
#pragma unroll
            for (int i = 0; i < KN / 16; ++i)
              if (i < steps) tile_mma_ts(tO, tP + i * 8, kv + mn_major_step(i), io, i > 0 ? 1u : more);
            tc_commit(BAR(PVDONE + y));
            if (frees) tc_commit(freed);
          }
          __syncwarp();
          ++block[i2];
        }
        s += 2;
        if (s >= NS) s = 1;
      }
    }
    if (elected()) tc_commit(BAR(DRAIN + 2 + lane0));
    wait_drain(BAR(DRAIN + 2 + lane0), 0, limit);
  } else if (warp >= Sm::kSoftWarp0) {
    // ------------------------------------------------------------------ softmax and output
    const int q4 = warp & 3, r = q4 * 32 + lane;  // lane quarter, row in the tile
    const uint32_t tO = tmem + (static_cast<uint32_t>(q4 * 32) << 16) + static_cast<uint32_t>(x) * 256;
    const uint32_t tS = tO + Sm::kColS, tP = tO + Sm::kColP;
    const float c = p.c;
    const uint64_t c2 = pair_of(c, c);
    int block = 0;
    bool ok = true;
    Item it;
    for (int k = 0; ok && take(k, it); ++k) {
      const Tile t = tile_of<KN>(it, number(it, x), p.group);
      const int nb = t.nb, head = t.head, tile0 = t.row_tile * kTile;
      if (!nb) continue;
      const int live = min(32, it.len - tile0 - q4 * 32);  // the warp's rows of the sequence, at most 0: none
      float m = -INFINITY, l = 0.f;
      for (int j = 0; j < nb; ++j, ++block) {
        if (!(ok = waitw(SFULL + x, block))) break;
        tc_fence_after();
        uint32_t s[KN];
        if (live > 0) {
#pragma unroll
          for (int i = 0; i + 32 <= KN; i += 32) tmem_ld32(tS + i, s + i);
          if constexpr (KN % 32) {
            uint32_t v[16];
            tmem_ld16(tS + KN - 16, v);
#pragma unroll
            for (int i = 0; i < 16; ++i) s[KN - 16 + i] = v[i];
          }
          tmem_wait_ld();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(BAR(SREAD + x));
        // (asked for early: the answer takes 100 to 200 cycles)
        const bool free_p = block == 0 || mbar_test_wait(BAR(PVDONE + x), (block - 1) & 1);
        float alpha = 1.f;
        if (live > 0) {
          if ((j + 1) * KN > tile0) {  // keys behind the row
            const int seen = tile0 + r - j * KN;
#pragma unroll
            for (int i = 0; i < KN; ++i) s[i] = i <= seen ? s[i] : 0xff800000u;
          }
          float top[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) top[i] = fmaxf(__uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1]));
#pragma unroll
          for (int i = 16; i < KN; i += 2)  // (three-input maxima)
            top[(i >> 1) & 7] = fmaxf(top[(i >> 1) & 7], fmaxf(__uint_as_float(s[i]), __uint_as_float(s[i + 1])));
          const float mb = fmaxf(fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])), fmaxf(fmaxf(top[4], top[5]), fmaxf(top[6], top[7])));
          // (a row whose keys so far all score -infinity has no reference yet: the first finite score sets it; -inf + inf is no move)
          if ((mb - m) * c > 8.f || j == 0) {
            alpha = j == 0 ? 0.f : ex2((m - mb) * c);
            m = mb;
            l *= alpha;
          }
        }
        // O and P are the last product's until it is done
        if (!__all_sync(0xffffffffu, free_p) && !(ok = waitw(PVDONE + x, block - 1))) break;
        tc_fence_after();
        if (live > 0) {
          if (j > 0 && __any_sync(0xffffffffu, alpha != 1.f)) {
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
          const float shift = m == -INFINITY ? p.offset : fmaf(-m, c, p.offset);
          const uint64_t shift2 = pair_of(shift, shift);
          uint64_t sum[4] = {0, 0, 0, 0};
          auto weights = [&](int i, auto count) {
            uint32_t w[count() / 2];
#pragma unroll
            for (int e = 0; e < count() / 2; ++e) {
              const float2 y = halves_of(fma2(pair_of(__uint_as_float(s[i + 2 * e]), __uint_as_float(s[i + 2 * e + 1])), c2, shift2));
              const float a = ex2(y.x), b = ex2(y.y);
              sum[e & 3] = add2(sum[e & 3], pair_of(a, b));
              w[e] = pack2<FP16>(a, b);
            }
            if constexpr (count() == 32)
              tmem_st16(tP + i / 2, w);
            else
              tmem_st8(tP + i / 2, w);
          };
#pragma unroll
          for (int i = 0; i + 32 <= KN; i += 32) weights(i, std::integral_constant<int, 32>());
          if constexpr (KN % 32) weights(KN - 16, std::integral_constant<int, 16>());
          const float2 both = halves_of(add2(add2(sum[0], sum[1]), add2(sum[2], sum[3])));
          l += both.x + both.y;
          tmem_wait_st();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(BAR(PFULL + x));
      }
      if (!ok || !(ok = waitw(PVDONE + x, block - 1))) break;
      tc_fence_after();
      if (live <= 0) continue;
      const int64_t row = it.begin + tile0 + q4 * 32;
      const bool bad = store_tile<FP16, HD / 32>(tO, l == 0.f ? 0.f : 1.f / l, elem(p.a.out, row * p.a.ldo + head * HD), p.a.ldo, live);
      if (p.a.lse && lane < live) p.a.lse[(row + lane) * p.a.n_q_heads + head] = (log2f(l) - fmaf(-m, c, p.offset)) * kLn2;
      __syncwarp();  // (attend_row's lanes read and write what other lanes have written here)
      // (l is no number: nor is the row, by its own scores; 0: no key has weight)
      uint32_t again = __ballot_sync(0xffffffffu, bad && l > 0.f && lane < live);
      if (again) again = spoilt_rows<HD, FP16>(p.a, static_cast<int>(row), head, it.begin, again, const_cast<int*>(abort_flag) + 1);
      again |= __ballot_sync(0xffffffffu, bad && l == 0.f && lane < live);
      while (again) {
        const int rr = __ffs(static_cast<int>(again)) - 1;
        again &= again - 1;
        attend_row<HD, FP16>(p.a, static_cast<int>(row) + rr, head, it.begin, const_cast<int*>(abort_flag) + 1);
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

// Sequences of fewer rows than this on average: a tile each for the two halves of a CTA.  32768 rows of bf16 in sequences of 128, 256, 384, 512, 640,
// 767, 1024 and 2048, pairs / halves in us: 32 and 8 heads of 128: 155/160, 179/176, 192/196, 213/217, 228/257, 240/249, 282/298, 441/489;
// 32 and 32 of 128: 263/173, 221/200, 219/213, 242/229, 259/268, 263/268, 301/328, 458/527; 16 and 4 of 64: 74/70, 86/83, 92/98, 102/100,
// 107/111, 113/113, 132/134, 209/227.  What the halves gain is with heads of their own; where they lose below the border it is by 2 to 13 %.
constexpr int kShort = 768;

template <int HD, bool FP16, bool PAIRED>
int launch(const PromptArgs& a, cudaStream_t s) {
  using Sm = Smem<HD, PAIRED>;
  Params p{};
  p.a = a;
  p.group = a.n_q_heads / a.n_kv_heads;
  p.c = a.scale * kLog2e;
  p.offset = FP16 ? 7.f : 0.f;
  p.wait_limit = g_wait_limit_ns.load(std::memory_order_relaxed);
  // as many items as well-formed sequences can have: a last row tile each (and a lone last tile)
  const int64_t seqs = std::min(a.n_seq, a.rows), tiles = (a.rows / kTile + seqs) * p.group;
  p.items_bound = static_cast<int>(std::min<int64_t>((PAIRED ? (tiles + seqs + 1) / 2 : tiles) * a.n_kv_heads, 0x7fffffff));
  CUtensorMap q, k, v;
  if (!make_tensor_map_2d(&q, a.q, a.rows, static_cast<int64_t>(a.n_q_heads) * HD, a.ldq, kTile, FP16) ||
      !make_tensor_map_2d(&k, a.k, a.rows, static_cast<int64_t>(a.n_kv_heads) * HD, a.ldk, Sm::kKeys, FP16) ||
      !make_tensor_map_2d(&v, a.v, a.rows, static_cast<int64_t>(a.n_kv_heads) * HD, a.ldv, Sm::kKeys, FP16))
    return cuda_fail(cudaErrorInvalidValue, "vla_prompt_attn: tensor maps");
  int sms = 0;
  if (const int rc = device_sms(&sms)) return rc;
  const auto kern = prompt_attn_kernel<HD, FP16, PAIRED>;
  static std::atomic<uint64_t> done{0};
  VLA_CUDA_TRY(set_smem_limit(kern, Sm::kTotal, done));
  VLA_CUDA_TRY(launch_at(Start::kInOrder, kern, dim3(static_cast<unsigned>(std::min(p.items_bound, sms))), dim3(Sm::kThreads), Sm::kTotal, s, q, k, v,
                         p));
  note_launch();
  return VLA_OK;
}
template <int HD, bool FP16>
int launch_for(const PromptArgs& a, cudaStream_t s) {
  return a.rows / std::min(a.n_seq, a.rows) < kShort ? launch<HD, FP16, false>(a, s) : launch<HD, FP16, true>(a, s);
}

}  // namespace

int prompt_attn_launch(const PromptArgs& a, cudaStream_t s) {
  if (a.head_dim == 128) return a.fp16 ? launch_for<128, true>(a, s) : launch_for<128, false>(a, s);
  return a.fp16 ? launch_for<64, true>(a, s) : launch_for<64, false>(a, s);
}

}  // namespace vla
