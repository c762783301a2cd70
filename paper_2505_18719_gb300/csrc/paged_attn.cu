// Attention of one new token per row over its environment's paged positions.
//
// For a row r, query head h and its key-value head g: s_p = scale q . K_p, out = sum_p 2^(s_p log2 e - m) V_p / l with
// l the sum of the weights, any m that keeps them in range.  Sums over disjoint sets of positions join by
// (m, l, o) = (max m_i, sum 2^(m_i - m) l_i, sum 2^(m_i - m) o_i).
//
// Each cached byte is used once per 8 query heads, so the kernel is bound by HBM (2 hd 2-byte reads for 4 hd
// flops a query head) or, for few short rows, by latency.  The work is the list of (row, key-value head, tile of
// 8 query heads, block of positions), in that order, shared out on the device from the rows' lengths, as many shares
// as the GPU holds CTAs at once.  A share is a number of whole items (all but the block) where that leaves no CTA with
// much more than the mean, else equal numbers of blocks: then however long or uneven the rows are, all CTAs end
// together, and an item that a share's end cuts is joined by the last CTA that arrives at its ticket, from partial
// results in the workspace.  The 4 warps of a CTA take a step of each block each; many short items go to
// single warps instead.
//
// Each warp has its own ring of 8 KB stages filled by cp.async, which runs on from item to item.  The pages of
// a step's positions are looked up one step before its copies are issued; 16-byte pieces are XOR-swizzled so that
// ldmatrix reads without bank conflicts.  Scores and outputs run on mma.sync m16n8k16 with the 8 query heads as
// rows 0-7; rows 8-15 hold the low parts, x - fp16(x) (or bf16), of fp32 queries and of the softmax weights, so that
// they keep 22 (16) significant bits at no further instruction.  fp16 weights are 2^15 times the true ones: a weight
// of 1e-5 beside one of 1 keeps its bits.  So do fp32 queries of any size: each head of them is taken times the power of two
// that brings its largest channel to [2^14, 2^15), and its scores times the inverse.
//
// The warps of a CTA meet in shared memory at an item's end, each query head joined by one warp.  With one or two heads
// a tile that is the warps in turn, over four buffers: the others only arrive at its barrier and go on.  (A warp has its
// turn within any four items and then waits for all to have arrived, so whoever writes a buffer again knows that
// it has been read.)
//
// What runs once an item or once a call is kept short and in one place: a cold instruction line costs as
// much as a load (a second copy of the join made calls of few long rows 10 us slower).
//
// Measured, heads of 128, each cached byte once: 64 rows x 32 heads over 273 to 311 positions 52 us (5.9 TB/s, 0.88 of the copy rate:
// 5 us before the first bytes arrive and after the last, and 7 items on the fullest CTA where the mean is 6.7), 256 rows x 32 heads
// over 1031 to 1097 positions 661 to 690 us (6.5 to 6.8 TB/s), 8 rows x 8 key-value heads over up to 131072 positions 279 to 286 us
// (6.8 TB/s); 4 rows x 4 heads of 64 over 80 positions 3.8 us, a chain of latencies.
#include <algorithm>
#include <type_traits>

#include "lm.h"
#include "ptx.cuh"

namespace vla {

namespace {

constexpr int kWarps = 4;
constexpr int kHeads = 8;        // query heads of a tile
constexpr int kMaxCtas = 512;
constexpr int kJoin = 32;        // partial results that one warp joins at a time
constexpr int kMinBlocks = 4;    // a share of cut items is no smaller while items are longer
constexpr int kCutBlocks = 8;    // blocks that the join of a cut item costs
constexpr int kItem = 1;         // what an item costs beside its blocks, in blocks: its queries and its join
constexpr int kLastPosition = 0x7fffff00;  // a whole block past it still fits 32 bits
// Single warps take items of up to kAlone steps where that is less than all warps of a CTA take, an item counted as its steps
// and kEnds more (bf16 heads of 128, device time of single warps and of whole CTAs: 1152 items of 2 / 60 / 250 positions 5.0, 10.2,
// 27.0 us and 9.7, 12.6, 27.8; 360 items 4.7, 7.8, 18.5 and 6.5, 7.0, 15.0; 1536 items of 250 38 and 36, 3000 items 63 and 62)
constexpr int kAlone = 16, kEnds = 2;

// Workspace: tickets of the first level [kSlots][8], of the second as many, then the partial results: per slot
// o [8][hd], (m, l) [8].  Two slots a CTA: the item that it found begun, and the one that it leaves.
constexpr int kSlots = 2 * kMaxCtas;
constexpr size_t kTicketBytes = 2 * kSlots * kHeads * sizeof(int);
__host__ __device__ constexpr int slot_floats(int hd) { return kHeads * hd + 2 * kHeads; }

template <int HD>
struct Ring {
  // hd 64 has twice the softmax per byte and needs the warps more than the depth: 76 rows of 6400 positions x 10 heads
  // take 185 us with three CTAs of two stages, 204 with two of three (hd 128: 64 rows 54 us with two of three, 90 with
  // three of two)
  static constexpr int kStages = HD == 64 ? 2 : 3, kCtasPerSm = HD == 64 ? 3 : 2;
  static constexpr int kStep = 2048 / HD;             // positions of a warp's step: 16 or 32, 8 KB of keys and values
  static constexpr int kRow = HD * 2;                 // bytes of a position's channels
  static constexpr int kPlane = kStep * kRow;         // keys or values of a step
  static constexpr int kStage = 2 * kPlane;
  static constexpr int kBytes = kWarps * kStages * kStage;
};

__device__ __forceinline__ void cp16(uint32_t dst, const void* src, uint32_t bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void ldsm(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldsm_t(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
template <bool BF16>
__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if constexpr (BF16)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// 2^(m - top) of a set whose maximum is m within one whose maximum is top; 0 for an empty set.
__device__ __forceinline__ float join_weight(float m, float top) { return m == -INFINITY ? 0.f : exp2_approx(m - top); }
// Two values as (high, low) words of the cache's type.
template <bool BF16>
__device__ __forceinline__ void split2(float a, float b, uint32_t& hi, uint32_t& lo) {
  if constexpr (BF16) {
    hi = pack_bf16x2(a, b);
    const float2 h = unpack_bf16x2(hi);
    lo = pack_bf16x2(a - h.x, b - h.y);
  } else {
    hi = pack_f16x2(a, b);
    const float2 h = unpack_f16x2(hi);
    lo = pack_f16x2(a - h.x, b - h.y);
  }
}

__device__ __forceinline__ int add_acq_rel(int* p, int n) {
  int v;
  asm volatile("atom.acq_rel.gpu.global.add.s32 %0, [%1], %2;" : "=r"(v) : "l"(p), "r"(n) : "memory");
  return v;
}

// The channels of a head that a lane joins.
template <int HD>
struct Channels {
  static constexpr int kN = HD / 32;
  alignas(16) float v[kN];
  __device__ __forceinline__ Channels() {
#pragma unroll
    for (int i = 0; i < kN; ++i) v[i] = 0.f;
  }
  __device__ __forceinline__ void add(float f, const Channels& x) {
#pragma unroll
    for (int i = 0; i < kN; ++i) v[i] = fmaf(f, x.v[i], v[i]);
  }
  template <typename T>
  __device__ __forceinline__ void set(T x) {
    *reinterpret_cast<T*>(v) = x;
  }
  using Word = typename std::conditional<HD == 128, float4, float2>::type;
  static __device__ __forceinline__ Channels load(const float* p) {
    Channels c;
    c.set(*reinterpret_cast<const Word*>(p));
    return c;
  }
  static __device__ __forceinline__ Channels load_l2(const float* p) {
    Channels c;
    c.set(__ldcg(reinterpret_cast<const Word*>(p)));
    return c;
  }
  __device__ __forceinline__ void store(float* p) const { *reinterpret_cast<Word*>(p) = *reinterpret_cast<const Word*>(v); }
  __device__ __forceinline__ void write(void* p, int64_t i, float f, int dtype) const {
    if (dtype == VLA_F32) {
      Channels c;
      c.add(f, *this);
      c.store(static_cast<float*>(p) + i);
      return;
    }
    uint32_t w[kN / 2];
#pragma unroll
    for (int j = 0; j < kN / 2; ++j)
      w[j] = dtype == VLA_F16 ? pack_f16x2(f * v[2 * j], f * v[2 * j + 1]) : pack_bf16x2(f * v[2 * j], f * v[2 * j + 1]);
    if constexpr (kN == 4)
      *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p) + i) = make_uint2(w[0], w[1]);
    else
      *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(p) + i) = w[0];
  }
};

// An item as far as a share takes it, handed from the loading to the computing side of a warp.
struct Segment {
  int row, kv, tile, steps;  // (row, key-value head, tile); its blocks in this share, 0 = the share is done
  int from, blocks;          // the first of them; the item's blocks
};

enum Pages : int { kAnyPage = 0, kEights = 1, kShifted = 2 };  // kEights: multiples of 8 positions; kShifted: and powers of two

// Pages of multiples of 8 positions: 8 rows of ldmatrix share a page.  ONE: a query head for each key-value head (known when compiled: 64
// rows x 32 heads 51.7 us, 52.3 without; 150 rows x 20 heads over 4 positions 9.3 and 10.2).
template <int HD, bool BF16, bool PAIR, int PAGES, bool ONE>
__global__ void __launch_bounds__(32 * kWarps, Ring<HD>::kCtasPerSm) paged_attn_kernel(const PagedAttnArgs a, const int page_shift, const int tiles) {
  using R = Ring<HD>;
  using Some = Channels<HD>;
  constexpr int kStep = R::kStep, kStages = R::kStages;
  constexpr bool ALIGNED = PAGES != kAnyPage;
  constexpr float kShift = BF16 ? 0.f : 15.f;
  extern __shared__ __align__(128) uint8_t sm_raw[];
  uint8_t* sm = sm_raw + (-smem_u32(sm_raw) & 255u);  // rows of 256 bytes at multiples of 256
  float* const join_all = reinterpret_cast<float*>(sm + R::kBytes);  // [buffers][kWarps][tile_heads][HD], or a part for each warp
  constexpr int kJoinFloats = kWarps * kHeads * HD;
  __shared__ float2 join_ml[kWarps * kHeads];
  __shared__ uint32_t seen[kWarps][kStages];
  __shared__ Segment queue[kWarps][4];  // the loading side is at most two segments ahead
  __shared__ int64_t sums[kWarps];
  __shared__ int longest[kWarps];
  __shared__ int start_row;
  __shared__ int64_t start_units;
  pdl_launch_dependents();
  pdl_wait();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int items = ONE ? a.kv.n_heads : a.kv.n_heads * tiles, group = ONE ? 1 : a.n_q_heads / a.kv.n_heads, all_items = a.rows * items;

  // positions of a row, 0 where it has none or what it says of itself is out of range
  auto length_of = [&](int row, int& env) {
    const int pos = a.row_pos[row];
    env = a.row_env[row];
    const int col = PAGES == kShifted ? pos >> page_shift : pos / a.kv.page_size;
    const bool ok = pos >= 0 && pos <= kLastPosition && col < a.max_pages && static_cast<unsigned>(env) < static_cast<unsigned>(a.n_env);
    if (!ok && pos != -1) raise_status(a.status, VLA_STATUS_PAGES);
    return ok ? pos + 1 : 0;
  };

  // ---- this CTA's share.  Each thread sums a run of rows.
  int crew = kWarps;   // warps that share an item
  int item, end_item;  // this worker's items
  int block = 0;       // of the first one
  int64_t to_load;     // blocks after which the share ends
  int64_t share;       // a share's units: blocks, and kItem more before the first block of each item
  {
    const int run = (a.rows + 32 * kWarps - 1) / (32 * kWarps), r0 = tid * run, r1 = min(r0 + run, a.rows);
    int64_t sum = 0;
    int most = 1, env;
    for (int r = r0; r < r1; ++r) {
      const int steps = max(1, (length_of(r, env) + kStep - 1) / kStep);
      most = max(most, steps);
      sum += (steps + kWarps - 1) / kWarps + kItem;
    }
    int64_t upto = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t u = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += u;
    }
    most = __reduce_max_sync(0xffffffffu, most);
    if (lane == 31) {
      sums[warp] = upto;
      longest[warp] = most;
    }
    __syncthreads();
    int64_t total = 0, before = upto - sum;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) before += sums[w];
      total += sums[w];
      most = max(most, longest[w]);
    }
    total *= items;
    const int ctas = static_cast<int>(gridDim.x), me = static_cast<int>(blockIdx.x);
    // at least the mean, without a 64-bit division
    share = static_cast<int64_t>(static_cast<float>(total - 1) * 1.000001f / static_cast<float>(ctas)) + 1;
    to_load = INT64_MAX;
    const int per = (all_items - 1) / ctas + 1, per_warp = (per + kWarps - 1) / kWarps, longest_item = (most + kWarps - 1) / kWarps;
    if (most <= kAlone && static_cast<int64_t>(per_warp) * (most + kEnds) < static_cast<int64_t>(per) * (longest_item + kEnds)) {
      crew = 1;
      item = min(all_items, (me * kWarps + warp) * per_warp);
      end_item = min(all_items, item + per_warp);
    } else if (static_cast<int64_t>(per) * (longest_item + kItem) <= share + kCutBlocks || share > (1 << 30)) {
      item = min(all_items, me * per);
      end_item = min(all_items, item + per);
    } else {
      const int64_t mean = static_cast<int64_t>(static_cast<float>(total) / static_cast<float>(all_items)) + 1;
      share = max(share, min(static_cast<int64_t>(kMinBlocks + kItem), mean));
      const int64_t first = share * me, left = min(share, total - first);
      if (left <= 0) return;
      // the thread whose run of rows has the share's first unit finds its row
      if (before * items <= first && first < (before + sum) * items) {
        int r = r0;
        for (;; ++r) {
          const int units = max(1, (length_of(r, env) + kStep * kWarps - 1) / (kStep * kWarps)) + kItem;
          if (r + 1 >= r1 || first < (before + units) * items) break;
          before += units;
        }
        start_row = r;
        start_units = first - before * items;
      }
      __syncthreads();
      const int units = max(1, (length_of(start_row, env) + kStep * kWarps - 1) / (kStep * kWarps)) + kItem;
      int in_row = static_cast<int>(static_cast<float>(start_units) / static_cast<float>(units));
      if (static_cast<int64_t>(in_row) * units > start_units) --in_row;  // a float quotient of up to 2^20 items is at most 1 off
      if (static_cast<int64_t>(in_row + 1) * units <= start_units) ++in_row;
      block = static_cast<int>(start_units - static_cast<int64_t>(in_row) * units) - kItem;
      item = start_row * items + in_row;
      end_item = all_items;
      to_load = left + min(block, 0);
      block = max(block, 0);
      if (to_load <= 0) return;
    }
    if (item >= end_item) return;
  }
  const int sub = warp & (crew - 1), block_len = kStep * crew;

  // ---- loading side: the pages of a step's positions (of 8 at a time, or of each lane's) are known one step ahead
  int row = item / items, n, blocks, env;
  int kv = ONE ? item - row * items : (item - row * items) / tiles, tile = ONE ? 0 : item - row * items - kv * tiles, segments = 0;
  int next_page = -1;
  const uint32_t ring = smem_u32(sm) + warp * kStages * R::kStage;
  constexpr int kChunks = HD / 8, kRows = 32 / kChunks;   // 16-byte pieces of a position, positions per instruction
  constexpr int kGroupLanes = 32 / (kStep / 8);           // lanes that look up the page of the same 8 positions
  const int chunk = lane % kChunks, my_row = lane / kChunks;
  const int my_key = sub * kStep + (ALIGNED ? lane / kGroupLanes * 8 : lane);
  bool fresh_row = true, fresh_item = true;
  // goes over to the next step's item and page
  auto look_up = [&]() {
    if (fresh_row) {
      n = length_of(row, env);
      blocks = max(1, (n + block_len - 1) / block_len);
    }
    if (fresh_item) {
      const bool more = item < end_item && to_load > 0;
      if (lane == 0) queue[warp][segments & 3] = Segment{row, kv, tile, more ? static_cast<int>(min(static_cast<int64_t>(blocks - block), to_load)) : 0, block, blocks};
      ++segments;
      // its queries on their way into L1, a line a lane: read two steps from now, 1 us from L2 or memory
      constexpr int kLine = 128 / (PAIR ? 4 : 2), kLines = HD / kLine;
      const int h = tile * kHeads + lane / kLines;
      if (more && sub == 0 && lane < kHeads * kLines && h < group) {
        const int64_t at = row * a.ldq + static_cast<int64_t>(kv * group + h) * HD + lane % kLines * kLine;
        uint32_t unused;
        asm volatile("ld.global.b32 %0, [%1];" : "=r"(unused) : "l"(static_cast<const char*>(a.q) + at * (PAIR ? 4 : 2)));
      }
    }
    next_page = -1;
    const int key = block * block_len + my_key;
    if (item < end_item && to_load > 0 && (ALIGNED || lane < kStep) && key < n) {
      const int col = PAGES == kShifted ? key >> page_shift : key / a.kv.page_size;
      next_page = a.table[static_cast<int64_t>(env) * a.max_pages + col];
      if (static_cast<unsigned>(next_page) >= static_cast<unsigned>(a.kv.n_pages)) {
        raise_status(a.status, VLA_STATUS_PAGES);
        next_page = -1;
      }
    }
  };
  auto issue = [&](int stage) {
    const int key = block * block_len + my_key;
    const int slot = PAGES == kShifted ? key & ((1 << page_shift) - 1) : key % a.kv.page_size;
    int64_t off = next_page * a.kv.page_stride + slot * a.kv.slot_stride + kv * a.kv.head_stride;
    const uint32_t dst0 = ring + stage * R::kStage + my_row * R::kRow;
    const uint16_t *const k0 = static_cast<const uint16_t*>(a.kv.k), *const v0 = static_cast<const uint16_t*>(a.kv.v);
    uint32_t mask;
    if constexpr (ALIGNED) {
      const int some = next_page >= 0 ? min(8, n - key) : 0;  // of the 8 positions of this lane's page
      mask = __reduce_or_sync(0xffffffffu, ((1u << some) - 1u) << (lane / kGroupLanes * 8));
    } else {
      mask = __ballot_sync(0xffffffffu, next_page >= 0);
    }
    if (mask) {
      const int64_t pitch = kRows * a.kv.slot_stride, mine = chunk * 8 + my_row * a.kv.slot_stride;
      int64_t from = 0;
#pragma unroll
      for (int i = 0; i < kStep / kRows; ++i) {
        const int r = i * kRows + my_row;
        if constexpr (ALIGNED)
          from = i * kRows % 8 == 0 ? __shfl_sync(0xffffffffu, off, i * kRows / 8 * kGroupLanes) + mine : from + pitch;
        else
          from = __shfl_sync(0xffffffffu, off, r) + chunk * 8;
        // a position past the last is not read: zeros, from an address that is not used
        const bool ok = (mask >> r) & 1u;
        const uint32_t dst = dst0 + i * kRows * R::kRow + ((chunk ^ (r & 7)) << 4);
        cp16(dst, ok ? k0 + from : k0, ok ? 16u : 0u);
        cp16(dst + R::kPlane, ok ? v0 + from : v0, ok ? 16u : 0u);
      }
    }
    if (lane == 0) seen[warp][stage] = mask;
    asm volatile("cp.async.commit_group;" ::: "memory");
    fresh_row = fresh_item = false;
    if (item < end_item && to_load > 0) {
      --to_load;
      if (++block == blocks) {
        block = 0;
        ++item;
        to_load -= kItem;
        fresh_item = true;
        if (ONE || ++tile == tiles) {
          tile = 0;
          if (++kv == a.kv.n_heads) {
            kv = 0;
            ++row;
            fresh_row = item < end_item;
          }
        }
      } else if (to_load == 0) {
        fresh_item = true;
      }
    }
    look_up();
  };
  look_up();
#pragma unroll 1
  for (int i = 0; i < kStages - 1; ++i) issue(i);

  // ---- computing side
  const int g = lane >> 2, t = lane & 3;
  float to_log2 = a.scale * 1.44269504f;  // of this lane's query head
  const int tile_heads = ONE ? 1 : min(group, kHeads), buffers = ONE || tile_heads <= 2 ? 4 : tile_heads <= 4 ? 2 : 1;
  uint32_t q[HD / 16][PAIR ? 4 : 2];
  // outputs: c0, c1 of the query head, c2, c3 of the weights' low parts; PAIR: both, added after each step
  constexpr int kOut = PAIR ? 2 : 4;
  float o[HD / 8][kOut], m = -INFINITY, l = 0.f;
  Segment seg{};
  int head0 = 0, heads = 0, turn = -1, left = 0, stage = 0;
  float *crew_o = nullptr, *my_o = nullptr;
  float2* crew_ml = nullptr;
  while (true) {
    __syncwarp();
    if (left == 0) {  // the next item
      ++turn;
      seg = queue[warp][turn & 3];
      left = seg.steps;
      if (left == 0) break;
      const int buffer = turn & (buffers - 1);
      // the crew's and this warp's part of the join's memory
      crew_o = crew == 1 ? join_all + warp * (kHeads * HD) : join_all + buffer * (kJoinFloats / buffers);
      crew_ml = crew == 1 ? join_ml + warp * kHeads : join_ml + buffer * (kWarps * kHeads / buffers);
      my_o = crew_o + sub * tile_heads * HD;
      head0 = ONE ? seg.kv : seg.kv * group + seg.tile * kHeads;
      heads = ONE ? 1 : min(kHeads, group - seg.tile * kHeads);
      if constexpr (PAIR) {
        // four channels a lane, split and laid out in this warp's part as each lane's operands (high and low words of
        // two pairs of channels): idle lanes would repeat the split otherwise
        uint32_t* mine = reinterpret_cast<uint32_t*>(my_o);
        constexpr int kLanes = HD / 4;
        const int c = lane % kLanes * 4;
        constexpr int kApart = 32 / kLanes, kMine = ONE ? 1 : kHeads / kApart;  // this lane's heads, whose loads wait together
        const int h0 = lane / kLanes;
        const float* from = static_cast<const float*>(a.q) + seg.row * a.ldq + static_cast<int64_t>(head0 + h0) * HD + c;
        float4 x[kMine];
#pragma unroll
        for (int i = 0; i < kMine; ++i)
          if (h0 + i * kApart < heads) x[i] = *reinterpret_cast<const float4*>(from + i * kApart * HD);
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
          if (i * kApart >= heads) break;
          // exponents of the largest channel from 2^-112 on (below, the two powers of two would leave fp32)
          uint32_t most = 0;
          if (h0 + i * kApart < heads) {
            const float near = fmaxf(fmaxf(fabsf(x[i].x), fabsf(x[i].y)), fmaxf(fabsf(x[i].z), fabsf(x[i].w)));
            most = __float_as_uint(near);
          }
          const uint32_t first = __reduce_max_sync(0xffffffffu, h0 == 0 ? most : 0u);
          if constexpr (kApart == 2) {
            const uint32_t second = __reduce_max_sync(0xffffffffu, h0 == 0 ? 0u : most);
            most = h0 == 0 ? first : second;
          } else {
            most = first;
          }
          if (h0 + i * kApart >= heads) continue;
          const uint32_t exponent = min(max(most >> 23, 15u), 254u);
          const float up = __uint_as_float((268u - exponent) << 23);
          if (c == 0) crew_ml[sub * tile_heads + h0 + i * kApart].x = __uint_as_float((exponent - 14u) << 23);
          uint2 u, v;
          split2<false>(x[i].x * up, x[i].y * up, u.x, u.y);
          split2<false>(x[i].z * up, x[i].w * up, v.x, v.y);
          // channels 16k + 8 half + 2t: lane t, words 2 half of the k-th step
          uint32_t* dst = mine + (h0 + i * kApart) * HD + c / 16 * 16 + c % 8 * 2 + (c & 8) / 4;
          *reinterpret_cast<uint2*>(dst) = u;
          *reinterpret_cast<uint2*>(dst + 4) = v;
        }
        __syncwarp();
        if (g < heads) to_log2 = crew_ml[sub * tile_heads + g].x * a.scale * 1.44269504f;
#pragma unroll
        for (int k = 0; k < HD / 16; ++k) {
          uint4 x = make_uint4(0u, 0u, 0u, 0u);
          if (g < heads) x = *reinterpret_cast<const uint4*>(mine + g * HD + k * 16 + t * 4);
          q[k][0] = x.x;
          q[k][1] = x.y;
          q[k][2] = x.z;
          q[k][3] = x.w;
        }
      } else {
        const int64_t q_at = seg.row * a.ldq + static_cast<int64_t>(head0 + g) * HD + 2 * t;
#pragma unroll
        for (int k = 0; k < HD / 16; ++k) {
          q[k][0] = q[k][1] = 0u;
          if (g < heads) {
            q[k][0] = *reinterpret_cast<const uint32_t*>(static_cast<const uint16_t*>(a.q) + q_at + 16 * k);
            q[k][1] = *reinterpret_cast<const uint32_t*>(static_cast<const uint16_t*>(a.q) + q_at + 16 * k + 8);
          }
        }
      }
#pragma unroll
      for (int i = 0; i < HD / 8; ++i)
#pragma unroll
        for (int e = 0; e < kOut; ++e) o[i][e] = 0.f;
      m = -INFINITY;
      l = 0.f;
    }

    asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
    __syncwarp();  // the stage has arrived, and the one before has been read by all lanes
    issue(stage == 0 ? kStages - 1 : stage - 1);
    const uint32_t mask = seen[warp][stage];
    const uint32_t keys = ring + stage * R::kStage, values = keys + R::kPlane;
    stage = stage + 1 == kStages ? 0 : stage + 1;
    if (mask) {
      constexpr int kTiles = kStep / 8;  // of 8 positions
      // The tensor cores truncate what they add to an accumulator; fp32 outputs keep more of their bits with two
      // chains for the scores and a fresh accumulator a step for the outputs, added in fp32.
      constexpr int kChains = PAIR ? 2 : 1;
      float s[kChains][kTiles][4] = {};
      {
        // piece 2k + b of row r lies at (2k + b) ^ (r & 7): the k-th step flips bits of one address
        const int r = (lane & 7) + ((lane >> 4) << 3);
        const uint32_t at = (keys + r * R::kRow) | ((((lane >> 3) & 1) ^ (r & 7)) << 4);
#pragma unroll
        for (int k = 0; k < HD / 16; ++k) {
#pragma unroll
          for (int i = 0; i < kTiles; i += 2) {
            uint32_t b[4];
            ldsm(b, (at ^ (k << 5)) + i * 8 * R::kRow);
            if constexpr (PAIR) {
              mma<BF16>(s[k & 1][i], q[k][0], q[k][1], q[k][2], q[k][3], b[0], b[1]);
              mma<BF16>(s[k & 1][i + 1], q[k][0], q[k][1], q[k][2], q[k][3], b[2], b[3]);
            } else {
              mma<BF16>(s[0][i], q[k][0], 0u, q[k][1], 0u, b[0], b[1]);
              mma<BF16>(s[0][i + 1], q[k][0], 0u, q[k][1], 0u, b[2], b[3]);
            }
          }
        }
      }
      float p[2 * kTiles], top = -INFINITY;
      const uint32_t mine = mask >> (2 * t);
#pragma unroll
      for (int i = 0; i < 2 * kTiles; ++i) {
        float x = s[0][i >> 1][i & 1];
        if constexpr (PAIR) x = (x + s[1][i >> 1][i & 1]) + (s[0][i >> 1][2 + (i & 1)] + s[1][i >> 1][2 + (i & 1)]);
        p[i] = (mine >> ((i >> 1) * 8 + (i & 1))) & 1u ? x * to_log2 : -INFINITY;
        top = fmaxf(top, p[i]);
      }
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(m, fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2)));
      if (__any_sync(0xffffffffu, top > m)) {
        const float keep = join_weight(m, top);
        l *= keep;
#pragma unroll
        for (int i = 0; i < HD / 8; ++i)
#pragma unroll
          for (int e = 0; e < kOut; ++e) o[i][e] *= keep;
        m = top;
      }
      const float base = (m == -INFINITY ? 0.f : m) - kShift;
#pragma unroll
      for (int i = 0; i < 2 * kTiles; ++i) {
        p[i] = exp2_approx(p[i] - base);
        l += p[i];
      }
      {
        const int r = (lane & 7) + (((lane >> 3) & 1) << 3);
        const uint32_t at = (values + r * R::kRow) | (((lane >> 4) ^ (r & 7)) << 4);
        uint32_t w[2 * kTiles];  // the weights as operands: high and low words
#pragma unroll
        for (int i = 0; i < kTiles; ++i) split2<BF16>(p[2 * i], p[2 * i + 1], w[2 * i], w[2 * i + 1]);
#pragma unroll
        for (int j = 0; j < HD / 16; ++j) {
          float c[2][4] = {};
#pragma unroll
          for (int i = 0; i < kTiles; i += 2) {
            uint32_t b[4];
            ldsm_t(b, (at ^ (j << 5)) + i * 8 * R::kRow);
            if constexpr (PAIR) {
              mma<BF16>(c[0], w[2 * i], w[2 * i + 1], w[2 * i + 2], w[2 * i + 3], b[0], b[1]);
              mma<BF16>(c[1], w[2 * i], w[2 * i + 1], w[2 * i + 2], w[2 * i + 3], b[2], b[3]);
            } else {
              mma<BF16>(o[2 * j], w[2 * i], w[2 * i + 1], w[2 * i + 2], w[2 * i + 3], b[0], b[1]);
              mma<BF16>(o[2 * j + 1], w[2 * i], w[2 * i + 1], w[2 * i + 2], w[2 * i + 3], b[2], b[3]);
            }
          }
          if constexpr (PAIR) {
#pragma unroll
            for (int e = 0; e < 4; ++e) o[2 * j + (e >> 1)][e & 1] += c[e >> 1][e & 1] + c[e >> 1][2 + (e & 1)];
          }
        }
      }
    }
    if (--left > 0) continue;

    // ---- the item's end: the crew's results meet
    l += __shfl_xor_sync(0xffffffffu, l, 1);
    l += __shfl_xor_sync(0xffffffffu, l, 2);
    if (g < heads) {
      if (t == 0) crew_ml[sub * tile_heads + g] = make_float2(m, l);
      float* dst = my_o + g * HD + 2 * t;
#pragma unroll
      for (int i = 0; i < HD / 8; ++i)
        *reinterpret_cast<float2*>(dst + 8 * i) = PAIR ? make_float2(o[i][0], o[i][1]) : make_float2(o[i][0] + o[i][kOut - 2], o[i][1] + o[i][kOut - 1]);
    }
    int h0 = 0, h_step = 1;  // this warp joins heads h0, h0 + h_step, ..
    if (crew == 1) {
      __syncwarp();
    } else if (buffers == 4) {
      const bool joins = warp == (turn & 3);
      if (joins)
        asm volatile("bar.sync %0, %1;" ::"r"(1 + (turn & 3)), "n"(32 * kWarps) : "memory");
      else
        asm volatile("bar.arrive %0, %1;" ::"r"(1 + (turn & 3)), "n"(32 * kWarps) : "memory");
      h0 = joins ? 0 : heads;
    } else {
      __syncthreads();
      h0 = warp;
      h_step = kWarps;
    }
    const int at = lane * Some::kN;  // this lane's channels of a head
    // two heads at a time, so that they wait for memory together
#pragma unroll 1
    for (; h0 < heads; h0 += 2 * h_step) {
      const bool both = !ONE && h0 + h_step < heads;
      float top[2], sum[2];
      Some val[2];
#pragma unroll
      for (int i = 0; i < (ONE ? 1 : 2); ++i) {
        const int h = i == 0 || both ? h0 + i * h_step : h0;
        float2 x[kWarps];
#pragma unroll
        for (int w = 0; w < kWarps; ++w) x[w] = w < crew ? crew_ml[w * tile_heads + h] : make_float2(-INFINITY, 0.f);
        top[i] = fmaxf(fmaxf(x[0].x, x[1].x), fmaxf(x[2].x, x[3].x));
        sum[i] = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          if (w >= crew) break;
          const float f = join_weight(x[w].x, top[i]);
          sum[i] = fmaf(f, x[w].y, sum[i]);
          val[i].add(f, Some::load(crew_o + (w * tile_heads + h) * HD + at));
        }
      }
      if (seg.from > 0 || seg.from + seg.steps < seg.blocks) {
        // CTAs c0 .. c1 have parts of the item; share s begins at unit s * share, so the distances from here tell
        float* const slots = reinterpret_cast<float*>(static_cast<uint8_t*>(a.workspace) + kTicketBytes);
        const int me = static_cast<int>(blockIdx.x), s32 = static_cast<int>(min(share, static_cast<int64_t>(0x7fffffff)));
        // blocks of the item before this share, and from this share's start to the item's last
        const int c0 = seg.from > 0 ? me - (seg.from - 1) / s32 - 1 : me;
        const int to_last = seg.from > 0 ? seg.blocks - 1 - seg.from : s32 - seg.steps + seg.blocks - 1;
        const int c1 = me + to_last / s32, parts = c1 - c0 + 1;
        // up to 32 parts are joined at once; more in groups, each group's result in its first member's slot, then the groups
        bool first_level = parts > kJoin, mine_last = true;
        int slot_cta = me;
        while (true) {
          const int step = first_level ? 1 : parts > kJoin ? kJoin : 1;
          const int lo = first_level ? c0 + (me - c0) / kJoin * kJoin : c0;
          const int count = first_level ? min(kJoin, c1 + 1 - lo) : (parts + step - 1) / step;
          auto slot_of = [&](int c) { return slots + static_cast<size_t>(2 * c + (c == c0 ? 1 : 0)) * slot_floats(HD); };
          float* const slot = slot_of(slot_cta);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            if (i == 1 && !both) break;
            val[i].store(slot + (h0 + i * h_step) * HD + at);
            if (lane == 0) reinterpret_cast<float2*>(slot + kHeads * HD)[h0 + i * h_step] = make_float2(top[i], sum[i]);
          }
          __syncwarp();  // it and the release order all lanes' parts before the ticket
          int there = 0;
          if (lane == 0) {
            int* ticket = static_cast<int*>(a.workspace) + ((!first_level && parts > kJoin ? kSlots : 0) + 2 * lo + (lo == c0 ? 1 : 0)) * kHeads + h0;
            there = add_acq_rel(ticket, 1);
            if (there == count - 1) *ticket = 0;
          }
          mine_last = __shfl_sync(0xffffffffu, there, 0) == count - 1;
          if (!mine_last) break;
          __syncwarp();
          float f[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            float2 y = make_float2(-INFINITY, 0.f);
            if (lane < count) y = __ldcg(reinterpret_cast<const float2*>(slot_of(lo + lane * step) + kHeads * HD) + (i == 0 || both ? h0 + i * h_step : h0));
            top[i] = warp_max(y.x);
            f[i] = join_weight(y.x, top[i]);
            sum[i] = warp_sum(f[i] * y.y);
            val[i] = Some();
          }
#pragma unroll 4
          for (int j = 0; j < count; ++j) {
            const float* part = slot_of(lo + j * step) + h0 * HD + at;
            const Some x = Some::load_l2(part), y = Some::load_l2(part + (both ? h_step * HD : 0));
            val[0].add(__shfl_sync(0xffffffffu, f[0], j), x);
            val[1].add(__shfl_sync(0xffffffffu, f[1], j), y);
          }
          if (!first_level) break;
          first_level = false;
          slot_cta = lo;
        }
        if (!mine_last) continue;
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (i == 1 && !both) break;
        const int h = head0 + h0 + i * h_step;
        const float inv = sum[i] > 0.f ? 1.f / sum[i] : sum[i] == sum[i] ? 0.f : sum[i];
        val[i].write(a.out, seg.row * a.ldo + static_cast<int64_t>(h) * HD + at, inv, a.dtype);
        if (a.lse && lane == 0) a.lse[static_cast<int64_t>(seg.row) * a.n_q_heads + h] = (top[i] + log2f(sum[i]) - kShift) * 0.693147181f;
      }
    }
    if (crew != 1 && buffers == 1) __syncthreads();
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
}

}  // namespace

size_t paged_attn_workspace(int hd) { return kTicketBytes + static_cast<size_t>(kSlots) * slot_floats(hd) * sizeof(float); }

int paged_attn_launch(const PagedAttnArgs& a, cudaStream_t s) {
  int dev = 0, sms = 0;
  VLA_CUDA_TRY(cudaGetDevice(&dev));
  VLA_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  const int group = a.n_q_heads / a.kv.n_heads, tiles = (group + kHeads - 1) / kHeads;
  const int ps = a.kv.page_size, shift = __builtin_ctz(ps);
  const bool pair = a.dtype == VLA_F32, bf = a.kv.dtype == VLA_BF16, eights = ps % 8 == 0, shifted = eights && !(ps & (ps - 1));
  auto go = [&](auto ring, auto kern, std::atomic<uint64_t>& done) -> int {
    using R = decltype(ring);
    // no more CTAs than have a step to take at the longest rows that the table holds
    const int64_t most = static_cast<int64_t>(a.rows) * a.kv.n_heads * tiles * ((static_cast<int64_t>(a.max_pages) * ps + R::kStep - 1) / R::kStep);
    const int grid = static_cast<int>(std::min<int64_t>(std::min(R::kCtasPerSm * sms, kMaxCtas), most));
    const int smem = 128 + R::kBytes + kWarps * kHeads * a.kv.head_dim * static_cast<int>(sizeof(float));
    VLA_CUDA_TRY(set_smem_limit(kern, smem, done));
    VLA_CUDA_TRY(launch_pdl(kern, dim3(grid), dim3(32 * kWarps), smem, s, a, shift, tiles));
    note_launch();
    VLA_CUDA_TRY(cudaGetLastError());
    return VLA_OK;
  };
  static std::atomic<uint64_t> done[24] = {};
#define VLA_PAGED(HD, BF, PAIR, I)                                                                             \
  (shifted && group == 1 ? go(Ring<HD>(), paged_attn_kernel<HD, BF, PAIR, kShifted, true>, done[4 * (I)])      \
   : shifted             ? go(Ring<HD>(), paged_attn_kernel<HD, BF, PAIR, kShifted, false>, done[4 * (I) + 1]) \
   : eights              ? go(Ring<HD>(), paged_attn_kernel<HD, BF, PAIR, kEights, false>, done[4 * (I) + 2])  \
                         : go(Ring<HD>(), paged_attn_kernel<HD, BF, PAIR, kAnyPage, false>, done[4 * (I) + 3]))
  if (a.kv.head_dim == 128) return bf ? VLA_PAGED(128, true, false, 0) : pair ? VLA_PAGED(128, false, true, 1) : VLA_PAGED(128, false, false, 2);
  return bf ? VLA_PAGED(64, true, false, 3) : pair ? VLA_PAGED(64, false, true, 4) : VLA_PAGED(64, false, false, 5);
#undef VLA_PAGED
}

}  // namespace vla
