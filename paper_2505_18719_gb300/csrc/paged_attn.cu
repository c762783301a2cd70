// Attention of one new token per row over its environment's paged positions.
//
// For a row r, query head h and its key-value head g: s_p = scale q . K_p, out = sum_p 2^(s_p log2 e - m) V_p / l with
// l the sum of the weights, any m that keeps them in range.  Sums over disjoint sets of positions join by
// (m, l, o) = (max m_i, sum 2^(m_i - m) l_i, sum 2^(m_i - m) o_i).
//
// Each cached byte is used once per 8 query heads, so the kernel is bound by HBM (2 hd 2-byte reads for 4 hd
// flops a query head) or, for few short rows, by latency.  The work is the list of (row, key-value head, tile of
// 8 query heads, block of 64 positions), in that order; one CTA per resident place takes an equal share of the
// list, however long or uneven the rows are, found from the rows' lengths on the device.  An item that
// a share's end cuts is joined by the last CTA that arrives at its ticket, from partial results in the workspace.
//
// In a CTA each of the 4 warps takes 16 of the 64 positions, with its own ring of stages filled by
// cp.async (no barrier between warps but at an item's end, where their results join).  The page of a step's
// positions is looked up one step before its copies are issued; 16-byte pieces are XOR-swizzled so that ldmatrix
// reads without bank conflicts.  Scores and outputs run on mma.sync m16n8k16 with the 8 query heads as rows 0-7;
// rows 8-15 hold the low parts, x - fp16(x) (or bf16), of fp32 queries and of the softmax weights, so that
// they keep 22 (16) significant bits at no further instruction.  fp16 weights are 2^15 times the true ones:
// a weight of 1e-5 beside one of 1 keeps its bits.
#include <algorithm>

#include "lm.h"
#include "ptx.cuh"

namespace vla {

namespace {

constexpr int kWarps = 4;
constexpr int kStep = 16;                 // positions of a warp's step
constexpr int kBlock = kStep * kWarps;    // positions of a CTA's step
constexpr int kHeads = 8;                 // query heads of a tile
constexpr int kCtasPerSm = 2;
constexpr int kMaxCtas = 1024;
constexpr int kJoin = 16;                 // partial results that one CTA joins at a time
constexpr int kMinBlocks = 4;             // a share is no smaller while items are longer

// Workspace: tickets of the first level [2 kMaxCtas], of the second [2 kMaxCtas], then the partial results:
// per slot o [8][hd], m [8], l [8].  Two slots a CTA: the item that it found begun, and the one that it leaves.
constexpr size_t kTicketBytes = 4 * kMaxCtas * sizeof(int);
__host__ __device__ constexpr int slot_floats(int hd) { return kHeads * hd + 2 * kHeads; }

template <int HD, int STAGES>
struct Ring {
  static constexpr int kRow = HD * 2;              // bytes of a position's channels
  static constexpr int kPlane = kStep * kRow;      // keys or values of a step
  static constexpr int kStage = 2 * kPlane;
  static constexpr int kBytes = kWarps * STAGES * kStage;
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

__device__ __forceinline__ int load_acquire(const int* p) {
  int v;
  asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ int add_acq_rel(int* p, int n) {
  int v;
  asm volatile("atom.acq_rel.gpu.global.add.s32 %0, [%1], %2;" : "=r"(v) : "l"(p), "r"(n) : "memory");
  return v;
}

// Where a CTA is in the list of work.
struct Cursor {
  int row, kv, tile, block;  // an item is (row, key-value head, tile); block within the item
  int n, blocks, env;        // the row's positions, their blocks (at least 1), its environment
};

// ALIGNED: pages are multiples of 16 positions, so that a step's positions share a page.
template <int HD, bool BF16, bool PAIR, bool ALIGNED, int STAGES>
__global__ void __launch_bounds__(32 * kWarps, kCtasPerSm) paged_attn_kernel(const PagedAttnArgs a, const int page_shift, const int tiles) {
  using R = Ring<HD, STAGES>;
  constexpr float kShift = BF16 ? 0.f : 15.f;
  extern __shared__ __align__(128) uint8_t sm_raw[];
  uint8_t* sm = sm_raw + (-smem_u32(sm_raw) & 255u);  // rows of 256 bytes at multiples of 256
  float* join_o = reinterpret_cast<float*>(sm + R::kBytes);  // [kWarps][kHeads][HD]
  __shared__ float join_m[kWarps][kHeads], join_l[kWarps][kHeads];
  __shared__ uint32_t seen[kWarps][STAGES];
  __shared__ int64_t scan[kWarps];
  __shared__ int start_row;
  __shared__ int64_t start_sum;
  __shared__ int last_here;
  pdl_launch_dependents();
  pdl_wait();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int items = a.kv.n_heads * tiles, group = a.n_q_heads / a.kv.n_heads;

  auto row_of = [&](Cursor& c) {
    const int pos = a.row_pos[c.row];
    c.env = a.row_env[c.row];
    const int col = page_shift >= 0 ? pos >> page_shift : pos / a.kv.page_size;
    const bool ok = pos >= 0 && col < a.max_pages && static_cast<unsigned>(c.env) < static_cast<unsigned>(a.n_env);
    c.n = ok ? pos + 1 : 0;
    c.blocks = ok ? pos / kBlock + 1 : 1;
    return ok || pos == -1;
  };
  auto advance = [&](Cursor& c) {
    if (++c.block < c.blocks) return;
    c.block = 0;
    if (++c.tile < tiles) return;
    c.tile = 0;
    if (++c.kv < a.kv.n_heads) return;
    c.kv = 0;
    if (++c.row < a.rows) row_of(c);
  };

  // ---- this CTA's share: exclusive sums of the rows' blocks, each thread a run of rows
  int64_t total;
  {
    const int run = (a.rows + 32 * kWarps - 1) / (32 * kWarps);
    const int r0 = min(tid * run, a.rows), r1 = min(r0 + run, a.rows);
    int64_t sum = 0;
    Cursor c{};
    for (c.row = r0; c.row < r1; ++c.row) {
      if (!row_of(c) && blockIdx.x == 0) raise_status(a.status, VLA_STATUS_PAGES);
      sum += c.blocks;
    }
    int64_t inc = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t u = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += u;
    }
    if (lane == 31) scan[warp] = inc;
    __syncthreads();
    int64_t before = 0, all = 0;
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) before += scan[w];
      all += scan[w];
    }
    total = all * items;
    const int64_t want = (total + gridDim.x - 1) / gridDim.x, mean = (all + a.rows - 1) / a.rows;
    const int64_t share = max(want, min(static_cast<int64_t>(kMinBlocks), mean));
    const int64_t active = (total + share - 1) / share;
    if (blockIdx.x >= active) return;
    const int64_t first = total * blockIdx.x / active;
    int64_t at = (before + inc - sum) * items;
    if (at <= first && first < at + sum * items) {
      for (c.row = r0; c.row < r1; ++c.row) {
        row_of(c);
        if (first < at + static_cast<int64_t>(c.blocks) * items) break;
        at += static_cast<int64_t>(c.blocks) * items;
      }
      start_row = c.row;
      start_sum = at;
    }
    __syncthreads();
  }
  const int64_t want = (total + gridDim.x - 1) / gridDim.x;
  const int64_t mean = (total / items + a.rows - 1) / a.rows;
  const int64_t share = max(want, min(static_cast<int64_t>(kMinBlocks), mean));
  const int64_t active = (total + share - 1) / share;
  const int64_t first = total * blockIdx.x / active, end = total * (blockIdx.x + 1) / active;
  auto cta_of = [&](int64_t block) { return static_cast<int>(((block + 1) * active - 1) / total); };

  Cursor use{};
  use.row = start_row;
  row_of(use);
  {
    const int64_t in_row = first - start_sum;
    const int item = static_cast<int>(in_row / use.blocks);
    use.block = static_cast<int>(in_row % use.blocks);
    use.kv = item / tiles;
    use.tile = item % tiles;
  }

  // ---- loading: the page of the step's positions (of lane i's position i, where they may differ) is known
  // one step ahead
  Cursor load = use;
  int64_t to_load = end - first;
  int next_page = -1;
  const uint32_t ring = smem_u32(sm) + warp * STAGES * R::kStage;
  constexpr int kChunks = HD / 8, kRows = 32 / kChunks;  // 16-byte pieces of a position, positions per instruction
  const int chunk = lane % kChunks, my_row = lane / kChunks;
  auto look_up = [&]() {
    next_page = -1;
    const int key = load.block * kBlock + warp * kStep + (ALIGNED ? 0 : lane);
    if (to_load > 0 && (ALIGNED || lane < kStep) && key < load.n) {
      const int col = page_shift >= 0 ? key >> page_shift : key / a.kv.page_size;
      next_page = a.table[static_cast<int64_t>(load.env) * a.max_pages + col];
      if (static_cast<unsigned>(next_page) >= static_cast<unsigned>(a.kv.n_pages)) {
        raise_status(a.status, VLA_STATUS_PAGES);
        next_page = -1;
      }
    }
  };
  auto issue = [&](int stage) {
    const int key = load.block * kBlock + warp * kStep + (ALIGNED ? 0 : lane);
    const int slot = page_shift >= 0 ? key & ((1 << page_shift) - 1) : key % a.kv.page_size;
    int64_t off = next_page * a.kv.page_stride + slot * a.kv.slot_stride + load.kv * a.kv.head_stride;
    const uint32_t dst0 = ring + stage * R::kStage + my_row * R::kRow;
    uint32_t mask;
    if constexpr (ALIGNED) {
      const int some = next_page >= 0 ? min(kStep, load.n - key) : 0;
      mask = (1u << some) - 1u;
      if (some > 0) {
        off += chunk * 8 + my_row * a.kv.slot_stride;
        const uint16_t* k = static_cast<const uint16_t*>(a.kv.k) + off;
        const uint16_t* v = static_cast<const uint16_t*>(a.kv.v) + off;
        const int64_t pitch = kRows * a.kv.slot_stride;
#pragma unroll
        for (int i = 0; i < kStep / kRows; ++i) {
          // a position past the last is not read: zeros, from an address that is not used
          const bool ok = i * kRows + my_row < some;
          const uint32_t dst = dst0 + i * kRows * R::kRow + ((chunk ^ ((i * kRows + my_row) & 7)) << 4);
          cp16(dst, ok ? k : static_cast<const uint16_t*>(a.kv.k), ok ? 16u : 0u);
          cp16(dst + R::kPlane, ok ? v : static_cast<const uint16_t*>(a.kv.v), ok ? 16u : 0u);
          k += pitch;
          v += pitch;
        }
      }
    } else {
      mask = __ballot_sync(0xffffffffu, next_page >= 0);
      if (mask) {
#pragma unroll
        for (int i = 0; i < kStep / kRows; ++i) {
          const int r = i * kRows + my_row;
          const int64_t o = __shfl_sync(0xffffffffu, off, r);
          const bool ok = (mask >> r) & 1u;
          const uint32_t dst = dst0 + i * kRows * R::kRow + ((chunk ^ (r & 7)) << 4);
          const int64_t from = ok ? o + chunk * 8 : 0;
          cp16(dst, static_cast<const uint16_t*>(a.kv.k) + from, ok ? 16u : 0u);
          cp16(dst + R::kPlane, static_cast<const uint16_t*>(a.kv.v) + from, ok ? 16u : 0u);
        }
      }
    }
    if (lane == 0) seen[warp][stage] = mask;
    asm volatile("cp.async.commit_group;" ::: "memory");
    if (to_load > 0) {
      --to_load;
      if (to_load > 0) advance(load);
    }
    look_up();
  };
  look_up();
#pragma unroll
  for (int i = 0; i < STAGES - 1; ++i) issue(i);

  // ---- the share, item by item
  const int g = lane >> 2, t = lane & 3;
  const float to_log2 = a.scale * 1.44269504f;
  int stage = 0;
  int64_t done = first;
  while (done < end) {
    const int from = use.block;
    const int steps = static_cast<int>(min(static_cast<int64_t>(use.blocks - from), end - done));
    const int head0 = use.kv * group + use.tile * kHeads;
    const int heads = min(kHeads, group - use.tile * kHeads);
    uint32_t q[HD / 16][PAIR ? 4 : 2];
    {
      if constexpr (PAIR) {
        // four channels a lane, split and laid out in this warp's part of join_o as each lane's operands (high
        // and low words of two pairs of channels): 8 idle rows of lanes would repeat the split otherwise
        uint32_t* mine = reinterpret_cast<uint32_t*>(join_o + warp * kHeads * HD);
        constexpr int kLanes = HD / 4;
        const int c = lane % kLanes * 4;
        uint32_t sat = 0;
        for (int h = lane / kLanes; h < heads; h += 32 / kLanes) {
          const float4 x = *reinterpret_cast<const float4*>(static_cast<const float*>(a.q) + use.row * a.ldq + static_cast<int64_t>(head0 + h) * HD + c);
          uint2 u, v;
          split_pack2_f16(x.x, x.y, u.x, u.y, sat);
          split_pack2_f16(x.z, x.w, v.x, v.y, sat);
          // channels 16k + 8 half + 2t: lane t, words 2 half of the k-th step
          uint32_t* dst = mine + h * HD + c / 16 * 16 + c % 8 * 2 + (c & 8) / 4;
          *reinterpret_cast<uint2*>(dst) = u;
          *reinterpret_cast<uint2*>(dst + 4) = v;
        }
        report_saturation(a.status, sat);
        __syncwarp();
#pragma unroll
        for (int k = 0; k < HD / 16; ++k) {
          uint4 x = make_uint4(0u, 0u, 0u, 0u);
          if (g < heads) x = *reinterpret_cast<const uint4*>(mine + g * HD + k * 16 + t * 4);
          q[k][0] = x.x;
          q[k][1] = x.y;
          q[k][2] = x.z;
          q[k][3] = x.w;
        }
        __syncwarp();
      } else {
        const int64_t q_at = use.row * a.ldq + static_cast<int64_t>(head0 + g) * HD + 2 * t;
#pragma unroll
        for (int k = 0; k < HD / 16; ++k) {
          q[k][0] = q[k][1] = 0u;
          if (g < heads) {
            q[k][0] = *reinterpret_cast<const uint32_t*>(static_cast<const uint16_t*>(a.q) + q_at + 16 * k);
            q[k][1] = *reinterpret_cast<const uint32_t*>(static_cast<const uint16_t*>(a.q) + q_at + 16 * k + 8);
          }
        }
      }
    }
    // the next item's queries on their way into L1 (one line a lane): read at its start, 1 us from L2 or memory
    if (warp == 0 && done + steps < end) {
      constexpr int kLine = 128 / (PAIR ? 4 : 2), kLines = HD / kLine;
      Cursor next = use;
      next.block = use.blocks - 1;
      advance(next);
      const int h = next.tile * kHeads + lane / kLines;
      if (lane < kHeads * kLines && h < group) {
        const int64_t at = next.row * a.ldq + static_cast<int64_t>(next.kv * group + h) * HD + lane % kLines * kLine;
        uint32_t unused;
        asm volatile("ld.global.b32 %0, [%1];" : "=r"(unused) : "l"(static_cast<const char*>(a.q) + at * (PAIR ? 4 : 2)));
      }
    }
    float o[HD / 8][4];
#pragma unroll
    for (int i = 0; i < HD / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
    float m = -INFINITY, l = 0.f;

    for (int step = 0; step < steps; ++step) {
      asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 2) : "memory");
      __syncwarp();
      issue(stage == 0 ? STAGES - 1 : stage - 1);
      const uint32_t mask = seen[warp][stage];
      const uint32_t keys = ring + stage * R::kStage, values = keys + R::kPlane;
      stage = stage + 1 == STAGES ? 0 : stage + 1;
      if (!mask) continue;
      float s[2][4] = {};
      {
        // piece 2k + b of row r lies at (2k + b) ^ (r & 7): the k-th step flips bits of one address
        const int r = (lane & 7) + ((lane >> 4) << 3);
        const uint32_t row = (keys + r * R::kRow) | ((((lane >> 3) & 1) ^ (r & 7)) << 4);
#pragma unroll
        for (int k = 0; k < HD / 16; ++k) {
          uint32_t b[4];
          ldsm(b, row ^ (k << 5));
          if constexpr (PAIR) {
            mma<BF16>(s[0], q[k][0], q[k][1], q[k][2], q[k][3], b[0], b[1]);
            mma<BF16>(s[1], q[k][0], q[k][1], q[k][2], q[k][3], b[2], b[3]);
          } else {
            mma<BF16>(s[0], q[k][0], 0u, q[k][1], 0u, b[0], b[1]);
            mma<BF16>(s[1], q[k][0], 0u, q[k][1], 0u, b[2], b[3]);
          }
        }
      }
      float p[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = PAIR ? s[i >> 1][i & 1] + s[i >> 1][2 + (i & 1)] : s[i >> 1][i & 1];
        p[i] = (mask >> ((i >> 1) * 8 + 2 * t + (i & 1))) & 1u ? x * to_log2 : -INFINITY;
      }
      float top = fmaxf(fmaxf(p[0], p[1]), fmaxf(p[2], p[3]));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(m, fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2)));
      if (__any_sync(0xffffffffu, top > m)) {
        const float keep = join_weight(m, top);
        l *= keep;
#pragma unroll
        for (int i = 0; i < HD / 8; ++i) {
          o[i][0] *= keep;
          o[i][1] *= keep;
          o[i][2] *= keep;
          o[i][3] *= keep;
        }
        m = top;
      }
      const float base = (m == -INFINITY ? 0.f : m) - kShift;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[i] = exp2_approx(p[i] - base);
        l += p[i];
      }
      uint32_t p0, p1, p2, p3;
      split2<BF16>(p[0], p[1], p0, p1);
      split2<BF16>(p[2], p[3], p2, p3);
      {
        const int r = (lane & 7) + (((lane >> 3) & 1) << 3);
        const uint32_t row = (values + r * R::kRow) | (((lane >> 4) ^ (r & 7)) << 4);
#pragma unroll
        for (int j = 0; j < HD / 16; ++j) {
          uint32_t b[4];
          ldsm_t(b, row ^ (j << 5));
          mma<BF16>(o[2 * j], p0, p1, p2, p3, b[0], b[1]);
          mma<BF16>(o[2 * j + 1], p0, p1, p2, p3, b[2], b[3]);
        }
      }
    }

    // ---- the four warps' results, then the parts of other CTAs
    l += __shfl_xor_sync(0xffffffffu, l, 1);
    l += __shfl_xor_sync(0xffffffffu, l, 2);
    if (t == 0) {
      join_m[warp][g] = m;
      join_l[warp][g] = l;
    }
    if (g < heads) {
      float* dst = join_o + (warp * kHeads + g) * HD + 2 * t;
#pragma unroll
      for (int i = 0; i < HD / 8; ++i)
        *reinterpret_cast<float2*>(dst + 8 * i) = make_float2(o[i][0] + o[i][2], o[i][1] + o[i][3]);
    }
    // the item's share of other CTAs: the CTAs c0 .. c1 take part
    int* tickets = static_cast<int*>(a.workspace);
    float* slots = reinterpret_cast<float*>(static_cast<uint8_t*>(a.workspace) + kTicketBytes);
    const int me = static_cast<int>(blockIdx.x);
    int c0 = me, c1 = me;
    if (from > 0) c0 = cta_of(done - from);
    if (from + steps < use.blocks) c1 = cta_of(done - from + use.blocks - 1);
    const int parts = c1 - c0 + 1;
    const bool two = parts > kJoin;  // levels of joins
    auto slot_of = [&](int c) { return slots + static_cast<size_t>(2 * c + (c == c0 ? 1 : 0)) * slot_floats(HD); };
    auto ticket_of = [&](int c) { return tickets + 2 * c + (c == c0 ? 1 : 0); };
    // where all others have already left their parts, this CTA joins them without leaving its own
    if (parts > 1 && !two && tid == 0) last_here = load_acquire(ticket_of(c0)) == parts - 1;
    __syncthreads();
    const bool ready = parts > 1 && !two && last_here;
    constexpr int kAhead = 32 * kWarps / HD;  // heads handled at a time
    const int d = tid % HD;
    auto store = [&](int h, float top, float sum, float val) {
      const float inv = sum > 0.f ? 1.f / sum : sum == sum ? 0.f : sum;
      store_from_float(a.out, use.row * a.ldo + static_cast<int64_t>(head0 + h) * HD + d, val * inv, a.dtype);
      if (a.lse && d == 0)
        a.lse[static_cast<int64_t>(use.row) * a.n_q_heads + head0 + h] = (top + log2f(sum) - kShift) * 0.693147181f;
    };
    // the parts of `count` CTAs lo, lo + step, ..; `mine` >= 0: that one's from the arguments
    auto join = [&](int h, int lo, int step, int count, int mine, float& top, float& sum, float& val) {
      const float m0 = top, l0 = sum, v0 = val;
      for (int i = 0; i < count; ++i)
        if (i != mine) top = fmaxf(top, __ldcg(slot_of(lo + i * step) + kHeads * HD + h));
      sum = val = 0.f;
      for (int i = 0; i < count; ++i) {
        const float* slot = slot_of(lo + i * step);
        const float mi = i == mine ? m0 : __ldcg(slot + kHeads * HD + h), li = i == mine ? l0 : __ldcg(slot + kHeads * HD + kHeads + h);
        const float vi = i == mine ? v0 : __ldcg(slot + h * HD + d), f = join_weight(mi, top);
        sum += f * li;
        val += f * vi;
      }
    };
    auto leave = [&](int c, int h, float top, float sum, float val) {
      float* slot = slot_of(c);
      slot[h * HD + d] = val;
      if (d == 0) {
        slot[kHeads * HD + h] = top;
        slot[kHeads * HD + kHeads + h] = sum;
      }
    };
    for (int h = tid / HD; h < heads; h += kAhead) {
      float top = -INFINITY, sum = 0.f, val = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) top = fmaxf(top, join_m[w][h]);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float f = join_weight(join_m[w][h], top);
        sum += f * join_l[w][h];
        val += f * join_o[(w * kHeads + h) * HD + d];
      }
      if (ready) join(h, c0, 1, parts, me - c0, top, sum, val);
      if (parts == 1 || ready)
        store(h, top, sum, val);
      else
        leave(me, h, top, sum, val);
    }
    if (ready) {
      if (tid == 0) *ticket_of(c0) = 0;
    } else if (parts > 1) {
      // groups of kJoin CTAs first, each group's result in its first member's slot, then the groups
      for (int level = two ? 0 : 1; level < 2; ++level) {
        const int lo = level == 0 ? c0 + (me - c0) / kJoin * kJoin : c0, step = level == 1 && two ? kJoin : 1;
        const int count = level == 0 ? min(kJoin, c1 + 1 - lo) : (parts + step - 1) / step;
        int* ticket = ticket_of(lo) + (level == 1 && two ? 2 * kMaxCtas : 0);
        __syncthreads();
        if (tid == 0) {
          // the barrier and the release order all threads' parts before the ticket
          last_here = add_acq_rel(ticket, 1) == count - 1;
          if (last_here) *ticket = 0;
        }
        __syncthreads();
        if (!last_here) break;
        for (int h = tid / HD; h < heads; h += kAhead) {
          float top = -INFINITY, sum = 0.f, val = 0.f;
          join(h, lo, step, count, -1, top, sum, val);
          if (level == 1) {
            store(h, top, sum, val);
          } else {
            // this head's m and l are read by all its threads above
            asm volatile("bar.sync %0, %1;" ::"r"(1 + tid / HD), "r"(HD) : "memory");
            leave(lo, h, top, sum, val);
          }
        }
      }
    }
    __syncthreads();
    done += steps;
    use.block += steps - 1;
    if (done < end) advance(use);
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
}

}  // namespace

size_t paged_attn_workspace(int hd) { return kTicketBytes + static_cast<size_t>(2 * kMaxCtas) * slot_floats(hd) * sizeof(float); }

int paged_attn_launch(const PagedAttnArgs& a, cudaStream_t s) {
  int dev = 0, sms = 0;
  VLA_CUDA_TRY(cudaGetDevice(&dev));
  VLA_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  const int group = a.n_q_heads / a.kv.n_heads, tiles = (group + kHeads - 1) / kHeads;
  const int ps = a.kv.page_size, shift = (ps & (ps - 1)) ? -1 : __builtin_ctz(ps);
  const int64_t most = static_cast<int64_t>(a.rows) * a.kv.n_heads * tiles * ((static_cast<int64_t>(a.max_pages) * ps + kBlock - 1) / kBlock);
  const int grid = static_cast<int>(std::min<int64_t>(std::min(kCtasPerSm * sms, kMaxCtas), most));
  auto go = [&](auto kern, int ring_bytes, std::atomic<uint64_t>& done) -> int {
    const int smem = 256 + ring_bytes + kWarps * kHeads * a.kv.head_dim * static_cast<int>(sizeof(float));
    VLA_CUDA_TRY(set_smem_limit(kern, smem, done));
    VLA_CUDA_TRY(launch_pdl(kern, dim3(grid), dim3(32 * kWarps), smem, s, a, shift, tiles));
    note_launch();
    VLA_CUDA_TRY(cudaGetLastError());
    return VLA_OK;
  };
  static std::atomic<uint64_t> done[12] = {};
  const bool pair = a.dtype == VLA_F32, bf = a.kv.dtype == VLA_BF16, aligned = ps % kStep == 0;
#define VLA_PAGED(HD, BF, PAIR, ST, I)                                                                \
  (aligned ? go(paged_attn_kernel<HD, BF, PAIR, true, ST>, Ring<HD, ST>::kBytes, done[2 * (I)])       \
           : go(paged_attn_kernel<HD, BF, PAIR, false, ST>, Ring<HD, ST>::kBytes, done[2 * (I) + 1]))
  if (a.kv.head_dim == 128) return bf ? VLA_PAGED(128, true, false, 3, 0) : pair ? VLA_PAGED(128, false, true, 3, 1) : VLA_PAGED(128, false, false, 3, 2);
  return bf ? VLA_PAGED(64, true, false, 4, 3) : pair ? VLA_PAGED(64, false, true, 4, 4) : VLA_PAGED(64, false, false, 4, 5);
#undef VLA_PAGED
}

}  // namespace vla
