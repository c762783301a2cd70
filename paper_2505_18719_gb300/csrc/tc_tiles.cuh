// Tiles of 128 rows for the tensor cores: descriptors, MMAs with an operand in tensor memory, wide tensor-memory accesses, and
// the tiles' layout in shared memory.
//
// A tile of `rows` x HD 16-bit elements lies as HD / 64 column blocks one behind the other, each `rows` rows of 128 bytes, 16-byte
// pieces XOR-ed with the row modulo 8 (what a TMA load with 128-byte swizzle writes).  The same tile serves as a K-major operand (rows
// x channels, summed over channels) and as an MN-major one (channels x rows, summed over rows).
#pragma once
#include "ptx.cuh"

namespace vla {

constexpr int kTile = 128;
constexpr uint32_t kBlockBytes = kTile * 128;  // a column block of a tile

// Low word of a tile's descriptor (the address, column blocks block_bytes apart); the high word is the same for all: groups of 8 rows
// 1024 bytes apart, version 1, 128-byte swizzle.
constexpr uint32_t kDescHigh = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t tile_desc(uint32_t saddr, uint32_t block_bytes = kBlockBytes) {
  return ((saddr & 0x3FFFFu) >> 4) | ((block_bytes >> 4) << 16);
}
// Offsets (in descriptor units of 16 bytes) of the k-th 16 elements along the sum: channels of a K-major operand, rows of an MN-major one.
__device__ __forceinline__ constexpr uint32_t k_major_step(int k, uint32_t block_bytes = kBlockBytes) {
  return (static_cast<uint32_t>(k >> 2) * block_bytes + (k & 3) * 32) >> 4;
}
__device__ __forceinline__ constexpr uint32_t mn_major_step(int k) { return static_cast<uint32_t>(k) * (2048 >> 4); }

// kind::f16, f32 sums, M = 128, N; A K-major (or in tensor memory), B K-major or MN-major.
__device__ __forceinline__ uint32_t tile_idesc(int N, bool fp16, bool b_mn_major) {
  return (1u << 4) | (fp16 ? 0u : (1u << 7) | (1u << 10)) | (b_mn_major ? 1u << 16 : 0u) | (static_cast<uint32_t>(N >> 3) << 17) |
         (static_cast<uint32_t>(kTile >> 4) << 24);
}
// D (tensor memory) (+)= A B, both in shared memory, or A in tensor memory.
__device__ __forceinline__ void tile_mma(uint32_t d_tmem, uint32_t a_desc, uint32_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "mov.b64 a, {%1, %5};\n\tmov.b64 b, {%2, %5};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n\t}" ::"r"(d_tmem),
      "r"(a_desc), "r"(b_desc), "r"(idesc), "r"(accumulate), "n"(kDescHigh)
      : "memory");
}
__device__ __forceinline__ void tile_mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint32_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 b;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "mov.b64 b, {%2, %5};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n\t}" ::"r"(d_tmem),
      "r"(a_tmem), "r"(b_desc), "r"(idesc), "r"(accumulate), "n"(kDescHigh)
      : "memory");
}

// The warp that issues MMAs runs as a whole, with its state in uniform registers (what the MMA takes its operands from; from one thread's
// registers each operand costs a move and its latency, 70 cycles an MMA), and one thread of it, always the same, issues.
__device__ __forceinline__ bool elected() {
  uint32_t p;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
  return p != 0;
}
__device__ __forceinline__ int uniform(int v) { return __reduce_max_sync(0xffffffffu, v); }
// All of an SM's tensor memory, by one warp; `slot` (shared memory) gets its address.
constexpr uint32_t kTmemAll = 512;
__device__ __forceinline__ void tmem_take(uint32_t slot) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(kTmemAll) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_give(uint32_t tmem) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemAll) : "memory");
}

// 32 consecutive columns of this thread's lane.
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
        "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
        "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr));
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, "
      "%13, %14, %15, %16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
      "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, uint32_t* r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr));
}
__device__ __forceinline__ void tmem_st4(uint32_t taddr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1, %2, %3, %4};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3])
               : "memory");
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(r[0]), "r"(r[1]),
               "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
// N columns (a multiple of 8) from tensor memory; N / 2 to it.
template <int N>
__device__ __forceinline__ void tmem_load(uint32_t taddr, uint32_t* r) {
#pragma unroll
  for (int i = 0; i + 32 <= N; i += 32) tmem_ld32(taddr + i, r + i);
#pragma unroll
  for (int i = N / 32 * 32; i < N; i += 8) tmem_ld8(taddr + i, r + i);
}
template <int N>
__device__ __forceinline__ void tmem_store(uint32_t taddr, const uint32_t* r) {
#pragma unroll
  for (int i = 0; i + 16 <= N; i += 16) tmem_st16(taddr + i, r + i);
#pragma unroll
  for (int i = N / 16 * 16; i < N; i += 4) tmem_st4(taddr + i, r + i);
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// Earlier kernels' ordinary stores before this thread's TMA and bulk loads of them (a kernel that starts beside another has no launch between).
__device__ __forceinline__ void fence_async_global() { asm volatile("fence.proxy.async.global;" ::: "memory"); }
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// 2^x (2^-inf = 0; results below the smallest normal number are 0)
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t y;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(y) : "l"(a), "l"(b));
  return y;
}
template <bool FP16>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  return FP16 ? pack_f16x2(a, b) : pack_bf16x2(a, b);
}

// Bounded wait of a whole warp: all lanes ask at once.  (Asked by one lane with the others waiting for it, the answer comes 600 cycles later.)  The
// clock, which takes longer to read than the wait lasts as a rule, comes in after 1024 tries.  abort_flag[0]: a wait of the CTA has given up;
// abort_flag[1]: grows while a warp is at something that may take longer than the limit (attend_row, whose loop ends by itself), which
// begins anew each time.
__device__ __forceinline__ bool warp_waits(uint32_t bar, uint32_t parity, volatile int* abort_flag, uint32_t* status, uint64_t limit) {
  uint64_t t0 = 0;
  int work = 0;
  for (uint32_t n = 1; !__all_sync(0xffffffffu, mbar_try_wait(bar, parity)); ++n) {
    if (n & 1023u) continue;
    if (const int now = uniform(abort_flag[1]); n == 1024 || now != work) {
      t0 = globaltimer();
      work = now;
    }
    const bool late = globaltimer() - t0 > limit, given_up = *abort_flag != 0;
    if (__any_sync(0xffffffffu, late) && (threadIdx.x & 31) == 0) {
      *abort_flag = 1;
      if (status) atomicOr(status, VLA_STATUS_TIMEOUT);
    }
    if (__any_sync(0xffffffffu, late || given_up)) return false;
  }
  return true;
}

// Rows `from` .. `to` - 1 of a tile in shared memory become zeros (one warp).
template <int HD>
__device__ __forceinline__ void zero_tile_rows(uint8_t* tile, int from, int to, uint32_t block_bytes = kBlockBytes) {
  for (int i = threadIdx.x & 31; i < (to - from) * (HD / 8); i += 32) {
    const int row = from + i / (HD / 8), c = i % (HD / 8);
    *reinterpret_cast<uint4*>(tile + (c >> 3) * block_bytes + row * 128 + (c & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
  }
}

}  // namespace vla
