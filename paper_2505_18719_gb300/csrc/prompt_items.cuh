// The work of a persistent kernel over packed sequences, found on the device from the sequences' starts.
#pragma once
#include "prompt_rows.cuh"
#include "tc_tiles.cuh"

namespace vla {

constexpr int kItems = 8;  // descriptors in flight between the warp that finds them and those that work on them

struct Item {
  int begin, len;  // a sequence; len < 0: no more items
  int a, b;        // what of it
};

// Items `next`, `next` + step, .. of all sequences in order, `count(len)` of each: put(begin, len, number in the sequence) by a whole warp, which
// reads the lengths of 32 sequences at a time.  Stops at `bound` (more than well-formed starts can give) or when put says no.
template <class Count, class Put>
__device__ __forceinline__ bool find_items(const int* seq_start, int n_seq, int rows, int64_t next, int64_t step, int64_t bound,
                                           const Count& count, const Put& put) {
  const int lane = threadIdx.x & 31;
  int64_t before = 0;  // items of the sequences before these 32
  for (int c0 = 0; c0 < n_seq && next < bound; c0 += 32) {
    Span sp{0, 0};
    if (c0 + lane < n_seq) sp = span_of(seq_start, c0 + lane, rows);
    const int64_t mine = count(sp.end - sp.begin);
    int64_t upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t y = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += y;
    }
    upto += before;
    while (next < bound) {
      const uint32_t past = __ballot_sync(0xffffffffu, next < upto);
      if (!past) break;
      const int src = __ffs(static_cast<int>(past)) - 1;
      const int begin = __shfl_sync(0xffffffffu, sp.begin, src), end = __shfl_sync(0xffffffffu, sp.end, src);
      if (!put(begin, end - begin, static_cast<int>(next - __shfl_sync(0xffffffffu, upto - mine, src)))) return false;
      next += step;
    }
    before = __shfl_sync(0xffffffffu, upto, 31);
  }
  return true;
}

// Rows of no sequence, shared out over the CTAs: zeros in `n` elements from each of them on (one warp).
struct Outside {
  int first, last, rows;
  __device__ __forceinline__ Outside(const int* seq_start, int n_seq, int n) : rows(n) {
    first = min(max(seq_start[0], 0), n);
    last = min(max(seq_start[n_seq], first), n);
  }
  __device__ __forceinline__ int count() const { return first + rows - last; }
  __device__ __forceinline__ int row(int i) const { return i < first ? i : last + i - first; }
};
__device__ __forceinline__ void zero_row(void* row, int n) {
  for (int e = threadIdx.x & 31; e < n / 8; e += 32) static_cast<uint4*>(row)[e] = make_uint4(0u, 0u, 0u, 0u);
}

// CHUNKS x 32 columns of this warp's 32 rows of tensor memory, times `scale`, to rows of `dst` (ld elements apart), of which `live` exist; each
// thread its own row, 32 bytes a store where rows lie for it (`wide`).  (Through shared memory, with lanes side by side in a row, the
// products' operands were in the way: 4000 cycles a tile.)  Whether this thread's row has a NaN or an infinity.
__device__ __forceinline__ bool wide_rows(const void* dst, int64_t ld) { return !((reinterpret_cast<uintptr_t>(dst) & 31) | (ld & 15)); }
template <bool FP16, int CHUNKS>
__device__ __forceinline__ bool store_tile(uint32_t tmem, float scale, void* dst, int64_t ld, int live) {
  const int lane = threadIdx.x & 31;
  const bool wide = wide_rows(dst, ld);
  uint4* row = static_cast<uint4*>(elem(dst, lane * ld));
  float bad = 0.f;
#pragma unroll
  for (int b = 0; b < CHUNKS; ++b) {
    uint32_t v[32], w[16];
    __syncwarp();  // (lanes without a row stored nothing; the load is the whole warp's)
    tmem_ld32(tmem + 32 * b, v);
    tmem_wait_ld();
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float y0 = __uint_as_float(v[2 * i]) * scale, y1 = __uint_as_float(v[2 * i + 1]) * scale;
      bad = fmaf(y0, 0.f, fmaf(y1, 0.f, bad));
      w[i] = pack2<FP16>(y0, y1);
    }
    if (lane < live && wide) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(row + 4 * b + 2 * h), "r"(w[8 * h]), "r"(w[8 * h + 1]),
                     "r"(w[8 * h + 2]), "r"(w[8 * h + 3]), "r"(w[8 * h + 4]), "r"(w[8 * h + 5]), "r"(w[8 * h + 6]), "r"(w[8 * h + 7])
                     : "memory");
    } else if (lane < live) {
#pragma unroll
      for (int h = 0; h < 4; ++h) row[4 * b + h] = make_uint4(w[4 * h], w[4 * h + 1], w[4 * h + 2], w[4 * h + 3]);
    }
  }
  return bad != 0.f;
}

}  // namespace vla
