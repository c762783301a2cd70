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

// `chunks` x 32 columns of this warp's 32 rows of tensor memory, times `scale`, to rows of `dst` (ld elements apart), of which `live` exist:
// through 2 KB of shared memory, 8 rows of 64 bytes a store.  Whether this thread's row has a NaN or an infinity.
template <bool FP16, int CHUNKS>
__device__ __forceinline__ bool store_tile(uint32_t tmem, uint8_t* staging, float scale, void* dst, int64_t ld, int live) {
  const int lane = threadIdx.x & 31;
  float bad = 0.f;
#pragma unroll
  for (int b = 0; b < CHUNKS; ++b) {
    uint32_t v[32];
    tmem_ld32(tmem + 32 * b, v);
    tmem_wait_ld();
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float y0 = __uint_as_float(v[8 * e + 2 * i]) * scale, y1 = __uint_as_float(v[8 * e + 2 * i + 1]) * scale;
        bad = fmaf(y0, 0.f, fmaf(y1, 0.f, bad));
        w[i] = pack2<FP16>(y0, y1);
      }
      *reinterpret_cast<uint4*>(staging + lane * 64 + ((e ^ ((lane >> 1) & 3)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int rr = 8 * i + (lane >> 2), e = lane & 3;
      if (rr < live)
        *reinterpret_cast<uint4*>(elem(dst, rr * ld + b * 32 + e * 8)) =
            *reinterpret_cast<const uint4*>(staging + rr * 64 + ((e ^ ((rr >> 1) & 3)) << 4));
    }
    __syncwarp();
  }
  return bad != 0.f;
}

}  // namespace vla
