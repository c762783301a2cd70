// How a row of any alignment comes to shared memory by a bulk copy, whose addresses and size are multiples of 16 bytes, without a read outside
// its tensor: the copy takes the bytes around the row up to the next multiple where the tensor has them, else single elements come beside it.
#pragma once
#include <stdint.h>

#ifdef __CUDACC__
#define VLA_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define VLA_HOST_DEVICE inline
#endif

namespace vla {

struct RowCopy {
  uintptr_t from;       // of the bulk copy
  uint32_t bytes;       // of it (may be 0)
  uint32_t head, tail;  // bytes at the row's begin and end that come by themselves, below 16
};
// The row of n bytes at p of a tensor that lies from lo up to hi (its last row's end).
VLA_HOST_DEVICE RowCopy row_copy(uintptr_t p, uint32_t n, uintptr_t lo, uintptr_t hi) {
  constexpr uintptr_t kMask = ~static_cast<uintptr_t>(15);
  const uintptr_t end = p + n, down = p & kMask, up = (p + 15) & kMask, end_down = end & kMask, end_up = (end + 15) & kMask;
  const bool head = down < lo, tail = end_up > hi;
  const uintptr_t from = head ? up : down, to = tail ? end_down : end_up;
  const uintptr_t head_end = head ? (up < end ? up : end) : p;
  const uintptr_t tail_begin = tail ? (end_down > head_end ? end_down : head_end) : end;
  return RowCopy{from, to > from ? static_cast<uint32_t>(to - from) : 0u, static_cast<uint32_t>(head_end - p),
                 static_cast<uint32_t>(end - tail_begin)};
}

}  // namespace vla
