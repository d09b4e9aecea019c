// Host interface of the 16-bit products (grouped.hip, adapter.hip,
// orthogonalise.hip).  Arguments were checked by the entry points.
#pragma once

#include "half_tile.hpp"

namespace oz {
namespace half {

struct GroupedRows {
  const void* x;  // rows x depth
  int64_t ldx;
  const void* w;  // a stack of cols x depth (or, transposed, depth x cols)
  int64_t ldw, group_stride;
  const int32_t* ends;
  void* y;  // rows x cols
  int64_t ldy;
  int rows, cols, depth, groups;
  bool vec;  // 16-byte stores of y (set by the launch)
};

struct GroupedWeights {
  const void* dy;  // rows x n
  int64_t lddy;
  const void* x;  // rows x k
  int64_t ldx;
  const int32_t* ends;
  void* dw;  // a stack of n x k
  int64_t lddw, group_stride;
  int rows, n, k, groups;
  bool vec;  // 16-byte stores of a 16-bit dw (set by the launch)
};

// Whether a matrix of `cols` columns can go to LDS by DMA: 16-byte rows, and a
// tile's offsets below 2^31.
inline bool dma_operand(const void* p, int64_t ld, int64_t cols) {
  return (uintptr_t)p % 16 == 0 && ld % 8 == 0 && cols % 8 == 0 && ld < ((int64_t)1 << 21);
}

hipError_t launch_grouped_rows(GroupedRows g, int type, bool transposed, hipStream_t s);
hipError_t launch_grouped_weights(GroupedWeights g, int type, int out, hipStream_t s);

}  // namespace half
}  // namespace oz
