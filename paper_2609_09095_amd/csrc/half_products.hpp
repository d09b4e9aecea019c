// Host interface of the 16-bit products (grouped.hip, adapter.hip,
// orthogonalise.hip).  Arguments were checked by the entry points.
#pragma once

#include "half_rules.hpp"
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
  bool stream;  // y past the caches (set by the launch)
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
  bool stream;  // a 16-bit dw past the caches (set by the launch)
};

struct Adapter {
  const void* x;  // rows x k
  int64_t ldx;
  const void* w;  // n x k
  int64_t ldw;
  const int32_t* ids;  // rows
  const void* a;       // a stack of rank x k
  int64_t lda, a_stride;
  const void* b;  // a stack of n x rank
  int64_t ldb, b_stride;
  const float* scales;  // adapters, or null: 1
  void* y;              // rows x n
  int64_t ldy;
  int rows, n, k, adapters, rank;
  // workspace (set by the launch)
  float* h;          // parts x rows x rank_pad
  void* h16;         // rows x 2 rank_pad
  float* factors;    // rows: what a row's h16 was divided by (half)
  float* partials;   // base_splits x rows x n_pad
  int rank_pad;      // rank rounded up to 16
  int n_pad;         // n rounded up to 4
  int splits;        // parts of the depth of X A^T
  int serve_splits;  // the same in the few-row form
  int base_splits;   // parts of the depth of X W^T in the few-row form
  bool stream;       // y past the caches
};

struct Orthogonalise {
  const void* g;  // count matrices m x n
  int64_t ldg, g_stride;
  void* x;  // the same, bfloat16
  int64_t ldx, x_stride;
  int count, m, n;
  int mp, np;  // m, n padded to multiples of 8
  float a, b, c, eps;
  bool diagonal_in_32_bits;  // P's, in this step (set by the launch)
  // workspace
  double* squares;  // count x orthogonalise_parts
  float* x32;       // count x mp x np
  void* x16[2];     // the same
  void* s16;        // count x s x s, s the shorter padded side; zero diagonal
  void* p16;        // the same; the diagonal in steps that round it
  float* d32;       // count x s: the diagonal of S
  float* p32;       // P's diagonal, or what its rounding left
};

// Matrices of at most this side run in one launch that needs no workspace.
constexpr int kOneLaunchSide = 128;
inline bool orthogonalise_in_one_launch(int64_t m, int64_t n) { return m <= kOneLaunchSide && n <= kOneLaunchSide; }

// Blocks (and partial sums) per matrix of the norm.
inline int orthogonalise_parts(int64_t m, int64_t n) {
  const int64_t p = m * ((n + 7) / 8) / 512;
  return (int)(p < 1 ? 1 : p > 1024 ? 1024 : p);
}

// Outputs that the 32 MiB of L2 do not hold are stored past it.
inline bool past_caches(int64_t bytes) { return bytes > ((int64_t)32 << 20); }

// Whether a matrix of `cols` columns can go to LDS by DMA: 16-byte rows, and a
// tile's offsets below 2^31.
inline bool dma_operand(const void* p, int64_t ld, int64_t cols) {
  return (uintptr_t)p % 16 == 0 && ld % 8 == 0 && cols % 8 == 0 && ld < ((int64_t)1 << 21);
}

hipError_t launch_grouped_rows(GroupedRows g, int type, bool transposed, hipStream_t s);
hipError_t launch_grouped_weights(GroupedWeights g, int type, int out, hipStream_t s);
hipError_t launch_adapter(Adapter p, const AdapterPlan& plan, char* room, int type, hipStream_t s);
hipError_t launch_orthogonalise(Orthogonalise o, int type, int steps, hipStream_t s);

}  // namespace half
}  // namespace oz
