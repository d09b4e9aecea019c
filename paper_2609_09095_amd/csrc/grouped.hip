// Products of ragged groups of rows with a stack of weights: the forward
// product, the gradient of its input and that of the weights.
//
//   Y[r, :]  = X[r, :] W_g^T          for the rows r of group g
//   dX[r, :] = dY[r, :] W_g
//   dW_g     = sum of dY[r, :]^T X[r, :] over the rows r of g
//
// The group ends are device memory: the host launches the most row tiles that
// any ends could need (rows / BM + groups + 1) and every block finds its group
// from the ends with two wavefront scans per 64 groups; blocks past the last
// tile leave at once.
#include "half_products.hpp"
#include "half_rules.hpp"

namespace oz {
namespace half {
namespace {

// Y (rows x cols) = X (rows x depth) times the group's weights: kAlong for
// weights cols x depth, kAcross for depth x cols.
//
// 2 rows cols depth operations on operands read about once per XCD: bound by the
// matrix cores and the clock they leave.  8192 x 8192 x 8192, one group: 815 us (1350
// TFLOP/s) in either layout, the library's own product of that size 765 us.
// 16384 rows of 16 uneven groups, 4096 x 2048: 294 us (935 TFLOP/s): each group's
// last tile is partly filled, and the tiles are 4.3 rounds of the CUs.
template <class T>
__global__ __launch_bounds__(T::THREADS, 1) void grouped_rows_kernel(GroupedRows g) {
  __shared__ __attribute__((aligned(1024))) char lds[T::LDS];
  const uint32_t tiles_n = ((uint32_t)g.cols + T::BN - 1) / T::BN;
  RowTiles<T::BM> all;
  const uint32_t tiles_m = all.init(g.ends, g.groups, g.rows);
  uint32_t place, tm, tn;
  if (!block_place(blockIdx.x, tiles_m * tiles_n, place)) return;
  place_to_tile(place, tiles_m, tiles_n, tm, tn);
  RowTile t;
  if (!all.find((int)tm, t)) return;
  const int c0 = (int)tn * T::BN;
  const int cols = g.cols - c0 < T::BN ? g.cols - c0 : T::BN;
  const bool none = t.group == g.groups;  // rows of no group: zeros
  const char* w = (const char*)g.w + (none ? 0 : t.group * g.group_stride * 2);
  const Operand a{(const char*)g.x + t.row * g.ldx * 2, g.ldx, t.rows, g.depth};
  const Operand b{w + (T::LB == kAlong ? c0 * g.ldw : (int64_t)c0) * 2, g.ldw, cols,
                  T::LB == kAlong ? g.depth : g.cols};
  v16f acc[T::MB][T::NB] = {};
  if (!product<T>(a, b, none ? 0 : g.depth, lds, acc)) return;
  store<T>(acc, lds, (char*)g.y + (t.row * g.ldy + c0) * 2, g.ldy, t.rows, cols, g.stream);
}

// The same for few rows per group (serving): a block reads 16 NB columns of a
// group's weights once, for at most 16 TB of its rows.  Bound by that read: 256
// rows of 64 groups, 1024 x 2048: 42 us (6.3 TB/s; a large copy reads and writes at
// 4.9).  With little to read by the launch and the chain of loads: 2 rows, two of 8
// groups, 2048 x 1024: 4.5 us.
template <int TYPE, int NB, int TB, int WAVES, int U>
__global__ __launch_bounds__(WAVES * 64) void grouped_few_kernel(GroupedRows g) {
  using O = typename Out<TYPE>::type;
  __shared__ v4f lds[WAVES * TB * 16 * NB * 4];
  const uint32_t tiles_n = ((uint32_t)g.cols + 16 * NB - 1) / (16 * NB);
  RowTiles<16 * TB> all;
  const uint32_t tiles_m = all.init(g.ends, g.groups, g.rows);
  uint32_t place;
  if (!block_place(blockIdx.x, tiles_m * tiles_n, place)) return;
  // a group's row tiles side by side: they share the weights
  const uint32_t tn = place / tiles_m, tm = place - tn * tiles_m;
  RowTile t;
  if (!all.find((int)tm, t)) return;
  const int c0 = (int)tn * (16 * NB), cols = g.cols - c0 < 16 * NB ? g.cols - c0 : 16 * NB;
  v4f acc[NB][TB] = {};
  if (t.group < g.groups && g.depth > 0) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int steps = (g.depth + 31) / 32;
    const char* w = (const char*)g.w + (t.group * g.group_stride + c0 * g.ldw) * 2;
    skinny<TYPE, NB, TB, U>(w, g.ldw, cols, (const char*)g.x + t.row * g.ldx * 2, g.ldx, t.rows, g.depth,
                         steps * wave / WAVES, steps * (wave + 1) / WAVES, acc);
  }
  O* const y = (O*)g.y + t.row * g.ldy + c0;
  skinny_join<NB, TB, WAVES>(acc, lds, [&](int row, int c, v4f v) {
    if (row >= t.rows || c >= cols) return;
    O* const q = y + row * g.ldy + c;
    if (c + 4 <= cols) {
      const uint2 w = pack4<TYPE>(v[0], v[1], v[2], v[3]);
      __builtin_memcpy(q, &w, 8);  // any alignment
    } else {
#pragma unroll
      for (int e = 0; e < 3; ++e)
        if (c + e < cols) q[e] = (O)v[e];
    }
  });
}

// dW_g (n x k) = dY_g^T X_g; a group without rows gets zeros.  One tile sums over
// all of its group's rows, so nothing is joined between blocks.  8192 x 8192 x
// 8192: 820 us (1340 TFLOP/s).  32768 rows of 32 groups, 2048 x 4096, 32-bit
// output: about 610 us (900 TFLOP/s): 1 GB of outputs leave past the caches
// between the tiles' products.
template <class T>
__global__ __launch_bounds__(T::THREADS, 1) void grouped_weights_kernel(GroupedWeights g) {
  __shared__ __attribute__((aligned(1024))) char lds[T::LDS];
  const uint32_t tiles_m = ((uint32_t)g.n + T::BM - 1) / T::BM, tiles_n = ((uint32_t)g.k + T::BN - 1) / T::BN;
  // every group's tiles are spread over the XCDs by themselves: groups differ in depth
  const uint32_t per = (tiles_m * tiles_n + 7) & ~7u;
  const uint32_t group = blockIdx.x / per;
  uint32_t place, tm, tn;
  if (!block_place(blockIdx.x - group * per, tiles_m * tiles_n, place)) return;
  place_to_tile(place, tiles_m, tiles_n, tm, tn);
  const int lane = threadIdx.x & 63;
  int last = 0, first = 0, end = 0;
  for (int g0 = 0; g0 <= (int)group; g0 += 64)
    group_rows(group_end(g.ends, g.groups, g.rows, g0, lane), lane, last, first, end);
  first = __builtin_amdgcn_readlane(first, group & 63);
  end = __builtin_amdgcn_readlane(end, group & 63);
  const int r0 = (int)tm * T::BM, c0 = (int)tn * T::BN;
  const int rows = g.n - r0 < T::BM ? g.n - r0 : T::BM, cols = g.k - c0 < T::BN ? g.k - c0 : T::BN;
  const Operand a{(const char*)g.dy + (first * g.lddy + r0) * 2, g.lddy, rows, g.n};
  const Operand b{(const char*)g.x + (first * g.ldx + c0) * 2, g.ldx, cols, g.k};
  v16f acc[T::MB][T::NB] = {};
  if (!product<T>(a, b, end - first, lds, acc)) return;
  constexpr int E = sizeof(typename Out<T::OUT>::type);
  store<T>(acc, lds, (char*)g.dw + (group * g.group_stride + r0 * g.lddw + c0) * E, g.lddw, rows, cols, g.stream);
}

template <class T>
hipError_t run_rows(const GroupedRows& g, hipStream_t s) {
  const int64_t tiles = ((int64_t)g.rows / T::BM + g.groups + 1) * ((g.cols + T::BN - 1) / T::BN);
  if (tiles * T::THREADS >= ((int64_t)1 << 32)) return hipErrorInvalidConfiguration;
  grouped_rows_kernel<T><<<dim3((uint32_t)tiles), dim3(T::THREADS), 0, s>>>(g);
  return hipGetLastError();
}

template <int TYPE, int NB, int TB, int WAVES, int U>
hipError_t run_few(const GroupedRows& g, hipStream_t s) {
  // a tile holds at least one row, and all but each group's last (and that of no group) are full
  const int64_t most = (int64_t)g.rows / (16 * TB) + g.groups + 1;
  const int64_t tiles = (most < g.rows ? most : g.rows) * ((g.cols + 16 * NB - 1) / (16 * NB));
  if (tiles * WAVES * 64 >= ((int64_t)1 << 32)) return hipErrorInvalidConfiguration;
  grouped_few_kernel<TYPE, NB, TB, WAVES, U><<<dim3((uint32_t)((tiles + 7) & ~(int64_t)7)), dim3(WAVES * 64), 0, s>>>(g);
  return hipGetLastError();
}

template <class T>
hipError_t run_weights(const GroupedWeights& g, hipStream_t s) {
  const int64_t each = (int64_t)((g.n + T::BM - 1) / T::BM) * ((g.k + T::BN - 1) / T::BN);
  const int64_t tiles = g.groups * ((each + 7) & ~(int64_t)7);
  if (tiles * T::THREADS >= ((int64_t)1 << 32)) return hipErrorInvalidConfiguration;
  grouped_weights_kernel<T><<<dim3((uint32_t)tiles), dim3(T::THREADS), 0, s>>>(g);
  return hipGetLastError();
}

template <int TYPE, int LB>
hipError_t rows_of_type(const GroupedRows& g, bool dma, hipStream_t s) {
  const bool few = few_rows(g.rows, g.groups) && (dma || few_rows_masked(g.rows, g.groups, g.cols, g.depth));
  if (LB == kAlong && few) switch (few_form(g.rows, g.groups, g.cols)) {
      case kFew16: return run_few<TYPE, 1, 1, 8, 8>(g, s);
      case kFew32: return run_few<TYPE, 2, 2, 8, 4>(g, s);
      case kFew64x32: return run_few<TYPE, 4, 2, 4, 2>(g, s);
      case kFew64x64: return run_few<TYPE, 4, 4, 4, 2>(g, s);
    }
  if (!dma) {
    if (masked_sets(expected_row_tiles(g.rows, g.groups, 64) * ceil_div(g.cols, 64), g.depth))
      return run_rows<Tile<TYPE, kAlong, LB, 2, 2, 1, 1, false, TYPE, 2, 4>>(g, s);
    if (masked_small(false, expected_row_tiles(g.rows, g.groups, 128) * ceil_div(g.cols, 128)))
      return run_rows<Tile<TYPE, kAlong, LB, 2, 2, 1, 1, false, TYPE>>(g, s);
    return run_rows<Tile<TYPE, kAlong, LB, 2, 4, 2, 1, false, TYPE>>(g, s);
  }
  switch (rows_tile(g.rows, g.groups, g.cols)) {
    case kSmallTile: return run_rows<Tile<TYPE, kAlong, LB, 2, 2, 1, 1, true, TYPE, 3>>(g, s);
    case kMiddleTile: return run_rows<Tile<TYPE, kAlong, LB, 2, 2, 2, 2, true, TYPE>>(g, s);
    default: return run_rows<Tile<TYPE, kAlong, LB, 2, 4, 4, 2, true, TYPE>>(g, s);
  }
}

template <int TYPE, int OUT>
hipError_t weights_of_type(const GroupedWeights& g, bool dma, hipStream_t s) {
  if (!dma) {
    if (masked_sets(g.groups * ceil_div(g.n, 64) * ceil_div(g.k, 64), g.rows / g.groups))  // their average depth
      return run_weights<Tile<TYPE, kAcross, kAcross, 2, 2, 1, 1, false, OUT, 2, 4>>(g, s);
    if (masked_small(true, g.groups * ceil_div(g.n, 128) * ceil_div(g.k, 128)))
      return run_weights<Tile<TYPE, kAcross, kAcross, 2, 2, 1, 1, false, OUT>>(g, s);
    return run_weights<Tile<TYPE, kAcross, kAcross, 2, 4, 2, 1, false, OUT>>(g, s);
  }
  switch (weights_tile(g.n, g.k, g.groups)) {
    case kSmallTile: return run_weights<Tile<TYPE, kAcross, kAcross, 2, 2, 1, 1, true, OUT, 3>>(g, s);
    case kMiddleTile: return run_weights<Tile<TYPE, kAcross, kAcross, 2, 2, 2, 2, true, OUT>>(g, s);
    default: return run_weights<Tile<TYPE, kAcross, kAcross, 2, 4, 4, 2, true, OUT>>(g, s);
  }
}

}  // namespace

hipError_t launch_grouped_rows(GroupedRows g, int type, bool transposed, hipStream_t s) {
  g.stream = past_caches((int64_t)g.rows * g.cols * 2);
  const bool dma = dma_operand(g.x, g.ldx, g.depth) && dma_operand(g.w, g.ldw, transposed ? g.cols : g.depth) &&
                   g.group_stride % 8 == 0 && g.cols % 8 == 0 && g.depth % 8 == 0;
  if (type == kBF16)
    return transposed ? rows_of_type<kBF16, kAcross>(g, dma, s) : rows_of_type<kBF16, kAlong>(g, dma, s);
  return transposed ? rows_of_type<kF16, kAcross>(g, dma, s) : rows_of_type<kF16, kAlong>(g, dma, s);
}

hipError_t launch_grouped_weights(GroupedWeights g, int type, int out, hipStream_t s) {
  g.stream = past_caches((int64_t)g.groups * g.n * g.k * 2);
  const bool dma = dma_operand(g.dy, g.lddy, g.n) && dma_operand(g.x, g.ldx, g.k);
  if (type == kBF16)
    return out == kF32 ? weights_of_type<kBF16, kF32>(g, dma, s) : weights_of_type<kBF16, kBF16>(g, dma, s);
  return out == kF32 ? weights_of_type<kF16, kF32>(g, dma, s) : weights_of_type<kF16, kF16>(g, dma, s);
}

}  // namespace half
}  // namespace oz
