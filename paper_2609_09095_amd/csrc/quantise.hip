// Matrices in 8 bits with a scale per block of 128: blocks of 1 x 128 along the
// rows, of 128 x 1 along the columns (the transposed matrix's rows), or of
// 128 x 128; along the rows, transposed, or both from one read.
//
// Bound by its read and writes.  A block of threads holds a tile of 128 x 128 in
// registers, 8 x 8 elements a thread; the transposed bytes go through LDS once,
// 8 rows of a column in one 64-bit word.  16384 x 4096 bfloat16 to both layouts, scales
// per vector: 58 us, 4.7 TB/s (a large copy: 5.1).
#include "eight_bits.hpp"
#include "eight_products.hpp"

namespace oz {
namespace eight {
namespace {

template <int TYPE, bool SQUARES, bool DIRECT, bool TURNED>
__global__ __launch_bounds__(256) void quantise_kernel(Quantise p) {
  constexpr int E = kBytes<TYPE>;
  __shared__ uint32_t most_of[4][kBlock];
  __shared__ uint2 turned_bytes[TURNED ? kBlock * 16 : 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int c = threadIdx.x & 15, g = threadIdx.x >> 4;  // 8 columns, 8 rows
  const uint32_t kb = ((uint32_t)p.cols + kBlock - 1) / kBlock;  // blocks along the columns, along the rows
  const int64_t nb = ((uint32_t)p.rows + kBlock - 1) / kBlock;
  const int64_t rb = blockIdx.x / kb, cb = blockIdx.x % kb, m = blockIdx.y;
  const int64_t r0 = rb * kBlock + g * 8, c0 = cb * kBlock + c * 8;
  const int cols = (int)(p.cols - c0 < 8 ? p.cols - c0 : 8), rows = (int)(p.rows - r0 < 8 ? p.rows - r0 : 8);
  Raw<TYPE> raw[8];
  const char* const x = (const char*)p.x + (m * p.x_stride + r0 * p.ldx + c0) * E;
#pragma unroll
  for (int i = 0; i < 8; ++i) raw[i] = load_raw<TYPE>(x + i * p.ldx * E, i < rows ? cols : 0);
  float v[8][8];
#pragma unroll
  for (int i = 0; i < 8; ++i) values<TYPE>(raw[i], v[i]);

  Scale all;  // squares: the tile's
  if constexpr (SQUARES) {
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) most = umax(most, size_bits(v[i][j]));
    most = max16(most);
    most = umax(most, (uint32_t)__shfl_xor((int)most, 16));
    most = umax(most, (uint32_t)__shfl_xor((int)most, 32));
    if (lane == 0) most_of[wave][0] = most;
    __syncthreads();
    most = umax(umax(most_of[0][0], most_of[1][0]), umax(most_of[2][0], most_of[3][0]));
    all = scale_of(most);
    if (threadIdx.x == 0) {
      if constexpr (DIRECT) p.scales[(m * nb + rb) * kb + cb] = all.s;
      if constexpr (TURNED) p.scales_t[(m * kb + cb) * nb + rb] = all.s;
    }
  }
  if constexpr (DIRECT) {
    uint8_t* const q = p.q + m * p.q_stride + r0 * p.ldq + c0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      Scale s = all;
      if constexpr (!SQUARES) {
        uint32_t most = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) most = umax(most, size_bits(v[i][j]));
        s = scale_of(max16(most));
        if (c == 0 && i < rows) p.scales[(m * kb + cb) * p.rows + r0 + i] = s.s;
      }
      uint2 b;
      b.x = pack_e4m3(quotient(v[i][0], s), quotient(v[i][1], s), quotient(v[i][2], s), quotient(v[i][3], s));
      b.y = pack_e4m3(quotient(v[i][4], s), quotient(v[i][5], s), quotient(v[i][6], s), quotient(v[i][7], s));
      store_bytes(q + i * p.ldq, b, i < rows ? cols : 0);
    }
  }
  if constexpr (TURNED) {
    if constexpr (!SQUARES) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) most = umax(most, size_bits(v[i][j]));
        most = umax(most, (uint32_t)__shfl_xor((int)most, 16));
        most = umax(most, (uint32_t)__shfl_xor((int)most, 32));
        if (lane < 16) most_of[wave][c * 8 + j] = most;
      }
      __syncthreads();
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      Scale s = all;
      if constexpr (!SQUARES) {
        const int at = c * 8 + j;
        s = scale_of(umax(umax(most_of[0][at], most_of[1][at]), umax(most_of[2][at], most_of[3][at])));
        if (g == 0 && j < cols) p.scales_t[(m * nb + rb) * p.cols + c0 + j] = s.s;
      }
      uint2 b;
      b.x = pack_e4m3(quotient(v[0][j], s), quotient(v[1][j], s), quotient(v[2][j], s), quotient(v[3][j], s));
      b.y = pack_e4m3(quotient(v[4][j], s), quotient(v[5][j], s), quotient(v[6][j], s), quotient(v[7][j], s));
      // a column's 16 words, rotated by its place so that 16 columns of 8 apart meet no bank twice
      turned_bytes[(c * 8 + j) * 16 + (g ^ c)] = b;
    }
    __syncthreads();
    uint8_t* const q = p.qt + m * p.qt_stride + cb * kBlock * p.ldqt + rb * kBlock;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int col = i * 16 + (threadIdx.x >> 4), word = threadIdx.x & 15;
      const int64_t left = p.rows - rb * kBlock - word * 8;
      if (cb * kBlock + col < p.cols)
        store_bytes(q + col * p.ldqt + word * 8, turned_bytes[col * 16 + (word ^ (col >> 3))], (int)(left < 8 ? left : 8));
    }
  }
}

template <int TYPE, bool SQUARES>
hipError_t run(const Quantise& p, hipStream_t s) {
  const int64_t tiles = ceil_div(p.cols, kBlock) * ceil_div(p.rows, kBlock);
  if (tiles * 256 >= ((int64_t)1 << 32)) return hipErrorInvalidConfiguration;
  const dim3 grid((uint32_t)tiles, (uint32_t)p.count);
  if (p.q && p.qt)
    quantise_kernel<TYPE, SQUARES, true, true><<<grid, dim3(256), 0, s>>>(p);
  else if (p.q)
    quantise_kernel<TYPE, SQUARES, true, false><<<grid, dim3(256), 0, s>>>(p);
  else
    quantise_kernel<TYPE, SQUARES, false, true><<<grid, dim3(256), 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_quantise(const Quantise& p, int type, bool squares, hipStream_t s) {
  if (type == kBF16) return squares ? run<kBF16, true>(p, s) : run<kBF16, false>(p, s);
  if (type == kF16) return squares ? run<kF16, true>(p, s) : run<kF16, false>(p, s);
  return squares ? run<kF32, true>(p, s) : run<kF32, false>(p, s);
}

}  // namespace eight
}  // namespace oz
