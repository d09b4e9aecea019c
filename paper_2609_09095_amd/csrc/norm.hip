// Root-mean-square norm of rows, with the residual's addition before it and, if
// asked for, the result in 8 bits with a scale per row and 128 columns; and its
// gradient.
//
//   h = x + r (rounded to its type),  y = h rho w,  rho = 1 / sqrt(mean h^2 + eps)
//   dx = rho (g - h rho^2 mean(g h)) + dh,  g = dy w,    dw = sum over rows of dy h rho
//
// Both are bound by their reads and writes.  A row's elements stay in the
// registers of LANES threads (8 CH each) from the load to the store, so each is
// read and written once; the next row's loads are in flight meanwhile.
#include "eight_bits.hpp"
#include "eight_products.hpp"

namespace oz {
namespace eight {
namespace {

// Sums over the LANES threads of a row, in all of them; the order is fixed.
// room: 2 x N x 16 floats; `turn` alternates between its halves, so one barrier
// keeps a row's sums apart from the next one's.
template <int LANES, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float* room, int turn) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    v[i] = sum16(v[i]);
    if constexpr (LANES > 16) v[i] += __shfl_xor(v[i], 16);
    if constexpr (LANES > 32) v[i] += __shfl_xor(v[i], 32);
  }
  if constexpr (LANES > 64) {
    constexpr int WAVES = LANES / 64;
    float* const mine = room + turn * (N * 16);
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) mine[i * 16 + (threadIdx.x >> 6)] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float t = mine[i * 16];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) t += mine[i * 16 + w];
      v[i] = t;
    }
  }
}

template <int TYPE, int LANES, int CH, bool RES, bool EIGHT>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void norm_kernel(Norm p) {
  constexpr int THREADS = LANES < 256 ? 256 : LANES, GROUPS = THREADS / LANES, E = kBytes<TYPE>;
  __shared__ float room[2 * 16];
  const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
  int have[CH];
  float w[CH][8];
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    have[i] = p.width - (lane + i * LANES) * 8;
    if (p.weight) {
      values<TYPE>(load_raw<TYPE>((const char*)p.weight + (int64_t)(lane + i * LANES) * 8 * E, have[i]), w[i]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) w[i][j] = 1.0f;
    }
  }
  Raw<TYPE> x[CH], r[CH];
  auto load = [&](int64_t row) {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int n = row < p.rows ? have[i] : 0;
      const int64_t c = (int64_t)(lane + i * LANES) * 8;
      x[i] = load_raw<TYPE>((const char*)p.x + (row * p.ldx + c) * E, n);
      if constexpr (RES) r[i] = load_raw<TYPE>((const char*)p.residual + (row * p.ldr + c) * E, n);
    }
  };
  const int64_t step = (int64_t)gridDim.x * GROUPS;
  load((int64_t)blockIdx.x * GROUPS + group);
  int turn = 0;
  for (int64_t first = (int64_t)blockIdx.x * GROUPS; first < p.rows; first += step) {
    const int64_t row = first + group;
    const bool any = row < p.rows;
    float h[CH][8], sum[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      values<TYPE>(x[i], h[i]);
      if constexpr (RES) {
        float b[8];
        values<TYPE>(r[i], b);
#pragma unroll
        for (int j = 0; j < 8; ++j) h[i][j] += b[j];
        const Raw<TYPE> kept = rounded<TYPE>(h[i]);
        if (any) store_raw<TYPE>((char*)p.h + (row * p.ldh + (int64_t)(lane + i * LANES) * 8) * E, kept, have[i]);
        values<TYPE>(kept, h[i]);  // the norm is that of the sum as it is kept
      }
    }
    load(row + step);
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[0] = __builtin_fmaf(h[i][j], h[i][j], sum[0]);
    row_sums<LANES, 1>(sum, room, turn);
    turn ^= 1;
    const float rho = 1.0f / sqrtf(sum[0] / (float)p.width + p.eps);
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int64_t c = (int64_t)(lane + i * LANES) * 8;
      float y[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = h[i][j] * rho * w[i][j];
      if constexpr (EIGHT) {
        uint32_t most = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) most = umax(most, j < have[i] ? size_bits(y[j]) : 0);
        const Scale s = scale_of(max16(most));
        uint2 b;
        b.x = pack_e4m3(quotient(y[0], s), quotient(y[1], s), quotient(y[2], s), quotient(y[3], s));
        b.y = pack_e4m3(quotient(y[4], s), quotient(y[5], s), quotient(y[6], s), quotient(y[7], s));
        if (any) {
          store_bytes((uint8_t*)p.y + row * p.ldy + c, b, have[i]);
          if ((lane & 15) == 0 && have[i] > 0) p.scales[(c / kBlock) * p.lds + row] = s.s;
        }
      } else {
        if (any) store_raw<TYPE>((char*)p.y + (row * p.ldy + c) * E, rounded<TYPE>(y), have[i]);
      }
    }
  }
}

// Each block adds up dw over its rows in registers and leaves one row of
// partial sums; dw_kernel adds those.
template <int TYPE, int LANES, int CH, bool DH>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void norm_gradient_kernel(NormGradient p) {
  constexpr int THREADS = LANES < 256 ? 256 : LANES, GROUPS = THREADS / LANES, E = kBytes<TYPE>;
  __shared__ float room[GROUPS > 1 ? GROUPS * LANES * CH * 8 : 2 * 2 * 16];
  const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
  int have[CH];
  float dw[CH][8] = {};
  Raw<TYPE> w[CH];
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    have[i] = p.width - (lane + i * LANES) * 8;
    if (p.weight) {
      w[i] = load_raw<TYPE>((const char*)p.weight + (int64_t)(lane + i * LANES) * 8 * E, have[i]);
    } else {
      const float one[8] = {1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f};
      w[i] = rounded<TYPE>(one);
    }
  }
  Raw<TYPE> y[CH], x[CH], d[CH];
  auto load = [&](int64_t row) {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int n = row < p.rows ? have[i] : 0;
      const int64_t c = (int64_t)(lane + i * LANES) * 8;
      y[i] = load_raw<TYPE>((const char*)p.dy + (row * p.lddy + c) * E, n);
      x[i] = load_raw<TYPE>((const char*)p.h + (row * p.ldh + c) * E, n);
      if constexpr (DH) d[i] = load_raw<TYPE>((const char*)p.dh + (row * p.lddh + c) * E, n);
    }
  };
  const int64_t step = (int64_t)gridDim.x * GROUPS;
  load((int64_t)blockIdx.x * GROUPS + group);
  int turn = 0;
  for (int64_t first = (int64_t)blockIdx.x * GROUPS; first < p.rows; first += step) {
    const int64_t row = first + group;
    float h[CH][8], dy[CH][8], b[CH][8], sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      values<TYPE>(x[i], h[i]);
      values<TYPE>(y[i], dy[i]);
      if constexpr (DH) values<TYPE>(d[i], b[i]);
    }
    load(row + step);
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      float f[8];
      values<TYPE>(w[i], f);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        sum[0] = __builtin_fmaf(h[i][j], h[i][j], sum[0]);
        sum[1] = __builtin_fmaf(dy[i][j] * f[j], h[i][j], sum[1]);
      }
    }
    row_sums<LANES, 2>(sum, room, turn);
    turn ^= 1;
    const float rho = 1.0f / sqrtf(sum[0] / (float)p.width + p.eps), mean = rho * rho * (sum[1] / (float)p.width);
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      float f[8], dx[8];
      values<TYPE>(w[i], f);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        dx[j] = rho * __builtin_fmaf(-h[i][j], mean, dy[i][j] * f[j]);
        if constexpr (DH) dx[j] += b[i][j];
        if (row < p.rows) dw[i][j] = __builtin_fmaf(dy[i][j] * h[i][j], rho, dw[i][j]);
      }
      if (row < p.rows)
        store_raw<TYPE>((char*)p.dx + (row * p.lddx + (int64_t)(lane + i * LANES) * 8) * E, rounded<TYPE>(dx), have[i]);
    }
  }
  float* const part = p.parts + (int64_t)blockIdx.x * p.width;
  if constexpr (GROUPS > 1) {
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) room[(group * CH + i) * LANES * 8 + lane * 8 + j] = dw[i][j];
    __syncthreads();
    for (int c = threadIdx.x; c < p.width; c += THREADS) {
      float t = room[c];
#pragma unroll
      for (int g = 1; g < GROUPS; ++g) t += room[g * CH * LANES * 8 + c];
      part[c] = t;
    }
  } else {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const Raw<kF32> r = rounded<kF32>(dw[i]);
      store_raw<kF32>((char*)(part + (int64_t)(lane + i * LANES) * 8), r, have[i]);
    }
  }
}

// 16 columns a block, the parts over 16 sets of lanes
__global__ __launch_bounds__(256) void dw_kernel(const float* parts, int count, int width, float* dw) {
  __shared__ float room[16][17];
  const int c = blockIdx.x * 16 + (threadIdx.x & 15), set = threadIdx.x >> 4;
  float t = 0.0f;
  if (c < width) {
#pragma unroll 8
    for (int i = set; i < count; i += 16) t += parts[(int64_t)i * width + c];
  }
  room[set][threadIdx.x & 15] = t;
  __syncthreads();
  if (set == 0 && c < width) {
#pragma unroll
    for (int i = 1; i < 16; ++i) t += room[i][threadIdx.x];
    dw[c] = t;
  }
}

__global__ __launch_bounds__(256) void zeros_kernel(float* p, int64_t count) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < count) p[i] = 0.0f;
}

template <int TYPE, int LANES, int CH>
hipError_t run_norm(const Norm& p, hipStream_t s) {
  const dim3 grid((uint32_t)norm_blocks(p.rows, p.width, kNormThreads)), block(LANES < 256 ? 256 : LANES);
  if (p.residual) {
    if (p.scales)
      norm_kernel<TYPE, LANES, CH, true, true><<<grid, block, 0, s>>>(p);
    else
      norm_kernel<TYPE, LANES, CH, true, false><<<grid, block, 0, s>>>(p);
  } else {
    if (p.scales)
      norm_kernel<TYPE, LANES, CH, false, true><<<grid, block, 0, s>>>(p);
    else
      norm_kernel<TYPE, LANES, CH, false, false><<<grid, block, 0, s>>>(p);
  }
  return hipGetLastError();
}

template <int TYPE, int LANES, int CH>
hipError_t run_gradient(const NormGradient& p, hipStream_t s) {
  const int64_t parts = norm_parts(p.rows, p.width);
  const dim3 grid((uint32_t)parts), block(LANES < 256 ? 256 : LANES);
  if (p.dh)
    norm_gradient_kernel<TYPE, LANES, CH, true><<<grid, block, 0, s>>>(p);
  else
    norm_gradient_kernel<TYPE, LANES, CH, false><<<grid, block, 0, s>>>(p);
  if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  dw_kernel<<<dim3((uint32_t)ceil_div(p.width, 16)), dim3(256), 0, s>>>(p.parts, (int)parts, p.width, p.dw);
  return hipGetLastError();
}

// calls f<LANES, CH>() for the form of this width
template <class F>
hipError_t of_form(int width, F f) {
  const NormForm g = norm_form(width);
  switch (g.lanes * 8 + g.chunks) {
    case 16 * 8 + 1: return f.template operator()<16, 1>();
    case 32 * 8 + 1: return f.template operator()<32, 1>();
    case 64 * 8 + 1: return f.template operator()<64, 1>();
    case 64 * 8 + 2: return f.template operator()<64, 2>();
    case 256 * 8 + 1: return f.template operator()<256, 1>();
    case 512 * 8 + 1: return f.template operator()<512, 1>();
    case 1024 * 8 + 1: return f.template operator()<1024, 1>();
    case 1024 * 8 + 2: return f.template operator()<1024, 2>();
    default: return f.template operator()<1024, 4>();
  }
}

template <class F>
hipError_t of_type(int type, F f) {
  if (type == kBF16) return f.template operator()<kBF16>();
  if (type == kF16) return f.template operator()<kF16>();
  return f.template operator()<kF32>();
}

}  // namespace

hipError_t launch_zeros(float* p, int64_t count, hipStream_t s) {
  zeros_kernel<<<dim3((uint32_t)ceil_div(count, 256)), dim3(256), 0, s>>>(p, count);
  return hipGetLastError();
}

hipError_t launch_norm(const Norm& p, int type, hipStream_t s) {
  return of_type(type, [&]<int TYPE>() {
    return of_form(p.width, [&]<int LANES, int CH>() { return run_norm<TYPE, LANES, CH>(p, s); });
  });
}

hipError_t launch_norm_gradient(const NormGradient& p, int type, hipStream_t s) {
  return of_type(type, [&]<int TYPE>() {
    return of_form(p.width, [&]<int LANES, int CH>() { return run_gradient<TYPE, LANES, CH>(p, s); });
  });
}

}  // namespace eight
}  // namespace oz
