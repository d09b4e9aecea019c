// Root-mean-square norm of rows, with the residual's addition before it and, if
// asked for, the result in 8 bits with a scale per row and 128 columns; and its
// gradient.
//
//   h = x + r (rounded to its type),  y = h rho w,  rho = 1 / sqrt(mean h^2 + eps)
//   dx = rho (g - h rho^2 mean(g h)) + dh,  g = dy w,    dw = sum over rows of dy h rho
//
// Both are bound by their reads and writes.  A row's elements stay in the
// registers of LANES threads (8 CH each) from the load to the store, so each is
// read and written once; the next row's loads are in flight meanwhile.  8192 x 4096
// bfloat16 with residual to e4m3: 44 us, 5.4 TB/s; the gradients of 16384 x 4096: 97
// us, 5.5 TB/s (a large copy: 5.1).  4096 x 16384: 121 us, 4.4 TB/s (with the row read
// twice 154).  Rows of more than 16384 elements are read twice by the gradient: 2048 x
// 20000 151 us, 2.2 TB/s of what has to be moved.
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

// A thread's chunks of 8 columns of a row.  The chunk that the row's end cuts is read
// as the row's last 8 elements and moved down when it is used, and one past the end
// reads them too: a branch around a load would wait for its data and leave none in
// flight.  Rows of fewer than 8 elements are read one by one.
template <int TYPE, int LANES>
struct Columns {
  int width, lane;
  bool narrow;
  __device__ __forceinline__ void init(int w, int l) {
    width = w, lane = l;
    narrow = w < 8;
  }
  __device__ __forceinline__ int column(int i) const { return (lane + i * LANES) * 8; }
  // elements of the chunk that exist; below 1: none
  __device__ __forceinline__ int have(int i) const { return width - column(i); }
  __device__ __forceinline__ Raw<TYPE> load(const void* p, int64_t first, int i) const {
    constexpr int E = kBytes<TYPE>;
    const int off = narrow || have(i) >= 8 ? column(i) : width - 8;
    const char* const q = (const char*)p + (first + off) * E;
    return narrow ? load_raw<TYPE>(q, have(i)) : load_raw<TYPE>(q, 8);
  }
  __device__ __forceinline__ void get(const Raw<TYPE>& r, int i, float (&v)[8]) const {
    values<TYPE>(r, v);
    const int n = have(i);
    if (!narrow && __builtin_amdgcn_ballot_w64(n < 8)) {
      const int s = n >= 8 ? 0 : n <= 0 ? 8 : 8 - n;  // elements to drop
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = s & 8 ? 0.0f : s & 4 ? (j < 4 ? v[(j + 4) & 7] : 0.0f) : v[j];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = s & 2 ? (j < 6 ? v[(j + 2) & 7] : 0.0f) : v[j];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = s & 1 ? (j < 7 ? v[(j + 1) & 7] : 0.0f) : v[j];
    }
  }
};

template <int TYPE, int LANES, int CH, bool RES, bool EIGHT>
__global__ __launch_bounds__(norm_threads(LANES)) void norm_kernel(Norm p) {
  constexpr int THREADS = norm_threads(LANES), GROUPS = THREADS / LANES, E = kBytes<TYPE>;
  constexpr bool AHEAD = CH < 4;  // registers for the next row
  __shared__ float room[2 * 16];
  const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
  Columns<TYPE, LANES> cols;
  cols.init(p.width, lane);
  float w[CH][8];
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    if (p.weight) {
      cols.get(cols.load(p.weight, 0, i), i, w[i]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) w[i][j] = 1.0f;
    }
  }
  Raw<TYPE> x[CH], r[CH];
  auto load = [&](int64_t row) {
    row = row < p.rows ? row : p.rows - 1;  // one past the last is read again and not used
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      x[i] = cols.load(p.x, row * p.ldx, i);
      if constexpr (RES) r[i] = cols.load(p.residual, row * p.ldr, i);
    }
  };
  const int64_t step = (int64_t)gridDim.x * GROUPS;
  if constexpr (AHEAD) load((int64_t)blockIdx.x * GROUPS + group);
  int turn = 0;
  for (int64_t first = (int64_t)blockIdx.x * GROUPS; first < p.rows; first += step) {
    const int64_t row = first + group;
    const bool any = row < p.rows;
    if constexpr (!AHEAD) load(row);
    float h[CH][8], sum[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      cols.get(x[i], i, h[i]);
      if constexpr (RES) {
        float b[8];
        cols.get(r[i], i, b);
#pragma unroll
        for (int j = 0; j < 8; ++j) h[i][j] += b[j];
        const Raw<TYPE> kept = rounded<TYPE>(h[i]);
        if (any) store_raw<TYPE>((char*)p.h + (row * p.ldh + cols.column(i)) * E, kept, cols.have(i));
        values<TYPE>(kept, h[i]);  // the norm is that of the sum as it is kept
      }
    }
    if constexpr (AHEAD) load(row + step);
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[0] = __builtin_fmaf(h[i][j], h[i][j], sum[0]);
    row_sums<LANES, 1>(sum, room, turn);
    turn ^= 1;
    const float rho = 1.0f / sqrtf(sum[0] / (float)p.width + p.eps);
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int c = cols.column(i), have = cols.have(i);
      float y[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = h[i][j] * rho * w[i][j];
      if constexpr (EIGHT) {
        uint32_t most = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) most = umax(most, j < have ? size_bits(y[j]) : 0);
        const Scale s = scale_of(max16(most));
        uint2 b;
        b.x = pack_e4m3(quotient(y[0], s), quotient(y[1], s), quotient(y[2], s), quotient(y[3], s));
        b.y = pack_e4m3(quotient(y[4], s), quotient(y[5], s), quotient(y[6], s), quotient(y[7], s));
        if (any) {
          store_bytes((uint8_t*)p.y + row * p.ldy + c, b, have);
          if ((lane & 15) == 0 && have > 0) p.scales[(c / kBlock) * p.lds + row] = s.s;
        }
      } else {
        if (any) store_raw<TYPE>((char*)p.y + (row * p.ldy + c) * E, rounded<TYPE>(y), have);
      }
    }
  }
}

// Each block adds up dw over its rows in registers and leaves one row of
// partial sums; dw_kernel adds those, in an order that the sizes fix: no atomics.
template <int TYPE, int LANES, int CH, bool DH>
__global__ __launch_bounds__(norm_threads(LANES)) void norm_gradient_kernel(NormGradient p) {
  constexpr int THREADS = norm_threads(LANES), GROUPS = THREADS / LANES, E = kBytes<TYPE>;
  __shared__ float room[GROUPS > 1 ? LANES * CH * 8 : 2 * 2 * 16];
  const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
  Columns<TYPE, LANES> cols;
  cols.init(p.width, lane);
  // of more than a chunk in LDS, so that the row stays in registers
  constexpr bool WIDE = CH > 1;
  __shared__ v4f wide[WIDE ? CH * LANES * 2 : 1];
  float dw[WIDE ? 1 : CH][8] = {};
  if constexpr (WIDE) {
    for (int i = 0; i < 2 * CH; ++i) wide[i * LANES + lane] = v4f{};  // a thread's own from here on
  }
  const void* weight = p.weight;
  auto weights = [&](int i) {
    const float one[8] = {1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f};
    return weight ? cols.load(weight, 0, i) : rounded<TYPE>(one);
  };
  auto add = [&](const float (&h)[8], const float (&dy)[8], const float (&f)[8], float (&sum)[2]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      sum[0] = __builtin_fmaf(h[j], h[j], sum[0]);
      sum[1] = __builtin_fmaf(dy[j] * f[j], h[j], sum[1]);
    }
  };
  auto finish = [&](int64_t row, int i, float rho, float mean, const float (&h)[8], const float (&dy)[8], const float (&f)[8],
                    const float (&b)[8]) {
    float dx[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      dx[j] = rho * __builtin_fmaf(-h[j], mean, dy[j] * f[j]);
      if constexpr (DH) dx[j] += b[j];
    }
    if constexpr (WIDE) {
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        v4f t = wide[(2 * i + q) * LANES + lane];
#pragma unroll
        for (int j = 0; j < 4; ++j) t[j] = __builtin_fmaf(dy[4 * q + j] * h[4 * q + j], rho, t[j]);
        wide[(2 * i + q) * LANES + lane] = t;
      }
    } else if (row < p.rows) {
#pragma unroll
      for (int j = 0; j < 8; ++j) dw[i][j] = __builtin_fmaf(dy[j] * h[j], rho, dw[i][j]);
    }
    if (row < p.rows)
      store_raw<TYPE>((char*)p.dx + (row * p.lddx + cols.column(i)) * E, rounded<TYPE>(dx), cols.have(i));
  };
  const int64_t step = (int64_t)gridDim.x * GROUPS;
  int turn = 0;
  if constexpr (CH == 1) {
    const Raw<TYPE> w = weights(0);
    Raw<TYPE> y, x, d;
    auto load = [&](int64_t row) {
      row = row < p.rows ? row : p.rows - 1;  // one past the last is read again and not used
      y = cols.load(p.dy, row * p.lddy, 0);
      x = cols.load(p.h, row * p.ldh, 0);
      if constexpr (DH) d = cols.load(p.dh, row * p.lddh, 0);
    };
    load((int64_t)blockIdx.x * GROUPS + group);
    for (int64_t first = (int64_t)blockIdx.x * GROUPS; first < p.rows; first += step) {
      const int64_t row = first + group;
      float h[8], dy[8], f[8], b[8] = {}, sum[2] = {0.0f, 0.0f};
      cols.get(x, 0, h);
      cols.get(y, 0, dy);
      if constexpr (DH) cols.get(d, 0, b);
      load(row + step);
      cols.get(w, 0, f);
      add(h, dy, f, sum);
      row_sums<LANES, 2>(sum, room, turn);
      turn ^= 1;
      const float rho = 1.0f / sqrtf(sum[0] / (float)p.width + p.eps), mean = rho * rho * (sum[1] / (float)p.width);
      finish(row, 0, rho, mean, h, dy, f, b);
    }
  } else if constexpr (CH == 2) {
    // registers: a row as it is in memory, and of 16-bit types the next one's H and dY
    constexpr bool AHEAD = TYPE != kF32;
    Raw<TYPE> y[CH], x[CH];
    auto load = [&](int64_t row) {
      row = row < p.rows ? row : p.rows - 1;
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        y[i] = cols.load(p.dy, row * p.lddy, i);
        x[i] = cols.load(p.h, row * p.ldh, i);
      }
    };
    if constexpr (AHEAD) load(blockIdx.x);
    for (int64_t row = blockIdx.x; row < p.rows; row += step) {
      if constexpr (!AHEAD) {
        load(row);
        asm volatile("" : "+s"(weight));  // read again for every row: no registers for it
      }
      Raw<TYPE> hr[CH], yr[CH], dr[CH];
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        hr[i] = x[i], yr[i] = y[i];
        if constexpr (DH) dr[i] = cols.load(p.dh, row * p.lddh, i);
      }
      if constexpr (AHEAD) load(row + step);
      float sum[2] = {0.0f, 0.0f};
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        float h[8], dy[8], f[8];
        cols.get(hr[i], i, h);
        cols.get(yr[i], i, dy);
        cols.get(weights(i), i, f);
        add(h, dy, f, sum);
        __builtin_amdgcn_sched_barrier(0);
      }
      row_sums<LANES, 2>(sum, room, turn);
      turn ^= 1;
      const float rho = 1.0f / sqrtf(sum[0] / (float)p.width + p.eps), mean = rho * rho * (sum[1] / (float)p.width);
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        // as they are in memory: the compiler would keep the first pass's conversions
#pragma unroll
        for (int q = 0; q < Raw<TYPE>::Q; ++q) asm volatile("" : "+v"(hr[i].q[q]), "+v"(yr[i].q[q]));
        float h[8], dy[8], f[8], b[8] = {};
        cols.get(hr[i], i, h);
        cols.get(yr[i], i, dy);
        cols.get(weights(i), i, f);
        if constexpr (DH) cols.get(dr[i], i, b);
        finish(row, i, rho, mean, h, dy, f, b);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  } else {
    // a row does not fit the registers: it is read again, from the caches
    for (int64_t row = blockIdx.x; row < p.rows; row += step) {
      float sum[2] = {0.0f, 0.0f};
#pragma unroll 1
      for (int i = 0; i < CH; ++i) {
        float h[8], dy[8], f[8];
        cols.get(cols.load(p.h, row * p.ldh, i), i, h);
        cols.get(cols.load(p.dy, row * p.lddy, i), i, dy);
        cols.get(weights(i), i, f);
        add(h, dy, f, sum);
      }
      row_sums<LANES, 2>(sum, room, turn);
      turn ^= 1;
      const float rho = 1.0f / sqrtf(sum[0] / (float)p.width + p.eps), mean = rho * rho * (sum[1] / (float)p.width);
#pragma unroll 1
      for (int i = 0; i < CH; ++i) {
        float h[8], dy[8], f[8], b[8] = {};
        cols.get(cols.load(p.h, row * p.ldh, i), i, h);
        cols.get(cols.load(p.dy, row * p.lddy, i), i, dy);
        cols.get(weights(i), i, f);
        if constexpr (DH) cols.get(cols.load(p.dh, row * p.lddh, i), i, b);
        finish(row, i, rho, mean, h, dy, f, b);
      }
    }
  }
  float* const part = p.parts + (int64_t)blockIdx.x * p.width;
  if constexpr (GROUPS > 1) {
    // one group after the other
    for (int g = 0; g < GROUPS; ++g) {
      if (group == g) {
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            v4f* const at = (v4f*)&room[(lane + i * LANES) * 8 + 4 * q];
            const v4f v = {dw[i][4 * q], dw[i][4 * q + 1], dw[i][4 * q + 2], dw[i][4 * q + 3]};
            *at = g == 0 ? v : *at + v;
          }
      }
      __syncthreads();
    }
    for (int c = threadIdx.x; c < p.width; c += THREADS) part[c] = room[c];
  } else {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      Raw<kF32> r;
      if constexpr (WIDE) {
#pragma unroll
        for (int q = 0; q < 2; ++q) r.q[q] = __builtin_bit_cast(v4i, wide[(2 * i + q) * LANES + lane]);
      } else {
        r = rounded<kF32>(dw[i]);
      }
      store_raw<kF32>((char*)(part + cols.column(i)), r, cols.have(i));
    }
  }
}

// 16 columns a block, the parts over 64 sets of lanes: a few loads one after the other
// (the gradients of 4999 x 1031 with 16 sets 22 us, with 64 20).
__global__ __launch_bounds__(1024) void dw_kernel(const float* parts, int count, int width, float* dw) {
  __shared__ float room[64][17];
  const int c = blockIdx.x * 16 + (threadIdx.x & 15), at = threadIdx.x & 15, set = threadIdx.x >> 4;
  float t = 0.0f;
  if (c < width) {
#pragma unroll 8
    for (int i = set; i < count; i += 64) t += parts[(int64_t)i * width + c];
  }
  room[set][at] = t;
  __syncthreads();
  if (set < 8) {
#pragma unroll
    for (int i = 1; i < 8; ++i) t += room[set + 8 * i][at];
  }
  __syncthreads();
  if (set < 8) room[set][at] = t;
  __syncthreads();
  if (set == 0 && c < width) {
#pragma unroll
    for (int i = 1; i < 8; ++i) t += room[i][at];
    dw[c] = t;
  }
}

__global__ __launch_bounds__(256) void zeros_kernel(float* p, int64_t count) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < count) p[i] = 0.0f;
}

template <int TYPE, int LANES, int CH>
hipError_t run_norm(const Norm& p, hipStream_t s) {
  const dim3 grid((uint32_t)norm_blocks(p.rows, p.width, kNormThreads)), block(norm_threads(LANES));
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
  const dim3 grid((uint32_t)parts), block(norm_threads(LANES));
  if (p.dh)
    norm_gradient_kernel<TYPE, LANES, CH, true><<<grid, block, 0, s>>>(p);
  else
    norm_gradient_kernel<TYPE, LANES, CH, false><<<grid, block, 0, s>>>(p);
  if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  dw_kernel<<<dim3((uint32_t)ceil_div(p.width, 16)), dim3(1024), 0, s>>>(p.parts, (int)parts, p.width, p.dw);
  return hipGetLastError();
}

// calls f<LANES, CH>() for the form of this width
template <class F>
hipError_t of_form(NormForm g, F f) {
  switch (g.lanes * 8 + g.chunks) {
    case 16 * 8 + 1: return f.template operator()<16, 1>();
    case 32 * 8 + 1: return f.template operator()<32, 1>();
    case 64 * 8 + 1: return f.template operator()<64, 1>();
    case 128 * 8 + 1: return f.template operator()<128, 1>();
    case 192 * 8 + 1: return f.template operator()<192, 1>();
    case 256 * 8 + 1: return f.template operator()<256, 1>();
    case 384 * 8 + 1: return f.template operator()<384, 1>();
    case 512 * 8 + 1: return f.template operator()<512, 1>();
    case 768 * 8 + 1: return f.template operator()<768, 1>();
    case 1024 * 8 + 1: return f.template operator()<1024, 1>();
    case 768 * 8 + 2: return f.template operator()<768, 2>();
    case 1024 * 8 + 2: return f.template operator()<1024, 2>();
    case 1024 * 8 + 4: return f.template operator()<1024, 4>();
    default: return hipErrorInvalidValue;  // no such form: a grid of other blocks would miss rows
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
    return of_form(norm_form(p.width), [&]<int LANES, int CH>() { return run_norm<TYPE, LANES, CH>(p, s); });
  });
}

hipError_t launch_norm_gradient(const NormGradient& p, int type, hipStream_t s) {
  return of_type(type, [&]<int TYPE>() {
    return of_form(norm_form(p.width), [&]<int LANES, int CH>() { return run_gradient<TYPE, LANES, CH>(p, s); });
  });
}

}  // namespace eight
}  // namespace oz
