// Orthogonalisation of a stack of matrices by Newton-Schulz products:
//
//   X_0 = G / (|G|_F + eps);   S = X X^T,  P = b S + c S^2,  X <- a X + P X
//
// with the transposed form S = X^T X, X <- a X + X P for matrices of more rows
// than columns.  The polynomial a s + b s^3 + c s^5 acts on every singular
// value; a small one grows by a factor of up to a per step, and a rounding
// error of X with it, so X itself is kept in 32 bits from step to step: P X is
// the part that is formed from 16-bit operands, whose rounding errors come in
// multiplied by P, which is small where the singular values are.
//
// The operands X, S and P are IEEE half: their entries are bounded (|X| by the
// polynomial's largest value, S by its square), so powers of two place them
// in half's range, and its 11 bits round eight times finer than the bfloat16
// of the result.  Stored as X 2^8, S 2^10, P 2^8.
//
// Matrices are padded with zero rows and columns to multiples of 8 (zeros stay
// zeros through every step), so all loads are DMA.
#include "half_products.hpp"

namespace oz {
namespace half {
namespace {

constexpr float kScaleX = 256.0f, kScaleS = 1024.0f, kScaleP = 256.0f;

template <int TYPE>
__device__ __forceinline__ float to_float(const void* p, int64_t i) {
  using E = typename Out<TYPE>::type;
  return (float)((const E*)p)[i];
}

// Sums of squares of a matrix, one per block, in 64 bits: no overflow or
// underflow for any 32-bit input.  grid (blocks, count)
template <int TYPE>
__global__ __launch_bounds__(256) void squares_kernel(Orthogonalise o) {
  const int64_t total = (int64_t)o.m * o.n;
  const int64_t per = (total + gridDim.x - 1) / gridDim.x;
  const int64_t end = per * (blockIdx.x + 1) < total ? per * (blockIdx.x + 1) : total;
  double sum = 0;
  for (int64_t i = per * blockIdx.x + threadIdx.x; i < end; i += 256) {
    const int64_t r = i / o.n, c = i - r * o.n;
    const double x = to_float<TYPE>(o.g, blockIdx.y * o.g_stride + r * o.ldg + c);
    sum += x * x;
  }
  __shared__ double part[4];
  for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) o.squares[blockIdx.y * gridDim.x + blockIdx.x] = part[0] + part[1] + part[2] + part[3];
}

// X_0 in both forms, padding included.  grid (blocks, count)
template <int TYPE>
__global__ __launch_bounds__(256) void start_kernel(Orthogonalise o, int parts) {
  double sum = 0;
  for (int i = 0; i < parts; ++i) sum += o.squares[blockIdx.y * parts + i];
  const float scale = (float)(1.0 / (sqrt(sum) + (double)o.eps));
  const int64_t total = (int64_t)o.mp * o.np;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / o.np, c = i - r * o.np;
    float x = 0.0f;
    if (r < o.m && c < o.n) x = to_float<TYPE>(o.g, blockIdx.y * o.g_stride + r * o.ldg + c) * scale;
    o.x32[blockIdx.y * total + i] = x;
    ((_Float16*)o.x16[0])[blockIdx.y * total + i] = (_Float16)(x * kScaleX);
  }
}

// The tile of the upper triangle number t among tiles x tiles: column by
// column, tm <= tn.
__device__ __forceinline__ void triangle_tile(uint32_t t, uint32_t& tm, uint32_t& tn) {
  uint32_t c = (uint32_t)((sqrtf(8.0f * (float)t + 1.0f) - 1.0f) * 0.5f);
  while (c * (c + 1) / 2 > t) --c;
  while ((c + 1) * (c + 2) / 2 <= t) ++c;
  tn = c;
  tm = t - c * (c + 1) / 2;
}

// A symmetric product C = A A^T (kAlong, A s x depth) or A^T A (kAcross, A
// depth x s), the tiles on and above the diagonal, each stored twice.  With
// SQUARE, A = S and P = b S + c S^2 is stored.  grid (tiles, count)
template <class T, bool SQUARE>
__global__ __launch_bounds__(T::THREADS, 1) void gram_kernel(Orthogonalise o, const char* in, char* out, int s,
                                                            int depth, int64_t ld, float c) {
  __shared__ __attribute__((aligned(1024))) char lds[T::LDS];
  static_assert(T::BM == T::BN && T::LA == T::LB, "square tiles");
  uint32_t tm, tn;
  triangle_tile(blockIdx.x, tm, tn);
  const int r0 = (int)tm * T::BM, c0 = (int)tn * T::BN;
  const int rows = s - r0 < T::BM ? s - r0 : T::BM, cols = s - c0 < T::BN ? s - c0 : T::BN;
  const char* a = in + blockIdx.y * ((int64_t)o.mp * o.np * 2);
  if constexpr (SQUARE) a = in + blockIdx.y * ((int64_t)s * s * 2);
  const int64_t step = T::LA == kAlong ? ld : 1;
  v16f acc[T::MB][T::NB] = {};
  product<T>(Operand{a + r0 * step * 2, ld, rows, (int)ld}, Operand{a + c0 * step * 2, ld, cols, (int)ld}, depth, lds, acc);
  char* const o16 = out + blockIdx.y * ((int64_t)s * s * 2);
  const _Float16* const S = (const _Float16*)a;
  store_wide<T>(acc, lds, o16 + ((int64_t)r0 * s + c0) * 2, s, rows, cols, true, [&](int r, int q, float* v) {
    if constexpr (SQUARE) {
      const bool in = r < rows && q < cols;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float x = in ? (float)S[(int64_t)(r0 + r) * s + c0 + q + j] : 0.0f;
        v[j] = v[j] * c + x * (o.b * kScaleP / kScaleS);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] *= c;
    }
  });
  if (tm == tn) return;
  // the mirror image: the wavefront's blocks transposed, 32 rows at a time
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = wave / T::WC * T::MB * 32, wc = wave % T::WC * T::NB * 32;
  _Float16* const m16 = (_Float16*)o16 + (int64_t)(c0 + wc) * s + r0 + wr;
#pragma unroll
  for (int x = 0; x < T::MB; ++x)
#pragma unroll
    for (int y = 0; y < T::NB; ++y)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int r = x * 32 + (lane & 31), q = y * 32 + 8 * (i >> 2) + 4 * (lane >> 5) + (i & 3);
        if (wr + r < rows && wc + q < cols) {
          float v = acc[x][y][i] * c;
          if constexpr (SQUARE) v += (float)S[(int64_t)(r0 + wr + r) * s + c0 + wc + q] * (o.b * kScaleP / kScaleS);
          m16[(int64_t)q * s + r] = (_Float16)v;
        }
      }
}

// X <- a X + P X (WIDE_ matrices, kAlong x kAcross) or a X + X P (kAlong x
// kAlong: P is symmetric).  LAST: the result to the caller's matrix.
// grid (tiles, count)
template <class T, bool TALL, bool LAST>
__global__ __launch_bounds__(T::THREADS, 1) void update_kernel(Orthogonalise o, const char* x16, char* next) {
  __shared__ __attribute__((aligned(1024))) char lds[T::LDS];
  const int s = TALL ? o.np : o.mp;
  const uint32_t tiles_n = ((uint32_t)o.np + T::BN - 1) / T::BN;
  const int r0 = (int)(blockIdx.x / tiles_n) * T::BM, c0 = (int)(blockIdx.x % tiles_n) * T::BN;
  const int rows = o.mp - r0 < T::BM ? o.mp - r0 : T::BM, cols = o.np - c0 < T::BN ? o.np - c0 : T::BN;
  const int64_t each = (int64_t)o.mp * o.np;
  const char* const X = x16 + blockIdx.y * each * 2;
  const char* const P = (const char*)o.p16 + blockIdx.y * ((int64_t)s * s * 2);
  v16f acc[T::MB][T::NB] = {};
  if constexpr (TALL)
    product<T>(Operand{X + (int64_t)r0 * o.np * 2, o.np, rows, o.np}, Operand{P + (int64_t)c0 * s * 2, s, cols, s}, s, lds, acc);
  else
    product<T>(Operand{P + (int64_t)r0 * s * 2, s, rows, s}, Operand{X + (int64_t)c0 * 2, o.np, cols, o.np}, s, lds, acc);
  float* const x32 = o.x32 + blockIdx.y * each + (int64_t)r0 * o.np + c0;
  auto value = [&](int r, int q, float* v) {
    if (r < rows && q < cols) {
      float4* const p = (float4*)(x32 + (int64_t)r * o.np + q);
      const float4 x = *p;
      const float k = 1.0f / (kScaleX * kScaleP);
      v[0] = o.a * x.x + k * v[0];
      v[1] = o.a * x.y + k * v[1];
      v[2] = o.a * x.z + k * v[2];
      v[3] = o.a * x.w + k * v[3];
      if constexpr (!LAST) {
        *p = float4{v[0], v[1], v[2], v[3]};
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] *= kScaleX;
      }
    }
  };
  if constexpr (LAST)
    store_wide<T>(acc, lds, (char*)o.x + (blockIdx.y * o.x_stride + r0 * o.ldx + c0) * 2, o.ldx, o.m - r0, o.n - c0,
                  o.vec, value);
  else
    store_wide<T>(acc, lds, next + (blockIdx.y * each + (int64_t)r0 * o.np + c0) * 2, o.np, rows, cols, true, value);
}

template <int TYPE>
hipError_t start(const Orthogonalise& o, hipStream_t s) {
  const int64_t total = (int64_t)o.mp * o.np;
  const int parts = orthogonalise_parts(o.m, o.n);
  squares_kernel<TYPE><<<dim3(parts, o.count), dim3(256), 0, s>>>(o);
  const int blocks = (int)((total + 2047) / 2048 < 4096 ? (total + 2047) / 2048 : 4096);
  start_kernel<TYPE><<<dim3(blocks, o.count), dim3(256), 0, s>>>(o, parts);
  return hipGetLastError();
}

template <int WR, int WC, int MB, int NB>
hipError_t steps(const Orthogonalise& o, int steps, hipStream_t s) {
  const bool tall = o.m > o.n;
  const int sh = tall ? o.np : o.mp, lo = tall ? o.mp : o.np;
  using G0 = Tile<kF16, kAlong, kAlong, WR, WC, MB, NB, true, kF16>;
  using G1 = Tile<kF16, kAcross, kAcross, WR, WC, MB, NB, true, kF16>;
  const uint32_t t = (uint32_t)((sh + G0::BM - 1) / G0::BM);
  const dim3 tri(t * (t + 1) / 2, o.count), block(G0::THREADS);
  const dim3 all((uint32_t)((o.mp + G0::BM - 1) / G0::BM) * (uint32_t)((o.np + G0::BN - 1) / G0::BN), o.count);
  for (int i = 0; i < steps; ++i) {
    const char* x = (const char*)o.x16[i & 1];
    char* next = (char*)o.x16[(i + 1) & 1];
    const float cs = kScaleS / (kScaleX * kScaleX), cp = o.c * kScaleP / (kScaleS * kScaleS);
    if (tall)
      gram_kernel<G1, false><<<tri, block, 0, s>>>(o, x, (char*)o.s16, sh, lo, o.np, cs);
    else
      gram_kernel<G0, false><<<tri, block, 0, s>>>(o, x, (char*)o.s16, sh, lo, o.np, cs);
    gram_kernel<G0, true><<<tri, block, 0, s>>>(o, (const char*)o.s16, (char*)o.p16, sh, sh, sh, cp);
    const bool last = i + 1 == steps;
    using U0 = Tile<kF16, kAlong, kAcross, WR, WC, MB, NB, true, kF16>;
    using L0 = Tile<kF16, kAlong, kAcross, WR, WC, MB, NB, true, kBF16>;
    using L1 = Tile<kF16, kAlong, kAlong, WR, WC, MB, NB, true, kBF16>;
    if (tall && last)
      update_kernel<L1, true, true><<<all, block, 0, s>>>(o, x, next);
    else if (tall)
      update_kernel<G0, true, false><<<all, block, 0, s>>>(o, x, next);
    else if (last)
      update_kernel<L0, false, true><<<all, block, 0, s>>>(o, x, next);
    else
      update_kernel<U0, false, false><<<all, block, 0, s>>>(o, x, next);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_orthogonalise(Orthogonalise o, int type, int count_steps, hipStream_t s) {
  o.vec = (uintptr_t)o.x % 16 == 0 && o.ldx % 8 == 0 && o.x_stride % 8 == 0 && o.n % 8 == 0;
  hipError_t e = type == kBF16 ? start<kBF16>(o, s) : type == kF16 ? start<kF16>(o, s) : start<kF32>(o, s);
  if (e != hipSuccess) return e;
  const int64_t big = (int64_t)((o.mp + 255) / 256) * ((o.np + 255) / 256) * o.count;
  return big >= 256 ? steps<2, 4, 4, 2>(o, count_steps, s) : steps<2, 2, 2, 2>(o, count_steps, s);
}

}  // namespace half
}  // namespace oz
