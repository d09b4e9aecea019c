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
// S and P come close to multiples of the identity, and a rounding of their
// diagonals would be an error of every vector: the diagonals d and p are kept
// in 32 bits beside the matrices, whose own diagonals are stored as zeros, and
//   (S^2)_ij = (So^2)_ij + (d_i + d_j) So_ij,  (S^2)_ii = (So^2)_ii + d_i^2,
//   (P X)_ij = (Po X)_ij + p_i X_ij.
//
// Matrices are padded with zero rows and columns to multiples of 8 (zeros stay
// zeros through every step), so all loads are DMA.
#include "half_products.hpp"

namespace oz {
namespace half {
namespace {

constexpr float kScaleX = 256.0f, kScaleS = 1024.0f, kScaleP = 256.0f;

// Elements c .. c + 7 of a row of n; zeros past its end.
template <int TYPE>
__device__ __forceinline__ void row8(const void* g, int64_t row, int c, int n, float (&x)[8]) {
  if constexpr (TYPE == kF32) {
    const auto q = (const __attribute__((address_space(1))) float*)(global_bytes)g + row;
    if (__builtin_amdgcn_ballot_w64(c + 8 > n) == 0) {
      const char* const at = (const char*)g + (row + c) * 4;
      const float4 lo = __builtin_bit_cast(float4, load_whole(at)), hi = __builtin_bit_cast(float4, load_whole(at + 16));
      x[0] = lo.x, x[1] = lo.y, x[2] = lo.z, x[3] = lo.w, x[4] = hi.x, x[5] = hi.y, x[6] = hi.z, x[7] = hi.w;
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float v = q[c + j < n ? c + j : n - 1];
        x[j] = c + j < n ? v : 0.0f;
      }
    }
  } else {
    typedef typename Out<TYPE>::type v8 __attribute__((ext_vector_type(8)));
    const v8 v = __builtin_bit_cast(v8, load8((const char*)g + row * 2, c, n));
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = (float)v[j];
  }
}

// Sums of squares of a matrix, one per block, in 64 bits: no overflow or
// underflow for any 32-bit input.  grid (parts, count)
template <int TYPE>
__global__ __launch_bounds__(256) void squares_kernel(Orthogonalise o) {
  const uint32_t chunks = (uint32_t)o.np / 8, total = chunks * (uint32_t)o.m;
  double sum = 0;
#pragma unroll 4
  for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < total; i += gridDim.x * 256) {
    const uint32_t r = i / chunks, c = (i - r * chunks) * 8;
    float x[8];
    row8<TYPE>(o.g, blockIdx.y * o.g_stride + r * o.ldg, c, o.n, x);
#pragma unroll
    for (int j = 0; j < 8; ++j) sum += (double)x[j] * (double)x[j];
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
  for (int i = threadIdx.x & 63; i < parts; i += 64) sum += o.squares[blockIdx.y * parts + i];
  for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
  const float scale = (float)(1.0 / (sqrt(sum) + (double)o.eps));
  const uint32_t chunks = (uint32_t)o.np / 8, total = chunks * (uint32_t)o.mp;
  const int64_t each = (int64_t)o.mp * o.np;
  for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < total; i += gridDim.x * 256) {
    const uint32_t r = i / chunks, c = (i - r * chunks) * 8;
    float x[8] = {};
    if ((int)r < o.m) row8<TYPE>(o.g, blockIdx.y * o.g_stride + r * o.ldg, c, o.n, x);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = (int)(c + j) < o.n && (int)r < o.m ? x[j] * scale : 0.0f;
    float4* const p = (float4*)(o.x32 + blockIdx.y * each + (int64_t)i * 8);
    p[0] = float4{x[0], x[1], x[2], x[3]};
    p[1] = float4{x[4], x[5], x[6], x[7]};
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] *= kScaleX;
    const uint2 lo = pack4<kF16>(x[0], x[1], x[2], x[3]), hi = pack4<kF16>(x[4], x[5], x[6], x[7]);
    *(uint4*)((_Float16*)o.x16[0] + blockIdx.y * each + (int64_t)i * 8) = uint4{lo.x, lo.y, hi.x, hi.y};
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

// The wavefront's place in a WIDE tile: a lane holds, of block (a, b), row
// row0 + 32 a and the columns col0 + 32 b + 8 q .. + 3.
template <class T>
struct WidePlace {
  int row0, col0;
  __device__ __forceinline__ WidePlace() {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    row0 = wave / T::WC * T::MB * 32 + (lane & 31);
    col0 = wave % T::WC * T::NB * 32 + 4 * (lane >> 5);
  }
};

// A symmetric product A A^T (kAlong, A s x depth) or A^T A (kAcross, A
// depth x s), the tiles on and above the diagonal, each stored twice: S, or with
// SQUARE (A = So) P = b S + c S^2, their diagonals apart.  Block b takes the
// (b / sub^2)-th tile from `first` on, of the matrices' triangles of tiles one
// after the other, or its b % sub^2-th part where tiles of sub^2 times this size
// are meant.
template <class T, bool SQUARE>
__global__ __launch_bounds__(T::THREADS, 1) void gram_kernel(Orthogonalise o, const char* in, int s, int depth,
                                                            int64_t ld, uint32_t first, uint32_t sub) {
  __shared__ __attribute__((aligned(1024))) char lds[T::LDS];
  static_assert(T::BM == T::BN && T::LA == T::LB && T::OUT == kF16, "square tiles");
  const uint32_t side = ((uint32_t)s + T::BM * sub - 1) / (T::BM * sub), triangle = side * (side + 1) / 2;
  const uint32_t tile = first + blockIdx.x / (sub * sub), part = blockIdx.x % (sub * sub);
  const uint32_t z = tile / triangle;
  uint32_t tm, tn;
  triangle_tile(tile - z * triangle, tm, tn);
  tm = tm * sub + part / sub;
  tn = tn * sub + part % sub;
  const int r0 = (int)tm * T::BM, c0 = (int)tn * T::BN;
  if (tm > tn || c0 >= s) return;  // parts below the diagonal or past the edge
  const int rows = s - r0 < T::BM ? s - r0 : T::BM, cols = s - c0 < T::BN ? s - c0 : T::BN;
  const int64_t square = (int64_t)s * s;
  const char* const a = in + z * (SQUARE ? square : (int64_t)o.mp * o.np) * 2;
  _Float16* const out = (_Float16*)(SQUARE ? o.p16 : o.s16) + z * square + (int64_t)r0 * s + c0;
  const float* const d = o.d32 + (int64_t)z * s;
  float* const diagonal = (SQUARE ? o.p32 : o.d32) + (int64_t)z * s;
  const int64_t step = T::LA == kAlong ? ld : 1;
  const WidePlace<T> w;
  // So of the tile's own outputs, from clamped places and without a branch, so
  // that all loads are in flight; before the product where registers allow
  constexpr bool EARLY = T::MB * T::NB <= 4;
  const _Float16* const S = (const _Float16*)a + (int64_t)r0 * s + c0;
  uint2 own[EARLY ? T::MB : 1][T::NB][4];
  auto load_own = [&](int x, uint2 (&v)[T::NB][4]) __attribute__((always_inline)) {
    const int r = w.row0 + 32 * x < rows ? w.row0 + 32 * x : rows - 1;
#pragma unroll
    for (int b = 0; b < T::NB; ++b)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int c = w.col0 + 32 * b + 8 * q;
        v[b][q] = *(const uint2*)(S + (int64_t)r * s + (c < cols ? c : 0));
      }
  };
  if constexpr (SQUARE && EARLY) {
#pragma unroll
    for (int x = 0; x < T::MB; ++x) load_own(x, own[x]);
  }
  v16f acc[T::MB][T::NB] = {};
  product<T>(Operand{a + r0 * step * 2, ld, rows, (int)ld}, Operand{a + c0 * step * 2, ld, cols, (int)ld}, depth, lds,
             acc);
  if constexpr (SQUARE) {
    const float ks = kScaleP / kScaleS, kc = o.c * kScaleP / (kScaleS * kScaleS);
    float4 dc[T::NB][4];
#pragma unroll
    for (int b = 0; b < T::NB; ++b)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int c = w.col0 + 32 * b + 8 * q;
        dc[b][q] = *(const float4*)(d + c0 + (c < cols ? c : 0));
      }
#pragma unroll
    for (int x = 0; x < T::MB; ++x) {
      const float di = d[r0 + (w.row0 + 32 * x < rows ? w.row0 + 32 * x : rows - 1)];
      if constexpr (!EARLY) load_own(x, own[0]);
#pragma unroll
      for (int b = 0; b < T::NB; ++b)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          typedef _Float16 h4 __attribute__((ext_vector_type(4)));
          const h4 e = __builtin_bit_cast(h4, own[EARLY ? x : 0][b][q]);
          const float dj[4] = {dc[b][q].x, dc[b][q].y, dc[b][q].z, dc[b][q].w};
#pragma unroll
          for (int j = 0; j < 4; ++j)
            acc[x][b][4 * q + j] = kc * acc[x][b][4 * q + j] + (o.b + o.c * (di + dj[j])) * ks * (float)e[j];
        }
    }
  } else {
#pragma unroll
    for (int x = 0; x < T::MB; ++x)
#pragma unroll
      for (int b = 0; b < T::NB; ++b) acc[x][b] *= kScaleS / (kScaleX * kScaleX);
  }
  if (tm == tn) {
#pragma unroll
    for (int x = 0; x < T::MB; ++x)
#pragma unroll
      for (int b = 0; b < T::NB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int r = w.row0 + 32 * x;
          if (r != w.col0 + 32 * b + 8 * (i >> 2) + (i & 3)) continue;
          if (r < rows) {
            // acc: S_ii 2^10, or c (So^2)_ii 2^8 (So_ii is zero)
            if constexpr (SQUARE) {
              const float di = d[r0 + r];
              diagonal[r0 + r] = (o.b + o.c * di) * di + acc[x][b][i] * (1.0f / kScaleP);
            } else {
              diagonal[r0 + r] = acc[x][b][i] * (1.0f / kScaleS);
            }
          }
          acc[x][b][i] = 0.0f;
        }
  }
  store_wide<T>(acc, lds, out, s, rows, cols, true, false, [](int, int, float*) {});
  if (tm == tn) return;
  // the mirror image: a half wavefront has 32 consecutive rows of one column
  _Float16* const mirror = (_Float16*)(SQUARE ? o.p16 : o.s16) + z * square + (int64_t)c0 * s + r0;
#pragma unroll
  for (int x = 0; x < T::MB; ++x)
#pragma unroll
    for (int b = 0; b < T::NB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int r = w.row0 + 32 * x, c = w.col0 + 32 * b + 8 * (i >> 2) + (i & 3);
        if (r < rows && c < cols) mirror[(int64_t)c * s + r] = (_Float16)acc[x][b][i];
      }
}

// X <- a X + P X (kAlong x kAcross) or, TALL, a X + X P (kAlong x kAlong: P is
// symmetric).  LAST: the result to the caller's matrix.  grid (tiles, count)
template <class T, bool TALL, bool LAST>
__global__ __launch_bounds__(T::THREADS, 1) void update_kernel(Orthogonalise o, const char* x16, char* next) {
  __shared__ __attribute__((aligned(1024))) char lds[T::LDS];
  const int s = TALL ? o.np : o.mp;
  const uint32_t tiles_n = ((uint32_t)o.np + T::BN - 1) / T::BN, tiles_m = ((uint32_t)o.mp + T::BM - 1) / T::BM;
  uint32_t place, tm, tn;
  if (!block_place(blockIdx.x, tiles_m * tiles_n, place)) return;
  place_to_tile(place, tiles_m, tiles_n, tm, tn);
  const int r0 = (int)tm * T::BM, c0 = (int)tn * T::BN;
  const int rows = o.mp - r0 < T::BM ? o.mp - r0 : T::BM, cols = o.np - c0 < T::BN ? o.np - c0 : T::BN;
  const int64_t each = (int64_t)o.mp * o.np;
  const char* const X = x16 + blockIdx.y * each * 2;
  const char* const P = (const char*)o.p16 + blockIdx.y * ((int64_t)s * s * 2);
  const float* const p = o.p32 + (int64_t)blockIdx.y * s;
  float* const x32 = o.x32 + blockIdx.y * each + (int64_t)r0 * o.np + c0;
  const WidePlace<T> w;
  constexpr bool EARLY = T::MB * T::NB <= 4;
  float4 own[EARLY ? T::MB : 1][T::NB][4];
  auto load_own = [&](int x, float4 (&v)[T::NB][4]) __attribute__((always_inline)) {
    const int r = w.row0 + 32 * x < rows ? w.row0 + 32 * x : rows - 1;
#pragma unroll
    for (int b = 0; b < T::NB; ++b)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int c = w.col0 + 32 * b + 8 * q;
        v[b][q] = *(const float4*)(x32 + (int64_t)r * o.np + (c < cols ? c : 0));
      }
  };
  if constexpr (EARLY) {
#pragma unroll
    for (int x = 0; x < T::MB; ++x) load_own(x, own[x]);
  }
  v16f acc[T::MB][T::NB] = {};
  if constexpr (TALL)
    product<T>(Operand{X + (int64_t)r0 * o.np * 2, o.np, rows, o.np}, Operand{P + (int64_t)c0 * s * 2, s, cols, s}, s,
               lds, acc);
  else
    product<T>(Operand{P + (int64_t)r0 * s * 2, s, rows, s}, Operand{X + (int64_t)c0 * 2, o.np, cols, o.np}, s, lds,
               acc);
  const float k = 1.0f / (kScaleX * kScaleP);
#pragma unroll
  for (int x = 0; x < T::MB; ++x) {
    const int r = w.row0 + 32 * x < rows ? w.row0 + 32 * x : rows - 1;
    const float pi = TALL ? 0.0f : p[r0 + r];
    if constexpr (!EARLY) load_own(x, own[0]);
#pragma unroll
    for (int b = 0; b < T::NB; ++b)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int c = w.col0 + 32 * b + 8 * q;
        const float4 v = own[EARLY ? x : 0][b][q];
        const float4 pj = TALL ? *(const float4*)(p + c0 + (c < cols ? c : 0)) : float4{pi, pi, pi, pi};
        float4 y;
        y.x = (o.a + pj.x) * v.x + k * acc[x][b][4 * q];
        y.y = (o.a + pj.y) * v.y + k * acc[x][b][4 * q + 1];
        y.z = (o.a + pj.z) * v.z + k * acc[x][b][4 * q + 2];
        y.w = (o.a + pj.w) * v.w + k * acc[x][b][4 * q + 3];
        if constexpr (!LAST)
          if (w.row0 + 32 * x < rows && c < cols) *(float4*)(x32 + (int64_t)r * o.np + c) = y;
        const float scale = LAST ? 1.0f : kScaleX;
        acc[x][b][4 * q] = y.x * scale;
        acc[x][b][4 * q + 1] = y.y * scale;
        acc[x][b][4 * q + 2] = y.z * scale;
        acc[x][b][4 * q + 3] = y.w * scale;
      }
  }
  auto as_is = [](int, int, float*) {};
  if constexpr (LAST)
    store_wide<T>(acc, lds, (char*)o.x + (blockIdx.y * o.x_stride + r0 * o.ldx + c0) * 2, o.ldx, o.m - r0, o.n - c0,
                  o.vec, true, as_is);
  else
    store_wide<T>(acc, lds, next + (blockIdx.y * each + (int64_t)r0 * o.np + c0) * 2, o.np, rows, cols, true, false, as_is);
}

template <int TYPE>
hipError_t start(const Orthogonalise& o, hipStream_t s) {
  const int parts = orthogonalise_parts(o.m, o.n);
  squares_kernel<TYPE><<<dim3(parts, o.count), dim3(256), 0, s>>>(o);
  const int64_t chunks = (int64_t)o.mp * o.np / 8, blocks = ceil_div(chunks, 256);
  start_kernel<TYPE><<<dim3((uint32_t)(blocks < 2048 ? blocks : 2048), o.count), dim3(256), 0, s>>>(o, parts);
  return hipGetLastError();
}

// tile shapes: WR, WC, MB, NB, stages
template <int WR, int WC, int MB, int NB, int BUFS>
struct Shape {
  template <int LA, int LB, int OUT>
  using Of = Tile<kF16, LA, LB, WR, WC, MB, NB, true, OUT, BUFS>;
};
using Large = Shape<2, 4, 4, 2, 2>;
using Middle = Shape<2, 2, 2, 2, 2>;
using Small = Shape<2, 2, 1, 1, 4>;

// `tiles` tiles of sub times the shape's side, from `first` on
template <class H, int L, bool SQUARE>
void gram(const Orthogonalise& o, const char* in, int s, int depth, int64_t ld, int64_t first, int64_t tiles, int sub,
          hipStream_t st) {
  using T = typename H::template Of<L, L, kF16>;
  gram_kernel<T, SQUARE><<<dim3((uint32_t)(tiles * sub * sub)), dim3(T::THREADS), 0, st>>>(
      o, in, s, depth, ld, (uint32_t)first, (uint32_t)sub);
}

template <int L, bool SQUARE>
void gram(const Orthogonalise& o, const char* in, int s, int depth, int64_t ld, hipStream_t st) {
  auto tiles = [&](int64_t b) { return o.count * ceil_div(s, b) * (ceil_div(s, b) + 1) / 2; };
  const int64_t large = tiles(256), over = large_tiles_over(large);
  if (over > 0) {
    gram<Large, L, SQUARE>(o, in, s, depth, ld, 0, large - over, 1, st);
    return gram<Small, L, SQUARE>(o, in, s, depth, ld, large - over, over, 4, st);
  }
  switch (tile_of(tiles(128), large)) {
    case kSmallTile: return gram<Small, L, SQUARE>(o, in, s, depth, ld, 0, tiles(64), 1, st);
    case kMiddleTile: return gram<Middle, L, SQUARE>(o, in, s, depth, ld, 0, tiles(128), 1, st);
    default: return gram<Large, L, SQUARE>(o, in, s, depth, ld, 0, large, 1, st);
  }
}

template <class H, bool TALL, bool LAST>
void update(const Orthogonalise& o, const char* x, char* next, hipStream_t st) {
  using T = typename H::template Of<kAlong, TALL ? kAlong : kAcross, LAST ? kBF16 : kF16>;
  const int64_t tiles = ceil_div(o.mp, T::BM) * ceil_div(o.np, T::BN);
  update_kernel<T, TALL, LAST><<<dim3((uint32_t)((tiles + 7) & ~(int64_t)7), o.count), dim3(T::THREADS), 0, st>>>(o, x, next);
}

template <bool TALL, bool LAST>
void update(const Orthogonalise& o, const char* x, char* next, hipStream_t st) {
  auto tiles = [&](int64_t b) { return o.count * ceil_div(o.mp, b) * ceil_div(o.np, b); };
  switch (tile_of(tiles(128), tiles(256))) {
    case kSmallTile: return update<Small, TALL, LAST>(o, x, next, st);
    case kMiddleTile: return update<Middle, TALL, LAST>(o, x, next, st);
    default: return update<Large, TALL, LAST>(o, x, next, st);
  }
}

template <bool TALL>
hipError_t steps(const Orthogonalise& o, int count, hipStream_t st) {
  const int s = TALL ? o.np : o.mp, l = TALL ? o.mp : o.np;
  for (int i = 0; i < count; ++i) {
    const char* x = (const char*)o.x16[i & 1];
    char* next = (char*)o.x16[(i + 1) & 1];
    gram<TALL ? kAcross : kAlong, false>(o, x, s, l, o.np, st);
    gram<kAlong, true>(o, (const char*)o.s16, s, s, s, st);
    if (i + 1 < count)
      update<TALL, false>(o, x, next, st);
    else
      update<TALL, true>(o, x, next, st);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_orthogonalise(Orthogonalise o, int type, int count_steps, hipStream_t s) {
  o.vec = (uintptr_t)o.x % 16 == 0 && o.ldx % 8 == 0 && o.x_stride % 8 == 0 && o.n % 8 == 0;
  const hipError_t e = type == kBF16 ? start<kBF16>(o, s) : type == kF16 ? start<kF16>(o, s) : start<kF32>(o, s);
  if (e != hipSuccess) return e;
  return o.m > o.n ? steps<true>(o, count_steps, s) : steps<false>(o, count_steps, s);
}

}  // namespace half
}  // namespace oz
