// A shared projection with low-rank adapters of many requests at once:
//
//   Y[t, :] = X[t, :] W^T + s_a (X[t, :] A_a^T) B_a^T,   a = ids[t]
//
// Two launches.  The first forms H[t, :] = X[t, :] A_a^T, partial sums of a
// split depth, in FP32.  The second runs the projection's tiles and, before a
// tile is stored, adds for each adapter that its rows name the product of
// those rows of H with that adapter's B_a: the projection's
// output is written once and never read.  s_a H goes into that product as
// two 16-bit numbers, its rounded value and the rest, so that H keeps at least
// 16 bits and the rounding of the output stays the only one that shows.
#include "half_products.hpp"
#include "ozaki25.h"

namespace oz {
namespace half {
namespace {

// The least adapter above `after` among `count` ids (at most 64 N) in LDS;
// `adapters` where there is none.  Ids outside [0, adapters) name none.
template <int N>
__device__ __forceinline__ int next_adapter(const int* ids, int count, int after, int adapters) {
  const int lane = threadIdx.x & 63;
  int least = adapters;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int t = i * 64 + lane;
    const int a = t < count ? ids[t] : -1;
    least = a > after && a < least ? a : least;
  }
  // the minimum, as the maximum of what is missing to `adapters`
  const int most = scan64(adapters - least, [](int a, int b) { return a > b ? a : b; });
  return adapters - __builtin_amdgcn_readlane(most, 63);
}

// H partial sums.  A block: TB tiles of 16 rows, 16 RB ranks, one part of the
// depth split again over its four wavefronts, the adapters of its rows in
// turn (every gridDim.y-th).  grid (row tiles, adapter slots, splits x rank
// chunks)
template <int TYPE, int RB, int TB>
__global__ __launch_bounds__(256) void shrink_kernel(Adapter p) {
  constexpr int ROWS = 16 * TB;
  __shared__ int ids[64];
  __shared__ float part[4][TB][RB][16][17];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int t0 = blockIdx.x * ROWS;
  const int rows = p.rows - t0 < ROWS ? p.rows - t0 : ROWS;
  const int split = blockIdx.z % p.splits, rank0 = blockIdx.z / p.splits * (16 * RB);
  if (threadIdx.x < ROWS) ids[threadIdx.x] = (int)threadIdx.x < rows ? p.ids[t0 + threadIdx.x] : -1;
  __syncthreads();
  // whole K steps of 32: this wavefront's range
  const int steps = (p.k + 31) / 32, q = split * 4 + wave;
  const int s0 = (int)((int64_t)steps * q / (p.splits * 4)), s1 = (int)((int64_t)steps * (q + 1) / (p.splits * 4));
  const int row = lane & 15, half = lane >> 4;
  int a = -1;
  for (uint32_t slot = 0;; ++slot) {
    a = next_adapter<1>(ids, ROWS, a, p.adapters);
    if (a == p.adapters) break;
    if (slot % gridDim.y != blockIdx.y) continue;
    v4f acc[RB][TB] = {};
    const char* const A = (const char*)p.a + (int64_t)a * p.a_stride * 2;
    for (int s = s0; s < s1; ++s) {
      const int c = s * 32 + half * 8;
      v4i fa[RB], fx[TB];
#pragma unroll
      for (int i = 0; i < RB; ++i) {
        const int r = rank0 + i * 16 + row;
        fa[i] = r < p.rank ? load8(A + (int64_t)r * p.lda * 2, c, p.k) : v4i{};
      }
#pragma unroll
      for (int j = 0; j < TB; ++j) {
        const int t = j * 16 + row;
        fx[j] = t < rows && ids[t] == a ? load8((const char*)p.x + (t0 + t) * p.ldx * 2, c, p.k) : v4i{};
      }
#pragma unroll
      for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int j = 0; j < TB; ++j) acc[i][j] = mfma16<TYPE>(fa[i], fx[j], acc[i][j]);
    }
    // lane l of a 16 x 16 block: row tile's row l % 16, ranks 4 (l / 16) .. + 3
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
      for (int j = 0; j < TB; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) part[wave][j][i][row][half * 4 + e] = acc[i][j][e];
    __syncthreads();
    for (int o = threadIdx.x; o < TB * 16 * RB * 16; o += 256) {
      const int r = o % (RB * 16), t = o / (RB * 16);
      if (t < rows && ids[t] == a && rank0 + r < p.rank_pad) {
        float v = 0;
#pragma unroll
        for (int w = 0; w < 4; ++w) v += part[w][t >> 4][r >> 4][t & 15][r & 15];
        p.h[((int64_t)split * p.rows + t0 + t) * p.rank_pad + rank0 + r] = v;
      }
    }
    __syncthreads();
  }
}

// The adapters' share of a tile, added to its sums.  ids: the tile's rows.
template <class T>
__device__ __forceinline__ void expand(const Adapter& p, int r0, int rows, int c0, int cols, const int* ids, char* lds,
                                       v16f (&acc)[T::MB][T::NB]) {
  static_assert(T::LA == kAlong && T::LB == kAlong && T::BM <= 256);
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Fragments<kAlong, T::BM, T::MB> fa;
  Fragments<kAlong, T::BN, T::NB> fb;
  fa.init(wave / T::WC * T::MB, lane);
  fb.init(wave % T::WC * T::NB, lane);
  using O = typename Out<T::TYPE>::type;
  typedef O v8o __attribute__((ext_vector_type(8)));
  const int depth = 2 * p.rank_pad;  // the rounded values, then the rests
  int a = -1;
  for (;;) {
    a = next_adapter<T::BM / 64>(ids, rows, a, p.adapters);
    if (a == p.adapters) break;
    const float scale = p.scales ? p.scales[a] : 1.0f;
    const char* const B = (const char*)p.b + ((int64_t)a * p.b_stride + (int64_t)c0 * p.ldb) * 2;
    for (int d0 = 0; d0 < depth; d0 += kDepth) {
      const int chunks = (depth - d0 < kDepth ? depth - d0 : kDepth) / 8;
      for (int o = threadIdx.x; o < T::BM * chunks; o += T::THREADS) {
        const int r = o / chunks, c = o - r * chunks, d = d0 + c * 8;
        const bool rest = d >= p.rank_pad;
        v8o e{};
        if (r < rows && ids[r] == a) {
          const float* h = p.h + (int64_t)(r0 + r) * p.rank_pad + (rest ? d - p.rank_pad : d);
          float v[8] = {};
          for (int s = 0; s < p.splits; ++s) {
            const float4 x = *(const float4*)h, y = *(const float4*)(h + 4);
            v[0] += x.x, v[1] += x.y, v[2] += x.z, v[3] += x.w;
            v[4] += y.x, v[5] += y.y, v[6] += y.z, v[7] += y.w;
            h += (int64_t)p.rows * p.rank_pad;
          }
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float x = v[j] * scale;
            const O hi = (O)x;
            // an overflowing value has no rest: it stays an infinity
            e[j] = !rest ? hi : __builtin_isfinite((float)hi) ? (O)(x - (float)hi) : (O)0.0f;
          }
        }
        *(v4i*)(lds + r * 128 + ((c ^ swz_along(r)) << 4)) = __builtin_bit_cast(v4i, e);
      }
      for (int o = threadIdx.x; o < T::BN * chunks; o += T::THREADS) {
        const int v = o / chunks, c = o - v * chunks, d = d0 + c * 8;
        const int r = d >= p.rank_pad ? d - p.rank_pad : d;
        v4i e{};
        if (v < cols) e = load8(B + (int64_t)v * p.ldb * 2, r, p.rank);
        *(v4i*)(lds + T::A_BYTES + v * 128 + ((c ^ swz_along(v)) << 4)) = e;
      }
      __syncthreads();
      // a lane's outputs of a block lie in one row: it takes the sums where
      // that row names this adapter (a product with zeros instead would pass
      // on an infinity of this adapter's B)
#pragma unroll
      for (int x = 0; x < T::MB; ++x) {
        const bool mine = ids[(wave / T::WC * T::MB + x) * 32 + (lane & 31)] == a;
        v4i xa[kDepth / 16];
#pragma unroll
        for (int ks = 0; ks < kDepth / 16; ++ks) xa[ks] = ks * 2 < chunks ? fa.read((lds_bytes)lds, ks, x) : v4i{};
#pragma unroll
        for (int y = 0; y < T::NB; ++y) {
          v16f t{};
#pragma unroll
          for (int ks = 0; ks < kDepth / 16; ++ks)
            if (ks * 2 < chunks) t = mfma<T::TYPE>(fb.read((lds_bytes)lds + T::A_BYTES, ks, y), xa[ks], t);
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[x][y][i] += mine ? t[i] : 0.0f;
        }
      }
      __syncthreads();
    }
  }
}

template <class T>
__global__ __launch_bounds__(T::THREADS, 1) void adapter_kernel(Adapter p) {
  __shared__ __attribute__((aligned(1024))) char lds[T::LDS];
  __shared__ int ids[T::BM];
  const uint32_t tiles_n = ((uint32_t)p.n + T::BN - 1) / T::BN, tiles_m = ((uint32_t)p.rows + T::BM - 1) / T::BM;
  uint32_t place, tm, tn;
  if (!block_place(blockIdx.x, tiles_m * tiles_n, place)) return;
  place_to_tile(place, tiles_m, tiles_n, tm, tn);
  const int r0 = (int)tm * T::BM, c0 = (int)tn * T::BN;
  const int rows = p.rows - r0 < T::BM ? p.rows - r0 : T::BM, cols = p.n - c0 < T::BN ? p.n - c0 : T::BN;
  for (int i = threadIdx.x; i < T::BM; i += T::THREADS) ids[i] = i < rows ? p.ids[r0 + i] : -1;
  v16f acc[T::MB][T::NB] = {};
  product<T>(Operand{(const char*)p.x + r0 * p.ldx * 2, p.ldx, rows, p.k}, Operand{(const char*)p.w + c0 * p.ldw * 2, p.ldw, cols, p.k},
             p.k, lds, acc);
  __syncthreads();
  if (p.rank > 0) expand<T>(p, r0, rows, c0, cols, ids, lds, acc);
  store<T>(acc, lds, (char*)p.y + (r0 * p.ldy + c0) * 2, p.ldy, rows, cols, p.vec);
}

// ---- few rows (serving): the weights are read once ------------------------------
// First launch: the projection's partial sums over parts of the depth, and
// beside them H[t, :], a block per row, 16 ranks and part.
constexpr int kServeWaves = 4;

template <int TYPE, int NB, int TB>
__global__ __launch_bounds__(kServeWaves * 64) void serve_partials_kernel(Adapter p, uint32_t shrink_blocks,
                                                                          uint32_t tiles_n) {
  __shared__ v4f lds[kServeWaves * TB * 16 * NB * 4];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int steps = (p.k + 31) / 32;
  auto range = [&](int part, int parts, int& s0, int& s1) {
    const int q = part * kServeWaves + wave;
    s0 = (int)((int64_t)steps * q / (parts * kServeWaves));
    s1 = (int)((int64_t)steps * (q + 1) / (parts * kServeWaves));
  };
  int s0, s1;
  if (blockIdx.x < shrink_blocks) {
    const uint32_t chunks = (uint32_t)p.rank_pad / 16;
    const int t = (int)(blockIdx.x / (chunks * p.splits)), in = (int)(blockIdx.x % (chunks * p.splits));
    const int chunk = in % chunks, split = in / chunks;
    const int a = p.ids[t];
    if (a < 0 || a >= p.adapters) return;
    const int ranks = p.rank - chunk * 16 < 16 ? p.rank - chunk * 16 : 16;
    range(split, p.splits, s0, s1);
    v4f acc[1][1] = {};
    skinny<TYPE, 1, 1>((const char*)p.a + ((int64_t)a * p.a_stride + chunk * 16 * p.lda) * 2, p.lda, ranks,
                       (const char*)p.x + t * p.ldx * 2, p.ldx, 1, p.k, s0, s1, acc);
    skinny_join<1, 1, kServeWaves>(acc, lds, [&](int row, int r, v4f v) {
      if (row > 0) return;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        p.h[((int64_t)split * p.rows + t) * p.rank_pad + chunk * 16 + r + e] = r + e < ranks ? v[e] : 0.0f;
    });
    return;
  }
  const uint32_t place = blockIdx.x - shrink_blocks, per = tiles_n * p.base_splits;
  const int t0 = (int)(place / per) * (16 * TB), in = (int)(place % per);
  const int split = in % p.base_splits, c0 = in / p.base_splits * (16 * NB);
  const int rows = p.rows - t0 < 16 * TB ? p.rows - t0 : 16 * TB, cols = p.n - c0 < 16 * NB ? p.n - c0 : 16 * NB;
  range(split, p.base_splits, s0, s1);
  v4f acc[NB][TB] = {};
  skinny<TYPE, NB, TB>((const char*)p.w + c0 * p.ldw * 2, p.ldw, cols, (const char*)p.x + t0 * p.ldx * 2, p.ldx, rows,
                       p.k, s0, s1, acc);
  float* const out = p.partials + (int64_t)split * p.rows * p.n_pad;
  skinny_join<NB, TB, kServeWaves>(acc, lds, [&](int row, int c, v4f v) {
    if (row < rows && c < cols) *(v4f*)(out + (int64_t)(t0 + row) * p.n_pad + c0 + c) = v;  // n_pad: a multiple of 4
  });
}

// Second launch: the partial sums in their order, then the row's adapter: a
// thread per output, s_a H and the sum over the ranks in FP32.
// grid (columns / 256, rows)
template <int TYPE>
__global__ __launch_bounds__(256) void serve_join_kernel(Adapter p) {
  using O = typename Out<TYPE>::type;
  typedef O v8o __attribute__((ext_vector_type(8)));
  __shared__ float h[OZAKI25_MAX_RANK];
  const int t = blockIdx.y, c = blockIdx.x * 256 + threadIdx.x;
  const int a = p.rank > 0 ? p.ids[t] : -1;
  const bool any = a >= 0 && a < p.adapters;
  if (any && (int)threadIdx.x < p.rank_pad) {
    float v = 0;
    for (int s = 0; s < p.splits; ++s) v += p.h[((int64_t)s * p.rows + t) * p.rank_pad + threadIdx.x];
    h[threadIdx.x] = v * (p.scales ? p.scales[a] : 1.0f);
  }
  float y = 0;
  if (c < p.n)
    for (int s = 0; s < p.base_splits; ++s) y += p.partials[((int64_t)s * p.rows + t) * p.n_pad + c];
  __syncthreads();
  if (c >= p.n) return;
  if (any) {
    const char* const B = (const char*)p.b + ((int64_t)a * p.b_stride + (int64_t)c * p.ldb) * 2;
    for (int r = 0; r < p.rank; r += 8) {
      const v8o b = __builtin_bit_cast(v8o, load8(B, r, p.rank));
#pragma unroll
      for (int e = 0; e < 8; ++e) y += h[r + e] * (float)b[e];
    }
  }
  ((O*)p.y)[(int64_t)t * p.ldy + c] = (O)y;
}

template <int TYPE, int NB, int TB>
hipError_t serve_tiles(const Adapter& p, hipStream_t s) {
  const uint32_t tiles_n = (uint32_t)(p.n + 16 * NB - 1) / (16 * NB), tiles_t = (uint32_t)(p.rows + 16 * TB - 1) / (16 * TB);
  const uint32_t shrinks = p.rank > 0 ? (uint32_t)p.rows * (p.rank_pad / 16) * p.splits : 0;
  serve_partials_kernel<TYPE, NB, TB><<<dim3(shrinks + tiles_n * tiles_t * p.base_splits), dim3(kServeWaves * 64), 0, s>>>(
      p, shrinks, tiles_n);
  serve_join_kernel<TYPE><<<dim3((p.n + 255) / 256, p.rows), dim3(256), 0, s>>>(p);
  return hipGetLastError();
}

template <int TYPE>
hipError_t serve(const Adapter& p, hipStream_t s) {
  if (p.rows <= 16) return serve_tiles<TYPE, 4, 1>(p, s);
  if (p.rows <= 32) return serve_tiles<TYPE, 4, 2>(p, s);
  return serve_tiles<TYPE, 4, 4>(p, s);
}

template <class T>
hipError_t run(const Adapter& p, hipStream_t s) {
  const int64_t tiles = (int64_t)((p.rows + T::BM - 1) / T::BM) * ((p.n + T::BN - 1) / T::BN);
  if (tiles * T::THREADS >= ((int64_t)1 << 32)) return hipErrorInvalidConfiguration;
  adapter_kernel<T><<<dim3((uint32_t)((tiles + 7) & ~(int64_t)7)), dim3(T::THREADS), 0, s>>>(p);
  return hipGetLastError();
}

template <int TYPE, int RB>
hipError_t shrink(const Adapter& p, hipStream_t s) {
  const uint32_t chunks = (uint32_t)(p.rank + 16 * RB - 1) / (16 * RB);
  if (p.rows <= 256)
    shrink_kernel<TYPE, RB, 1><<<dim3((p.rows + 15) / 16, 16, p.splits * chunks), dim3(256), 0, s>>>(p);
  else
    shrink_kernel<TYPE, RB, 4><<<dim3((p.rows + 63) / 64, 4, p.splits * chunks), dim3(256), 0, s>>>(p);
  return hipGetLastError();
}

template <int TYPE>
hipError_t of_type(const Adapter& p, bool dma, hipStream_t s) {
  if (p.base_splits > 0) return serve<TYPE>(p, s);
  if (p.rank > 0 && p.k > 0) {
    const hipError_t e = p.rank <= 16 ? shrink<TYPE, 1>(p, s) : p.rank <= 32 ? shrink<TYPE, 2>(p, s) : shrink<TYPE, 4>(p, s);
    if (e != hipSuccess) return e;
  }
  if (dma) return run<Tile<TYPE, kAlong, kAlong, 2, 4, 4, 2, true, TYPE>>(p, s);
  return run<Tile<TYPE, kAlong, kAlong, 2, 2, 2, 2, false, TYPE>>(p, s);
}

}  // namespace

hipError_t launch_adapter(Adapter p, int type, hipStream_t s) {
  const bool dma = dma_operand(p.x, p.ldx, p.k) && dma_operand(p.w, p.ldw, p.k);
  p.vec = (uintptr_t)p.y % 16 == 0 && p.ldy % 8 == 0 && p.n % 8 == 0;
  if (p.k == 0 || p.adapters == 0) p.rank = 0;  // X A^T is zero
  return type == kBF16 ? of_type<kBF16>(p, dma, s) : of_type<kF16>(p, dma, s);
}

}  // namespace half
}  // namespace oz
