// A shared projection with low-rank adapters of many requests at once:
//
//   Y[t, :] = X[t, :] W^T + s_a (X[t, :] A_a^T) B_a^T,   a = ids[t]
//
// Many rows: H[t, :] = X[t, :] A_a^T is formed first, in partial sums of a
// split depth, and s_a H written as two 16-bit numbers, a rounded value and the
// rest, so that it keeps 16 bits (bfloat16) or 22 (half, at a power of two of each
// row's own).  Then the projection's tiles
// run and, before a tile is stored, add for each adapter that its rows name
// the product of those rows of H with that adapter's B_a: the projection's
// output is written once and never read.
//
// Few rows, and some more that name many adapters (which a tile would go through
// one by one): the projection's weights are what has to be read.  One launch
// reads them once into partial sums over parts of the depth and forms H beside
// it; a second one adds the parts up and the adapters' share, in FP32.
//
// A few rows that would cost the tiles a round of their own take the few-row
// form behind them.
#include "half_products.hpp"
#include "half_rules.hpp"
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

// ---- many rows: whole tiles --------------------------------------------------
// Partial sums of X A_a^T: a block has 32 rows, 16 RB ranks and a part of the
// depth, split again over its wavefronts; the adapters that its rows name in
// turn.  Little work, bound by the chain of loads: 333 rows, k = 1111, rank 24:
// 11 us.  grid (row tiles, parts x rank chunks)
constexpr int kShrinkRows = 32, kShrinkTiles = 1024;  // rows of a block; from how many rows on tiles

template <int TYPE, int RB>
__global__ __launch_bounds__(256) void shrink_kernel(Adapter p) {
  constexpr int TB = kShrinkRows / 16;
  __shared__ int ids[kShrinkRows];
  __shared__ v4f lds[4 * TB * 16 * RB * 4];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t0 = blockIdx.x * kShrinkRows;
  const int rows = p.rows - t0 < kShrinkRows ? p.rows - t0 : kShrinkRows;
  const int split = blockIdx.y % p.splits, rank0 = blockIdx.y / p.splits * (16 * RB);
  const int ranks = p.rank - rank0 < 16 * RB ? p.rank - rank0 : 16 * RB;
  if (threadIdx.x < kShrinkRows) ids[threadIdx.x] = (int)threadIdx.x < rows ? p.ids[t0 + threadIdx.x] : -1;
  __syncthreads();
  const int steps = (p.k + 31) / 32, q = split * 4 + wave;
  const int s0 = (int)((int64_t)steps * q / (p.splits * 4)), s1 = (int)((int64_t)steps * (q + 1) / (p.splits * 4));
  for (int a = -1;;) {
    a = next_adapter<1>(ids, rows, a, p.adapters);
    if (a == p.adapters) break;
    v4f acc[RB][TB] = {};
    skinny<TYPE, RB, TB, 4>((const char*)p.a + (a * p.a_stride + rank0 * p.lda) * 2, p.lda, ranks,
                         (const char*)p.x + t0 * p.ldx * 2, p.ldx, rows, p.k, s0, s1, acc);
    skinny_join<RB, TB, 4>(acc, lds, [&](int t, int r, v4f v) {
      if (t >= rows || ids[t] != a || rank0 + r >= p.rank_pad) return;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = r + e < ranks ? v[e] : 0.0f;
      *(v4f*)(p.h + ((int64_t)split * p.rows + t0 + t) * p.rank_pad + rank0 + r) = v;
    });
    __syncthreads();
  }
}

// The same with whole tiles, 64 rows x 64 ranks, for many rows whose operands
// can go to LDS by DMA: k = 4096, rank 64, 4096 rows 19 us against 32, the whole
// call with 8192 rows 262 / 277; with 512 rows of rank 16 17.8 / 16.2.
// grid (row tiles, parts x rank chunks)
template <class T>
__global__ __launch_bounds__(T::THREADS, 1) void shrink_tiles_kernel(Adapter p) {
  static_assert(!T::WIDE && T::BM == 64);
  __shared__ __attribute__((aligned(1024))) char lds[T::LDS + T::BM * 4];
  int* const ids = (int*)(lds + T::LDS);
  const int t0 = blockIdx.x * T::BM;
  const int rows = p.rows - t0 < T::BM ? p.rows - t0 : T::BM;
  const int split = blockIdx.y % p.splits, rank0 = blockIdx.y / p.splits * T::BN;
  const int ranks = p.rank - rank0 < T::BN ? p.rank - rank0 : T::BN;
  const int stages = (p.k + kDepth - 1) / kDepth;
  const int d0 = stages * split / p.splits * kDepth, d1 = stages * (split + 1) / p.splits * kDepth;
  const int depth = (d1 < p.k ? d1 : p.k) - d0;
  if ((int)threadIdx.x < T::BM) ids[threadIdx.x] = (int)threadIdx.x < rows ? p.ids[t0 + threadIdx.x] : -1;
  __syncthreads();
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = wave / T::WC * T::MB * 32 + 4 * (lane >> 5), col = wave % T::WC * T::NB * 32 + (lane & 31);
  for (int a = -1;;) {
    a = next_adapter<1>(ids, rows, a, p.adapters);
    if (a == p.adapters) break;
    v16f acc[T::MB][T::NB] = {};
    product<T>(Operand{(const char*)p.x + (t0 * p.ldx + d0) * 2, p.ldx, rows, p.k},
               Operand{(const char*)p.a + (a * p.a_stride + rank0 * p.lda + d0) * 2, p.lda, ranks, p.k}, depth, lds, acc);
    // lane l of a block: rank l % 32, rows 8 (i / 4) + 4 (l / 32) + i % 4; ranks past the last are zeros
#pragma unroll
    for (int x = 0; x < T::MB; ++x)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int t = row + 32 * x + 8 * (i >> 2) + (i & 3);
        if (ids[t] != a) continue;
#pragma unroll
        for (int y = 0; y < T::NB; ++y)
          if (rank0 + col + 32 * y < p.rank_pad)
            p.h[((int64_t)split * p.rows + t0 + t) * p.rank_pad + rank0 + col + 32 * y] = acc[x][y][i];
      }
  }
}

// A number of 16 bits and the rest of x, of x's sign and neither zero unless x is:
// an infinity that both are multiplied by stays one.  The number is x rounded toward
// zero, or the one before it where that would leave nothing; the rest is rounded
// to nearest.  Together they keep 16 bits of x in bfloat16 and 22 in half.
template <int TYPE>
__device__ __forceinline__ void split(float x, uint16_t& number, uint16_t& rest) {
  using O = typename Out<TYPE>::type;
  const float size = __builtin_fabsf(x);
  const uint16_t sign = __builtin_bit_cast(uint32_t, x) >> 16 & 0x8000;
  uint32_t n, r;
  if constexpr (TYPE == kF16)
    n = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(size, 0.0f));
  else
    n = __builtin_bit_cast(uint32_t, size) >> 16;
  const auto value = [](uint32_t u) { return (float)__builtin_bit_cast(O, (uint16_t)u); };
  n -= n > 1 && value(n) == size ? 1 : 0;
  r = __builtin_bit_cast(uint16_t, (O)(size - value(n)));
  if (size > 0.0f) n = n > 1 ? n : 1, r = r > 1 ? r : 1;
  if (!__builtin_isfinite(size)) n = r = __builtin_bit_cast(uint16_t, (O)size);
  number = n | sign;
  rest = r | sign;
}

// s_a H from its partial sums, as two 16-bit numbers (rank_pad of a row and
// rank_pad more); rows without an adapter are not written.  One would round what the
// result's own rounding has not asked for; two cost 64 more ranks of the matrix
// cores.  4096 rows, rank 64: 5.0 us, mostly the launch.
//
// Half's range is not that of s_a H: a row's values are divided by a power of
// two that brings its largest finite one to [2^14, 2^15), and the tiles multiply
// its sums by that power in 32 bits.  No value overflows, and the least number,
// 2^-24, is 2^-38 of the row's largest value or less.  bfloat16 has float32's range.
// `lanes`, a power of two, hold a row, four ranks each.
template <int TYPE>
__global__ __launch_bounds__(256) void split_kernel(Adapter p, int lanes) {
  using O = typename Out<TYPE>::type;
  const int r = (int)(threadIdx.x & (lanes - 1)) * 4, per = 256 / lanes;
  for (int64_t t = (int64_t)blockIdx.x * per + threadIdx.x / lanes; t < p.rows; t += (int64_t)gridDim.x * per) {
    const int a = p.ids[t];
    if (a < 0 || a >= p.adapters) continue;
    v4f v{};
    if (r < p.rank_pad)
      for (int s = 0; s < p.splits; ++s) v += *(const v4f*)(p.h + ((int64_t)s * p.rows + t) * p.rank_pad + r);
    v *= p.scales ? p.scales[a] : 1.0f;
    // ranks past the last: zeros also behind an infinite scale or activation
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = r + e < p.rank ? v[e] : 0.0f;
    if constexpr (TYPE == kF16) {
      float most = 0.0f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float size = __builtin_fabsf(v[e]);
        most = size > most && __builtin_isfinite(size) ? size : most;
      }
      for (int d = lanes >> 1; d; d >>= 1) most = fmaxf(most, __shfl_xor(most, d));
      // most in [2^(e - 1), 2^e); below 2^-100 nothing is left of it in any product
      const int e = most > 0.0f ? __builtin_amdgcn_frexp_expf(most) : 0, power = (e < -100 ? -100 : e) - 15;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = __builtin_ldexpf(v[i], -power);
      if (r == 0) p.factors[t] = __builtin_ldexpf(1.0f, power);
    }
    if (r >= p.rank_pad) continue;
    uint16_t numbers[4], rests[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) split<TYPE>(v[e], numbers[e], rests[e]);
    char* const out = (char*)p.h16 + (t * 2 * p.rank_pad + r) * 2;
    __builtin_memcpy(out, numbers, 8);
    __builtin_memcpy(out + p.rank_pad * 2, rests, 8);
  }
}

// The adapters' share of a tile, added to its sums: 64 ranks at a time, H's
// rounded values, its rests and B_a in LDS.  A lane's outputs of a block lie in
// one row (WIDE): it takes the sums where that row names this adapter.  (Rows
// of other adapters as zeros would do without that choice, but pass on an
// infinity of this adapter's B.)  An infinity of the row's own B_a meets two
// numbers of one sign (split_kernel).
template <class T>
__device__ __forceinline__ void expand(const Adapter& p, int r0, int rows, int c0, int cols, const int* ids,
                                       const float* factors, char* lds, v16f (&acc)[T::MB][T::NB]) {
  static_assert(T::LA == kAlong && T::LB == kAlong && T::WIDE);
  static_assert(2 * T::A_BYTES + T::B_BYTES <= T::LDS);
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = wave / T::WC, wc = wave % T::WC;
  Fragments<kAlong, T::BM, T::MB> fa;
  Fragments<kAlong, T::BN, T::NB> fb;
  fa.init(wr * T::MB, lane);
  fb.init(wc * T::NB, lane);
  char* const rests = lds + T::A_BYTES;
  char* const bs = lds + 2 * T::A_BYTES;
  for (int a = -1;;) {
    a = next_adapter<(T::BM + 63) / 64>(ids, rows, a, p.adapters);
    if (a == p.adapters) break;
    const char* const B = (const char*)p.b + (a * p.b_stride + c0 * p.ldb) * 2;
    for (int d0 = 0; d0 < p.rank_pad; d0 += kDepth) {
      const int left = p.rank_pad - d0 < kDepth ? p.rank_pad - d0 : kDepth;
      const char* const h = (const char*)p.h16 + ((int64_t)r0 * 2 * p.rank_pad + d0) * 2;
      MaskedSide<kAlong, T::BM, T::ADMA> hi, lo;
      MaskedSide<kAlong, T::BN, T::BDMA> b;
      hi.init(Operand{h, 2 * p.rank_pad, rows, 2 * p.rank_pad}, left, wave, lane);
      lo.init(Operand{h + p.rank_pad * 2, 2 * p.rank_pad, rows, 2 * p.rank_pad}, left, wave, lane);
      b.init(Operand{B + d0 * 2, p.ldb, cols, p.rank}, p.rank - d0, wave, lane);
      hi.load(wave, lane, left);
      lo.load(wave, lane, left);
      b.load(wave, lane, p.rank - d0);
#pragma unroll
      for (int i = 0; i < T::ADMA; ++i) {
        hi.put(i, lds, wave, lane);
        lo.put(i, rests, wave, lane);
      }
#pragma unroll
      for (int i = 0; i < T::BDMA; ++i) b.put(i, bs, wave, lane);
      __syncthreads();
      const int ks_end = left / 16;
#pragma unroll
      for (int x = 0; x < T::MB; ++x) {
        const int row = (wr * T::MB + x) * 32 + (lane & 31);
        const bool mine = ids[row] == a;
        const float factor = T::TYPE == kF16 ? factors[row] : 1.0f;
        v16f t[T::NB] = {};
        for (int ks = 0; ks < ks_end; ++ks) {
          // the swizzle's K step term, as Fragments has it
          const v4i xh = *(const v4i*)(lds + fa.at(ks) + x * 4096), xl = *(const v4i*)(rests + fa.at(ks) + x * 4096);
#pragma unroll
          for (int y = 0; y < T::NB; ++y) {
            const v4i xb = *(const v4i*)(bs + fb.at(ks) + y * 4096);
            t[y] = mfma<T::TYPE>(xb, xh, t[y]);
            t[y] = mfma<T::TYPE>(xb, xl, t[y]);
          }
        }
#pragma unroll
        for (int y = 0; y < T::NB; ++y)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[x][y][i] += mine ? factor * t[y][i] : 0.0f;
      }
      __syncthreads();
    }
  }
}

// The projection's tiles with their adapters' share.  Bound by the matrix cores:
// 4096 x 4096 x 4096, rank 64, eight adapters in runs: 125 us in bfloat16 and 128 in
// half (137 + 4.3 GFLOP: 1130 and 1100 TFLOP/s), without adapters 117; the tiles are one
// round of the CUs, whose first loads and last stores overlap nothing.
template <class T>
__global__ __launch_bounds__(T::THREADS, 1) void adapter_kernel(Adapter p) {
  // one array: with two, the compiler would tell them apart by alias scopes of
  // its own and wait for the loads into LDS before every fragment
  __shared__ __attribute__((aligned(1024))) char lds[T::LDS + T::BM * 8];
  int* const ids = (int*)(lds + T::LDS);
  float* const factors = (float*)(ids + T::BM);
  const uint32_t tiles_n = ((uint32_t)p.n + T::BN - 1) / T::BN, tiles_m = ((uint32_t)p.rows + T::BM - 1) / T::BM;
  uint32_t place, tm, tn;
  if (!block_place(blockIdx.x, tiles_m * tiles_n, place)) return;
  place_to_tile(place, tiles_m, tiles_n, tm, tn);
  const int r0 = (int)tm * T::BM, c0 = (int)tn * T::BN;
  const int rows = p.rows - r0 < T::BM ? p.rows - r0 : T::BM, cols = p.n - c0 < T::BN ? p.n - c0 : T::BN;
  if (p.rank > 0)
    for (int i = threadIdx.x; i < T::BM; i += T::THREADS) {
      ids[i] = i < rows ? p.ids[r0 + i] : -1;
      if constexpr (T::TYPE == kF16) factors[i] = i < rows ? p.factors[r0 + i] : 1.0f;
    }
  v16f acc[T::MB][T::NB] = {};
  if (!product<T>(Operand{(const char*)p.x + r0 * p.ldx * 2, p.ldx, rows, p.k},
                  Operand{(const char*)p.w + c0 * p.ldw * 2, p.ldw, cols, p.k}, p.k, lds, acc))
    return;
  if (p.rank > 0) expand<T>(p, r0, rows, c0, cols, ids, factors, lds, acc);
  store<T>(acc, lds, (char*)p.y + (r0 * p.ldy + c0) * 2, p.ldy, rows, cols, p.stream);
}

// ---- few rows (serving): the weights are read once ------------------------------
// First launch: the projection's partial sums over parts of the depth, and
// beside them H[t, :], a block per row, 16 ranks and part.  4096 x 4096, rank 16:
// one row 8.1 us (33.6 MB of weights: 4.2 TB/s, the launch and first loads among
// it), 64 rows of 64 adapters 15.7.  (One launch for both, with a counter that
// tells the last block to join, would order the blocks' writes by fences; two
// launches need none and give the same sums in every run.)
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
    skinny<TYPE, 1, 1, 8>((const char*)p.a + ((int64_t)a * p.a_stride + chunk * 16 * p.lda) * 2, p.lda, ranks,
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
  skinny<TYPE, NB, TB, (NB + TB <= 6 ? 4 : 2)>((const char*)p.w + c0 * p.ldw * 2, p.ldw, cols, (const char*)p.x + t0 * p.ldx * 2, p.ldx, rows,
                       p.k, s0, s1, acc);
  float* const out = p.partials + (int64_t)split * p.rows * p.n_pad;
  skinny_join<NB, TB, kServeWaves>(acc, lds, [&](int row, int c, v4f v) {
    if (row < rows && c < cols) *(v4f*)(out + (int64_t)(t0 + row) * p.n_pad + c0 + c) = v;  // n_pad: a multiple of 4
  });
}

// Second launch: the partial sums in their order, then the row's adapter: a
// thread per output, s_a H and the sum over the ranks in FP32.  As long as its
// chain of loads: 4.4 us for one row, 5.2 for 64 (4096 columns, rank 16).
// grid (columns / 256, rows)
template <int TYPE>
__global__ __launch_bounds__(256) void serve_join_kernel(Adapter p) {
  using O = typename Out<TYPE>::type;
  typedef O v8o __attribute__((ext_vector_type(8)));
  __shared__ float h[OZAKI25_MAX_RANK];
  const int t = blockIdx.y, c = blockIdx.x * 256 + threadIdx.x;
  const int at = c < p.n ? c : p.n - 1;
  const int a = p.rank > 0 ? p.ids[t] : -1;
  const bool any = a >= 0 && a < p.adapters;
  // all loads first: the call is as long as its chain of loads
  float parts[8];  // base_splits of them
#pragma unroll
  for (int s = 0; s < 8; ++s)
    if (s < p.base_splits) parts[s] = p.partials[((int64_t)s * p.rows + t) * p.n_pad + at];
  constexpr int AHEAD = 8;  // chunks of 8 ranks
  v4i b[AHEAD];
  const char* const B = (const char*)p.b + ((int64_t)a * p.b_stride + (int64_t)at * p.ldb) * 2;
  if (any) {
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
      if (i * 8 < p.rank) b[i] = load8(B, i * 8, p.rank);
    if ((int)threadIdx.x < p.rank_pad) {
      float v = 0;
      for (int s = 0; s < p.splits; ++s) v += p.h[((int64_t)s * p.rows + t) * p.rank_pad + threadIdx.x];
      h[threadIdx.x] = (int)threadIdx.x < p.rank ? v * (p.scales ? p.scales[a] : 1.0f) : 0.0f;
    }
  }
  float y = 0;
#pragma unroll
  for (int s = 0; s < 8; ++s)
    if (s < p.base_splits) y += parts[s];
  __syncthreads();
  if (any) {
    auto add = [&](int r, v4i chunk) __attribute__((always_inline)) {
      const v8o w = __builtin_bit_cast(v8o, chunk);
#pragma unroll
      for (int e = 0; e < 8; ++e) y += h[r + e] * (float)w[e];
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
      if (i * 8 < p.rank) add(i * 8, b[i]);
    for (int r = AHEAD * 8; r < p.rank; r += 8) add(r, load8(B, r, p.rank));
  }
  if (c < p.n) ((O*)p.y)[(int64_t)t * p.ldy + c] = (O)y;
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
  // 32 / 64 columns per block: 1 row 13.1 / 14.0 us, 32 rows 19.0 / 16.2 (4096 x 4096, rank 16)
  if (p.rows <= 16) return serve_tiles<TYPE, 2, 1>(p, s);
  if (p.rows <= 32) return serve_tiles<TYPE, 4, 2>(p, s);
  return serve_tiles<TYPE, 4, 4>(p, s);
}

template <class T>
hipError_t run(const Adapter& p, hipStream_t s) {
  const int64_t tiles = ceil_div(p.rows, T::BM) * ceil_div(p.n, T::BN);
  const dim3 grid((uint32_t)((tiles + 7) & ~(int64_t)7));
  adapter_kernel<T><<<grid, dim3(T::THREADS), 0, s>>>(p);
  return hipGetLastError();
}

template <int TYPE, int RB>
hipError_t shrink(const Adapter& p, hipStream_t s) {
  if (p.rows >= kShrinkTiles && dma_operand(p.x, p.ldx, p.k) && dma_operand(p.a, p.lda, p.k) && p.a_stride % 8 == 0) {
    using T = Tile<TYPE, kAlong, kAlong, 2, 2, 1, 1, true, kF32, 3>;
    const dim3 grid((uint32_t)ceil_div(p.rows, T::BM), (uint32_t)(p.splits * ceil_div(p.rank, T::BN)));
    shrink_tiles_kernel<T><<<grid, dim3(T::THREADS), 0, s>>>(p);
  } else {
    const dim3 grid((uint32_t)ceil_div(p.rows, kShrinkRows), (uint32_t)(p.splits * ceil_div(p.rank, 16 * RB)));
    shrink_kernel<TYPE, RB><<<grid, dim3(256), 0, s>>>(p);
  }
  int lanes = 4;  // of a row: 16 to 256 ranks
  while (lanes * 4 < p.rank_pad) lanes *= 2;
  const int64_t blocks = ceil_div((int64_t)p.rows * lanes, 256);
  split_kernel<TYPE><<<dim3((uint32_t)(blocks < 1 << 20 ? blocks : 1 << 20)), dim3(256), 0, s>>>(p, lanes);
  return hipGetLastError();
}

template <int TYPE>
hipError_t tiles(const Adapter& p, hipStream_t s) {
  if (p.rank > 0) {
    const hipError_t e = p.rank <= 16 ? shrink<TYPE, 1>(p, s) : p.rank <= 32 ? shrink<TYPE, 2>(p, s) : shrink<TYPE, 4>(p, s);
    if (e != hipSuccess) return e;
  }
  const int64_t middle = ceil_div(p.rows, 128) * ceil_div(p.n, 128);
  if (!(dma_operand(p.x, p.ldx, p.k) && dma_operand(p.w, p.ldw, p.k))) {
    if (masked_sets(ceil_div(p.rows, 64) * ceil_div(p.n, 64), p.k))
      return run<Tile<TYPE, kAlong, kAlong, 2, 2, 1, 1, false, TYPE, 2, 4>>(p, s);
    if (masked_small(false, middle)) return run<Tile<TYPE, kAlong, kAlong, 2, 2, 1, 1, false, TYPE>>(p, s);
    return run<Tile<TYPE, kAlong, kAlong, 2, 4, 2, 1, false, TYPE>>(p, s);
  }
  switch (tile_of(middle, ceil_div(p.rows, 256) * ceil_div(p.n, 256))) {
    case kSmallTile: return run<Tile<TYPE, kAlong, kAlong, 2, 2, 1, 1, true, TYPE, 3>>(p, s);
    case kMiddleTile: return run<Tile<TYPE, kAlong, kAlong, 2, 2, 2, 2, true, TYPE>>(p, s);
    default: return run<Tile<TYPE, kAlong, kAlong, 2, 4, 4, 2, true, TYPE>>(p, s);
  }
}

template <int TYPE>
hipError_t both(Adapter p, int serve_rows, hipStream_t s) {
  const int whole = p.rows - serve_rows;
  if (whole > 0) {
    Adapter t = p;
    t.rows = whole;
    const hipError_t e = tiles<TYPE>(t, s);
    if (e != hipSuccess) return e;
  }
  if (serve_rows == 0) return hipSuccess;
  p.rows = serve_rows;
  p.x = (const char*)p.x + whole * p.ldx * 2;
  p.y = (char*)p.y + whole * p.ldy * 2;
  if (p.ids) p.ids += whole;
  p.splits = p.serve_splits;
  return serve<TYPE>(p, s);
}

}  // namespace

hipError_t launch_adapter(Adapter p, const AdapterPlan& plan, char* room, int type, hipStream_t s) {
  // more work-items than a launch holds (by the smallest tiles): before anything runs
  constexpr int64_t kMost = ((int64_t)1 << 32) - 4096;
  if (ceil_div(p.rows, 64) * ceil_div(p.n, 64) * 256 > kMost || ceil_div(p.rows, kShrinkRows) * 256 > kMost)
    return hipErrorInvalidConfiguration;
  p.stream = past_caches((int64_t)p.rows * p.n * 2);
  if (p.k == 0 || p.adapters == 0) p.rank = 0;  // X A^T is zero
  // the two parts run one after the other and share the room of their partial sums of H
  p.h = (float*)room;
  p.h16 = room + plan.h_bytes;
  p.factors = (float*)(room + plan.h_bytes + plan.h16_bytes);
  p.partials = (float*)(room + plan.h_bytes + plan.h16_bytes + plan.factor_bytes);
  p.splits = plan.splits, p.serve_splits = plan.serve_splits, p.base_splits = plan.base_splits;
  return type == kBF16 ? both<kBF16>(p, plan.serve_rows, s) : both<kF16>(p, plan.serve_rows, s);
}

}  // namespace half
}  // namespace oz
