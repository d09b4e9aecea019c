// Products of e4m3 matrices with a scale per block of 128 depths.
//
//   Y[r, c] = sum over b of a[b, r] s[b, c] (sum over l in block b of A[r, l] B[c, l])
//
// s[b, c] is B's scale of column c, or that of the 128 x 128 block it lies in.
// Forward: A activations, B weights in squares.  dX: A the output's gradient, B the
// weights' transposed bytes.  dW: A and B the transposed gradient and activations.
//
// Large products are bound by the matrix cores and the operands' way into LDS: 8192 x
// 8192 x 8192 2.3 to 2.4 PFLOP/s, 16384 x 4096 x 4096 233 to 250 us, as the card's clock is
// (with the loads left out 188, with the scaling left out 232 where whole 257); with FP32
// outputs and scales per vector, 2048 x 4096 x 8192, 126 to 138 us; rows that do not start on
// 16 bytes go through registers, 4096 x 4096 x 4095 181 us.  Tiles of 64 x 64 take 0.37 us a
// stage, a chain of barrier, LDS reads, products and scaling.  A few rows are a chain of
// loads: 1 x 4096 x 4096 6 us, 16 MB of weights.
#include "eight_products.hpp"
#include "eight_tile.hpp"

namespace oz {
namespace eight {
namespace {

// A tile, or (SPLIT) one of g.split parts of its depth, which leaves FP32 sums.
template <class T, bool SPLIT>
__global__ __launch_bounds__(T::THREADS, 2) void scaled_kernel(Scaled g) {
  __shared__ __attribute__((aligned(1024))) char lds[T::LDS];
  const uint32_t tiles_n = ((uint32_t)g.n + T::BN - 1) / T::BN, tiles_m = ((uint32_t)g.rows + T::BM - 1) / T::BM;
  const uint32_t tiles = tiles_m * tiles_n;
  uint32_t place, tm, tn;
  if (!half::block_place(blockIdx.x, SPLIT ? tiles * g.split : tiles, place)) return;
  uint32_t part = 0;
  int64_t b0 = 0;  // blocks of depths before the part
  int depth = g.k;
  if constexpr (SPLIT) {
    part = place / tiles;
    place -= part * tiles;
    const int64_t blocks = (g.k + kBlock - 1) / kBlock;
    b0 = blocks * part / g.split;
    const int64_t b1 = blocks * (part + 1) / g.split;
    depth = (int)((b1 * kBlock < g.k ? b1 * kBlock : g.k) - b0 * kBlock);
  }
  half::place_to_tile(place, tiles_m, tiles_n, tm, tn);
  const int r0 = (int)tm * T::BM, c0 = (int)tn * T::BN;
  const int rows = g.rows - r0 < T::BM ? g.rows - r0 : T::BM, cols = g.n - c0 < T::BN ? g.n - c0 : T::BN;
  const Bytes a{(const char*)g.a + r0 * g.lda + b0 * kBlock, g.lda, rows};
  const Bytes b{(const char*)g.b + c0 * g.ldb + b0 * kBlock, g.ldb, cols};
  const Scales sa{g.as + b0 * g.ldas + r0, g.ldas};
  const Scales sb{T::SQUARES ? g.bs + c0 / kBlock * g.ldbs + b0 : g.bs + b0 * g.ldbs + c0, g.ldbs};
  v16f acc[T::MB][T::NB] = {};
  product8<T>(a, b, sa, sb, cols, depth, lds, acc);
  if constexpr (SPLIT) {
    const int64_t ld = pad4(g.n);
    store_sums<T>(acc, g.parts + ((int64_t)part * g.rows + r0) * ld + c0, ld, rows, cols);
  } else if constexpr (T::OUT == kF32) {
    store_sums<T>(acc, (float*)g.y + r0 * g.ldy + c0, g.ldy, rows, cols);
  } else {
    half::store_wide<T>(acc, lds, (uint16_t*)g.y + r0 * g.ldy + c0, g.ldy, rows, cols, g.stream, [](int, int, float*) {});
  }
}

// The parts' sums in their order.
template <int OUT>
__global__ __launch_bounds__(256) void scaled_join_kernel(Scaled g) {
  using O = typename Out<OUT>::type;
  const int64_t ld = pad4(g.n), groups = ld / 4, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t r = i / groups, c = i % groups * 4;
  if (r >= g.rows) return;
  const float* p = g.parts + r * ld + c;
  v4f v = *(const v4f*)p;
#pragma unroll 8
  for (int q = 1; q < g.split; ++q) v += *(const v4f*)(p + q * g.rows * ld);
  O* const y = (O*)g.y + r * g.ldy + c;
  const int left = (int)(g.n - c);
  if (left >= 4) {
    if constexpr (OUT == kF32) {
      __builtin_memcpy(y, &v, 16);
    } else {
      const uint2 w = half::pack4<OUT>(v[0], v[1], v[2], v[3]);
      __builtin_memcpy(y, &w, 8);  // any alignment
    }
  } else {
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (e < left) y[e] = (O)v[e];
  }
}

// Few rows: a block reads 16 NB columns of B once, straight into fragments, for at
// most 16 TB rows; its wavefronts split the depth.  Lane l holds bytes 32 (l / 16)
// .. + 31 of a block of 128 depths of vector l % 16.
template <int OUT, bool SQUARES, int NB, int TB, int WAVES, int U>
__global__ __launch_bounds__(WAVES * 64) void scaled_few_kernel(Scaled g) {
  using O = typename Out<OUT>::type;
  __shared__ v4f lds[WAVES * TB * 16 * NB * 4];
  const uint32_t tiles_n = ((uint32_t)g.n + 16 * NB - 1) / (16 * NB), tiles_m = ((uint32_t)g.rows + 16 * TB - 1) / (16 * TB);
  uint32_t place;
  if (!half::block_place(blockIdx.x, tiles_m * tiles_n, place)) return;
  const uint32_t tn = place / tiles_m, tm = place - tn * tiles_m;
  const int c0 = (int)tn * (16 * NB), cols = g.n - c0 < 16 * NB ? g.n - c0 : 16 * NB;
  const int r0 = (int)tm * (16 * TB), rows = g.rows - r0 < 16 * TB ? g.rows - r0 : 16 * TB;
  const int lane = threadIdx.x & 63, at = lane & 15, part = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int steps = (g.k + kStage - 1) / kStage, whole = g.k / kStage;
  const int s0 = steps * wave / WAVES, s1 = steps * (wave + 1) / WAVES;
  const char *pw[NB], *px[TB];
  const float *sx[TB], *sw[NB];
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    const int c = c0 + (i * 16 + at < cols ? i * 16 + at : cols - 1);
    pw[i] = (const char*)g.b + c * g.ldb;
    const int first = c0 + (i * 16 < cols ? i * 16 : 0);  // sums' columns: first + 4 part ..
    sw[i] = SQUARES ? g.bs + first / kBlock * g.ldbs : g.bs;
  }
#pragma unroll
  for (int j = 0; j < TB; ++j) {
    const int r = r0 + (j * 16 + at < rows ? j * 16 + at : rows - 1);
    px[j] = (const char*)g.a + r * g.lda;
    sx[j] = g.as + r;
  }
  v4f acc[NB][TB] = {};
  auto add = [&](int s, const v8i (&fw)[NB], const v8i (&fx)[TB], const float (&fs)[TB], const v4f (&cs)[NB]) {
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int j = 0; j < TB; ++j) {
        const v4f t = mfma128<OUT>(fw[i], fx[j], v4f{});
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][j][e] = __builtin_fmaf(t[e], fs[j] * cs[i][e], acc[i][j][e]);
      }
  };
  auto scales = [&](int s, float (&fs)[TB], v4f (&cs)[NB]) {
#pragma unroll
    for (int j = 0; j < TB; ++j) fs[j] = sx[j][s * g.ldas];
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      if constexpr (SQUARES) {
        const float v = sw[i][s];
        cs[i] = v4f{v, v, v, v};
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int c = c0 + i * 16 + 4 * part + e;
          cs[i][e] = sw[i][s * g.ldbs + (c < g.n ? c : g.n - 1)];
        }
      }
    }
  };
  int s = s0;
  const int most = whole < s1 ? whole : s1;
  for (; s < most; s += U) {
    v8i fw[U][NB], fx[U][TB];
    float fs[U][TB];
    v4f cs[U][NB];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (s + u < most) {
        const int64_t o = (int64_t)(s + u) * kStage + part * 32;
#pragma unroll
        for (int i = 0; i < NB; ++i) fw[u][i] = two(half::load_whole(pw[i] + o), half::load_whole(pw[i] + o + 16));
#pragma unroll
        for (int j = 0; j < TB; ++j) fx[u][j] = two(half::load_whole(px[j] + o), half::load_whole(px[j] + o + 16));
        scales(s + u, fs[u], cs[u]);
      }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (s + u < most) add(s + u, fw[u], fx[u], fs[u], cs[u]);
  }
  if (whole < s1) {  // the step that the depth's end cuts
    const int64_t o = (int64_t)whole * kStage + part * 32;
    v8i fw[NB], fx[TB];
    float fs[TB];
    v4f cs[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i) fw[i] = two(load16(pw[i], o, g.k), load16(pw[i], o + 16, g.k));
#pragma unroll
    for (int j = 0; j < TB; ++j) fx[j] = two(load16(px[j], o, g.k), load16(px[j], o + 16, g.k));
    scales(whole, fs, cs);
    add(whole, fw, fx, fs, cs);
  }
  O* const y = (O*)g.y + r0 * g.ldy + c0;
  half::skinny_join<NB, TB, WAVES>(acc, lds, [&](int row, int c, v4f v) {
    if (row >= rows || c >= cols) return;
    O* const q = y + row * g.ldy + c;
    if (c + 4 <= cols) {
      if constexpr (OUT == kF32) {
        __builtin_memcpy(q, &v, 16);
      } else {
        const uint2 w = half::pack4<OUT>(v[0], v[1], v[2], v[3]);
        __builtin_memcpy(q, &w, 8);  // any alignment
      }
    } else {
#pragma unroll
      for (int e = 0; e < 3; ++e)
        if (c + e < cols) q[e] = (O)v[e];
    }
  });
}

// Y = 0 where the depth is empty
template <int OUT>
__global__ __launch_bounds__(256) void scaled_zero_kernel(Scaled g) {
  using O = typename Out<OUT>::type;
  const int64_t total = (int64_t)g.rows * g.n;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256)
    ((O*)g.y)[i / g.n * g.ldy + i % g.n] = (O)0.0f;
}

// PARTS: of forms whose depth may be split
template <class T, bool PARTS = true>
hipError_t run_tiles(const Scaled& g, hipStream_t s) {
  const int64_t tiles = ceil_div(g.rows, T::BM) * ceil_div(g.n, T::BN) * g.split;
  if ((tiles + 8) * T::THREADS >= ((int64_t)1 << 32)) return hipErrorInvalidConfiguration;
  const dim3 grid((uint32_t)((tiles + 7) & ~(int64_t)7)), block(T::THREADS);
  if constexpr (PARTS) {
    if (g.split > 1) {
      scaled_kernel<T, true><<<grid, block, 0, s>>>(g);
      if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
      scaled_join_kernel<T::OUT><<<dim3((uint32_t)ceil_div(g.rows * (pad4(g.n) / 4), 256)), dim3(256), 0, s>>>(g);
      return hipGetLastError();
    }
  }
  scaled_kernel<T, false><<<grid, block, 0, s>>>(g);
  return hipGetLastError();
}

template <int OUT, bool SQUARES, int NB, int TB, int WAVES, int U>
hipError_t run_few(const Scaled& g, hipStream_t s) {
  const int64_t tiles = ceil_div(g.rows, 16 * TB) * ceil_div(g.n, 16 * NB);
  if ((tiles + 8) * WAVES * 64 >= ((int64_t)1 << 32)) return hipErrorInvalidConfiguration;
  scaled_few_kernel<OUT, SQUARES, NB, TB, WAVES, U>
      <<<dim3((uint32_t)((tiles + 7) & ~(int64_t)7)), dim3(WAVES * 64), 0, s>>>(g);
  return hipGetLastError();
}

template <int OUT, bool SQUARES>
hipError_t of_type(const Scaled& g, hipStream_t s) {
  if (g.k == 0) {
    scaled_zero_kernel<OUT><<<dim3(2048), dim3(256), 0, s>>>(g);
    return hipGetLastError();
  }
  switch (g.form) {
    case kScaledFew16: return run_few<OUT, SQUARES, 1, 1, 8, 4>(g, s);
    case kScaledFew32: return run_few<OUT, SQUARES, 1, 2, 8, 4>(g, s);
    case kScaledFew48: return run_few<OUT, SQUARES, 1, 3, 8, 2>(g, s);
    default: break;
  }
  if (!g.dma) {
    if (g.form == kScaledSmall) return run_tiles<Tile8<2, 2, 1, 1, false, OUT, SQUARES>>(g, s);
    return run_tiles<Tile8<2, 4, 2, 1, false, OUT, SQUARES>>(g, s);
  }
  if (g.form == kScaledSmall) return run_tiles<Tile8<2, 2, 1, 1, true, OUT, SQUARES, 3>>(g, s);
  if constexpr (OUT != kF32 && SQUARES) {
    if (g.form == kScaledLarge) return run_tiles<Tile8<2, 4, 4, 2, true, OUT, SQUARES>, false>(g, s);
  } else {
    if (g.split == 1 && scaled_tall(g.rows, g.n)) return run_tiles<Tile8<4, 2, 2, 2, true, OUT, SQUARES>, false>(g, s);
  }
  return run_tiles<Tile8<2, 2, 2, 2, true, OUT, SQUARES>>(g, s);
}

template <int OUT>
hipError_t of_scales(const Scaled& g, bool squares, hipStream_t s) {
  return squares ? of_type<OUT, true>(g, s) : of_type<OUT, false>(g, s);
}

}  // namespace

size_t plan_scaled(Scaled& g, int out) {
  // a single row starts where its matrix does, whatever the pitch says
  if (g.rows == 1) g.lda = (g.k + 15) / 16 * 16;
  if (g.n == 1) g.ldb = (g.k + 15) / 16 * 16;
  g.dma = scaled_dma((uintptr_t)g.a, g.lda, (uintptr_t)g.b, g.ldb);
  const bool words = scaled_words((uintptr_t)g.a, g.lda, (uintptr_t)g.b, g.ldb);
  const ScaledPlan plan = scaled_plan(g.rows, g.n, g.k, words);
  g.form = plan.form;
  g.split = plan.split;
  g.stream = (int64_t)g.rows * g.n * (out == kF32 ? 4 : 2) > ((int64_t)32 << 20);
  return scaled_room(g.rows, g.n, g.k, words);
}

hipError_t launch_scaled(const Scaled& g, bool squares, int out, hipStream_t s) {
  if (out == kBF16) return of_scales<kBF16>(g, squares, s);
  if (out == kF16) return of_scales<kF16>(g, squares, s);
  return of_scales<kF32>(g, squares, s);
}

}  // namespace eight
}  // namespace oz
