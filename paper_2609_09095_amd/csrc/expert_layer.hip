// A layer of experts for few tokens.
//
//   Y[t] = sum over j of gates[t, j] D_e act[t, e],   e = which[t, j]
//   act[t, e] = silu(G_e X[t]) * (U_e X[t]),  or silu(U_e X[t]) without G
//
// Two launches, the hidden values and the outputs (a third, which adds the experts'
// shares, for more than kTogether tokens).  Bound by the read of the weights that
// tokens reach, each once: a block reads 16 rows of an expert's weights straight
// into the matrix cores' fragments, for all tokens of that expert, and its
// wavefronts split the depth.  Every block reads `which` by itself, so the host
// needs no expert's tokens.
//
// The hidden values stay in FP32.  As operands they are two bfloat16 numbers, the
// rounded value and the rest (16 bits of it); half's weights then too (all 11 bits).
#include "eight_products.hpp"
#include "eight_bits.hpp"

namespace oz {
namespace eight {
namespace {

constexpr int kStep = 128;  // depths of a step; lane l has 32 (l / 16) .. + 31 of vector l % 16
constexpr int kMaxPairs = kMaxLayerTokens * kMaxTop;

// ---- which experts, and whose tokens -------------------------------------------
struct Reached {
  uint32_t bits[kMaxLayerExperts / 32];
  int before[kMaxLayerExperts / 32];  // experts reached in the words before
  int count;
};

// The experts that tokens reach.
template <int THREADS>
__device__ __forceinline__ void find_reached(const Layer& p, Reached& s) {
  constexpr int WORDS = kMaxLayerExperts / 32;
  for (int i = threadIdx.x; i < WORDS; i += THREADS) s.bits[i] = 0;
  __syncthreads();
  const int pairs = p.tokens * p.top;
  for (int i = threadIdx.x; i < pairs; i += THREADS) {
    const int e = p.which[i];
    if (e >= 0 && e < p.experts) atomicOr(&s.bits[e >> 5], 1u << (e & 31));
  }
  __syncthreads();
  if (threadIdx.x < 64) {
    int total = 0;
#pragma unroll
    for (int w0 = 0; w0 < WORDS; w0 += 64) {
      const int mine = __builtin_popcount(s.bits[w0 + threadIdx.x]);
      const int incl = half::scan64(mine, [](int a, int b) { return a + b; });
      s.before[w0 + threadIdx.x] = total + incl - mine;
      total += __builtin_amdgcn_readlane(incl, 63);
    }
    if (threadIdx.x == 0) s.count = total;
  }
  __syncthreads();
}

__device__ __forceinline__ int rank_of(const Reached& s, int e) {
  return s.before[e >> 5] + __builtin_popcount(s.bits[e >> 5] & ((1u << (e & 31)) - 1));
}

// One expert's tokens, in order.
struct Tokens {
  int expert, count;
  uint16_t list[kMaxPairs];  // t top + j
};

// The reached expert number `rank` and its tokens; false past the last.
template <int THREADS>
__device__ __forceinline__ bool find_tokens(const Layer& p, const Reached& s, int rank, Tokens& t) {
  if (rank >= s.count) return false;
  for (int w = threadIdx.x; w < kMaxLayerExperts / 32; w += THREADS) {
    int nth = rank - s.before[w];
    uint32_t b = s.bits[w];
    if (nth >= 0 && nth < __builtin_popcount(b)) {
      for (; nth > 0; --nth) b &= b - 1;
      t.expert = w * 32 + __builtin_ctz(b);
    }
  }
  __syncthreads();
  if (threadIdx.x < 64) {
    const int pairs = p.tokens * p.top, e = t.expert;
    int n = 0;
    for (int i0 = 0; i0 < pairs; i0 += 64) {
      const int i = i0 + threadIdx.x;
      const bool is = i < pairs && p.which[i] == e;
      const uint64_t m = __builtin_amdgcn_ballot_w64(is);
      if (is) t.list[n + __builtin_popcountll(m & (((uint64_t)1 << threadIdx.x) - 1))] = (uint16_t)i;
      n += __builtin_popcountll(m);
    }
    if (threadIdx.x == 0) t.count = n;
  }
  __syncthreads();
  return true;
}

// ---- operands --------------------------------------------------------------------
// A lane's 32 elements of a step: four chunks of 8 for four products of depth 32.
template <bool EIGHT>
struct Weights {
  v4i q[EIGHT ? 2 : 4];
};

// row: the vector's first element; o: the lane's first depth
template <bool EIGHT>
__device__ __forceinline__ Weights<EIGHT> load_weights(const char* row, int64_t o, int depth, bool whole) {
  Weights<EIGHT> r;
  if constexpr (EIGHT) {
#pragma unroll
    for (int j = 0; j < 2; ++j) r.q[j] = whole ? half::load_whole(row + o + 16 * j) : load16(row, o + 16 * j, depth);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) r.q[j] = whole ? half::load_whole(row + (o + 8 * j) * 2) : half::load8(row, (int)o + 8 * j, depth);
  }
  return r;
}

// Chunk j as MFMA operand of the 16-bit type TYPE (e4m3 weights), or as it is.
template <int TYPE, bool EIGHT>
__device__ __forceinline__ v4i chunk(const Weights<EIGHT>& w, int j) {
  if constexpr (EIGHT)
    return widened<TYPE>(w.q[j >> 1][(j & 1) * 2], w.q[j >> 1][(j & 1) * 2 + 1]);
  else
    return w.q[j];
}

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

// v as two bfloat16 numbers, the rounded value and the (rounded) rest
__device__ __forceinline__ void split(const float (&v)[8], v4i& hi, v4i& lo) {
  v8bf a, b;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    a[j] = (__bf16)v[j];
    b[j] = (__bf16)(v[j] - (float)a[j]);
  }
  hi = __builtin_bit_cast(v4i, a);
  lo = __builtin_bit_cast(v4i, b);
}

// c + 32 depths of weights times hidden values, which are hi + lo
template <int TYPE, bool EIGHT>
__device__ __forceinline__ v4f down_product(const Weights<EIGHT>& w, int j, v4i hi, v4i lo, v4f c) {
  if constexpr (EIGHT || TYPE == kBF16) {
    const v4i a = chunk<kBF16>(w, j);
    c = half::mfma16<kBF16>(a, lo, c);
    return half::mfma16<kBF16>(a, hi, c);
  } else {
    Raw<kF16> r;
    r.q[0] = w.q[j];
    float v[8];
    values<kF16>(r, v);
    v4i wh, wl;
    split(v, wh, wl);
    c = half::mfma16<kBF16>(wh, lo, c);
    c = half::mfma16<kBF16>(wl, hi, c);
    return half::mfma16<kBF16>(wh, hi, c);
  }
}

__device__ __forceinline__ float silu(float x) { return x / (1.0f + expf(-x)); }

// Hidden values h[o .. o + 8), zeros past `inner`, times g.
__device__ __forceinline__ void load_hidden(const float* h, int64_t o, int inner, float g, float (&v)[8]) {
  const Raw<kF32> r = load_raw<kF32>((const char*)(h + o), (int)(inner - o));
  values<kF32>(r, v);
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] *= g;
}

// ---- hidden values ---------------------------------------------------------------
// A block: 16 NB rows of one expert's weights.  GATED: the first half of them G's,
// the others U's, of the same 8 NB hidden columns (of one product's 16 rows where
// NB is 1).
template <int TYPE, bool EIGHT, bool GATED, int NB, int TB, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void hidden_kernel(Layer p) {
  constexpr int COLS = GATED ? 8 * NB : 16 * NB, E = EIGHT ? 1 : 2, Q = NB * 4, ROWS = TB * 16;
  __shared__ Reached reached;
  __shared__ Tokens tokens;
  __shared__ v4f lds[WAVES * ROWS * Q];
  const int tiles = (p.inner + COLS - 1) / COLS;
  const int rank = blockIdx.x / tiles, c0 = (blockIdx.x - rank * tiles) * COLS;
  find_reached<WAVES * 64>(p, reached);
  if (!find_tokens<WAVES * 64>(p, reached, rank, tokens)) return;
  const int64_t e = tokens.expert;
  const int lane = threadIdx.x & 63, at = lane & 15, part = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int steps = (p.width + kStep - 1) / kStep, s0 = steps * wave / WAVES, s1 = steps * (wave + 1) / WAVES;
  const char* pw[NB];
  const float* sw[NB];  // scales of the lane's sums
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    // the matrix and column of product row r
    auto place = [&](int r, bool& g) {
      const int all = i * 16 + r;
      g = GATED && all < COLS;
      const int c = c0 + (GATED && !g ? all - COLS : all);
      return c < p.inner ? c : p.inner - 1;
    };
    bool g;
    int c = place(at, g);
    const ExpertWeights& m = g ? p.gate : p.up;
    pw[i] = (const char*)m.w + (e * m.stride + c * m.ld) * E;
    c = place(4 * part, g);
    const ExpertWeights& n = g ? p.gate : p.up;
    sw[i] = EIGHT ? n.scales + e * n.scales_stride + c / kBlock * n.scales_ld : nullptr;
  }
  for (int r0 = 0; r0 < tokens.count; r0 += ROWS) {
    const int rows = tokens.count - r0 < ROWS ? tokens.count - r0 : ROWS;
    const char* px[TB];
#pragma unroll
    for (int j = 0; j < TB; ++j) {
      const int r = j * 16 + at < rows ? j * 16 + at : rows - 1;
      px[j] = (const char*)p.x + tokens.list[r0 + r] / p.top * p.ldx * 2;
    }
    v4f acc[NB][TB] = {};
    auto run = [&](int s, bool whole) {
      const int64_t o = (int64_t)s * kStep + part * 32;
      Weights<EIGHT> w[NB];
      Weights<false> x[TB];
#pragma unroll
      for (int i = 0; i < NB; ++i) w[i] = load_weights<EIGHT>(pw[i], o, p.width, whole);
#pragma unroll
      for (int j = 0; j < TB; ++j) x[j] = load_weights<false>(px[j], o, p.width, whole);
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        v4f t[TB];
#pragma unroll
        for (int j = 0; j < TB; ++j) t[j] = EIGHT ? v4f{} : acc[i][j];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const v4i a = chunk<TYPE>(w[i], k);
#pragma unroll
          for (int j = 0; j < TB; ++j) t[j] = half::mfma16<TYPE>(a, x[j].q[k], t[j]);
        }
#pragma unroll
        for (int j = 0; j < TB; ++j) {
          if constexpr (EIGHT)
            acc[i][j] += t[j] * sw[i][s];
          else
            acc[i][j] = t[j];
        }
      }
    };
    const int most = p.width / kStep < s1 ? p.width / kStep : s1;
    int s = s0;
#pragma unroll 2
    for (; s < most; ++s) run(s, true);
    if (s < s1) run(s, false);
    // the wavefronts' sums in their order
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int j = 0; j < TB; ++j) {
        const int row = j * 16 + at, q = i * 4 + part;
        lds[(wave * ROWS + row) * Q + ((q + row) & (Q - 1))] = acc[i][j];
      }
    __syncthreads();
    auto sum = [&](int row, int q) {
      v4f v{};
#pragma unroll
      for (int w = 0; w < WAVES; ++w) v += lds[(w * ROWS + row) * Q + ((q + row) & (Q - 1))];
      return v;
    };
    constexpr int QO = COLS / 4;
    for (int o = threadIdx.x; o < ROWS * QO; o += WAVES * 64) {
      const int row = o / QO, q = o % QO, c = c0 + q * 4;
      if (row >= rows || c >= p.inner) continue;
      v4f g = sum(row, q), u{1.0f, 1.0f, 1.0f, 1.0f};
      if constexpr (GATED) u = sum(row, q + QO);
      v4f h;
#pragma unroll
      for (int k = 0; k < 4; ++k) h[k] = silu(g[k]) * u[k];
      // the row's padding to a multiple of 4 takes what lies past its end
      *(v4f*)(p.hidden + (int64_t)tokens.list[r0 + row] * p.inner_pad + c) = h;
    }
    __syncthreads();
  }
}

// ---- outputs of at most kTogether tokens -----------------------------------------
// A block: COLS output columns of every reached expert, whose sums stay in one set of
// registers: product column t is token t, left out where it does not reach the expert.
struct Table {
  int expert[kTogether * kMaxTop];
  float gate[kTogether * kMaxTop][kTogether];
  int16_t pair[kTogether * kMaxTop][kTogether];  // -1: not reached
};

template <int TYPE, bool EIGHT, int COLS, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void together_kernel(Layer p) {
  constexpr int E = EIGHT ? 1 : 2;
  using O = typename Out<TYPE>::type;
  __shared__ Reached reached;
  __shared__ Table table;
  __shared__ v4f lds[WAVES * 16 * 4];
  find_reached<WAVES * 64>(p, reached);
  const int count = reached.count;
  for (int i = threadIdx.x; i < count * kTogether; i += WAVES * 64) {
    table.gate[i / kTogether][i % kTogether] = 0.0f;
    table.pair[i / kTogether][i % kTogether] = -1;
  }
  __syncthreads();
  if ((int)threadIdx.x < p.tokens) {
    // a token that names an expert twice has it with the sum of the gates
    for (int j = 0; j < p.top; ++j) {
      const int i = threadIdx.x * p.top + j, e = p.which[i];
      if (e < 0 || e >= p.experts) continue;
      const int r = rank_of(reached, e);
      table.expert[r] = e;
      table.gate[r][threadIdx.x] += p.gates[i];
      if (table.pair[r][threadIdx.x] < 0) table.pair[r][threadIdx.x] = (int16_t)i;
    }
  }
  __syncthreads();
  const int lane = threadIdx.x & 63, at = lane & 15, part = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c0 = blockIdx.x * COLS, c = c0 + (at < COLS ? at : COLS - 1) < p.out ? c0 + (at < COLS ? at : COLS - 1) : p.out - 1;
  const int each = (p.inner + kStep - 1) / kStep, whole = p.inner / kStep;  // steps of an expert
  const int64_t all = (int64_t)count * each;
  const int s0 = (int)(all * wave / WAVES), s1 = (int)(all * (wave + 1) / WAVES);
  v4f acc{};
  int r = s0 / each, s = s0 - r * each;
#pragma unroll 2
  for (int i = s0; i < s1; ++i) {
    const int64_t e = table.expert[r];
    const int64_t o = (int64_t)s * kStep + part * 32;
    const Weights<EIGHT> w =
        load_weights<EIGHT>((const char*)p.down.w + (e * p.down.stride + c * p.down.ld) * E, o, p.inner, s < whole);
    const int pair = table.pair[r][at];
    const float g = table.gate[r][at];
    const float* const h = p.hidden + (int64_t)(pair < 0 ? 0 : pair) * p.inner_pad;
    v4f t{};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float v[8];
      load_hidden(h, o + 8 * j, p.inner, g, v);
      v4i hi, lo;
      split(v, hi, lo);
      t = down_product<TYPE>(w, j, hi, lo, t);
    }
    if constexpr (EIGHT) t *= p.down.scales[e * p.down.scales_stride + c0 / kBlock * p.down.scales_ld + s];
    // a token that does not reach the expert sees nothing of it, not even a NaN
#pragma unroll
    for (int k = 0; k < 4; ++k) acc[k] = pair < 0 ? acc[k] : acc[k] + t[k];
    if (++s == each) s = 0, ++r;
  }
  lds[(wave * 16 + at) * 4 + ((part + at) & 3)] = acc;
  __syncthreads();
  if (threadIdx.x < 64) {
    const int row = threadIdx.x >> 2, q = threadIdx.x & 3, col = c0 + q * 4;
    v4f v{};
#pragma unroll
    for (int w = 0; w < WAVES; ++w) v += lds[(w * 16 + row) * 4 + ((q + row) & 3)];
    if (row < p.tokens && q * 4 < COLS) {
      O* const y = (O*)p.y + row * p.ldy + col;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (col + k < p.out) y[k] = (O)v[k];
    }
  }
}

// ---- outputs of more tokens --------------------------------------------------------
// A block: 16 NB output columns of one expert, for its tokens; combine_kernel adds a
// token's shares in the order of its choices.
template <int TYPE, bool EIGHT, int NB, int TB, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void share_kernel(Layer p) {
  constexpr int COLS = 16 * NB, E = EIGHT ? 1 : 2, Q = NB * 4, ROWS = TB * 16;
  __shared__ Reached reached;
  __shared__ Tokens tokens;
  __shared__ v4f lds[WAVES * ROWS * Q];
  const int tiles = (p.out + COLS - 1) / COLS;
  const int rank = blockIdx.x / tiles, c0 = (blockIdx.x - rank * tiles) * COLS;
  find_reached<WAVES * 64>(p, reached);
  if (!find_tokens<WAVES * 64>(p, reached, rank, tokens)) return;
  const int64_t e = tokens.expert;
  const int lane = threadIdx.x & 63, at = lane & 15, part = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int steps = (p.inner + kStep - 1) / kStep, s0 = steps * wave / WAVES, s1 = steps * (wave + 1) / WAVES;
  const char* pw[NB];
  const float* sw[NB];
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    const int c = c0 + i * 16 + at < p.out ? c0 + i * 16 + at : p.out - 1;
    pw[i] = (const char*)p.down.w + (e * p.down.stride + c * p.down.ld) * E;
    const int first = c0 + i * 16 < p.out ? c0 + i * 16 : c0;
    sw[i] = EIGHT ? p.down.scales + e * p.down.scales_stride + first / kBlock * p.down.scales_ld : nullptr;
  }
  for (int r0 = 0; r0 < tokens.count; r0 += ROWS) {
    const int rows = tokens.count - r0 < ROWS ? tokens.count - r0 : ROWS;
    const float *ph[TB], one = 1.0f;
#pragma unroll
    for (int j = 0; j < TB; ++j) {
      const int r = j * 16 + at < rows ? j * 16 + at : rows - 1;
      ph[j] = p.hidden + (int64_t)tokens.list[r0 + r] * p.inner_pad;
    }
    v4f acc[NB][TB] = {};
    for (int s = s0; s < s1; ++s) {
      const int64_t o = (int64_t)s * kStep + part * 32;
      const bool whole = s < p.inner / kStep;
      Weights<EIGHT> w[NB];
#pragma unroll
      for (int i = 0; i < NB; ++i) w[i] = load_weights<EIGHT>(pw[i], o, p.inner, whole);
      v4f t[NB][TB];
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < TB; ++j) t[i][j] = EIGHT ? v4f{} : acc[i][j];
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int j = 0; j < TB; ++j) {
          float v[8];
          load_hidden(ph[j], o + 8 * k, p.inner, one, v);
          v4i hi, lo;
          split(v, hi, lo);
#pragma unroll
          for (int i = 0; i < NB; ++i) t[i][j] = down_product<TYPE>(w[i], k, hi, lo, t[i][j]);
        }
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < TB; ++j) {
          if constexpr (EIGHT)
            acc[i][j] += t[i][j] * sw[i][s];
          else
            acc[i][j] = t[i][j];
        }
    }
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int j = 0; j < TB; ++j) {
        const int row = j * 16 + at, q = i * 4 + part;
        lds[(wave * ROWS + row) * Q + ((q + row) & (Q - 1))] = acc[i][j];
      }
    __syncthreads();
    for (int o = threadIdx.x; o < ROWS * Q; o += WAVES * 64) {
      const int row = o / Q, q = o % Q, c = c0 + q * 4;
      if (row >= rows || c >= p.out) continue;
      v4f v{};
#pragma unroll
      for (int w = 0; w < WAVES; ++w) v += lds[(w * ROWS + row) * Q + ((q + row) & (Q - 1))];
      const int pair = tokens.list[r0 + row];
      *(v4f*)(p.parts + (int64_t)pair * p.out_pad + c) = v * p.gates[pair];
    }
    __syncthreads();
  }
}

template <int TYPE>
__global__ __launch_bounds__(256) void combine_kernel(Layer p) {
  using O = typename Out<TYPE>::type;
  const int groups = p.out_pad / 4;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int t = (int)(i / groups), c = (int)(i % groups) * 4;
  if (t >= p.tokens) return;
  v4f v{};
  for (int j = 0; j < p.top; ++j) {
    const int pair = t * p.top + j, e = p.which[pair];
    if (e >= 0 && e < p.experts) v += *(const v4f*)(p.parts + (int64_t)pair * p.out_pad + c);
  }
  O* const y = (O*)p.y + t * p.ldy + c;
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (c + k < p.out) y[k] = (O)v[k];
}

template <int TYPE, bool EIGHT, bool GATED, int NB, int TB>
hipError_t run_hidden(const Layer& p, hipStream_t s) {
  constexpr int COLS = GATED ? 8 * NB : 16 * NB, WAVES = 8;
  const int64_t pairs = (int64_t)p.tokens * p.top, most = p.experts < pairs ? p.experts : pairs;
  const int64_t blocks = most * ceil_div(p.inner, COLS);
  if (blocks * WAVES * 64 >= ((int64_t)1 << 32)) return hipErrorInvalidConfiguration;
  hidden_kernel<TYPE, EIGHT, GATED, NB, TB, WAVES><<<dim3((uint32_t)blocks), dim3(WAVES * 64), 0, s>>>(p);
  return hipGetLastError();
}

template <int TYPE, bool EIGHT>
hipError_t run_layer(const Layer& p, hipStream_t s) {
  hipError_t e;
  const bool many = p.tokens > kTogether;
  if (p.gate.w)
    e = many ? run_hidden<TYPE, EIGHT, true, 2, 2>(p, s) : run_hidden<TYPE, EIGHT, true, 1, 1>(p, s);
  else
    e = many ? run_hidden<TYPE, EIGHT, false, 1, 2>(p, s) : run_hidden<TYPE, EIGHT, false, 1, 1>(p, s);
  if (e != hipSuccess) return e;
  if (!many) {
    constexpr int WAVES = 8, COLS = 8;
    together_kernel<TYPE, EIGHT, COLS, WAVES><<<dim3((uint32_t)ceil_div(p.out, COLS)), dim3(WAVES * 64), 0, s>>>(p);
    return hipGetLastError();
  }
  constexpr int WAVES = 8, NB = 1, TB = 2;
  const int64_t pairs = (int64_t)p.tokens * p.top, most = p.experts < pairs ? p.experts : pairs;
  const int64_t blocks = most * ceil_div(p.out, 16 * NB);
  if (blocks * WAVES * 64 >= ((int64_t)1 << 32)) return hipErrorInvalidConfiguration;
  share_kernel<TYPE, EIGHT, NB, TB, WAVES><<<dim3((uint32_t)blocks), dim3(WAVES * 64), 0, s>>>(p);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  combine_kernel<TYPE><<<dim3((uint32_t)ceil_div((int64_t)p.tokens * (p.out_pad / 4), 256)), dim3(256), 0, s>>>(p);
  return hipGetLastError();
}

// Y = 0: no expert, no choice, or nothing between the projections
template <int TYPE>
__global__ __launch_bounds__(256) void nothing_kernel(Layer p) {
  using O = typename Out<TYPE>::type;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < (int64_t)p.tokens * p.out) ((O*)p.y)[i / p.out * p.ldy + i % p.out] = (O)0.0f;
}

template <int TYPE>
hipError_t of_type(const Layer& p, bool eight, hipStream_t s) {
  if (p.top == 0 || p.experts == 0 || p.inner == 0 || p.width == 0) {
    nothing_kernel<TYPE><<<dim3((uint32_t)ceil_div((int64_t)p.tokens * p.out, 256)), dim3(256), 0, s>>>(p);
    return hipGetLastError();
  }
  return eight ? run_layer<TYPE, true>(p, s) : run_layer<TYPE, false>(p, s);
}

}  // namespace

hipError_t launch_layer(const Layer& p, int type, bool eight, hipStream_t s) {
  return type == kBF16 ? of_type<kBF16>(p, eight, s) : of_type<kF16>(p, eight, s);
}

}  // namespace eight
}  // namespace oz
