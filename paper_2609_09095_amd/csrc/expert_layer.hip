// A layer of experts for few tokens.
//
//   Y[t] = sum over j of gates[t, j] D_e act[t, e],   e = which[t, j]
//   act[t, e] = silu(G_e X[t]) * (U_e X[t]),  or silu(U_e X[t]) without G
//
// Two launches, the hidden values and the outputs (a third, which adds the experts'
// shares, for more than kTogether choices).  Bound by the read of the weights that
// tokens reach, each once: a block reads 16 to 64 rows of an expert's weights straight
// into the matrix cores' fragments, for all tokens of that expert, and its
// wavefronts split the depth.  Every block reads `which` by itself, so the host
// needs no expert's tokens.  64 tokens with 4 of 64 experts, 2048 x 1024 in e4m3: 46 +
// 38 + 4 us, 4.5 TB/s; 16 such tokens, bfloat16: 88 us, 5.9 TB/s.  One token's launches,
// 7 and 5 us, are chains of loads: its choices, then weights.
//
// The hidden values stay in FP32.  As operands they are two bfloat16 numbers, the
// rounded value and the rest (16 bits of it); half's weights then too (all 11 bits).
#include "eight_bits.hpp"
#include "eight_products.hpp"

namespace oz {
namespace eight {
namespace {

constexpr int kStep = 128;  // depths of a step; lane l has four chunks of 8 of vector l % 16
constexpr int kMaxPairs = kMaxLayerTokens * kMaxTop;

// ---- which experts, and whose tokens -------------------------------------------
// Up to 64 choices are one lane's each, and a wavefront finds its way by itself: the
// experts in the order of their first choice, an expert's choices as a mask.
struct FewChoices {
  int mine;       // the lane's choice, -1 for none
  uint64_t left;  // choices of experts that were not taken yet
  __device__ __forceinline__ void init(const Layer& p, int lane) {
    const int e = lane < p.tokens * p.top ? p.which[lane] : -1;
    mine = e >= 0 && e < p.experts ? e : -1;
    left = __builtin_amdgcn_ballot_w64(mine >= 0);
  }
  // the next expert and its choices; 0 choices past the last
  __device__ __forceinline__ int take(uint64_t& choices) {
    choices = 0;
    if (!left) return 0;
    const int e = __builtin_amdgcn_readlane(mine, __builtin_ctzll(left));
    choices = __builtin_amdgcn_ballot_w64(mine == e);
    left &= ~choices;
    return e;
  }
};

// More choices: the experts reached as bits in LDS, in ascending order.
constexpr int kWords = kMaxLayerExperts / 32;

constexpr int kAtOnce = 8;  // choices that a thread holds

struct Reached {
  uint32_t bits[kWords];
  int counts[kAtOnce][16];
};

// Choices i0 + k THREADS + threadIdx.x, -1 past the last: their loads are in flight
// together.
template <int THREADS>
__device__ __forceinline__ void load_choices(const Layer& p, int i0, int (&mine)[kAtOnce]) {
  const int pairs = p.tokens * p.top;
#pragma unroll
  for (int k = 0; k < kAtOnce; ++k) {
    mine[k] = -1;
    const int i = i0 + k * THREADS + threadIdx.x;
    if (i < pairs) mine[k] = p.which[i];
  }
}

// How many of a thread's choices there may be.
template <int THREADS>
__device__ __forceinline__ int sets_of_choices(const Layer& p, int i0) {
  const int n = (p.tokens * p.top - i0 + THREADS - 1) / THREADS;
  return n < kAtOnce ? n : kAtOnce;
}

// Sets the bits; leaves the first choices in `mine`.
template <int THREADS>
__device__ __forceinline__ void find_reached(const Layer& p, Reached& s, int (&mine)[kAtOnce]) {
  const int pairs = p.tokens * p.top;
  auto set = [&](const int (&c)[kAtOnce], int sets) {
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      if (k >= sets) break;
      if (c[k] >= 0 && c[k] < p.experts) atomicOr(&s.bits[c[k] >> 5], 1u << (c[k] & 31));
    }
  };
  load_choices<THREADS>(p, 0, mine);
  for (int i = threadIdx.x; i < kWords; i += THREADS) s.bits[i] = 0;
  __syncthreads();
  set(mine, sets_of_choices<THREADS>(p, 0));
  for (int i0 = kAtOnce * THREADS; i0 < pairs; i0 += kAtOnce * THREADS) {
    int more[kAtOnce];
    load_choices<THREADS>(p, i0, more);
    set(more, sets_of_choices<THREADS>(p, i0));
  }
  __syncthreads();
}

// The lane's words, and how many experts the words before them hold; returns all.
__device__ __forceinline__ int count_reached(const Reached& s, int lane, uint64_t& mine, int& before) {
  static_assert(kWords == 128);
  mine = (uint64_t)s.bits[2 * lane + 1] << 32 | s.bits[2 * lane];
  const int own = __builtin_popcountll(mine), incl = half::scan64(own, [](int a, int b) { return a + b; });
  before = incl - own;
  return __builtin_amdgcn_readlane(incl, 63);
}

// One expert's choices, in order (t top + j).
struct Tokens {
  Reached reached;
  uint16_t list[kMaxPairs];
};

// The expert number `rank` of a block and its choices in s.list; `count` of them, 0
// past the last expert.
template <int THREADS>
__device__ __forceinline__ int find_tokens(const Layer& p, int rank, Tokens& s, int& count) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, pairs = p.tokens * p.top;
  count = 0;
  if (pairs <= 64) {
    FewChoices c;
    c.init(p, lane);
    uint64_t m;
    int e = c.take(m);
    for (int i = 0; i < rank && m; ++i) e = c.take(m);
    if (!m) return 0;
    // every wavefront writes the same
    if (c.mine == e) s.list[__builtin_popcountll(m & (((uint64_t)1 << lane) - 1))] = (uint16_t)lane;
    count = __builtin_popcountll(m);
    __syncthreads();
    return e;
  }
  int mine_of[kAtOnce];
  find_reached<THREADS>(p, s.reached, mine_of);
  uint64_t mine;
  int before;
  if (rank >= count_reached(s.reached, lane, mine, before)) return 0;
  // the word that holds it is one lane's
  const uint64_t holds = __builtin_amdgcn_ballot_w64(rank >= before && rank < before + __builtin_popcountll(mine));
  const int at = __builtin_ctzll(holds);
  uint64_t b = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(mine >> 32), at) << 32 |
               (uint32_t)__builtin_amdgcn_readlane((int)mine, at);
  for (int nth = rank - __builtin_amdgcn_readlane(before, at); nth > 0; --nth) b &= b - 1;
  const int e = at * 64 + __builtin_ctzll(b);
  for (int i0 = 0; i0 < pairs; i0 += kAtOnce * THREADS) {
    if (i0) load_choices<THREADS>(p, i0, mine_of);
    const int sets = sets_of_choices<THREADS>(p, i0);
    // all the ballots, then one exchange of their counts
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      if (k >= sets) break;
      const uint64_t m = __builtin_amdgcn_ballot_w64(mine_of[k] == e);
      if (lane == 0) s.reached.counts[k][wave] = __builtin_popcountll(m);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      if (k >= sets) break;
      const bool is = mine_of[k] == e;
      const uint64_t m = __builtin_amdgcn_ballot_w64(is);
      int n = count;
#pragma unroll
      for (int w = 0; w < THREADS / 64; ++w) {
        const int c = s.reached.counts[k][w];
        n += w < wave ? c : 0;
        count += c;
      }
      if (is)
        s.list[n + __builtin_popcountll(m & (((uint64_t)1 << lane) - 1))] = (uint16_t)(i0 + k * THREADS + threadIdx.x);
    }
    __syncthreads();
  }
  return e;
}

// ---- operands --------------------------------------------------------------------
// A lane's 32 elements of a step: four chunks of 8 for four products of depth 32.
template <bool EIGHT>
struct Weights {
  v4i q[EIGHT ? 2 : 4];
};

// Where chunk j (8 elements) of a step lies for the lanes of part `part`: a load's lanes
// of one vector read 64 bytes in a row of its weights.
template <bool EIGHT>
__device__ __forceinline__ int depth_of(int part, int j) {
  return EIGHT ? 64 * (j >> 1) + 16 * part + 8 * (j & 1) : 32 * j + 8 * part;
}

// row: the vector's first element; o: the step's first depth
template <bool EIGHT>
__device__ __forceinline__ Weights<EIGHT> load_weights(const char* row, int64_t o, int part, int depth, bool whole) {
  Weights<EIGHT> r;
  if constexpr (EIGHT) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int64_t at = o + depth_of<true>(part, 2 * j);
      r.q[j] = whole ? half::load_whole(row + at) : load16(row, at, depth);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t at = o + depth_of<false>(part, j);
      r.q[j] = whole ? half::load_whole(row + at * 2) : half::load8(row, (int)at, depth);
    }
  }
  return r;
}

// The same depths of a vector of 16-bit numbers beside weights of either kind.
template <bool EIGHT>
__device__ __forceinline__ Weights<false> load_beside(const char* row, int64_t o, int part, int depth, bool whole) {
  Weights<false> r;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int64_t at = o + depth_of<EIGHT>(part, j);
    r.q[j] = whole ? half::load_whole(row + at * 2) : half::load8(row, (int)at, depth);
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

// Hidden values h[o .. o + 8), zeros past `inner`.
__device__ __forceinline__ void load_hidden(const float* h, int64_t o, int inner, bool whole, float (&v)[8]) {
  const Raw<kF32> r = load_raw<kF32>((const char*)(h + o), whole ? 8 : (int)(inner - o));
  values<kF32>(r, v);
}

// Steps s0 .. s1 - 1, those below `whole` without an end inside.
template <class F>
__device__ __forceinline__ void each_step(int s0, int s1, int whole, F step) {
  const int most = whole < s1 ? whole : s1;
  int s = s0;
#pragma unroll 2
  for (; s < most; ++s) step(s, true);
  if (s < s1) step(s, false);
}

// ---- hidden values ---------------------------------------------------------------
// A block: 16 NB rows of one expert's weights.  GATED: the first half of them G's,
// the others U's, of the same 8 NB hidden columns (of one product's 16 rows where
// NB is 1).
template <int TYPE, bool EIGHT, bool GATED, int NB, int TB, int WAVES>
__global__ __launch_bounds__(WAVES * 64, NB * TB > 4 ? 2 : 4) void hidden_kernel(Layer p) {
  constexpr int COLS = GATED ? 8 * NB : 16 * NB, E = EIGHT ? 1 : 2, Q = NB * 4, ROWS = TB * 16;
  __shared__ Tokens tokens;
  __shared__ v4f lds[WAVES * ROWS * Q];
  const int tiles = (p.inner + COLS - 1) / COLS;
  const int rank = blockIdx.x / tiles, c0 = (blockIdx.x - rank * tiles) * COLS;
  int count;
  const int64_t e = find_tokens<WAVES * 64>(p, rank, tokens, count);
  if (count == 0) return;
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
  for (int r0 = 0; r0 < count; r0 += ROWS) {
    const int rows = count - r0 < ROWS ? count - r0 : ROWS;
    const char* px[TB];
#pragma unroll
    for (int j = 0; j < TB; ++j) {
      const int r = j * 16 + at < rows ? j * 16 + at : rows - 1;
      px[j] = (const char*)p.x + tokens.list[r0 + r] / p.top * p.ldx * 2;
    }
    v4f acc[NB][TB] = {};
    each_step(s0, s1, p.width / kStep, [&](int s, bool whole) {
      const int64_t o = (int64_t)s * kStep;
      Weights<EIGHT> w[NB];
      Weights<false> x[TB];
#pragma unroll
      for (int i = 0; i < NB; ++i) w[i] = load_weights<EIGHT>(pw[i], o, part, p.width, whole);
#pragma unroll
      for (int j = 0; j < TB; ++j) x[j] = load_beside<EIGHT>(px[j], o, part, p.width, whole);
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
    });
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

// ---- outputs of at most kTogether choices ----------------------------------------
// A block: COLS output columns of every reached expert, whose sums stay in one set of
// registers: product column t is token t, left out where it does not reach the expert.
template <int TYPE, bool EIGHT, int COLS, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void together_kernel(Layer p) {
  constexpr int E = EIGHT ? 1 : 2;
  using O = typename Out<TYPE>::type;
  __shared__ v4f lds[WAVES * 16 * 4];
  const int lane = threadIdx.x & 63, at = lane & 15, part = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const float gates = lane < p.tokens * p.top ? p.gates[lane] : 0.0f;
  FewChoices choices;
  choices.init(p, lane);
  const uint64_t valid = choices.left;
  int count = 0;
  for (uint64_t m; choices.take(m), m;) ++count;
  choices.left = valid;
  int taken = 0;
  // expert number r (of ascending calls), and the lane's token's choice of it (-1: none)
  // with its gate; a token that names it twice has the sum of the gates
  auto look_up = [&](int r, int64_t& e, int& pair, float& gate) {
    uint64_t all = 0;
    for (; taken <= r; ++taken) e = choices.take(all);
    uint64_t m = at < p.tokens ? all >> (at * p.top) & (((uint64_t)1 << p.top) - 1) : 0;
    pair = m ? at * p.top + __builtin_ctzll(m) : -1;
    gate = 0.0f;
    while (__builtin_amdgcn_ballot_w64(m != 0)) {
      const float g = __shfl(gates, m ? at * p.top + __builtin_ctzll(m) : 0);
      gate += m ? g : 0.0f;
      m &= m - 1;
    }
  };
  const int c0 = blockIdx.x * COLS, c = c0 + (at < COLS ? at : COLS - 1) < p.out ? c0 + (at < COLS ? at : COLS - 1) : p.out - 1;
  const int each = (p.inner + kStep - 1) / kStep, whole = p.inner / kStep;  // steps of an expert
  const int64_t all = (int64_t)count * each;
  const int s0 = (int)(all * wave / WAVES), s1 = (int)(all * (wave + 1) / WAVES);
  v4f acc{};
  for (int i = s0; i < s1;) {
    const int r = i / each, first = i - r * each, end = s1 - r * each < each ? s1 - r * each : each;
    int64_t e;
    int pair;
    float gate;
    look_up(r, e, pair, gate);
    const char* const w = (const char*)p.down.w + (e * p.down.stride + c * p.down.ld) * E;
    const float* const h = p.hidden + (int64_t)(pair < 0 ? 0 : pair) * p.inner_pad;
    const float* const scales = EIGHT ? p.down.scales + e * p.down.scales_stride + c0 / kBlock * p.down.scales_ld : nullptr;
    each_step(first, end, whole, [&](int s, bool is_whole) {
      const int64_t o = (int64_t)s * kStep;
      const Weights<EIGHT> q = load_weights<EIGHT>(w, o, part, p.inner, is_whole);
      float values[4][8];
#pragma unroll
      for (int j = 0; j < 4; ++j) load_hidden(h, o + depth_of<EIGHT>(part, j), p.inner, is_whole, values[j]);
      v4f t{};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = values[j][k] * gate;
        v4i hi, lo;
        split(v, hi, lo);
        t = down_product<TYPE>(q, j, hi, lo, t);
      }
      if constexpr (EIGHT) t *= scales[s];
      // a token that does not reach the expert sees nothing of it, not even a NaN
#pragma unroll
      for (int k = 0; k < 4; ++k) acc[k] = pair < 0 ? acc[k] : acc[k] + t[k];
    });
    i += end - first;
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

// ---- outputs of more choices --------------------------------------------------------
// A block: 16 NB output columns of one expert, for its tokens; combine_kernel adds a
// token's shares in the order of its choices.
template <int TYPE, bool EIGHT, int NB, int TB, int WAVES>
__global__ __launch_bounds__(WAVES * 64, NB * TB > 2 ? 2 : 4) void share_kernel(Layer p) {
  constexpr int COLS = 16 * NB, E = EIGHT ? 1 : 2, Q = NB * 4, ROWS = TB * 16;
  __shared__ Tokens tokens;
  __shared__ v4f lds[WAVES * ROWS * Q];
  const int tiles = (p.out + COLS - 1) / COLS;
  const int rank = blockIdx.x / tiles, c0 = (blockIdx.x - rank * tiles) * COLS;
  int count;
  const int64_t e = find_tokens<WAVES * 64>(p, rank, tokens, count);
  if (count == 0) return;
  const int lane = threadIdx.x & 63, at = lane & 15, part = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int steps = (p.inner + kStep - 1) / kStep, s0 = steps * wave / WAVES, s1 = steps * (wave + 1) / WAVES;
  const char* pw[NB];
  const float* sw[NB];
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    const int c = c0 + i * 16 + at < p.out ? c0 + i * 16 + at : p.out - 1;
    pw[i] = (const char*)p.down.w + (e * p.down.stride + c * p.down.ld) * E;
    const int square = c0 + i * 16 < p.out ? c0 + i * 16 : c0;
    sw[i] = EIGHT ? p.down.scales + e * p.down.scales_stride + square / kBlock * p.down.scales_ld : nullptr;
  }
  for (int r0 = 0; r0 < count; r0 += ROWS) {
    const int rows = count - r0 < ROWS ? count - r0 : ROWS;
    const float* ph[TB];
#pragma unroll
    for (int j = 0; j < TB; ++j) {
      const int r = j * 16 + at < rows ? j * 16 + at : rows - 1;
      ph[j] = p.hidden + (int64_t)tokens.list[r0 + r] * p.inner_pad;
    }
    v4f acc[NB][TB] = {};
    each_step(s0, s1, p.inner / kStep, [&](int s, bool whole) {
      const int64_t o = (int64_t)s * kStep;
      Weights<EIGHT> w[NB];
      float h[TB][4][8];
#pragma unroll
      for (int i = 0; i < NB; ++i) w[i] = load_weights<EIGHT>(pw[i], o, part, p.inner, whole);
#pragma unroll
      for (int j = 0; j < TB; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k) load_hidden(ph[j], o + depth_of<EIGHT>(part, k), p.inner, whole, h[j][k]);
      v4f t[NB][TB];
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < TB; ++j) t[i][j] = EIGHT ? v4f{} : acc[i][j];
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int j = 0; j < TB; ++j) {
          v4i hi, lo;
          split(h[j][k], hi, lo);
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
    });
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
#pragma unroll 4
  for (int j = 0; j < p.top; ++j) {
    // what a choice of no expert left in the workspace is read and not used
    const int pair = t * p.top + j, e = p.which[pair];
    const v4f w = *(const v4f*)(p.parts + (int64_t)pair * p.out_pad + c);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] += e >= 0 && e < p.experts ? w[k] : 0.0f;
  }
  O* const y = (O*)p.y + t * p.ldy + c;
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (c + k < p.out) y[k] = (O)v[k];
}

template <int TYPE, bool EIGHT, bool GATED, int NB, int TB, int WAVES>
hipError_t run_hidden(const Layer& p, int64_t experts, hipStream_t s) {
  const int64_t blocks = experts * ceil_div(p.inner, GATED ? 8 * NB : 16 * NB);
  if (blocks * WAVES * 64 >= ((int64_t)1 << 32)) return hipErrorInvalidConfiguration;
  hidden_kernel<TYPE, EIGHT, GATED, NB, TB, WAVES><<<dim3((uint32_t)blocks), dim3(WAVES * 64), 0, s>>>(p);
  return hipGetLastError();
}

template <int TYPE, bool EIGHT, bool GATED>
hipError_t run_hidden(const Layer& p, int64_t experts, hipStream_t s) {
  switch (hidden_form(p.tokens * p.top, experts, p.inner, GATED, EIGHT)) {
    case kHiddenOne: return run_hidden<TYPE, EIGHT, GATED, 1, 1, 8>(p, experts, s);
    case kHiddenSmall: return run_hidden<TYPE, EIGHT, GATED, 1, 1, 4>(p, experts, s);
    case kHiddenWide: return run_hidden<TYPE, EIGHT, GATED, 2, 1, 4>(p, experts, s);
    case kHiddenRows: return run_hidden<TYPE, EIGHT, GATED, 2, 2, 4>(p, experts, s);
    default: return run_hidden<TYPE, EIGHT, GATED, 4, 2, 4>(p, experts, s);
  }
}

template <int TYPE, bool EIGHT, int COLS>
hipError_t run_together(const Layer& p, hipStream_t s) {
  constexpr int WAVES = 8;
  together_kernel<TYPE, EIGHT, COLS, WAVES><<<dim3((uint32_t)ceil_div(p.out, COLS)), dim3(WAVES * 64), 0, s>>>(p);
  return hipGetLastError();
}

template <int TYPE, bool EIGHT, int NB, int TB>
hipError_t run_share(const Layer& p, int64_t experts, hipStream_t s) {
  constexpr int WAVES = 4;
  const int64_t blocks = experts * ceil_div(p.out, 16 * NB);
  if (blocks * WAVES * 64 >= ((int64_t)1 << 32)) return hipErrorInvalidConfiguration;
  share_kernel<TYPE, EIGHT, NB, TB, WAVES><<<dim3((uint32_t)blocks), dim3(WAVES * 64), 0, s>>>(p);
  return hipGetLastError();
}

template <int TYPE, bool EIGHT>
hipError_t run_layer(const Layer& p, hipStream_t s) {
  const int64_t pairs = (int64_t)p.tokens * p.top, most = p.experts < pairs ? p.experts : pairs;
  hipError_t e = p.gate.w ? run_hidden<TYPE, EIGHT, true>(p, most, s) : run_hidden<TYPE, EIGHT, false>(p, most, s);
  if (e != hipSuccess) return e;
  if (layer_together(p.tokens, p.top))
    return together_wide(p.out) ? run_together<TYPE, EIGHT, 16>(p, s) : run_together<TYPE, EIGHT, 8>(p, s);
  e = share_rows(pairs, p.experts, p.out) ? run_share<TYPE, EIGHT, 4, 2>(p, most, s) : run_share<TYPE, EIGHT, 2, 1>(p, most, s);
  if (e != hipSuccess) return e;
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
