// Products of e4m3 matrices with a scale per block of 128 depths on gfx950's
// matrix cores: one output tile per block, FP32 sums in registers.
//
//   C[r, c] = sum over b of a[b, r] s[b, c] (sum over l in b of A[r, l] B[c, l])
//
// A stage is one block of depths: 128 bytes of each of the tile's vectors in LDS,
// laid out as the 16-bit tiles' 64 depths are, and the scales of its vectors.  A
// stage's products of a 32 x 32 block of outputs (two of depth 64, 128 cycles of a
// matrix core) go to registers of their own and are then added, scaled, to the
// block's sums: 16 fused multiply-adds (64 cycles of the vector unit), which run
// beside the next block's products.
//
// An output's two scales are multiplied first, in FP32.
#pragma once

#include "eight_bits.hpp"

namespace oz {
namespace eight {

typedef int v8i __attribute__((ext_vector_type(8)));
using half::kAlong;
using half::v16f;

constexpr int kStage = 128;  // depths, and bytes of a vector, per stage

// An operand's tile: p at its first vector and depth.
struct Bytes {
  const char* p;
  int64_t ld;  // bytes
  int vecs;    // that exist, at most the tile's
};

// Scales of a tile: element (b, v) at p[b step + v], or of squares p[b].
struct Scales {
  const float* p;
  int64_t step;
};

template <class T>
struct ByteDma;
template <class T>
struct ByteMasked;

// WR x WC wavefronts, each MB x NB blocks of 32 x 32 outputs; products are
// transposed, so a lane has four consecutive columns of a row.  SQUARES: B's
// scales are those of 128 x 128 blocks.  BUFS: stages in LDS.
template <int WR_, int WC_, int MB_, int NB_, bool DMA_, int OUT_, bool SQUARES_, int BUFS_ = 2>
struct Tile8 {
  static constexpr int WR = WR_, WC = WC_, MB = MB_, NB = NB_, OUT = OUT_, BUFS = BUFS_;
  static constexpr bool DMA = DMA_, SQUARES = SQUARES_;
  static constexpr int BM = WR * MB * 32, BN = WC * NB * 32;
  static constexpr int WAVES = WR * WC, THREADS = WAVES * 64;
  static constexpr int A_BYTES = BM * kStage, B_BYTES = BN * kStage;
  static constexpr int STAGE = A_BYTES + B_BYTES, SET = BUFS * STAGE;
  static constexpr int SLOT = (BM + BN) * 4, LDS = SET + 3 * SLOT;  // scales: three stages'
  static constexpr int ADMA = A_BYTES / 1024 / WAVES, BDMA = B_BYTES / 1024 / WAVES;
  using Loads = std::conditional_t<DMA, ByteDma<Tile8>, ByteMasked<Tile8>>;
  static_assert(ADMA * WAVES * 1024 == A_BYTES && BDMA * WAVES * 1024 == B_BYTES, "whole slabs per wavefront");
  static_assert(BM + BN <= THREADS, "a thread carries one scale");
  static_assert(NB * 32 <= 128 && 128 % (NB * 32) == 0, "a wavefront's columns lie in one square");
};

// Rows that start on 16 bytes, whatever their length: chunks past the depth are
// sent outside the descriptor and read as zero; the chunk that the depth's end
// cuts is read whole (its 16 aligned bytes lie in one page) and cleaned in LDS.
template <class T>
struct ByteDma {
  half::DmaSide<kAlong, T::BM, T::ADMA> a;
  half::DmaSide<kAlong, T::BN, T::BDMA> b;
  __amdgpu_buffer_rsrc_t ra, rb;
  int left;  // depths that remain, in pairs of bytes
  __device__ __forceinline__ void init(const Bytes& oa, const Bytes& ob, int depth, int wave, int lane) {
    left = (depth + 15) / 16 * 8;
    a.init(half::Operand{oa.p, oa.ld / 2, oa.vecs, left}, left, wave, lane);
    b.init(half::Operand{ob.p, ob.ld / 2, ob.vecs, left}, left, wave, lane);
  }
  __device__ __forceinline__ void early(int, int) {}
  __device__ __forceinline__ void begin() {
    ra = a.rsrc(left);
    rb = b.rsrc(left);
  }
  __device__ __forceinline__ void late(int j, char* buf, int wave, int) {
    if (j < T::ADMA)
      a.load(j, ra, buf, wave, left);
    else
      b.load(j - T::ADMA, rb, buf + T::A_BYTES, wave, left);
  }
  __device__ __forceinline__ void end() {
    left -= half::kDepth;
    a.advance();
    b.advance();
  }
  static constexpr int IN_FLIGHT = T::ADMA + T::BDMA;
};

// Any alignment and pitch, through registers.
template <int V, int N>
struct ByteSide {
  v4i reg[N];
  const char* p;
  int64_t ld;
  int vecs;
  __device__ __forceinline__ void load(int wave, int lane, int64_t at, int64_t depth) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      int r, c;
      half::chunk_at<kAlong, V>((wave * N + i) * 1024 + lane * 16, r, c);
      // a vector past the edge is read as the last one
      const bool is = r < vecs;
      reg[i] = load16(p + (int64_t)(is ? r : vecs - 1) * ld, at + c * 16, depth);
    }
  }
  __device__ __forceinline__ void put(int i, char* lds, int wave, int lane) const {
    *(v4i*)(lds + (wave * N + i) * 1024 + lane * 16) = reg[i];
  }
};

template <class T>
struct ByteMasked {
  ByteSide<T::BM, T::ADMA> a;
  ByteSide<T::BN, T::BDMA> b;
  int64_t at, depth;
  __device__ __forceinline__ void init(const Bytes& oa, const Bytes& ob, int d, int, int) {
    a.p = half::uniform(oa.p), a.ld = oa.ld, a.vecs = oa.vecs;
    b.p = half::uniform(ob.p), b.ld = ob.ld, b.vecs = ob.vecs;
    at = 0, depth = d;
  }
  __device__ __forceinline__ void early(int wave, int lane) {
    a.load(wave, lane, at, depth);
    b.load(wave, lane, at, depth);
    at += kStage;
  }
  __device__ __forceinline__ void begin() {}
  __device__ __forceinline__ void late(int j, char* buf, int wave, int lane) {
    if (j < T::ADMA)
      a.put(j, buf, wave, lane);
    else
      b.put(j - T::ADMA, buf + T::A_BYTES, wave, lane);
  }
  __device__ __forceinline__ void end() {}
  static constexpr int IN_FLIGHT = 0;
};

// A stage's scales: thread v < BM carries row v's, the next BN threads a column's
// each.  Vectors past the edge take the last one's (their sums are not stored).
template <class T>
struct ScaleLoads {
  const float* p;
  int64_t step;
  int stage, stages;
  float next;
  __device__ __forceinline__ void init(const Scales& sa, const Scales& sb, int rows, int cols, int n) {
    const int t = threadIdx.x;
    if (t < T::BM) {
      p = sa.p + (t < rows ? t : rows - 1);
      step = sa.step;
    } else {
      const int c = t - T::BM < cols ? t - T::BM : cols - 1;
      p = T::SQUARES ? sb.p + (int64_t)(c / kBlock) * sb.step : sb.p + c;
      step = T::SQUARES ? 1 : sb.step;
    }
    stage = 0, stages = n;
  }
  __device__ __forceinline__ void load() {
    next = stage < stages && threadIdx.x < T::BM + T::BN ? p[stage * step] : 0.0f;
    ++stage;
  }
  __device__ __forceinline__ void put(float* slot) const {
    if (threadIdx.x < T::BM + T::BN) slot[threadIdx.x] = next;
  }
};

__device__ __forceinline__ v8i two(v4i lo, v4i hi) {
  return v8i{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
}

// Lane l's 32 bytes of vector l % 32 and half h of a stage: chunks 4 h + 2 (l / 32)
// and the next, as they lie in LDS.
template <int N>
struct ByteFragments {
  int base[4];  // (half, chunk of the two)
  __device__ __forceinline__ void init(int w0, int lane) {
    const int v = w0 * 32 + (lane & 31);
#pragma unroll
    for (int j = 0; j < 4; ++j) base[j] = v * kStage + (((j >> 1) * 4 + 2 * (lane >> 5) + (j & 1)) ^ half::swz_along(v)) * 16;
  }
  __device__ __forceinline__ v8i read(half::lds_bytes lds, int h, int x) const {
    using q = const __attribute__((address_space(3))) v4i*;
    return two(*(q)(lds + base[2 * h] + x * 4096), *(q)(lds + base[2 * h + 1] + x * 4096));
  }
};

// c + a b, 64 depths of 32 x 32 outputs.  The 8-bit products add the eight products
// of neighbouring depths with 13 bits below the largest of them (measured: 1.4e-5 of
// a result's norm on normal numbers, whatever the depth), which a 16-bit output's
// rounding hides.  An FP32 output takes bfloat16 products of the same numbers, exact
// in FP32, at half the rate.
template <int OUT>
__device__ __forceinline__ v16f mfma64(v8i a, v8i b, v16f c) {
  if constexpr (OUT == kF32) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      c = half::mfma<kBF16>(widened<kBF16>(a[2 * j], a[2 * j + 1]), widened<kBF16>(b[2 * j], b[2 * j + 1]), c);
    return c;
  } else {
    // scale operands of 0 are 2^0
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 0, 0, 0, 0, 0, 0);
  }
}

// The same, 128 depths of 16 x 16 outputs.
template <int OUT>
__device__ __forceinline__ v4f mfma128(v8i a, v8i b, v4f c) {
  if constexpr (OUT == kF32) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      c = half::mfma16<kBF16>(widened<kBF16>(a[2 * j], a[2 * j + 1]), widened<kBF16>(b[2 * j], b[2 * j + 1]), c);
    return c;
  } else {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 0, 0, 0, 0);
  }
}

// Zeros past the depth's end in the chunk that it cuts, of every vector of a stage.
template <class T>
__device__ __forceinline__ void clean_tail(char* lds, int left) {
  const int c = left >> 4, keep = left & 15;
  for (int v = threadIdx.x; v < T::BM + T::BN; v += T::THREADS) {
    const int in = v < T::BM ? v : v - T::BM;
    v4i* const q = (v4i*)(lds + v * kStage + ((c ^ half::swz_along(in)) << 4));
    v4i x = *q;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int n = keep - 4 * i;  // bytes of this word that stay
      x[i] = n <= 0 ? 0 : n >= 4 ? x[i] : x[i] & ((1 << (8 * n)) - 1);
    }
    *q = x;
  }
}

template <class T>
__device__ __forceinline__ int next_stage(int cur) {
  return cur + T::STAGE < T::SET ? cur + T::STAGE : 0;
}

// acc += A B over `depth` (at least 1), scaled.  lds: T::LDS bytes, 1024-aligned.
//
// As in the 16-bit tiles the last column of products of a stage runs behind the
// barrier that hands over to the next stage, whose first fragments are read
// meanwhile, and the buffer just freed takes the loads of the stage BUFS later.
template <class T>
__device__ __forceinline__ void product8(const Bytes& oa, const Bytes& ob, const Scales& sa, const Scales& sb, int cols,
                                         int depth, char* lds, v16f (&acc)[T::MB][T::NB]) {
  constexpr int ND = T::ADMA + T::BDMA, MB = T::MB, NB = T::NB;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = wave / T::WC, wc = wave % T::WC;
  const int nst = (depth + kStage - 1) / kStage;
  const int tail = T::DMA && depth % 16 ? depth % kStage : 0;  // depths of a last stage whose end cuts a chunk
  typename T::Loads ld;
  ScaleLoads<T> sl;
  ld.init(oa, ob, depth, wave, lane);
  sl.init(sa, sb, oa.vecs, cols, nst);
  float* const slots = (float*)(lds + T::SET);
  sl.load();
  sl.put(slots);
  sl.load();
#pragma unroll
  for (int s = 0; s < T::BUFS; ++s) {
    ld.early(wave, lane);
    ld.begin();
#pragma unroll
    for (int j = 0; j < ND; ++j) ld.late(j, lds + s * T::STAGE, wave, lane);
    ld.end();
  }
  half::wait_loads_and_lds<(T::BUFS - 1) * T::Loads::IN_FLIGHT>();
  half::block_barrier();
  if (tail && nst == 1) {
    clean_tail<T>(lds, tail);
    __syncthreads();
  }
  const bool active = wr * MB * 32 < oa.vecs && wc * NB * 32 < cols;
  ByteFragments<MB> fa;
  ByteFragments<NB> fb;
  fa.init(wr * MB, lane);
  fb.init(wc * NB, lane);
  const auto l3 = (half::lds_bytes)lds;
  v8i af[2][2], bf[NB][2];
  if (active) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      af[0][h] = fa.read(l3, h, 0);
#pragma unroll
      for (int y = 0; y < NB; ++y) bf[y][h] = fb.read(l3 + T::A_BYTES, h, y);
    }
  }
  int cur = 0, slot = 0;
  for (int s = 0; s < nst; ++s) {
    const int next = next_stage<T>(cur), next_slot = slot == 2 ? 0 : slot + 1;
    ld.early(wave, lane);
    float fs[MB], cs[NB][T::SQUARES ? 1 : 16];
    if (active) {
      const float* const here = slots + slot * (T::SLOT / 4);
#pragma unroll
      for (int x = 0; x < MB; ++x) fs[x] = here[(wr * MB + x) * 32 + (lane & 31)];
      const float* const there = here + T::BM + wc * NB * 32;
      if constexpr (T::SQUARES) {
#pragma unroll
        for (int x = 0; x < MB; ++x) fs[x] *= there[0];
      } else {
#pragma unroll
        for (int y = 0; y < NB; ++y)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const v4f v = *(const v4f*)(there + y * 32 + 8 * q + 4 * (lane >> 5));
#pragma unroll
            for (int e = 0; e < 4; ++e) cs[y][4 * q + e] = v[e];
          }
      }
    }
    auto hand_over = [&] {
      // the next stage's scales, and (older than the loads that may be in flight) its bytes
      sl.put(slots + next_slot * (T::SLOT / 4));
      half::wait_loads_and_lds<(T::BUFS - 2) * T::Loads::IN_FLIGHT>();
      half::block_barrier();
      if (tail && s + 2 == nst) {
        clean_tail<T>(lds + next, tail);
        __syncthreads();
      }
      sl.load();
      ld.begin();
    };
    if (active) {
#pragma unroll
      for (int x = 0; x < MB; ++x) {
        const bool last = x + 1 == MB;
        if (last) hand_over();
        __builtin_amdgcn_sched_barrier(0);
        if (!last) {
#pragma unroll
          for (int h = 0; h < 2; ++h) af[(x + 1) & 1][h] = fa.read(l3 + cur, h, x + 1);
        }
        v16f t[NB];
#pragma unroll
        for (int y = 0; y < NB; ++y) {
          t[y] = mfma64<T::OUT>(bf[y][0], af[x & 1][0], v16f{});
          t[y] = mfma64<T::OUT>(bf[y][1], af[x & 1][1], t[y]);
        }
        if (last) {
#pragma unroll
          for (int j = 0; j < ND; ++j) ld.late(j, lds + cur, wave, lane);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            af[(x + 1) & 1][h] = fa.read(l3 + next, h, 0);
#pragma unroll
            for (int y = 0; y < NB; ++y) bf[y][h] = fb.read(l3 + next + T::A_BYTES, h, y);
          }
        }
#pragma unroll
        for (int y = 0; y < NB; ++y)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float f = T::SQUARES ? fs[x] : fs[x] * cs[y][T::SQUARES ? 0 : i];
            acc[x][y][i] = __builtin_fmaf(t[y][i], f, acc[x][y][i]);
          }
        __builtin_amdgcn_sched_barrier(0);
      }
      if constexpr (MB % 2) {
        af[0][0] = af[1][0];
        af[0][1] = af[1][1];
      }
    } else {
      hand_over();
#pragma unroll
      for (int j = 0; j < ND; ++j) ld.late(j, lds + cur, wave, lane);
    }
    ld.end();
    cur = next;
    slot = next_slot;
  }
  __builtin_amdgcn_s_waitcnt(0);  // the look-ahead past the end lands before LDS is used again
  __syncthreads();
}

// The tile to a row-major matrix of type T::OUT, rounded once.
template <class T>
__device__ __forceinline__ void store8(const v16f (&acc)[T::MB][T::NB], char* lds, void* out, int64_t ld, int rows, int cols,
                                       bool stream) {
  if constexpr (T::OUT != kF32) {
    half::store_wide<T>(acc, lds, out, ld, rows, cols, stream, [](int, int, float*) {});
  } else {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row = wave / T::WC * T::MB * 32 + (lane & 31), col = wave % T::WC * T::NB * 32 + 4 * (lane >> 5);
#pragma unroll
    for (int a = 0; a < T::MB; ++a) {
      float* const p = (float*)out + (int64_t)(row + a * 32) * ld + col;
      if (row + a * 32 >= rows) continue;
#pragma unroll
      for (int b = 0; b < T::NB; ++b)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int c = col + b * 32 + 8 * q;
          const v4f v = {acc[a][b][4 * q], acc[a][b][4 * q + 1], acc[a][b][4 * q + 2], acc[a][b][4 * q + 3]};
          if (c + 4 <= cols) {
            __builtin_memcpy(p + b * 32 + 8 * q, &v, 16);
          } else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
              if (c + e < cols) p[b * 32 + 8 * q + e] = v[e];
          }
        }
    }
  }
}

}  // namespace eight
}  // namespace oz
