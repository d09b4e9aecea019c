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
  // a stage's scales, a dword of every lane; a stage more than of bytes, since the last of
  // its products are added up behind the barrier that frees its bytes
  static constexpr int SLOT = THREADS * 4, SLOTS = (BUFS + 1) * SLOT, LDS = SET + SLOTS;
  static constexpr int ADMA = A_BYTES / 1024 / WAVES, BDMA = B_BYTES / 1024 / WAVES;
  // Loads issued right behind the barrier that frees their buffer; the others follow
  // beside the next stage's first products (all at once they keep the wavefront from
  // issuing products: 8192 x 8192 x 8192 484 / 458 us; but 128 x 128 tiles 2048 x 2048
  // x 2048 17.0 / 18.7, 256 x 128 tiles 2048 x 4096 x 8192 in FP32 139 / 148).
  static constexpr int SOON = DMA && BUFS == 2 && MB == 4 ? (ADMA + BDMA) / 2 : ADMA + BDMA;
  // Steps of a block's products, each followed by its part of the block before's additions.
  // With a scale per column an output takes a multiplication and a multiply-add, an FP32
  // one's operands their widening too: about the products' time, and whole blocks of either
  // leave the other's unit idle: 2048 x 4096 x 8192
  // with scales per vector, 256 x 128 tiles, FP32 in 1 / 4 / 8 steps 139.5 / 136.8 / 138.9 us,
  // bfloat16 in 1 / 2 85 / 82; but 128 x 128 tiles 2048 x 2048 x 2048 17.2 / 18.3.
  static constexpr int STEPS = WR < 4 ? 1 : OUT == kF32 ? 4 : 2;
  using Loads = std::conditional_t<DMA, ByteDma<Tile8>, ByteMasked<Tile8>>;
  static_assert(ADMA * WAVES * 1024 == A_BYTES && BDMA * WAVES * 1024 == B_BYTES, "whole slabs per wavefront");
  static_assert(BM + BN <= THREADS, "a lane brings one scale");
  static_assert(NB * 32 <= 128 && 128 % (NB * 32) == 0, "a wavefront's columns lie in one square");
};

// Rows that start on 16 bytes, whatever their length.  The last block of depths
// comes first: chunks past its end are sent outside the descriptor and read as zero,
// and the chunk that the end cuts is read whole (its 16 aligned bytes lie in one
// page) and cleaned in LDS, so that all later stages are whole.
template <int V, int N>
struct ByteDmaSide {
  static_assert(N % 2 == 0);
  const char* p;
  int64_t extent;  // bytes from p to the end of the last valid row
  int voff[2];     // of the lane's chunk of even and odd slabs, less the slab's rows
  int rows8;       // bytes from slab to slab
  __device__ __forceinline__ void init(const Bytes& op, int depth, int wave, int lane) {
    p = half::uniform(op.p);
    extent = op.vecs > 0 ? (op.vecs - 1) * op.ld + (depth + 15) / 16 * 16 : 0;
    rows8 = __builtin_amdgcn_readfirstlane((int)op.ld * 8);
    const int r = wave * N * 8 + (lane >> 3), c = (lane & 7) ^ (lane >> 3);  // the swizzle of row r, bar its bit 3
    voff[0] = (int)(r * op.ld) + c * 16;
    voff[1] = (int)(r * op.ld) + (c ^ 1) * 16;
  }
  // `depth`: of the stage, at most 128; all: bytes before the stage's first depth
  __device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc(int64_t all, bool any) const {
    const int64_t e = any ? extent - all : 0;
    const int n = (int)(e < 0x7ffffff0 ? e : 0x7ffffff0);
    return __builtin_amdgcn_make_buffer_rsrc((void*)(p + all), (short)0, __builtin_amdgcn_readfirstlane(n), 0x00020000);
  }
  __device__ __forceinline__ void load(int i, __amdgpu_buffer_rsrc_t r, char* lds, int wave) const {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (half::lds_ptr)(lds + (wave * N + i) * 1024), 16, voff[i & 1] + i * rows8, 0, 0, 0);
  }
  __device__ __forceinline__ void load_cut(int i, __amdgpu_buffer_rsrc_t r, char* lds, int wave, int lane, int depth) const {
    const int c = (lane & 7) ^ (lane >> 3) ^ (i & 1);
    const int off = c * 16 < depth ? voff[i & 1] + i * rows8 : 0x7ffffff8;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (half::lds_ptr)(lds + (wave * N + i) * 1024), 16, off, 0, 0, 0);
  }
};

template <class T>
struct ByteDma {
  ByteDmaSide<T::BM, T::ADMA> a;
  ByteDmaSide<T::BN, T::BDMA> b;
  __amdgpu_buffer_rsrc_t ra, rb;
  int stage, stages;
  int64_t at;
  __device__ __forceinline__ void init(const Bytes& oa, const Bytes& ob, int depth, int wave, int lane) {
    a.init(oa, depth, wave, lane);
    b.init(ob, depth, wave, lane);
    stages = (depth + kStage - 1) / kStage;
    stage = 1, at = 0;
  }
  __device__ __forceinline__ void first(char* buf, int depth, int wave, int lane) {
    const int64_t before = (int64_t)(stages - 1) * kStage;
    const __amdgpu_buffer_rsrc_t x = a.rsrc(before, true), y = b.rsrc(before, true);
#pragma unroll
    for (int i = 0; i < T::ADMA; ++i) a.load_cut(i, x, buf, wave, lane, depth - (int)before);
#pragma unroll
    for (int i = 0; i < T::BDMA; ++i) b.load_cut(i, y, buf + T::A_BYTES, wave, lane, depth - (int)before);
  }
  __device__ __forceinline__ void early(int, int) {}
  __device__ __forceinline__ void begin() {
    const bool any = stage < stages;
    ra = a.rsrc(at, any);
    rb = b.rsrc(at, any);
    ++stage;
    at += kStage;
  }
  __device__ __forceinline__ void late(int j, char* buf, int wave, int) {
    if (j < T::ADMA)
      a.load(j, ra, buf, wave);
    else
      b.load(j - T::ADMA, rb, buf + T::A_BYTES, wave);
  }
  static constexpr int IN_FLIGHT = T::ADMA + T::BDMA + 1;  // and the scales
};

// Any alignment and pitch, through registers.  A vector past the edge is read as the
// last one.
template <int V, int N>
struct ByteSide {
  v4i reg[N];
  const char* p;
  int64_t at[N];  // of the lane's chunks in a stage
  int vecs;
  __device__ __forceinline__ void init(const Bytes& op, int wave, int lane) {
    p = half::uniform(op.p);
    vecs = op.vecs;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      int r, c;
      half::chunk_at<kAlong, V>((wave * N + i) * 1024 + lane * 16, r, c);
      at[i] = (r < vecs ? r : vecs - 1) * op.ld + c * 16;
    }
  }
  __device__ __forceinline__ void load(const char* stage) {
#pragma unroll
    for (int i = 0; i < N; ++i) reg[i] = half::load_whole(stage + at[i]);
  }
  // the stage from depth o on, which the depth's end may cut
  __device__ __forceinline__ void load_cut(int wave, int lane, int64_t o, int64_t depth) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      int r, c;
      half::chunk_at<kAlong, V>((wave * N + i) * 1024 + lane * 16, r, c);
      reg[i] = load16(p + at[i] - c * 16, o + c * 16, depth);
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
  const char *pa, *pb;
  int stage, stages;
  __device__ __forceinline__ void init(const Bytes& oa, const Bytes& ob, int depth, int wave, int lane) {
    a.init(oa, wave, lane);
    b.init(ob, wave, lane);
    pa = a.p, pb = b.p;
    stages = (depth + kStage - 1) / kStage;
    stage = 1;
  }
  __device__ __forceinline__ void first(char* buf, int depth, int wave, int lane) {
    const int64_t o = (int64_t)(stages - 1) * kStage;
    a.load_cut(wave, lane, o, depth);
    b.load_cut(wave, lane, o, depth);
#pragma unroll
    for (int j = 0; j < T::ADMA + T::BDMA; ++j) late(j, buf, wave, lane);
  }
  __device__ __forceinline__ void early(int, int) {
    // later stages are whole; past the last the registers' old bytes are put and not used
    if (stage < stages) {
      a.load(pa);
      b.load(pb);
    }
    ++stage;
    pa += kStage, pb += kStage;
  }
  __device__ __forceinline__ void begin() {}
  __device__ __forceinline__ void late(int j, char* buf, int wave, int lane) {
    if (j < T::ADMA)
      a.put(j, buf, wave, lane);
    else
      b.put(j - T::ADMA, buf + T::A_BYTES, wave, lane);
  }
  static constexpr int IN_FLIGHT = 0;
};

// A stage's scales, straight into LDS beside its bytes: lane v < BM brings row v's, the
// next BN lanes a column's each.  Vectors past the edge take the last one's (their sums
// are not stored).  As early as the bytes: through a register they came a stage ahead, and
// small tiles waited for them (256 x 3648 x 5143 26 / 19.5 us, 1024 x 1024 x 4096 20 / 16).
template <class T>
struct ScaleLoads {
  const float* p;  // of the wavefront (uniform)
  int64_t step;
  int off;  // of the lane's vector, in bytes
  int stage, stages;
  static_assert(T::BM % 64 == 0 && T::BN % 64 == 0, "a wavefront brings one operand's scales");
  __device__ __forceinline__ void init(const Scales& sa, const Scales& sb, int rows, int cols, int n) {
    const int t = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    if (wave * 64 < T::BM) {
      off = (t < rows ? t : rows - 1) * 4;
      p = sa.p;
      step = sa.step;
    } else {
      const int c = t - T::BM < cols ? t - T::BM : cols - 1;
      off = T::SQUARES ? 0 : c * 4;
      p = T::SQUARES ? sb.p + (int64_t)(__builtin_amdgcn_readfirstlane(c) / kBlock) * sb.step : sb.p;
      step = T::SQUARES ? 1 : sb.step;
    }
    stage = 0, stages = n;
  }
  // the last block first, like the bytes
  __device__ __forceinline__ void load(char* slot, int wave) {
    const int64_t b = stage == 0 ? stages - 1 : stage < stages ? stage - 1 : stages - 1;
    const __amdgpu_buffer_rsrc_t r =
        __builtin_amdgcn_make_buffer_rsrc((void*)half::uniform((const char*)(p + b * step)), (short)0, 0x7ffffff0, 0x00020000);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (half::lds_ptr)(slot + wave * 256), 4, off, 0, 0, 0);
    ++stage;
  }
};

__device__ __forceinline__ v8i two(v4i lo, v4i hi) {
  return v8i{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
}

// Lane l's 32 bytes of vector l % 32 and half h of a stage: chunks 4 h + 2 (l / 32)
// and the next, as they lie in LDS.
template <int N>
struct ByteFragments {
  int base[2][2];
  __device__ __forceinline__ void init(int w0, int lane) {
    const int v = w0 * 32 + (lane & 31);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int j = 0; j < 2; ++j) base[h][j] = v * kStage + ((h * 4 + 2 * (lane >> 5) + j) ^ half::swz_along(v)) * 16;
  }
  __device__ __forceinline__ v8i read(half::lds_bytes lds, int h, int x) const {
    using q = const __attribute__((address_space(3))) v4i*;
    return two(*(q)(lds + base[h][0] + x * 4096), *(q)(lds + base[h][1] + x * 4096));
  }
};

// Step q of T::STEPS of the products of a 32 x 32 block over a stage's 128 depths; t is
// their sum after the last step.  The 8-bit products add those of depths 8 i .. 8 i + 7
// as whole multiples of 2^-13 of (the power of two below) the largest of them, the rest
// dropped, and FP32 from there on: an eight is off by at most 8 2^-13 of its largest
// product.  That bounds the error by the operands and not by the result (448 448 - 448
// 448 + 1 gives 0), and is what a 16-bit output gets; on normal numbers it is 1.4e-5 of
// a result's norm, whatever the depth (measured).  An FP32 output takes bfloat16 products
// of the same numbers, exact in FP32, at half the rate.
template <class T>
__device__ __forceinline__ void products(int q, v16f& t, const v8i (&b)[2], const v8i (&a)[2]) {
  constexpr int EACH = (T::OUT == kF32 ? 8 : 2) / T::STEPS;
#pragma unroll
  for (int i = q * EACH; i < (q + 1) * EACH; ++i) {
    const v16f c = i == 0 ? v16f{} : t;
    if constexpr (T::OUT == kF32) {
      const int h = i / 4, j = i % 4 * 2;
      t = half::mfma<kBF16>(widened<kBF16>(b[h][j], b[h][j + 1]), widened<kBF16>(a[h][j], a[h][j + 1]), c);
    } else {
      // scale operands of 0 are 2^0
      t = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b[i], a[i], c, 0, 0, 0, 0, 0, 0);
    }
  }
}

// c + a b, 128 depths of 16 x 16 outputs, by the same products.
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

__device__ __forceinline__ void wait_lds_and_barrier() {
  half::wait_lds();
  half::block_barrier();
}

template <class T>
__device__ __forceinline__ int next_stage(int cur) {
  return cur + T::STAGE < T::SET ? cur + T::STAGE : 0;
}

// The scales of a lane's 16 columns of a block.
template <class T>
__device__ __forceinline__ void column_scales(const float* cs, v4f (&c)[4]) {
  if constexpr (!T::SQUARES) {
#pragma unroll
    for (int q = 0; q < 4; ++q) c[q] = *(const v4f*)(cs + 8 * q);
  }
}

// Outputs e0 .. e0 + N - 1 of a lane's 16: a block's products, scaled, into its sums.
// fs: the lane's row's scale (times the squares').
template <class T, int N>
__device__ __forceinline__ void add_scaled(v16f& acc, const v16f& t, float fs, const v4f (&c)[4], int e0) {
#pragma unroll
  for (int e = e0; e < e0 + N; ++e) acc[e] = __builtin_fmaf(t[e], T::SQUARES ? fs : fs * c[e / 4][e % 4], acc[e]);
  // here and not later: the compiler would carry the products over the barrier
  if (e0 + N == 16) asm volatile("" : "+v"(acc));
}

// One stage's products, a block at a time, in T::STEPS steps: a step's products are
// issued, then its part of the block before, whose products have ended by then, is added
// up.  On entry the fragments of the first row of blocks are in af[0], of all columns in
// bf.  cur, next: this stage's and the next one's buffer; freed: cur, as the target of the
// loads; freed_before: next, as that of the loads which the stage before left (they are
// declared not to alias, or the compiler would wait for all loads in flight before every
// read of LDS: what keeps them apart is the barrier).  here: this stage's scales;
// scales_freed: those of the stage before, as the target of the loads.
template <class T, class Loader>
__device__ __forceinline__ void stage_products8(Loader& ld, ScaleLoads<T>& sl, const ByteFragments<T::MB>& fa,
                                                const ByteFragments<T::NB>& fb, half::lds_bytes __restrict__ cur,
                                                half::lds_bytes __restrict__ next, char* __restrict__ freed,
                                                char* __restrict__ freed_before, const float* __restrict__ here,
                                                char* __restrict__ scales_freed, int wave, int lane, v8i (&af)[2][2], v8i (&bf)[T::NB][2],
                                                v16f (&acc)[T::MB][T::NB]) {
  constexpr int ND = T::ADMA + T::BDMA, MB = T::MB, NB = T::NB, M = MB * NB;
  ld.early(wave, lane);
  float fs[MB];
  const int wr = wave / T::WC, wc = wave % T::WC;
  const float* const cs = here + T::BM + wc * NB * 32 + (T::SQUARES ? 0 : 4 * (lane >> 5));
  const float* const rs = here + wr * MB * 32 + (lane & 31);
#pragma unroll
  for (int x = 0; x < MB; ++x) fs[x] = rs[x * 32];
  if constexpr (T::SQUARES) {
    const float c = cs[0];
#pragma unroll
    for (int x = 0; x < MB; ++x) fs[x] *= c;
  }
  v16f t[2];
#pragma unroll
  for (int x = 0; x < MB; ++x) {
    const bool last = x + 1 == MB;
    if (last) {
      // the next stage's bytes and scales, older than the loads that may stay in flight
      half::wait_loads_and_lds<(T::BUFS - 2) * T::Loads::IN_FLIGHT>();
      half::block_barrier();
      sl.load(scales_freed, wave);
      ld.begin();
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int y = 0; y < NB; ++y) {
      const int i = x * NB + y;
      const int o = i - 1, ox = o / NB, oy = o % NB;  // the block before
      v4f c[4];
      if (i > 0) column_scales<T>(cs + oy * 32, c);
#pragma unroll
      for (int q = 0; q < T::STEPS; ++q) {
        products<T>(q, t[i & 1], bf[y], af[x & 1]);
        if (q + 1 == T::STEPS) {
          if (y == 0) {
#pragma unroll
            for (int h = 0; h < 2; ++h) af[(x + 1) & 1][h] = fa.read(last ? next : cur, h, last ? 0 : x + 1);
          }
          if (last) {
#pragma unroll
            for (int h = 0; h < 2; ++h) bf[y][h] = fb.read(next + T::A_BYTES, h, y);
#pragma unroll
            for (int j = y * T::SOON / NB; j < (y + 1) * T::SOON / NB; ++j) ld.late(j, freed, wave, lane);
          }
          if (x == 0) {
#pragma unroll
            for (int j = T::SOON + y * (ND - T::SOON) / NB; j < T::SOON + (y + 1) * (ND - T::SOON) / NB; ++j)
              ld.late(j, freed_before, wave, lane);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
        if (i > 0) {
          add_scaled<T, 16 / T::STEPS>(acc[ox][oy], t[o & 1], fs[ox], c, q * (16 / T::STEPS));
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
  }
  v4f c[4];
  column_scales<T>(cs + (NB - 1) * 32, c);
  add_scaled<T, 16>(acc[MB - 1][NB - 1], t[(M - 1) & 1], fs[MB - 1], c, 0);
  if constexpr (MB % 2) {
    af[0][0] = af[1][0];
    af[0][1] = af[1][1];
  }
  __builtin_amdgcn_sched_barrier(0);
}

// acc += A B over `depth` (at least 1), scaled.  lds: T::LDS bytes, 1024-aligned.
//
// As in the 16-bit tiles the last row of a stage's products runs behind the barrier
// that hands over to the next stage, whose first fragments are read meanwhile, and the
// buffer just freed takes the loads of the stage BUFS later.  Wavefronts whose outputs
// all lie past the tile's edge load and wait like the others.
template <class T>
__device__ __forceinline__ void product8(const Bytes& oa, const Bytes& ob, const Scales& sa, const Scales& sb, int cols,
                                         int depth, char* lds, v16f (&acc)[T::MB][T::NB]) {
  constexpr int ND = T::ADMA + T::BDMA, MB = T::MB, NB = T::NB;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = wave / T::WC, wc = wave % T::WC;
  const int nst = (depth + kStage - 1) / kStage;
  typename T::Loads ld;
  ScaleLoads<T> sl;
  ld.init(oa, ob, depth, wave, lane);
  sl.init(sa, sb, oa.vecs, cols, nst);
  char* const slots = lds + T::SET;
  sl.load(slots, wave);
  ld.first(lds, depth, wave, lane);
#pragma unroll
  for (int s = 1; s < T::BUFS; ++s) {
    ld.early(wave, lane);
    sl.load(slots + s * T::SLOT, wave);
    ld.begin();
#pragma unroll
    for (int j = 0; j < (s + 1 == T::BUFS ? T::SOON : ND); ++j) ld.late(j, lds + s * T::STAGE, wave, lane);
  }
  half::wait_loads_and_lds<(T::DMA ? (T::BUFS - 2) * T::Loads::IN_FLIGHT + T::SOON + 1 : 0)>();
  half::block_barrier();
  if (T::DMA && depth % 16) {
    clean_tail<T>(lds, depth % kStage);
    wait_lds_and_barrier();
  }
  int cur = 0, slot = 0;
  if (wr * MB * 32 >= oa.vecs || wc * NB * 32 >= cols) {
    for (int s = 0; s < nst; ++s) {
      const int before = slot == 0 ? T::BUFS * T::SLOT : slot - T::SLOT;
      slot = slot == T::BUFS * T::SLOT ? 0 : slot + T::SLOT;
      ld.early(wave, lane);
#pragma unroll
      for (int j = T::SOON; j < ND; ++j) ld.late(j, lds + next_stage<T>(cur), wave, lane);
      half::wait_loads_and_lds<(T::BUFS - 2) * T::Loads::IN_FLIGHT>();
      half::block_barrier();
      sl.load(slots + before, wave);
      ld.begin();
#pragma unroll
      for (int j = 0; j < T::SOON; ++j) ld.late(j, lds + cur, wave, lane);
      cur = next_stage<T>(cur);
    }
  } else {
    ByteFragments<MB> fa;
    ByteFragments<NB> fb;
    fa.init(wr * MB, lane);
    fb.init(wc * NB, lane);
    const auto l3 = (half::lds_bytes)lds;
    v8i af[2][2], bf[NB][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      af[0][h] = fa.read(l3, h, 0);
#pragma unroll
      for (int y = 0; y < NB; ++y) bf[y][h] = fb.read(l3 + T::A_BYTES, h, y);
    }
    for (int s = 0; s < nst; ++s) {
      const int next = next_stage<T>(cur), before = slot == 0 ? T::BUFS * T::SLOT : slot - T::SLOT;
      stage_products8<T>(ld, sl, fa, fb, l3 + cur, l3 + next, lds + cur, lds + next, (const float*)(slots + slot), slots + before,
                         wave, lane, af, bf, acc);
      cur = next;
      slot = slot == T::BUFS * T::SLOT ? 0 : slot + T::SLOT;
    }
  }
  __builtin_amdgcn_s_waitcnt(0);  // the look-ahead past the end lands before LDS is used again
  __syncthreads();
}

// The tile's sums to a row-major FP32 matrix.
template <class T>
__device__ __forceinline__ void store_sums(const v16f (&acc)[T::MB][T::NB], float* out, int64_t ld, int rows, int cols) {
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = wave / T::WC * T::MB * 32 + (lane & 31), col = wave % T::WC * T::NB * 32 + 4 * (lane >> 5);
#pragma unroll
  for (int a = 0; a < T::MB; ++a) {
    float* const p = out + (int64_t)(row + a * 32) * ld + col;
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

}  // namespace eight
}  // namespace oz
