// Products of 16-bit floating-point matrices (bfloat16 or IEEE half) on
// gfx950's matrix cores: one output tile of C = A B per block, FP32
// accumulation in registers.
//
// Every product of two 16-bit numbers is exact in FP32, so the only roundings
// are those of the FP32 sums and the one of the result.
//
// An operand is a set of vectors (rows of the output for A, columns for B)
// along a common depth.  In memory either the depth is contiguous (kAlong: a
// vector is a row of `ld` elements) or the vectors are (kAcross: a depth is a
// row of `ld` elements).  A stage is 64 depths of a tile's vectors, 128 bytes
// each, in LDS:
//  kAlong:  a row of 128 bytes per vector, its eight 16-byte chunks XOR-swizzled
//           by the vector, read as b128 fragments (8 depths of one vector);
//  kAcross: a row per depth, its 32-byte pieces (16 vectors) XOR-swizzled by
//           the depth, read with the LDS transpose loads (4 depths of one
//           vector for each of 16 lanes).
// Both give lane l of a 32 x 32 x 16 MFMA the depths 8 (l / 32) .. + 7 of
// vector l % 32, so any two layouts combine.
//
// Two ways into LDS:
//  DMA:    buffer loads with the lds bit, 16 bytes per lane, where every row
//          starts on 16 bytes and sizes are multiples of 8 elements.  Rows
//          past the edge fall outside the descriptor and read as zero; chunks
//          past the depth are sent outside it.
//  masked: through registers with element bounds, for any pitch, size and
//          2-byte alignment.
// Two stages; a stage's loads are issued while the previous one is multiplied.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace oz {
namespace half {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef short v8s __attribute__((ext_vector_type(8)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));
using lds_ptr = __attribute__((address_space(3))) void*;

constexpr int kBF16 = 0, kF16 = 1, kF32 = 2;  // element types (ozaki25_dtype)
constexpr int kAlong = 0, kAcross = 1;        // operand layouts
constexpr int kDepth = 64;                    // depths per stage

template <int TYPE>
__device__ __forceinline__ v16f mfma(v4i a, v4i b, v16f c) {
  if constexpr (TYPE == kBF16)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8b, a), __builtin_bit_cast(v8b, b), c, 0, 0,
                                                   0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0,
                                                  0);
}

// FP32 to the output type, round to nearest even
template <int TYPE>
struct Out;
template <>
struct Out<kBF16> {
  using type = __bf16;
};
template <>
struct Out<kF16> {
  using type = _Float16;
};
template <>
struct Out<kF32> {
  using type = float;
};

__device__ __forceinline__ int swz_along(int vec) { return (vec & 7) ^ ((vec >> 3) & 1); }
__device__ __forceinline__ int swz_across(int d) { return d & 3; }

__device__ __forceinline__ const char* uniform(const void* p) {
  const uint64_t v = (uint64_t)p;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
  return (const char*)(((uint64_t)hi << 32) | lo);
}

// One operand of a tile: p at its first vector and depth.
struct Operand {
  const char* p;
  int64_t ld;  // elements
  int vecs;    // vectors that exist, at most the tile's
};

// A tile's shape: WR x WC wavefronts, each MB x NB blocks of 32 x 32 outputs.
template <int TYPE_, int LA_, int LB_, int WR_, int WC_, int MB_, int NB_, bool DMA_>
struct Tile {
  static constexpr int TYPE = TYPE_, LA = LA_, LB = LB_, WR = WR_, WC = WC_, MB = MB_, NB = NB_;
  static constexpr bool DMA = DMA_;
  static constexpr int BM = WR * MB * 32, BN = WC * NB * 32;
  static constexpr int WAVES = WR * WC, THREADS = WAVES * 64;
  static constexpr int A_BYTES = BM * kDepth * 2, B_BYTES = BN * kDepth * 2;
  static constexpr int STAGE = A_BYTES + B_BYTES, LDS = 2 * STAGE;
  static constexpr int ADMA = A_BYTES / 1024 / WAVES, BDMA = B_BYTES / 1024 / WAVES;
  static_assert(ADMA * WAVES * 1024 == A_BYTES && BDMA * WAVES * 1024 == B_BYTES, "whole slabs per wavefront");
};

// LDS byte o of a kAlong (kAcross) stage of V vectors holds chunk `c` (8
// elements) of row `r`: row = vector (depth), chunk along the depth (vectors).
template <int L, int V>
__device__ __forceinline__ void chunk_at(int o, int& r, int& c) {
  if constexpr (L == kAlong) {
    r = o >> 7;
    c = ((o >> 4) & 7) ^ swz_along(r);
  } else {
    r = o / (V * 2);
    const int pos = (o >> 4) % (V / 8);
    c = ((pos >> 1) ^ swz_across(r)) << 1 | (pos & 1);
  }
}

// ---- DMA loader -----------------------------------------------------------
template <int L, int V, int N>
struct Dma {
  int voff[N];  // byte offset of each of the wavefront's N slabs' chunks
  int dep[N];   // first depth of that chunk (kAlong)
  const char* p;
  int64_t step;    // bytes from stage to stage
  int64_t extent;  // bytes from p to the end of the last valid row
  __device__ __forceinline__ void init(const Operand& op, int depth, int wave, int lane) {
    p = uniform(op.p);
    step = L == kAlong ? kDepth * 2 : op.ld * kDepth * 2;
    const int64_t rows = L == kAlong ? op.vecs : depth, cols = L == kAlong ? depth : op.vecs;
    extent = rows > 0 && cols > 0 ? ((rows - 1) * op.ld + cols) * 2 : 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      int r, c;
      chunk_at<L, V>((wave * N + i) * 1024 + lane * 16, r, c);
      voff[i] = (int)(r * op.ld * 2) + c * 16;
      dep[i] = c * 8;
    }
  }
  // the descriptor of the next stage's piece; `left`: depths that remain
  __device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc(int left) const {
    const int64_t e = left > 0 ? extent : 0;
    const int n = (int)(e < 0x7ffffff0 ? e : 0x7ffffff0);
    return __builtin_amdgcn_make_buffer_rsrc((void*)p, (short)0, __builtin_amdgcn_readfirstlane(n), 0x00020000);
  }
  __device__ __forceinline__ void load(int i, __amdgpu_buffer_rsrc_t r, char* lds, int wave, int left) const {
    int off = voff[i];
    if constexpr (L == kAlong) off = dep[i] < left ? off : 0x7ffffff8;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_ptr)(lds + (wave * N + i) * 1024), 16, off, 0, 0, 0);
  }
  __device__ __forceinline__ void advance() {
    p += step;
    extent -= step;
  }
};

// ---- masked loader --------------------------------------------------------
template <int L, int V, int N>
struct Masked {
  v4i reg[N];
  const char* p;
  int64_t ld;
  int vecs;
  __device__ __forceinline__ void init(const Operand& op) {
    p = uniform(op.p);
    ld = op.ld;
    vecs = op.vecs;
  }
  __device__ __forceinline__ void load(int wave, int lane, int left) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      int r, c;
      chunk_at<L, V>((wave * N + i) * 1024 + lane * 16, r, c);
      const int rows = L == kAlong ? vecs : left, cols = L == kAlong ? left : vecs;
      const int have = r < rows ? cols - c * 8 : 0;
      v4i v{};
      if (have > 0) {
        const char* q = p + ((int64_t)r * ld + c * 8) * 2;
        if (have >= 8) {
          __builtin_memcpy(&v, q, 16);
        } else {
          v8s e{};
#pragma unroll
          for (int j = 0; j < 7; ++j)
            if (j < have) e[j] = ((const short*)q)[j];
          v = __builtin_bit_cast(v4i, e);
        }
      }
      reg[i] = v;
    }
  }
  __device__ __forceinline__ void put(char* lds, int wave, int lane) const {
#pragma unroll
    for (int i = 0; i < N; ++i) *(v4i*)(lds + (wave * N + i) * 1024 + lane * 16) = reg[i];
  }
  __device__ __forceinline__ void advance() { p += L == kAlong ? kDepth * 2 : ld * kDepth * 2; }
};

// Fragment of the 32 vectors from v0 for depths 16 ks .. + 15 of a stage.
template <int L, int V>
__device__ __forceinline__ v4i frag(const char* lds, int v0, int ks, int lane) {
  if constexpr (L == kAlong) {
    const int v = v0 + (lane & 31);
    return *(const v4i*)(lds + v * 128 + (((2 * ks + (lane >> 5)) ^ swz_along(v)) << 4));
  } else {
    using tr = __attribute__((address_space(3))) v4s*;
    const int d = 16 * ks + 8 * (lane >> 5) + ((lane >> 2) & 3);
    const int piece = ((v0 >> 4) + ((lane >> 4) & 1)) ^ swz_across(d);
    const char* q = lds + d * (V * 2) + piece * 32 + (lane & 3) * 8;
    const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr)q);
    const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr)(q + 4 * V * 2));
    return __builtin_bit_cast(v4i, v8s{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
  }
}

// One stage's products; `issue(j)` starts the j-th of ND loads of the next
// stage among the first MFMAs.
template <class T, int ND, class F>
__device__ __forceinline__ void stage_mma(const char* la, const char* lb, int wr, int wc, int lane,
                                          v16f (&acc)[T::MB][T::NB], F issue) {
  v4i af[4][T::MB], bf[4][T::NB];
#pragma unroll
  for (int ks = 0; ks < 4; ++ks) {
#pragma unroll
    for (int x = 0; x < T::MB; ++x) af[ks][x] = frag<T::LA, T::BM>(la, (wr * T::MB + x) * 32, ks, lane);
#pragma unroll
    for (int x = 0; x < T::NB; ++x) bf[ks][x] = frag<T::LB, T::BN>(lb, (wc * T::NB + x) * 32, ks, lane);
  }
#pragma unroll
  for (int ks = 0; ks < 4; ++ks)
#pragma unroll
    for (int a = 0; a < T::MB; ++a)
#pragma unroll
      for (int b = 0; b < T::NB; ++b) {
        const int j = (ks * T::MB + a) * T::NB + b;
        if (j < ND) issue(j);
        acc[a][b] = mfma<T::TYPE>(af[ks][a], bf[ks][b], acc[a][b]);
      }
  // reads of K step ks + 1 among the MFMAs of step ks, the loads among step 0's
  constexpr int PER = (T::LA == kAcross ? 2 : 1) * T::MB + (T::LB == kAcross ? 2 : 1) * T::NB;  // reads per step
  constexpr int M = T::MB * T::NB;                                                           // MFMAs per step
  __builtin_amdgcn_sched_group_barrier(0x100, PER, 0);
#pragma unroll
  for (int ks = 0; ks < 4; ++ks)
#pragma unroll
    for (int i = 0; i < M; ++i) {
      if (ks < 3) __builtin_amdgcn_sched_group_barrier(0x100, (PER + M - 1) / M, 0);
      if (ks * M + i < ND) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    }
}

// acc += A B over `depth`; lds: T::LDS bytes, 1024-aligned.
template <class T>
__device__ __forceinline__ void product(const Operand& a, const Operand& b, int depth, char* lds,
                                        v16f (&acc)[T::MB][T::NB]) {
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = wave / T::WC, wc = wave % T::WC;
  const int nst = (depth + kDepth - 1) / kDepth;
  if (nst == 0) return;
  char* const buf0 = lds;
  char* const buf1 = lds + T::STAGE;
  if constexpr (T::DMA) {
    Dma<T::LA, T::BM, T::ADMA> da;
    Dma<T::LB, T::BN, T::BDMA> db;
    da.init(a, depth, wave, lane);
    db.init(b, depth, wave, lane);
    int left = depth;
    auto start = [&](char* buf) {
      const auto ra = da.rsrc(left), rb = db.rsrc(left);
#pragma unroll
      for (int i = 0; i < T::ADMA; ++i) da.load(i, ra, buf, wave, left);
#pragma unroll
      for (int i = 0; i < T::BDMA; ++i) db.load(i, rb, buf + T::A_BYTES, wave, left);
    };
    auto next = [&]() {
      left -= kDepth;
      da.advance();
      db.advance();
    };
    auto stage = [&](char* cur, char* nxt) __attribute__((always_inline)) {
      __builtin_amdgcn_s_waitcnt(0);
      __syncthreads();
      next();
      const auto ra = da.rsrc(left), rb = db.rsrc(left);
      stage_mma<T, T::ADMA + T::BDMA>(cur, cur + T::A_BYTES, wr, wc, lane, acc, [&](int j) {
        if (j < T::ADMA)
          da.load(j, ra, nxt, wave, left);
        else
          db.load(j - T::ADMA, rb, nxt + T::A_BYTES, wave, left);
      });
    };
    start(buf0);
    for (int s = 0; s < nst; s += 2) {
      stage(buf0, buf1);
      if (s + 1 >= nst) break;
      stage(buf1, buf0);
    }
    __builtin_amdgcn_s_waitcnt(0);  // the look-ahead past the end (zeros) lands before LDS is used again
    __syncthreads();
  } else {
    Masked<T::LA, T::BM, T::ADMA> ma;
    Masked<T::LB, T::BN, T::BDMA> mb;
    ma.init(a);
    mb.init(b);
    int left = depth;
    ma.load(wave, lane, left);
    mb.load(wave, lane, left);
    ma.put(buf0, wave, lane);
    mb.put(buf0 + T::A_BYTES, wave, lane);
    char* cur = buf0;
    char* nxt = buf1;
    for (int s = 0; s < nst; ++s) {
      __syncthreads();
      left -= kDepth;
      ma.advance();
      mb.advance();
      if (s + 1 < nst) {
        ma.load(wave, lane, left);
        mb.load(wave, lane, left);
      }
      stage_mma<T, 0>(cur, cur + T::A_BYTES, wr, wc, lane, acc, [](int) {});
      if (s + 1 < nst) {
        ma.put(nxt, wave, lane);
        mb.put(nxt + T::A_BYTES, wave, lane);
      }
      char* t = cur;
      cur = nxt;
      nxt = t;
    }
    __syncthreads();
  }
}

// Calls f(row, column, value) for every output of the wavefront's blocks: lane
// l of a 32 x 32 block holds column l % 32, rows 8 (i / 4) + 4 (l / 32) + i % 4.
template <class T, class F>
__device__ __forceinline__ void each_output(const v16f (&acc)[T::MB][T::NB], F f) {
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r0 = wave / T::WC * T::MB * 32 + 4 * (lane >> 5), c0 = wave % T::WC * T::NB * 32 + (lane & 31);
#pragma unroll
  for (int a = 0; a < T::MB; ++a)
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
      for (int b = 0; b < T::NB; ++b) f(r0 + a * 32 + 8 * (i >> 2) + (i & 3), c0 + b * 32, acc[a][b][i]);
}

// The tile's rows < rows and columns < cols to a row-major matrix, one
// rounding to its type.
template <class T, int OUT>
__device__ __forceinline__ void store(const v16f (&acc)[T::MB][T::NB], void* out, int64_t ld, int rows, int cols) {
  using O = typename Out<OUT>::type;
  O* const o = (O*)out;
  each_output<T>(acc, [&](int r, int c, float v) {
    if (r < rows && c < cols) o[(int64_t)r * ld + c] = (O)v;
  });
}

// ---- groups of rows ---------------------------------------------------------
// Inclusive scans over the 64 lanes of a wavefront (values of at least 0).
template <class F>
__device__ __forceinline__ int scan64(int v, F f) {
  v = f(v, __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false));  // row_shr:1
  v = f(v, __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false));  // row_shr:2
  v = f(v, __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false));  // row_shr:4
  v = f(v, __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false));  // row_shr:8
  v = f(v, __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false));  // row_bcast:15
  v = f(v, __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false));  // row_bcast:31
  return v;
}

// 64 groups from g0: the lane's group's rows [first, end), ends clamped to
// [the previous end, rows] whatever the array holds.  Group number `groups`
// is what no group covers, [last end, rows).  `last` carries from call to call.
__device__ __forceinline__ void group_rows(const int32_t* ends, int groups, int rows, int g0, int lane, int& last,
                                           int& first, int& end) {
  const int g = g0 + lane;
  int e = g < groups ? ends[g] : rows;
  e = e < 0 ? 0 : (e > rows ? rows : e);
  e = scan64(e > last ? e : last, [](int a, int b) { return a > b ? a : b; });
  const int before = __builtin_amdgcn_update_dpp(0, e, 0x138, 0xf, 0xf, false);  // wave_shr:1
  first = lane == 0 ? last : before;
  end = e;
  last = __builtin_amdgcn_readlane(e, 63);
}

// The row tile number t of a grouped product with tiles of BM rows: its group
// (`groups` for rows of no group), first row and number of rows; false past
// the last tile.  total: the number of row tiles.
template <int BM>
__device__ __forceinline__ int count_row_tiles(const int32_t* ends, int groups, int rows) {
  const int lane = threadIdx.x & 63;
  int last = 0, total = 0;
  for (int g0 = 0; g0 <= groups; g0 += 64) {
    int first, end;
    group_rows(ends, groups, rows, g0, lane, last, first, end);
    const int t = (end - first + BM - 1) / BM;
    total += __builtin_amdgcn_readlane(scan64(t, [](int a, int b) { return a + b; }), 63);
  }
  return total;
}

struct RowTile {
  int group, row, rows;
};

template <int BM>
__device__ __forceinline__ bool find_row_tile(const int32_t* ends, int groups, int rows, int t, RowTile& out) {
  const int lane = threadIdx.x & 63;
  int last = 0, before = 0;
  for (int g0 = 0; g0 <= groups; g0 += 64) {
    int first, end;
    group_rows(ends, groups, rows, g0, lane, last, first, end);
    const int mine = (end - first + BM - 1) / BM;
    const int incl = scan64(mine, [](int a, int b) { return a + b; });
    const uint64_t past = __builtin_amdgcn_ballot_w64(before + incl > t);
    if (past) {
      const int l = __builtin_ctzll(past);
      const int in = t - before - __builtin_amdgcn_readlane(incl - mine, l);
      out.group = g0 + l;
      out.row = __builtin_amdgcn_readlane(first, l) + in * BM;
      const int left = __builtin_amdgcn_readlane(end, l) - out.row;
      out.rows = left < BM ? left : BM;
      return true;
    }
    before += __builtin_amdgcn_readlane(incl, 63);
  }
  return false;
}

}  // namespace half
}  // namespace oz
