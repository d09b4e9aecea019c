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
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

namespace oz {
namespace half {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef short v8s __attribute__((ext_vector_type(8)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));
using lds_ptr = __attribute__((address_space(3))) void*;
using global_bytes = const __attribute__((address_space(1))) char*;
using lds_bytes = const __attribute__((address_space(3))) char*;

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
  int width;   // elements of a whole memory row
};

template <class T>
struct DmaLoads;
template <class T>
struct MaskedLoads;

// A tile's shape: WR x WC wavefronts, each MB x NB blocks of 32 x 32 outputs.
// OUT: the output type.  A 16-bit output's blocks are multiplied transposed
// (WIDE), which gives a lane four consecutive columns of one row.
// BUFS: stages in LDS.  KG: sets of such wavefronts, each with its own stages and
// a part of the depth; the first set adds up the sums and stores.
template <int TYPE_, int LA_, int LB_, int WR_, int WC_, int MB_, int NB_, bool DMA_, int OUT_, int BUFS_ = 2,
          int KG_ = 1>
struct Tile {
  static constexpr int TYPE = TYPE_, LA = LA_, LB = LB_, WR = WR_, WC = WC_, MB = MB_, NB = NB_, OUT = OUT_;
  static constexpr bool DMA = DMA_, WIDE = OUT_ != kF32;
  static constexpr int BM = WR * MB * 32, BN = WC * NB * 32;
  static constexpr int WAVES = WR * WC, KG = KG_, THREADS = KG * WAVES * 64;
  static constexpr int A_BYTES = BM * kDepth * 2, B_BYTES = BN * kDepth * 2;
  static constexpr int BUFS = BUFS_, STAGE = A_BYTES + B_BYTES, SET = BUFS * STAGE, LDS = KG * SET;
  static constexpr int ADMA = A_BYTES / 1024 / WAVES, BDMA = B_BYTES / 1024 / WAVES;
  using Loads = std::conditional_t<DMA, DmaLoads<Tile>, MaskedLoads<Tile>>;
  static_assert(KG == 1 || BM * BN * 4 <= SET, "a set's sums fit its stages' LDS");
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

// At most N vector loads in flight, no LDS access.
template <int N>
__device__ __forceinline__ void wait_loads_and_lds() {
  static_assert(N < 64);
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14));
}

// No LDS access in flight; any number of vector loads.
__device__ __forceinline__ void wait_lds() { __builtin_amdgcn_s_waitcnt(15 | 7 << 4 | 3 << 14); }

// A barrier that waits for nothing but the other wavefronts; no memory access
// moves over it.
__device__ __forceinline__ void block_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// ---- loaders ----------------------------------------------------------------
// Both fill the two stage buffers in prologue() and then, per stage,
//   early()                  while the stage is multiplied
//   begin(), late(j), end()  once its buffer is free: load j of the stage after next
template <int L, int V, int N>
struct DmaSide {
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

template <class T>
struct DmaLoads {
  DmaSide<T::LA, T::BM, T::ADMA> a;
  DmaSide<T::LB, T::BN, T::BDMA> b;
  __amdgpu_buffer_rsrc_t ra, rb;
  int left;
  __device__ __forceinline__ void init(const Operand& oa, const Operand& ob, int depth, int wave, int lane) {
    a.init(oa, depth, wave, lane);
    b.init(ob, depth, wave, lane);
    left = depth;
  }
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
    left -= kDepth;
    a.advance();
    b.advance();
  }
  __device__ __forceinline__ void early(int, int) {}
  __device__ __forceinline__ void prologue(char* lds, int wave, int lane) {
#pragma unroll
    for (int s = 0; s < T::BUFS; ++s) {
      begin();
#pragma unroll
      for (int j = 0; j < T::ADMA + T::BDMA; ++j) late(j, lds + s * T::STAGE, wave, lane);
      end();
    }
    wait();
    block_barrier();
  }
  // the first stage's loads have landed, or (a stage's own were the oldest) the
  // next one's; those of the stages behind it may be in flight
  __device__ __forceinline__ void wait() { wait_loads_and_lds<(T::BUFS - 1) * (T::ADMA + T::BDMA)>(); }
  __device__ __forceinline__ void wait_next() { wait_loads_and_lds<(T::BUFS - 2) * (T::ADMA + T::BDMA)>(); }
};

// The upper `have` (0 to 8) of 8 elements moved down, zeros above them.
__device__ __forceinline__ v4i keep_upper(v4i v, int have) {
  const int s = 16 * (8 - have);  // bits to drop; 128: all
  const uint4 x = __builtin_bit_cast(uint4, v);
  uint64_t lo = (uint64_t)x.y << 32 | x.x, hi = (uint64_t)x.w << 32 | x.z;
  const uint64_t up = hi << 1 << (63 - (s & 63));  // hi << (64 - s), also for s = 0
  lo = s < 64 ? lo >> (s & 63) | up : hi >> (s & 63);
  hi = s < 64 ? hi >> (s & 63) : 0;
  if (s == 128) lo = 0;
  return v4i{(int)lo, (int)(lo >> 32), (int)hi, (int)(hi >> 32)};
}

// Chunks of 8 elements at any alignment.  A chunk that the row's end cuts is
// read as the row's last 8 elements and shifted when it is put into LDS (one
// load like the others: reading it element by element cost the edge tiles
// three times the whole product's time).  Rows of fewer than 8 elements are
// read element by element.
template <int L, int V, int N>
struct MaskedSide {
  v4i reg[N];
  int have[N];      // elements of the chunk that exist
  int64_t whole[N];  // a stage with all 64 depths: bytes from its first element to what is read
  global_bytes p;
  int64_t ld;
  int64_t safe;  // bytes from the stage's first element to 8 elements that always exist
  int vecs;
  bool narrow;
  bool cuts;  // some lane's chunk is not whole
  __device__ __forceinline__ int existing(int r, int c, int left) const {
    const int rows = L == kAlong ? vecs : left, cols = L == kAlong ? left : vecs;
    const int n = cols - c * 8;
    return r < rows ? (n < 0 ? 0 : n < 8 ? n : 8) : 0;
  }
  __device__ __forceinline__ int64_t place(int r, int c, int n) const {
    return n > 0 ? (r * ld + c * 8 - (8 - n)) * 2 : safe;
  }
  __device__ __forceinline__ void init(const Operand& op, int depth, int wave, int lane) {
    p = (global_bytes)uniform(op.p);
    ld = op.ld;
    vecs = op.vecs;
    narrow = op.width < 8;
    const int first = L == kAlong ? depth : vecs;  // of the first row, from here on
    safe = first < 8 ? (first - 8) * 2 : 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      int r, c;
      chunk_at<L, V>((wave * N + i) * 1024 + lane * 16, r, c);
      // kAcross: a chunk that does not exist reads its row's last 8 elements,
      // wherever the stage is (kAlong: the first row's first ones, which `safe`
      // would move away from)
      have[i] = existing(r, c, kDepth);
      whole[i] = L == kAcross || have[i] > 0 ? (r * ld + (have[i] > 0 ? c * 8 - (8 - have[i]) : vecs - 8)) * 2 : 0;
    }
  }
  __device__ __forceinline__ void load(int wave, int lane, int left) {
    int64_t at[N];
    if (left >= kDepth) {
      // the common stage: nothing depends on how far the depth goes
      int least = 8;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        at[i] = whole[i];
        least = have[i] < least ? have[i] : least;
      }
      cuts = __builtin_amdgcn_ballot_w64(least < 8) != 0;
    } else {
      cuts = true;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        int r, c;
        chunk_at<L, V>((wave * N + i) * 1024 + lane * 16, r, c);
        have[i] = existing(r, c, left);
        at[i] = place(r, c, have[i]);
      }
    }
    if (!narrow) {
      // no branch around a load: its end would wait for the data
#pragma unroll
      for (int i = 0; i < N; ++i)
        __builtin_memcpy(&reg[i], (const __attribute__((address_space(1))) void*)(p + at[i]), 16);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        int r, c;
        chunk_at<L, V>((wave * N + i) * 1024 + lane * 16, r, c);
        const int n = existing(r, c, left < kDepth ? left : kDepth);
        v8s e{};
#pragma unroll
        for (int j = 0; j < 7; ++j)
          if (j < n) e[j] = ((const __attribute__((address_space(1))) short*)(p + (r * ld + c * 8) * 2))[j];
        reg[i] = __builtin_bit_cast(v4i, e);
      }
      cuts = false;
    }
    const int64_t step = (L == kAlong ? kDepth : ld * kDepth) * 2;
    p += step;
    safe -= step;
  }
  __device__ __forceinline__ void put(int i, char* lds, int wave, int lane) const {
    v4i v = reg[i];
    if (cuts) v = keep_upper(v, have[i]);
    *(v4i*)(lds + (wave * N + i) * 1024 + lane * 16) = v;
  }
};

template <class T>
struct MaskedLoads {
  MaskedSide<T::LA, T::BM, T::ADMA> a;
  MaskedSide<T::LB, T::BN, T::BDMA> b;
  int left;
  __device__ __forceinline__ void init(const Operand& oa, const Operand& ob, int depth, int wave, int lane) {
    a.init(oa, depth, wave, lane);
    b.init(ob, depth, wave, lane);
    left = depth;
  }
  __device__ __forceinline__ void early(int wave, int lane) {
    a.load(wave, lane, left);
    b.load(wave, lane, left);
    left -= kDepth;
  }
  __device__ __forceinline__ void begin() {}
  __device__ __forceinline__ void late(int j, char* buf, int wave, int lane) {
    if (j < T::ADMA)
      a.put(j, buf, wave, lane);
    else
      b.put(j - T::ADMA, buf + T::A_BYTES, wave, lane);
  }
  __device__ __forceinline__ void end() {}
  __device__ __forceinline__ void prologue(char* lds, int wave, int lane) {
#pragma unroll
    for (int s = 0; s < T::BUFS; ++s) {
      early(wave, lane);
#pragma unroll
      for (int j = 0; j < T::ADMA + T::BDMA; ++j) late(j, lds + s * T::STAGE, wave, lane);
    }
    __syncthreads();
  }
  __device__ __forceinline__ void wait_next() { wait_loads_and_lds<0>(); }
};

// Fragments of a wavefront's N blocks of 32 vectors from block w0 on.
template <int L, int V, int N>
struct Fragments {
  // kAlong: by K step (16 depths); kAcross: by block.  LDS byte offsets.
  int base[L == kAlong ? 4 : N];
  __device__ __forceinline__ void init(int w0, int lane) {
    if constexpr (L == kAlong) {
      const int v = w0 * 32 + (lane & 31);
      const int c = (lane >> 5) ^ swz_along(v);
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) base[ks] = v * 128 + ((c << 4) ^ (ks << 5));
    } else {
      const int d = 8 * (lane >> 5) + ((lane >> 2) & 3);
#pragma unroll
      for (int x = 0; x < N; ++x) {
        const int piece = (2 * (w0 + x) + ((lane >> 4) & 1)) ^ swz_across(d);
        base[x] = d * (V * 2) + piece * 32 + (lane & 3) * 8;
      }
    }
  }
  // kAlong: the offset of block 0 for a K step known at run time only
  __device__ __forceinline__ int at(int ks) const {
    static_assert(L == kAlong);
    return base[0] ^ (ks << 5);
  }
  // block x, K step ks of the stage at lds
  __device__ __forceinline__ v4i read(lds_bytes lds, int ks, int x) const {
    if constexpr (L == kAlong) {
      return *(const __attribute__((address_space(3))) v4i*)(lds + base[ks] + x * 4096);
    } else {
      using tr = __attribute__((address_space(3))) v4s*;
      const auto q = lds + base[x] + ks * (32 * V);
      const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr)q);
      const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr)(q + 8 * V));
      return __builtin_bit_cast(v4i, v8s{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
    }
  }
};

template <class T>
__device__ __forceinline__ int next_buffer(int cur) {
  if constexpr (T::BUFS == 2) return cur ^ T::STAGE;
  return cur + T::STAGE < T::SET ? cur + T::STAGE : 0;
}

// One stage's products; on entry the fragments of its first K step are in
// af[0], bf[0].  cur, next: this stage's and the next one's buffer; freed: cur,
// as the target of the loads.  The three are declared not to alias, or the
// compiler would wait for all loads in flight before every transposing read:
// what keeps them apart is the barrier.
template <class T, class Loader, class FA, class FB>
__device__ __forceinline__ void stage_products(Loader& ld, const FA& fa, const FB& fb, lds_bytes __restrict__ cur,
                                               lds_bytes __restrict__ next, char* __restrict__ freed, int wave,
                                               int lane, v4i (&af)[2][T::MB], v4i (&bf)[2][T::NB],
                                               v16f (&acc)[T::MB][T::NB]) {
  constexpr int ND = T::ADMA + T::BDMA, M = T::MB * T::NB, KS = kDepth / 16, R = T::MB + T::NB;
  ld.early(wave, lane);
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    const bool last = ks + 1 == KS;
    if (last) {
      ld.wait_next();
      block_barrier();
      ld.begin();
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < M; ++i) {
      // this product's share of the next step's fragments
#pragma unroll
      for (int f = i * R / M; f < (i + 1) * R / M; ++f) {
        if (f < T::MB)
          af[(ks + 1) & 1][f] = fa.read(last ? next : cur, (ks + 1) % KS, f);
        else
          bf[(ks + 1) & 1][f - T::MB] = fb.read((last ? next : cur) + T::A_BYTES, (ks + 1) % KS, f - T::MB);
      }
      if (last) {
#pragma unroll
        for (int j = i * ND / M; j < (i + 1) * ND / M; ++j) ld.late(j, freed, wave, lane);
      }
      const int x = i / T::NB, y = i % T::NB;
      acc[x][y] = T::WIDE ? mfma<T::TYPE>(bf[ks & 1][y], af[ks & 1][x], acc[x][y])
                          : mfma<T::TYPE>(af[ks & 1][x], bf[ks & 1][y], acc[x][y]);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  ld.end();
}

// acc += A B over `depth`; lds: T::LDS bytes, 1024-aligned.
//
// Two stages in LDS (three for small tiles).  The last K step's products of a
// stage run behind the barrier that hands over to the next stage: their
// fragments are in registers by then, so the matrix cores work while the next
// stage's first fragments are read, and the buffer just freed takes the loads
// of the stage that comes BUFS later, which then have BUFS - 1 stages' products
// to arrive.  The order of reads, loads and products is the written one
// (sched_barrier).
//
// Wavefronts whose rows all lie past the tile's edge load and wait like the
// others, but multiply nothing (the matrix cores and the clock are theirs).
//
// With KG sets of wavefronts all run the same number of stages (a set whose part
// is empty repeats the first one's and is left out of the sum).  The sums are
// added in the sets' order.  False: the wavefront's set is done.
template <class T>
__device__ __forceinline__ bool product(Operand a, Operand b, int depth, char* lds, v16f (&acc)[T::MB][T::NB]) {
  const int lane = threadIdx.x & 63;
  const int all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), set = all / T::WAVES, wave = all % T::WAVES;
  const int wr = wave / T::WC, wc = wave % T::WC;
  int nst = (depth + kDepth - 1) / kDepth;
  if (nst == 0) return set == 0;
  const int parts = nst;
  char* const sets = lds;
  if constexpr (T::KG > 1) {
    nst = (nst + T::KG - 1) / T::KG;
    const int first = set * nst < parts ? set * nst * kDepth : 0;
    a.p += (T::LA == kAlong ? (int64_t)first : first * a.ld) * 2;
    b.p += (T::LB == kAlong ? (int64_t)first : first * b.ld) * 2;
    depth -= first;
    lds += set * T::SET;
  }
  constexpr int ND = T::ADMA + T::BDMA;
  using Loader = typename T::Loads;
  Loader ld;
  ld.init(a, b, depth, wave, lane);
  ld.prologue(lds, wave, lane);
  const bool active = wr * T::MB * 32 < a.vecs;
  if (!active) {
    int cur = 0;
    for (int s = 0; s < nst; ++s) {
      ld.early(wave, lane);
      ld.wait_next();
      block_barrier();
      ld.begin();
#pragma unroll
      for (int j = 0; j < ND; ++j) ld.late(j, lds + cur, wave, lane);
      ld.end();
      cur = next_buffer<T>(cur);
    }
  } else {
    Fragments<T::LA, T::BM, T::MB> fa;
    Fragments<T::LB, T::BN, T::NB> fb;
    fa.init(wr * T::MB, lane);
    fb.init(wc * T::NB, lane);
    const auto l3 = (lds_bytes)lds;
    v4i af[2][T::MB], bf[2][T::NB];
#pragma unroll
    for (int x = 0; x < T::MB; ++x) af[0][x] = fa.read(l3, 0, x);
#pragma unroll
    for (int x = 0; x < T::NB; ++x) bf[0][x] = fb.read(l3 + T::A_BYTES, 0, x);
    int cur = 0;
    for (int s = 0; s < nst; ++s) {
      const int next = next_buffer<T>(cur);
      stage_products<T>(ld, fa, fb, l3 + cur, l3 + next, lds + cur, wave, lane, af, bf, acc);
      cur = next;
    }
  }
  __builtin_amdgcn_s_waitcnt(0);  // the look-ahead past the end (zeros) lands before LDS is used again
  __syncthreads();
  if constexpr (T::KG > 1) {
    constexpr int EACH = T::WAVES * 64;
    float* const mine = (float*)lds + wave * 64 + lane;
    if (set > 0) {
#pragma unroll
      for (int x = 0; x < T::MB; ++x)
#pragma unroll
        for (int y = 0; y < T::NB; ++y)
#pragma unroll
          for (int i = 0; i < 16; ++i) mine[((x * T::NB + y) * 16 + i) * EACH] = acc[x][y][i];
    }
    __syncthreads();
    if (set > 0) return false;
#pragma unroll
    for (int g = 1; g < T::KG; ++g) {
      if (g * nst >= parts) break;
      const float* const other = mine + g * (T::SET / 4);
#pragma unroll
      for (int x = 0; x < T::MB; ++x)
#pragma unroll
        for (int y = 0; y < T::NB; ++y)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[x][y][i] += other[((x * T::NB + y) * 16 + i) * EACH];
    }
  }
  return true;
}

// Four consecutive outputs of a row, rounded to 16 bits.
template <int OUT>
__device__ __forceinline__ uint2 pack4(float x, float y, float z, float w) {
  using O = typename Out<OUT>::type;
  typedef O o2 __attribute__((ext_vector_type(2)));
  const o2 lo = {(O)x, (O)y}, hi = {(O)z, (O)w};
  return uint2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
}

// What a wavefront wrote to its own part of LDS is there for all its lanes.
__device__ __forceinline__ void wave_lds_ready() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// The wavefront's blocks (WIDE tiles) through its part of LDS, which is free
// after the last stage, to a row-major 16-bit matrix: 16 bytes per lane, whole
// runs of 64 bytes.  rows, cols: what exists of the tile.  `stream`: past the caches, for outputs that do not fit them.
// value(r, c, v): the four outputs from row r, column c on, given the sums.
template <class T, class F>
__device__ __forceinline__ void store_wide(const v16f (&acc)[T::MB][T::NB], char* lds, void* out, int64_t ld, int rows,
                                           int cols, bool stream, F value) {
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r0 = wave / T::WC * T::MB * 32, c0 = wave % T::WC * T::NB * 32;
  constexpr int PITCH = T::NB * 64, CH = T::NB * 4;  // bytes and 16-byte chunks per row
  static_assert(T::MB * 32 * PITCH * T::WAVES <= T::LDS, "outputs fit the stages' LDS");
  char* const mine = lds + wave * (T::MB * 32 * PITCH);
  const int row = lane & 31, half = lane >> 5;
#pragma unroll
  for (int a = 0; a < T::MB; ++a)
#pragma unroll
    for (int b = 0; b < T::NB; ++b)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float v[4] = {acc[a][b][4 * q], acc[a][b][4 * q + 1], acc[a][b][4 * q + 2], acc[a][b][4 * q + 3]};
        value(r0 + a * 32 + row, c0 + b * 32 + 8 * q + 4 * half, v);
        char* p = mine + (a * 32 + row) * PITCH + (((b * 4 + q) ^ (row & (CH - 1))) << 4) + half * 8;
        *(uint2*)p = pack4<T::OUT>(v[0], v[1], v[2], v[3]);
      }
  wave_lds_ready();
  constexpr int RPI = 64 / CH, ROUNDS = T::MB * 32 / RPI;  // rows per instruction
  const int lr = lane / CH, ch = lane % CH;
  const int cleft = cols - c0 - ch * 8;
  short* const o = (short*)out + (int64_t)(r0 + lr) * ld + c0 + ch * 8;
  v4i v[ROUNDS];
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i) {
    const int r = i * RPI + lr;
    v[i] = *(const v4i*)(mine + r * PITCH + ((ch ^ (r & (CH - 1))) << 4));
  }
  const int rleft = cleft > 0 ? rows - r0 - lr : 0;
  // 16 bytes at any alignment; single elements where the row's end cuts them
  typedef v4i any_v4i __attribute__((aligned(2)));
  using to = __attribute__((address_space(1))) any_v4i*;
  if (cleft >= 8) {
    if (stream) {
#pragma unroll
      for (int i = 0; i < ROUNDS; ++i)
        if (i * RPI < rleft) __builtin_nontemporal_store((any_v4i)v[i], (to)(o + (int64_t)(i * RPI) * ld));
    } else {
#pragma unroll
      for (int i = 0; i < ROUNDS; ++i)
        if (i * RPI < rleft) *(to)(o + (int64_t)(i * RPI) * ld) = v[i];
    }
  } else if (cleft > 0) {
#pragma unroll
    for (int i = 0; i < ROUNDS; ++i)
      if (i * RPI < rleft) {
        short* const q = o + (int64_t)(i * RPI) * ld;
        const v8s e = __builtin_bit_cast(v8s, v[i]);
#pragma unroll
        for (int j = 0; j < 7; ++j)
          if (j < cleft) q[j] = e[j];
      }
  }
}

// The tile to a row-major matrix of type T::OUT, rounded once.  32-bit outputs
// are stored straight from registers, 32 consecutive columns per half wavefront,
// and always past the caches.  16384, 16, 4096, 2048 with and without: forward 275 /
// 287 us, weights' gradient in 32 bits 274 / 330, in 16 bits 249 / 287.
template <class T>
__device__ __forceinline__ void store(const v16f (&acc)[T::MB][T::NB], char* lds, void* out, int64_t ld, int rows,
                                      int cols, bool stream) {
  if constexpr (T::WIDE) {
    store_wide<T>(acc, lds, out, ld, rows, cols, stream, [](int, int, float*) {});
  } else {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // lane l of a block: column l % 32, rows 8 (i / 4) + 4 (l / 32) + i % 4
    const int row = wave / T::WC * T::MB * 32 + 4 * (lane >> 5), col = wave % T::WC * T::NB * 32 + (lane & 31);
    float* const o = (float*)out + (int64_t)row * ld + col;
#pragma unroll
    for (int a = 0; a < T::MB; ++a)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int r = a * 32 + 8 * (i >> 2) + (i & 3);
        float* const p = o + (int64_t)r * ld;
        if (row + r < rows) {
#pragma unroll
          for (int b = 0; b < T::NB; ++b)
            if (col + b * 32 < cols) __builtin_nontemporal_store(acc[a][b][i], p + b * 32);
        }
      }
  }
}

// ---- few rows ----------------------------------------------------------------
// The weights' columns as MFMA rows: 16 NB output columns x 16 TB rows of X,
// operands straight from memory into fragments.  Each weight is read once per
// block, so a block has few rows and its wavefronts split the depth.
typedef float v4f __attribute__((ext_vector_type(4)));

template <int TYPE>
__device__ __forceinline__ v4f mfma16(v4i a, v4i b, v4f c) {
  if constexpr (TYPE == kBF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8b, a), __builtin_bit_cast(v8b, b), c, 0, 0,
                                                   0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0,
                                                  0);
}

__device__ __forceinline__ v4i load_whole(const char* q) {
  v4i v;
  __builtin_memcpy(&v, (const __attribute__((address_space(1))) void*)(global_bytes)q, 16);
  return v;
}

// Elements c .. c + 7 of a row of `cols`; zeros past its end.  Any alignment;
// no branch around the load where rows have 8 elements.
__device__ __forceinline__ v4i load8(const char* row, int c, int cols) {
  const int n = cols - c, have = n < 0 ? 0 : n < 8 ? n : 8;
  if (cols >= 8) return keep_upper(load_whole(row + (int64_t)(have > 0 ? c - (8 - have) : 0) * 2), have);
  v8s e{};
  const auto q = (const __attribute__((address_space(1))) short*)(global_bytes)row;
#pragma unroll
  for (int j = 0; j < 7; ++j)
    if (j < have) e[j] = q[c + j];
  return __builtin_bit_cast(v4i, e);
}

// acc[i][j] += 16 columns of W (rows of its cols x k matrix, from w on) times
// 16 rows of X, over the depths 32 s0 .. 32 s1 (below k).  Rows past the last
// are read as the last one; their sums are not used.  U steps in flight.  Lane l of a block: row of
// X l % 16, columns 4 (l / 16) .. + 3.
template <int TYPE, int NB, int TB, int U>
__device__ __forceinline__ void skinny(const char* w, int64_t ldw, int cols, const char* x, int64_t ldx, int rows,
                                       int k, int s0, int s1, v4f (&acc)[NB][TB]) {
  const int lane = threadIdx.x & 63, at = lane & 15, c0 = (lane >> 4) * 8;
  const char *pw[NB], *px[TB];
#pragma unroll
  for (int i = 0; i < NB; ++i) pw[i] = w + (int64_t)(i * 16 + at < cols ? i * 16 + at : cols - 1) * ldw * 2;
#pragma unroll
  for (int j = 0; j < TB; ++j) px[j] = x + (int64_t)(j * 16 + at < rows ? j * 16 + at : rows - 1) * ldx * 2;
  const int whole = k / 32 < s1 ? k / 32 : s1;  // steps without an end inside
  int s = s0;
  for (; s + U <= whole; s += U) {
    v4i fw[U][NB], fx[U][TB];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t o = ((int64_t)(s + u) * 32 + c0) * 2;
#pragma unroll
      for (int i = 0; i < NB; ++i) fw[u][i] = load_whole(pw[i] + o);
#pragma unroll
      for (int j = 0; j < TB; ++j) fx[u][j] = load_whole(px[j] + o);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < TB; ++j) acc[i][j] = mfma16<TYPE>(fw[u][i], fx[u][j], acc[i][j]);
  }
  if (s < whole) {  // fewer than U: all loads, then all products
    v4i fw[U - 1][NB], fx[U - 1][TB];
#pragma unroll
    for (int u = 0; u < U - 1; ++u)
      if (s + u < whole) {
        const int64_t o = ((int64_t)(s + u) * 32 + c0) * 2;
#pragma unroll
        for (int i = 0; i < NB; ++i) fw[u][i] = load_whole(pw[i] + o);
#pragma unroll
        for (int j = 0; j < TB; ++j) fx[u][j] = load_whole(px[j] + o);
      }
#pragma unroll
    for (int u = 0; u < U - 1; ++u)
      if (s + u < whole) {
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
          for (int j = 0; j < TB; ++j) acc[i][j] = mfma16<TYPE>(fw[u][i], fx[u][j], acc[i][j]);
      }
    s = whole;
  }
  if (s < s1) {  // the step that the depth's end cuts
    v4i fw[NB], fx[TB];
#pragma unroll
    for (int i = 0; i < NB; ++i) fw[i] = load8(pw[i], s * 32 + c0, k);
#pragma unroll
    for (int j = 0; j < TB; ++j) fx[j] = load8(px[j], s * 32 + c0, k);
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int j = 0; j < TB; ++j) acc[i][j] = mfma16<TYPE>(fw[i], fx[j], acc[i][j]);
  }
}

// The WAVES wavefronts' sums added up in their order: calls f(row, column,
// four sums) once for every row and group of four columns of the block.
template <int NB, int TB, int WAVES, class F>
__device__ __forceinline__ void skinny_join(const v4f (&acc)[NB][TB], v4f* lds, F f) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  // [wave][row][column / 4], columns rotated by the row
  constexpr int Q = NB * 4;
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int j = 0; j < TB; ++j) {
      const int row = j * 16 + (lane & 15), q = i * 4 + (lane >> 4);
      lds[(wave * TB * 16 + row) * Q + ((q + row) & (Q - 1))] = acc[i][j];
    }
  __syncthreads();
  for (int o = threadIdx.x; o < TB * 16 * Q; o += WAVES * 64) {
    const int row = o / Q, q = o % Q;
    v4f v{};
#pragma unroll
    for (int w = 0; w < WAVES; ++w) v += lds[(w * TB * 16 + row) * Q + ((q + row) & (Q - 1))];
    f(row, q * 4, v);
  }
}

// ---- order of the tiles ------------------------------------------------------
// Place -> (row tile, column tile): row tiles in sets of kSet, column by column
// inside a set, so that the blocks an XCD runs at a time share panels.  Sets of
// 1, 2, 4, 8: 32768, 32, 2048, 4096 forward 535 / 540 / 560 / 562 us, 16384, 16,
// 4096, 2048 279 / 277 / 272 / 280, its input gradient 298 / 304 / 320 / 298, 8192^3
// 844 / 820 / 820 / 820.
constexpr uint32_t kSet = 2;
__device__ __forceinline__ void place_to_tile(uint32_t place, uint32_t tiles_m, uint32_t tiles_n, uint32_t& tm,
                                              uint32_t& tn) {
  const uint32_t per = kSet * tiles_n;
  const uint32_t s = place / per, in = place - s * per;
  const uint32_t first = s * kSet;
  const uint32_t size = tiles_m - first < kSet ? tiles_m - first : kSet;
  tn = in / size;
  tm = first + in - tn * size;
}

// Blocks are dealt round-robin over the 8 XCDs; each XCD takes one contiguous
// range of the places.  False: no place is left for this block.
__device__ __forceinline__ bool block_place(uint32_t b, uint32_t total, uint32_t& place) {
  const uint32_t x = b & 7, i = b >> 3, per = total >> 3, rem = total & 7;
  if (i >= per + (x < rem ? 1 : 0)) return false;
  place = x * per + (x < rem ? x : rem) + i;
  return true;
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
__device__ __forceinline__ int group_end(const int32_t* ends, int groups, int rows, int g0, int lane) {
  const int g = g0 + lane;
  const int e = g < groups ? ends[g] : rows;
  return e < 0 ? 0 : (e > rows ? rows : e);
}
__device__ __forceinline__ void group_rows(int e, int lane, int& last, int& first, int& end) {
  e = scan64(e > last ? e : last, [](int a, int b) { return a > b ? a : b; });
  const int before = __builtin_amdgcn_update_dpp(0, e, 0x138, 0xf, 0xf, false);  // wave_shr:1
  first = lane == 0 ? last : before;
  end = e;
  last = __builtin_amdgcn_readlane(e, 63);
}

// The row tiles of a grouped product with tiles of BM rows.  Up to 255 groups
// are read once, all loads in flight, and stay in registers.
struct RowTile {
  int group, row, rows;
};

template <int BM>
struct RowTiles {
  static constexpr int HELD = 4;
  const int32_t* ends;
  int groups, rows, lane;
  int first[HELD], end[HELD];

  // calls f(first group, first rows, ends) for each 64 groups until it returns true
  template <class F>
  __device__ __forceinline__ bool each(F f) {
    if (groups < HELD * 64) {
#pragma unroll
      for (int i = 0; i < HELD; ++i)
        if (i * 64 <= groups && f(i * 64, first[i], end[i])) return true;
      return false;
    }
    int last = 0;
    for (int g0 = 0; g0 <= groups; g0 += 64) {
      int a, b;
      group_rows(group_end(ends, groups, rows, g0, lane), lane, last, a, b);
      if (f(g0, a, b)) return true;
    }
    return false;
  }
  // returns the number of tiles
  __device__ __forceinline__ int init(const int32_t* e, int ng, int nr) {
    ends = e;
    groups = ng;
    rows = nr;
    lane = threadIdx.x & 63;
    if (groups < HELD * 64) {
      int v[HELD], last = 0;
#pragma unroll
      for (int i = 0; i < HELD; ++i) v[i] = i * 64 <= groups ? group_end(ends, groups, rows, i * 64, lane) : rows;
#pragma unroll
      for (int i = 0; i < HELD; ++i)
        if (i * 64 <= groups) group_rows(v[i], lane, last, first[i], end[i]);
    }
    int total = 0;
    each([&](int, int a, int b) {
      total += __builtin_amdgcn_readlane(scan64((b - a + BM - 1) / BM, [](int x, int y) { return x + y; }), 63);
      return false;
    });
    return total;
  }
  // tile number t: its group (`groups` for rows of no group), first row and
  // number of rows; false past the last
  __device__ __forceinline__ bool find(int t, RowTile& out) {
    int before = 0;
    return each([&](int g0, int a, int b) {
      const int mine = (b - a + BM - 1) / BM;
      const int incl = scan64(mine, [](int x, int y) { return x + y; });
      const uint64_t past = __builtin_amdgcn_ballot_w64(before + incl > t);
      if (past) {
        const int l = __builtin_ctzll(past);
        out.group = g0 + l;
        out.row = __builtin_amdgcn_readlane(a, l) + (t - before - __builtin_amdgcn_readlane(incl - mine, l)) * BM;
        const int left = __builtin_amdgcn_readlane(b, l) - out.row;
        out.rows = left < BM ? left : BM;
        return true;
      }
      before += __builtin_amdgcn_readlane(incl, 63);
      return false;
    });
  }
};

}  // namespace half
}  // namespace oz
