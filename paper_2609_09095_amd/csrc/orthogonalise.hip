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
// polynomial's largest value, S by its square), so powers of two place those of a
// polynomial that is meant to converge in half's range (singular values below 7.9,
// |P| below 255; larger ones become infinities), and its 11 bits round eight times
// finer than the bfloat16 of the result.  Stored as X 2^8, S 2^10, P 2^8.
//
// S and P come close to multiples of the identity, and a rounding of their
// diagonals would be an error of every vector: the diagonals d and p are kept
// in 32 bits beside the matrices So, whose diagonal is stored as zeros, and Po:
//   (S^2)_ij = (So^2)_ij + (d_i + d_j) So_ij,  (S^2)_ii = (So^2)_ii + d_i^2,
//   (P X)_ij = (Po X)_ij + p_i X_ij.
//
// Po meets X rounded to half, with an error e, and p meets it in 32 bits.  Near the
// end S is near a multiple of the identity, and what is beside P's diagonal is
// small, and so is its product with e.  But without the diagonal that product is
// full of directions that X may not have (P e is not), and every later step
// multiplies such noise by a: 128 x 40 of rank 1 was 9e-3 of its norm from 64 bits,
// and 4 x 12 after eight steps all of it.  So only the last two steps take p in 32
// bits; in the others Po has a diagonal, rounded, and p is what that rounding left.
// Distance from 64 bits before the result's rounding (1.7e-3), 128 x 128 of rank 16
// and 128: p in 32 bits in all steps 2.1e-3 and 0.8e-3, in none 0.8e-3 and 1.4e-3,
// in the last two 0.8e-3 and 1.0e-3.
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
// underflow for any 32-bit input.  Bound by the read: 2 x 4096 x 4096 bfloat16
// 18.7 us (3.6 TB/s).  grid (parts, count)
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

// Division by |G|_F + eps: its reciprocal may be no normal 32-bit number where
// G's own elements are, so it is kept as a factor in [1/2, 1] and a power of two.
// A matrix of zeros is divided by nothing, whatever eps is.
struct Scaling {
  float factor;
  int power;
  __device__ __forceinline__ Scaling(double squares, float eps) {
    const double scale = squares == 0.0 ? 0.0 : 1.0 / (sqrt(squares) + (double)eps);
    power = __builtin_amdgcn_frexp_exp(scale);
    factor = (float)__builtin_amdgcn_frexp_mant(scale);
  }
  __device__ __forceinline__ float operator()(float x) const { return __builtin_ldexpf(x, power) * factor; }
};

// X_0 in both forms, padding included.  Bound by memory: 2 x 4096 x 4096 53 us
// (268 MB: 5.1 TB/s).  grid (blocks, count)
template <int TYPE>
__global__ __launch_bounds__(256) void start_kernel(Orthogonalise o, int parts) {
  double sum = 0;
  for (int i = threadIdx.x & 63; i < parts; i += 64) sum += o.squares[blockIdx.y * parts + i];
  for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
  const Scaling scale(sum, o.eps);
  const uint32_t chunks = (uint32_t)o.np / 8, total = chunks * (uint32_t)o.mp;
  const int64_t each = (int64_t)o.mp * o.np;
  for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < total; i += gridDim.x * 256) {
    const uint32_t r = i / chunks, c = (i - r * chunks) * 8;
    float x[8] = {};
    if ((int)r < o.m) row8<TYPE>(o.g, blockIdx.y * o.g_stride + r * o.ldg, c, o.n, x);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = (int)(c + j) < o.n && (int)r < o.m ? scale(x[j]) : 0.0f;
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

// P_ii in two: what Po has of it, as it is stored, and the rest, in 32 bits all of it;
// c_s2: c (So^2)_ii.
struct Diagonal {
  float stored, rest;
  __device__ __forceinline__ Diagonal(float b, float c, float d, float c_s2, bool in_32_bits) {
    const float p = (b + c * d) * d + c_s2;
    stored = in_32_bits ? 0.0f : (float)(_Float16)(p * kScaleP);
    rest = p - stored * (1.0f / kScaleP);
  }
};

constexpr __host__ __device__ bool diagonal_in_32_bits(int step, int steps) { return step + 2 >= steps; }

// The diagonal element that the lane holds of a WIDE block on the diagonal, set
// to zero there; false: it holds none.
__device__ __forceinline__ bool take_diagonal(v16f& v, float& mine) {
  const int lane = threadIdx.x & 63, r = lane & 31, c0 = 4 * (lane >> 5);
  mine = 0.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const bool here = r == c0 + 8 * (i >> 2) + (i & 3);
    mine = here ? v[i] : mine;
    v[i] = here ? 0.0f : v[i];
  }
  return (r >> 2 & 1) == lane >> 5;
}

// And one put there.
__device__ __forceinline__ void give_diagonal(v16f& v, float mine) {
  const int lane = threadIdx.x & 63, r = lane & 31, c0 = 4 * (lane >> 5);
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = r == c0 + 8 * (i >> 2) + (i & 3) ? mine : v[i];
}

// What store_wide left in LDS, transposed: out[c, r], whose rows have `rows`
// elements (a multiple of 8, at 16 bytes).  Transposing loads give a lane 8 of
// them, and 4 lanes a run of 64 bytes.
template <class T>
__device__ __forceinline__ void mirror_wide(char* lds, _Float16* out, int64_t ld, int rows, int cols) {
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r0 = wave / T::WC * T::MB * 32, c0 = wave % T::WC * T::NB * 32;
  constexpr int PITCH = T::NB * 64, CH = T::NB * 4;
  const auto mine = (lds_bytes)lds + wave * (T::MB * 32 * PITCH);
  const int group = 8 * (lane >> 4), r = group + (lane >> 2 & 3), c = 4 * (lane & 3);
  using tr = __attribute__((address_space(3))) v4s*;
  auto at = [&](int row, int col) { return (tr)(mine + row * PITCH + (((col >> 3) ^ (row & (CH - 1))) << 4) + (col & 7) * 2); };
#pragma unroll
  for (int b = 0; b < T::NB * 2; ++b) {
    const int col = c0 + b * 16 + (lane & 15);
#pragma unroll
    for (int a = 0; a < T::MB; ++a) {
      const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(at(a * 32 + r, b * 16 + c));
      const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(at(a * 32 + r + 4, b * 16 + c));
      const int row = r0 + a * 32 + group;
      if (row < rows && col < cols)
        *(v4i*)(out + (int64_t)col * ld + row) = __builtin_bit_cast(v4i, v8s{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
    }
  }
}

// A symmetric product A A^T (kAlong, A s x depth) or A^T A (kAcross, A
// depth x s), the tiles on and above the diagonal, each stored twice: S, or with
// SQUARE (A = So) P = b S + c S^2, their diagonals apart.  Block b takes the
// (b / sub^2)-th tile from `first` on, of the matrices' triangles of tiles one
// after the other, or its b % sub^2-th part where tiles of sub^2 times this size
// are meant.
//
// Bound by the matrix cores and, as one round of tiles, by what they do not
// overlap (first loads, mirror image): 2 x 4096 x 4096, 256 of 272 tiles: S 127 us,
// P 136 (1080 and 1010 TFLOP/s), the 16 left 26 and 27.  A contiguous range of the
// triangle per XCD instead of every eighth tile: 8 x 512 x 2048 262 / 306 us in all.
template <class T, bool SQUARE>
__global__ __launch_bounds__(T::THREADS, 1) void gram_kernel(Orthogonalise o, const char* in, int s, int depth,
                                                            int64_t ld, uint32_t first, uint32_t tiles, uint32_t sub) {
  __shared__ __attribute__((aligned(1024))) char lds[T::LDS];
  static_assert(T::BM == T::BN && T::LA == T::LB && T::OUT == kF16, "square tiles");
  const uint32_t side = ((uint32_t)s + T::BM * sub - 1) / (T::BM * sub), triangle = side * (side + 1) / 2;
  uint32_t place;
  if (!block_place(blockIdx.x, tiles * sub * sub, place)) return;
  const uint32_t tile = first + place / (sub * sub), part = place % (sub * sub);
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
  const char* const S = uniform(a + ((int64_t)r0 * s + c0) * 2);  // a tile's offsets fit 32 bits
  uint2 own[EARLY ? T::MB : 1][T::NB][4];
  auto load_own = [&](int x, uint2 (&v)[T::NB][4]) __attribute__((always_inline)) {
    const int r = w.row0 + 32 * x < rows ? w.row0 + 32 * x : rows - 1;
#pragma unroll
    for (int b = 0; b < T::NB; ++b)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int c = w.col0 + 32 * b + 8 * q;
        v[b][q] = *(const uint2*)(S + (uint32_t)(r * s + (c < cols ? c : 0)) * 2);
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
    // (b + c (d_i + d_j)) So_ij in the operands' scales
    const float ks = kScaleP / kScaleS, cs = o.c * ks, kc = o.c * kScaleP / (kScaleS * kScaleS);
    float4 dc[T::NB][4];
#pragma unroll
    for (int b = 0; b < T::NB; ++b)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int c = w.col0 + 32 * b + 8 * q;
        const float4 v = *(const float4*)(d + c0 + (c < cols ? c : 0));
        dc[b][q] = float4{cs * v.x, cs * v.y, cs * v.z, cs * v.w};
      }
#pragma unroll
    for (int x = 0; x < T::MB; ++x) {
      const float di = o.b * ks + cs * d[r0 + (w.row0 + 32 * x < rows ? w.row0 + 32 * x : rows - 1)];
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
            acc[x][b][4 * q + j] = __builtin_fmaf(di + dj[j], (float)e[j], kc * acc[x][b][4 * q + j]);
        }
    }
  } else {
#pragma unroll
    for (int x = 0; x < T::MB; ++x)
#pragma unroll
      for (int b = 0; b < T::NB; ++b) acc[x][b] *= kScaleS / (kScaleX * kScaleX);
  }
  // the diagonal apart: at most one element per lane and row of blocks
  float stored[T::MB] = {};
  if (tm == tn) {
#pragma unroll
    for (int x = 0; x < T::MB; ++x) {
      const int r = w.row0 + 32 * x;
      float mine = 0.0f;
#pragma unroll
      for (int b = 0; b < T::NB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) mine = r == w.col0 + 32 * b + 8 * (i >> 2) + (i & 3) ? acc[x][b][i] : mine;
      const bool here = r >= w.col0 && r < w.col0 + T::NB * 32 && (r - w.col0 & 4) == 0 && r < rows;
      const int at = r0 + (r < rows ? r : rows - 1);
      if constexpr (SQUARE) {
        // c (So^2)_ii 2^8 (So_ii is zero)
        const Diagonal p(o.b, o.c, d[at], mine * (1.0f / kScaleP), o.diagonal_in_32_bits);
        stored[x] = p.stored;
        if (here) diagonal[at] = p.rest;
      } else if (here) {
        diagonal[at] = mine * (1.0f / kScaleS);  // S_ii 2^10
      }
    }
  }
  int call = 0;  // block row a, block b and quad q in order: known when unrolled
  store_wide<T>(acc, lds, out, s, rows, cols, false, [&](int r, int c, float* v) {
    const int x = call++ / (T::NB * 4);
    if (tm != tn) return;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = r == c + j ? stored[x] : v[j];
  });
  if (tm == tn) return;
  mirror_wide<T>(lds, (_Float16*)(SQUARE ? o.p16 : o.s16) + z * square + (int64_t)c0 * s + r0, s, rows, cols);
}

// The wavefront's part of a large tile of a 32-bit matrix, 64 rows of it at a
// time, between memory and the wavefront's part of LDS in whole rows of 256
// bytes, whose 16-byte chunks are XOR-swizzled by the row.  (16 bytes per lane
// and row straight to registers touch 32 rows at once: 297 us against 277 for
// an update of 2 x 4096 x 4096.)
template <class T>
struct TileRows {
  const int64_t ld;  // elements, at most OZAKI25_MAX_SIDE
  const int rows, cols;  // what exists of the tile
  int row, ch;  // the lane's row of 4, its place in it
  int r0, c0;   // of the wavefront in the tile
  char* mine;
  __device__ __forceinline__ TileRows(char* lds, int64_t ld, int rows, int cols) : ld(ld), rows(rows), cols(cols) {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    r0 = wave / T::WC * T::MB * 32, c0 = wave % T::WC * T::NB * 32;
    mine = lds + wave * (64 * 256);
    row = lane >> 4, ch = lane & 15;
  }
  __device__ __forceinline__ int column(int i) const { return c0 + (ch ^ (4 * i + row & 15)) * 4; }
  // rows `first` to first + 63 of the wavefront's part; places past the edge are
  // clamped.  What the wavefront still reads of the rows before them comes first:
  // a load into LDS does not wait for reads that are queued.
  __device__ __forceinline__ void load(const float* tile, int first) const {
    wave_lds_ready();
    wait_lds();
    const auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)uniform((const char*)tile), (short)0, 0x7ffffff0, 0x00020000);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int r = r0 + first + 4 * i + row, c = column(i);
      const int at = ((r < rows ? r : rows - 1) * (int)ld + (c < cols ? c : 0)) * 4;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_ptr)(mine + i * 1024), 16, at, 0, 0, 0);
    }
    __builtin_amdgcn_s_waitcnt(0);
    wave_lds_ready();
  }
  __device__ __forceinline__ void store(float* tile, int first) const {
    wave_lds_ready();
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int r = r0 + first + 4 * i + row, c = column(i);
      const v4i v = *(const v4i*)(mine + i * 1024 + (threadIdx.x & 63) * 16);
      if (r < rows && c < cols) *(v4i*)(tile + r * ld + c) = v;
    }
    __builtin_amdgcn_s_waitcnt(0);  // read before the next load overwrites it
    wave_lds_ready();
  }
  // four elements of row r (of 64) from column c on
  __device__ __forceinline__ float4* at(int r, int c) const {
    return (float4*)(mine + r * 256 + (((c >> 2) ^ (r & 15)) << 4));
  }
};

// X <- a X + P X (kAlong x kAcross) or, TALL, a X + X P (kAlong x kAlong: P is
// symmetric).  LAST: the result to the caller's matrix.  grid (tiles, count)
//
// 2 x 4096 x 4096: 280 us for 275 GFLOP and 335 MB of X in and out (two rounds of
// tiles, 100 us of products each); 3 x 1537 x 515: 15 us.
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
  static_assert(EARLY || (T::NB == 2 && T::MB % 2 == 0 && T::LDS >= T::WAVES * 64 * 256));
  const TileRows<T> whole(lds, o.np, rows, cols);
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
  const int lane_row = threadIdx.x & 31, lane_col = 4 * (threadIdx.x >> 5 & 1);
#pragma unroll
  for (int x = 0; x < T::MB; ++x) {
    const int r = w.row0 + 32 * x < rows ? w.row0 + 32 * x : rows - 1;
    const float pi = TALL ? 0.0f : p[r0 + r];
    if constexpr (!EARLY)
      if (x % 2 == 0) whole.load(x32, 32 * x);
#pragma unroll
    for (int b = 0; b < T::NB; ++b)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int c = w.col0 + 32 * b + 8 * q;
        float4 v;
        if constexpr (EARLY)
          v = own[x][b][q];
        else
          v = *whole.at(lane_row + 32 * (x & 1), lane_col + 32 * b + 8 * q);
        const float4 pj = TALL ? *(const float4*)(p + c0 + (c < cols ? c : 0)) : float4{pi, pi, pi, pi};
        float4 y;
        y.x = __builtin_fmaf(o.a + pj.x, v.x, k * acc[x][b][4 * q]);
        y.y = __builtin_fmaf(o.a + pj.y, v.y, k * acc[x][b][4 * q + 1]);
        y.z = __builtin_fmaf(o.a + pj.z, v.z, k * acc[x][b][4 * q + 2]);
        y.w = __builtin_fmaf(o.a + pj.w, v.w, k * acc[x][b][4 * q + 3]);
        if constexpr (!LAST && !EARLY) *whole.at(lane_row + 32 * (x & 1), lane_col + 32 * b + 8 * q) = y;
        if constexpr (!LAST && EARLY)
          if (w.row0 + 32 * x < rows && c < cols) *(float4*)(x32 + (int64_t)r * o.np + c) = y;
        const float scale = LAST ? 1.0f : kScaleX;
        acc[x][b][4 * q] = y.x * scale;
        acc[x][b][4 * q + 1] = y.y * scale;
        acc[x][b][4 * q + 2] = y.z * scale;
        acc[x][b][4 * q + 3] = y.w * scale;
      }
    if constexpr (!LAST && !EARLY)
      if (x % 2 == 1) whole.store(x32, 32 * (x - 1));
  }
  auto as_is = [](int, int, float*) {};
  if constexpr (LAST)
    store_wide<T>(acc, lds, (char*)o.x + (blockIdx.y * o.x_stride + r0 * o.ldx + c0) * 2, o.ldx, o.m - r0, o.n - c0,
                  true, as_is);
  else
    store_wide<T>(acc, lds, next + (blockIdx.y * each + (int64_t)r0 * o.np + c0) * 2, o.np, rows, cols, false, as_is);
}

// ---- matrices of at most 128 x 128: all steps in one block ---------------------
// Eight wavefronts of 64 x 32 outputs; X in registers (32 bits) and, as the
// operands are needed, in LDS, one array for X and one for S and then P.  Their
// rows of 256 bytes have their 16-byte chunks XOR-swizzled by the row and are
// read both ways, along a row and (transposing loads) across rows.  Tall
// matrices are transposed as they are read and written.  32 x 128 x 128: a launch
// of 35 us where the steps' launches took 95.
constexpr int kSide = kOneLaunchSide, kRow = kSide * 2;
constexpr float kBlockX = 32.0f;  // X's scale here, whose square is S's
static_assert(kBlockX * kBlockX == kScaleS);

__device__ __forceinline__ int block_offset(int row, int col) {
  return row * kRow + (((col >> 3) ^ (row & 15)) << 4) + (col & 7) * 2;
}

// acc = A B over `depth` from LDS: A's rows along, B's rows along or across.
template <bool ACROSS>
__device__ __forceinline__ void block_product(lds_bytes a, lds_bytes b, int row0, int col0, int depth, v16f (&acc)[2]) {
  const int lane = threadIdx.x & 63;
  acc[0] = acc[1] = v16f{};
#pragma unroll  // offsets known when compiled: 32 x 128 x 128 42.4 -> 38.9 us
  for (int k = 0; k < kSide; k += 16) {
    if (k >= depth) break;

    v4i fa[2], fb;
    const int d = k + 8 * (lane >> 5);
#pragma unroll
    for (int x = 0; x < 2; ++x)
      fa[x] = *(const __attribute__((address_space(3))) v4i*)(a + block_offset(row0 + 32 * x + (lane & 31), d));
    if constexpr (ACROSS) {
      using tr = __attribute__((address_space(3))) v4s*;
      const int r = d + ((lane >> 2) & 3), c = col0 + (lane & 16) + 4 * (lane & 3);
      const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr)(b + block_offset(r, c)));
      const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr)(b + block_offset(r + 4, c)));
      fb = __builtin_bit_cast(v4i, v8s{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
    } else {
      fb = *(const __attribute__((address_space(3))) v4i*)(b + block_offset(col0 + (lane & 31), d));
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) acc[x] = mfma<kF16>(fb, fa[x], acc[x]);  // as WIDE tiles
  }
}

template <int TYPE>
__global__ __launch_bounds__(512, 1) void small_kernel(Orthogonalise o, int steps) {
  using E = typename Out<TYPE>::type;
  __shared__ __attribute__((aligned(1024))) char lds[2 * kSide * kRow + 2 * kSide * 4 + 8 * 8];
  char* const xs = lds;
  char* const ss = lds + kSide * kRow;
  float* const diag_s = (float*)(lds + 2 * kSide * kRow);
  float* const diag_p = diag_s + kSide;
  double* const sums = (double*)(diag_p + kSide);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row0 = (wave >> 2) * 64, col0 = (wave & 3) * 32;
  const int row = row0 + (lane & 31), col = col0 + 4 * (lane >> 5);
  const bool tall = o.m > o.n;
  const int s = tall ? o.n : o.m, l = tall ? o.m : o.n;
  const int64_t along = tall ? o.ldg : 1, across = tall ? 1 : o.ldg;  // strides of X's columns and rows in G
  const auto g = (const __attribute__((address_space(1))) E*)(global_bytes)o.g + blockIdx.x * o.g_stride;
  v16f X[2];
  double sum = 0;
#pragma unroll
  for (int x = 0; x < 2; ++x)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int r = row + 32 * x, c = col + 8 * (i >> 2) + (i & 3);
      const bool in = r < s && c < l;
      const float v = (float)g[(in ? r : 0) * across + (in ? c : 0) * along];
      X[x][i] = in ? v : 0.0f;
      sum += (double)X[x][i] * (double)X[x][i];
    }
  for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
  if (lane == 0) sums[wave] = sum;
  __syncthreads();
  const double square =
      ((sums[0] + sums[1]) + (sums[2] + sums[3])) + ((sums[4] + sums[5]) + (sums[6] + sums[7]));
  const Scaling scale(square, o.eps);
#pragma unroll
  for (int x = 0; x < 2; ++x)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      // (not by the product alone: padding stays zero for an infinite or NaN scale)
      const bool in = row + 32 * x < s && col + 8 * (i >> 2) + (i & 3) < l;
      X[x][i] = in ? scale(X[x][i]) * kBlockX : 0.0f;
    }
  // the four outputs of group q of block x to LDS
  auto put = [&](char* to, int x, int q, float v0, float v1, float v2, float v3) __attribute__((always_inline)) {
    *(uint2*)(to + block_offset(row + 32 * x, col + 8 * q)) = pack4<kF16>(v0, v1, v2, v3);
  };
  const auto x3 = (lds_bytes)xs, s3 = (lds_bytes)ss;
  const int depth_s = (s + 15) / 16 * 16, depth_l = (l + 15) / 16 * 16;
  v16f acc[2];
  const float ks = kScaleP / kScaleS, cs = o.c * ks, kc = o.c * kScaleP / (kScaleS * kScaleS);
  // Wavefronts whose outputs all lie past the edge only wait.  (Blocks of 32 rows
  // past it that share a wavefront may then hold anything: they are nobody's
  // depth and not stored.)
  const bool in_x = row0 < s && col0 < l, in_s = row0 < s && col0 < s;
  for (int step = 0; step < steps; ++step) {
    if (in_x) {
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          put(xs, x, q, X[x][4 * q], X[x][4 * q + 1], X[x][4 * q + 2], X[x][4 * q + 3]);
    }
    __syncthreads();
    if (in_s) {
      block_product<false>(x3, x3, row0, col0, depth_l, acc);
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        float mine;
        if (row0 + 32 * x == col0 && take_diagonal(acc[x], mine)) diag_s[row + 32 * x] = mine * (1.0f / kScaleS);
#pragma unroll
        for (int q = 0; q < 4; ++q)
          put(ss, x, q, acc[x][4 * q], acc[x][4 * q + 1], acc[x][4 * q + 2], acc[x][4 * q + 3]);
      }
    }
    __syncthreads();
    if (in_s) {
      block_product<false>(s3, s3, row0, col0, depth_s, acc);
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int r = row + 32 * x;
        const float d = diag_s[r], di = o.b * ks + cs * d;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          typedef _Float16 h4 __attribute__((ext_vector_type(4)));
          const int c = col + 8 * q;
          const h4 e = *(const h4*)(ss + block_offset(r, c));
          const float4 dj = *(const float4*)(diag_s + c);
          const float dc[4] = {cs * dj.x, cs * dj.y, cs * dj.z, cs * dj.w};
#pragma unroll
          for (int j = 0; j < 4; ++j)
            acc[x][4 * q + j] = __builtin_fmaf(di + dc[j], (float)e[j], kc * acc[x][4 * q + j]);
        }
        float mine;
        if (row0 + 32 * x == col0) {
          const bool holds = take_diagonal(acc[x], mine);
          const Diagonal p(o.b, o.c, d, mine * (1.0f / kScaleP), diagonal_in_32_bits(step, steps));
          if (holds) diag_p[r] = p.rest;
          give_diagonal(acc[x], p.stored);
        }
      }
    }
    __syncthreads();
    if (in_s) {
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          put(ss, x, q, acc[x][4 * q], acc[x][4 * q + 1], acc[x][4 * q + 2], acc[x][4 * q + 3]);
    }
    __syncthreads();
    if (in_x) {
      block_product<true>(s3, x3, row0, col0, depth_s, acc);
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const float a = o.a + diag_p[row + 32 * x];
#pragma unroll
        for (int i = 0; i < 16; ++i) X[x][i] = __builtin_fmaf(a, X[x][i], (1.0f / kScaleP) * acc[x][i]);
      }
    }
    __syncthreads();
  }
  const int64_t out_c = tall ? o.ldx : 1, out_r = tall ? 1 : o.ldx;
  __bf16* const out = (__bf16*)o.x + blockIdx.x * o.x_stride;
#pragma unroll
  for (int x = 0; x < 2; ++x)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int r = row + 32 * x, c = col + 8 * (i >> 2) + (i & 3);
      if (r < s && c < l) out[r * out_r + c * out_c] = (__bf16)(X[x][i] * (1.0f / kBlockX));
    }
}

template <int TYPE>
hipError_t start(const Orthogonalise& o, hipStream_t s) {
  const int parts = orthogonalise_parts(o.m, o.n);
  squares_kernel<TYPE><<<dim3(parts, o.count), dim3(256), 0, s>>>(o);
  const int64_t chunks = (int64_t)o.mp * o.np / 8, blocks = ceil_div(chunks, 256);
  start_kernel<TYPE><<<dim3((uint32_t)(blocks < 2048 ? blocks : 2048), o.count), dim3(256), 0, s>>>(o, parts);
  return hipGetLastError();
}

// Tile shapes: WR, WC, MB, NB, stages.  Small tiles with 3 / 4 stages (3 / 2 blocks
// per CU): 1 x 2048 x 2048 438 / 494 us, 1 x 1024 x 1024 147 / 145.
template <int WR, int WC, int MB, int NB, int BUFS>
struct Shape {
  template <int LA, int LB, int OUT>
  using Of = Tile<kF16, LA, LB, WR, WC, MB, NB, true, OUT, BUFS>;
};
using Large = Shape<2, 4, 4, 2, 2>;
using Middle = Shape<2, 2, 2, 2, 2>;
using Small = Shape<2, 2, 1, 1, 3>;

// `tiles` tiles of sub times the shape's side, from `first` on
template <class H, int L, bool SQUARE>
void gram(const Orthogonalise& o, const char* in, int s, int depth, int64_t ld, int64_t first, int64_t tiles, int sub,
          hipStream_t st) {
  using T = typename H::template Of<L, L, kF16>;
  const uint32_t blocks = ((uint32_t)(tiles * sub * sub) + 7) & ~7u;
  gram_kernel<T, SQUARE><<<dim3(blocks), dim3(T::THREADS), 0, st>>>(o, in, s, depth, ld, (uint32_t)first,
                                                                    (uint32_t)tiles, (uint32_t)sub);
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
hipError_t steps(Orthogonalise o, int count, hipStream_t st) {
  const int s = TALL ? o.np : o.mp, l = TALL ? o.mp : o.np;
  for (int i = 0; i < count; ++i) {
    const char* x = (const char*)o.x16[i & 1];
    char* next = (char*)o.x16[(i + 1) & 1];
    o.diagonal_in_32_bits = diagonal_in_32_bits(i, count);
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
  if (orthogonalise_in_one_launch(o.m, o.n)) {
    if (type == kBF16)
      small_kernel<kBF16><<<dim3(o.count), dim3(512), 0, s>>>(o, count_steps);
    else if (type == kF16)
      small_kernel<kF16><<<dim3(o.count), dim3(512), 0, s>>>(o, count_steps);
    else
      small_kernel<kF32><<<dim3(o.count), dim3(512), 0, s>>>(o, count_steps);
    return hipGetLastError();
  }
  const hipError_t e = type == kBF16 ? start<kBF16>(o, s) : type == kF16 ? start<kF16>(o, s) : start<kF32>(o, s);
  if (e != hipSuccess) return e;
  return o.m > o.n ? steps<true>(o, count_steps, s) : steps<false>(o, count_steps, s);
}

}  // namespace half
}  // namespace oz
