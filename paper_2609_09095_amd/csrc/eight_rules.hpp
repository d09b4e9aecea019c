// The rules by which the 8-bit path chooses its kernels, from sizes alone.
// Plain C++, so that they also compile for the host's tests.
#pragma once

#include <cstddef>
#include <cstdint>

namespace oz {
namespace eight {

constexpr int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

constexpr int kMaxNormWidth = 32768;

// How a norm's row is spread: `lanes` threads with `chunks` times 8 elements each: one
// chunk a lane where a block has the lanes, in steps of 64 lanes up to 256 and as fine
// as the kernels' instances go beyond.  us, steps of 64 / powers of two: gradients of
// 4999 x 1031 halves 21.7 / 23.0, the norm of 8192 x 1031 18.6 / 20.8.  One chunk a lane
// / two on half the lanes: gradients of 16384 x 4096 bfloat16 103 / 158 (a second read
// of the row), of 4999 x 1031 22 / 31, the norms of 8192 x 4096 46 / 45, 8192 x 1031
// 18.6 / 22.  768 / 1024 lanes with two chunks: 4096 x 12288 bfloat16 71 / 73, gradients 94
// / 103, of 5852 x 9152 118 / 131.  Sums run over 16 lanes at least, and rows of 64 leave half
// of those idle: 262144 x 64 17.9 us, x 128 21.1.
struct NormForm {
  int lanes, chunks;
};

constexpr NormForm norm_form(int64_t width) {
  const int64_t c = ceil_div(width, 8);
  if (c <= 16) return {16, 1};
  if (c <= 32) return {32, 1};
  if (c <= 256) return {(int)ceil_div(c, 64) * 64, 1};
  if (c <= 512) return {c <= 384 ? 384 : 512, 1};
  if (c <= 1024) return {c <= 768 ? 768 : 1024, 1};
  if (c <= 1536) return {768, 2};
  return {1024, c <= 2048 ? 2 : 4};
}

// Threads of a block (more than one row's where a row is a wavefront's or less).
constexpr int norm_threads(int lanes) { return lanes <= 64 ? 256 : lanes; }

// Blocks of a norm's launch: as many as the card runs at once, each a row (or a set
// of rows) at a time, so that the weights are loaded once and the next row's loads are
// in flight while one is worked on.
constexpr int64_t norm_blocks(int64_t rows, int64_t width, int64_t per_cu) {
  const int lanes = norm_form(width).lanes, threads = norm_threads(lanes);
  const int64_t need = ceil_div(rows, threads / lanes), most = 256 * (per_cu > threads ? per_cu / threads : 1);
  return need < most ? need : most;
}

// Threads per CU: fewer keep too few loads in flight, more leave a block too few rows to
// load ahead (and in the gradient more partial sums).  us of 1024 / 1536 / 2048 / 4096:
// norms of 8192 x 4096 46 / 44 / 46 / 44, 2000 x 16384 43.1 / 42.9 / 46 / 52, 8192 x 1031
// 19.1 / 17.4 / 18.6 / 18.0.  Of 512 / 768 / 1024 / 2048: gradients of 16384 x 4096 97.4 /
// 97.3 / 103 / 107, 4999 x 1031 22.8 / 20.4 / 21.7 / 25.5, 16384 x 2048 49.7 / 51 / 54 / 58.
constexpr int64_t kNormThreads = 1536;         // the forward pass
constexpr int64_t kNormGradientThreads = 768;  // the gradient; its blocks leave a partial sum each

constexpr int64_t norm_parts(int64_t rows, int64_t width) { return norm_blocks(rows, width, kNormGradientThreads); }

constexpr int64_t pad4(int64_t n) { return (n + 3) / 4 * 4; }

// An 8-bit product's form: few rows, or tiles of 64 x 64, 128 x 128, 256 x 256; and the
// parts of the depth that its tiles are split into.  Times in us, bfloat16 outputs,
// squares.
enum ScaledForm { kScaledFew16, kScaledFew32, kScaledFew48, kScaledSmall, kScaledMiddle, kScaledLarge };
struct ScaledPlan {
  ScaledForm form;
  int split;
};

// A tile's stage takes its time however few tiles there are, so a long depth is split
// where that leaves CUs without one, into parts of at least 8 blocks of 128 depths; the
// second launch, which adds the parts, pays from 24 blocks on where most CUs are idle and
// from 48 on else.  Whole / split: 512, 512, 8192 26 / 16; 285, 128, 7355 24 / 12; 65,
// 4096, 4096 14.9 / 12.7; 1024, 1024, 16384 77 / 34; but 640, 128, 2048 9.0 / 11.3; 192, 1618,
// 4544 in parts for half the CUs 12.9, for all 14.1.
constexpr int scaled_parts(int64_t tiles, int64_t blocks) {
  if (blocks < 24) return 1;
  int64_t p = (blocks < 48 ? 256 : 768) / tiles;
  p = p < blocks / 8 ? p : blocks / 8;
  return (int)(p < 1 ? 1 : p > 8 ? 8 : p);
}

// Up to 16 rows, or 48 with a depth of up to 4096: the few-row form, which reads B once
// and the rows once per 16 columns.  Few-row form / tiles: 17, 4096, 4096 9.0 / 11.3; 33,
// 4096, 4096 10.0 / 10.8; 64, 4096, 4096 12.6 / 11.5; 32, 8192, 8192 28 / 17.5; 64, 1024, 8192
// 22 / 11.3.  Tiles of 256 x 256 for 205 of them and more (80 of 100 CUs), as for 16-bit
// operands.
//
// words: the operands' rows start on 4 bytes (scaled_words).  Of others a piece of 16 bytes
// takes the few-row form several loads.  Few-row form / tiles: 17, 64, 2000 4.3 / 10.3; 32,
// 4096, 4092 8.7 / 10.8; 48, 4096, 3001 7.5 / 11.6; 48, 64, 4092 10.7 / 10.1; but off 4 bytes 17,
// 64, 4095 17.3 / 10.0; 32, 256, 4095 23.8 / 10.6; 48, 4096, 2047 17.4 / 15.4; 16, 4096, 4095
// 16.8 / 11.0; 16, 4096, 3001 9.6 / 10.5; 8, 4096, 3843 11.3 / 13.2; 8, 4096, 4225 15.3 / 12.5; 1,
// 4096, 5001 9.7 / 12.6; 1, 4096, 8191 18.5 / 14.8 (against the rule 17, 64, 1111 5.4 / 7.9; 8, 4096,
// 4095 14.3 / 10.9; 4, 256, 5001 12.0 / 10.6).
constexpr ScaledPlan scaled_plan(int64_t rows, int64_t n, int64_t k, bool words = true) {
  if (rows <= 16 && (words || k <= (rows <= 4 ? 5120 : rows <= 8 ? 4096 : 3200))) return {kScaledFew16, 1};
  if (rows <= 48 && k <= 4096 && words) return {rows <= 32 ? kScaledFew32 : kScaledFew48, 1};
  const int64_t small = ceil_div(rows, 64) * ceil_div(n, 64), middle = ceil_div(rows, 128) * ceil_div(n, 128),
                large = ceil_div(rows, 256) * ceil_div(n, 256), blocks = ceil_div(k, 128);
  if (rows <= 16 || (rows <= 48 && k <= 4096)) return {kScaledSmall, scaled_parts(small, blocks)};
  if (middle >= 205) return {large >= 205 ? kScaledLarge : kScaledMiddle, 1};
  if (middle >= 64 && rows > 64 && blocks >= 64) return {kScaledMiddle, scaled_parts(middle, blocks)};
  return {kScaledSmall, scaled_parts(small, blocks)};
}

// FP32 outputs and scales per vector leave no registers for 256 x 256; 256 x 128 where
// there are as many of them.  128 x 128 / 256 x 128, scales per vector: 2048, 4096, 8192
// FP32 142 / 132, bfloat16 92 / 82; 16384, 4096, 4096 566 / 543, 362 / 331; 6500, 1031, 300
// 18.4 / 18.8, 12.3 / 12.0; with half as many tiles 2048, 2048, 2048 17.3 / 19.3.
constexpr bool scaled_tall(int64_t rows, int64_t n) { return ceil_div(rows, 256) * ceil_div(n, 128) >= 205; }

constexpr bool scaled_words(uintptr_t a, int64_t lda, uintptr_t b, int64_t ldb) {
  return ((a | b | (uintptr_t)lda | (uintptr_t)ldb) & 3) == 0;
}

// Whether tiles take their operands by DMA: rows that start on 16 bytes and are less than
// 2^22 bytes apart.
constexpr bool scaled_dma(uintptr_t a, int64_t lda, uintptr_t b, int64_t ldb) {
  return ((a | b | (uintptr_t)lda | (uintptr_t)ldb) & 15) == 0 && lda < (1 << 22) && ldb < (1 << 22);
}

// Bytes that the parts of a split depth take.
constexpr size_t scaled_room(int64_t rows, int64_t n, int64_t k, bool words = true) {
  const int split = scaled_plan(rows, n, k, words).split;
  return split > 1 ? (size_t)split * rows * pad4(n) * 4 : 0;
}

// A layer of experts for few tokens.  Times in us, of the kernel alone: tokens, top,
// experts, width, inner; "e" weights in e4m3.
constexpr int kMaxLayerTokens = 256, kMaxTop = 32, kMaxLayerExperts = 4096;

// Choices whose outputs are summed in one launch (a block goes through every expert),
// others in two (a block per expert, then the sum).  One / two launches: 1, 2, 8, 2048,
// 1024 5.6 / 4.7 + 2.6; 4, 2, 8, 4096, 2048 20.6 / 20.5 + 4.7; 16, 4, 64, 2048, 1024 e 46
// / 26 + 4.7.
constexpr int kTogether = 16;
constexpr bool layer_together(int64_t tokens, int64_t top) { return tokens * top <= kTogether; }
// Its blocks: 16 output columns, or 8 where that would leave CUs without one.  16 / 8:
// 4, 2, 8, 4096, 2048 20.6 / 35; 1, 2, 8, 2048, 1024 6.1 / 5.6.
constexpr bool together_wide(int64_t out) { return out >= 4096; }

// Hidden values: blocks of 16, 32 or 64 rows of weights (8 to 32 columns of both
// projections), 16 or 32 tokens, four or eight wavefronts.
enum HiddenForm { kHiddenOne, kHiddenSmall, kHiddenWide, kHiddenRows, kHiddenLarge };
// 16 / 32 rows: 4, 2, 8, 4096, 2048 33 / 36; 32, 2, 8, 4096, 1024 e 24 / 20; 64, 4, 64, 2048,
// 1024 e 61 / 49.  32 tokens where an expert has 12 on average: 64, 2, 8, 4096, 1024 44 /
// 52, but 32, 2, 8, 4096, 1024 e 26 / 20; then 32 / 64 rows, of the whole layer: 64, 8, 16,
// 2048, 1024 91 / 87, 32, 8, 8, 2048, 2048 e 48 / 42, but 64, 2, 8, 4096, 1024 76 / 88
// (256 blocks).  Eight wavefronts where CUs have one block:
// 1, 2, 8, 2048, 1024 7.2 / 7.5.
constexpr HiddenForm hidden_form(int64_t choices, int64_t experts, int64_t inner, bool gated, bool eight) {
  const int64_t wide = experts * ceil_div(inner, gated ? 16 : 32);
  if (wide < 256) return kHiddenOne;
  if (choices >= 12 * experts) return experts * ceil_div(inner, gated ? 32 : 64) >= 512 ? kHiddenLarge : kHiddenRows;
  return wide < (eight ? 512 : 1536) ? kHiddenSmall : kHiddenWide;
}

// Outputs of more choices: blocks of 32 columns and 16 choices of an expert, or 64 and 32
// where experts have 12 on average.  Of the whole layer: 64, 8, 16, 2048, 1024 102 / 92, 32,
// 8, 8, 2048, 2048 e 58 / 48, 256, 8, 64, 2048, 1024 e 272 / 243; but with few blocks 64, 1,
// 2, 2048, 2048 e 43 / 48.
constexpr bool share_rows(int64_t choices, int64_t experts, int64_t out) {
  return choices >= 12 * experts && experts * ceil_div(out, 64) >= 256;
}

constexpr size_t layer_hidden_bytes(int64_t tokens, int64_t top, int64_t inner) {
  return (size_t)(tokens * top * pad4(inner)) * 4;
}
constexpr size_t layer_part_bytes(int64_t tokens, int64_t top, int64_t out) {
  return layer_together(tokens, top) ? 0 : (size_t)(tokens * top * pad4(out)) * 4;
}

}  // namespace eight
}  // namespace oz
