// The rules by which the 8-bit path chooses its kernels, from sizes alone.
// Plain C++, so that they also compile for the host's tests.
#pragma once

#include <cstddef>
#include <cstdint>

namespace oz {
namespace eight {

constexpr int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

constexpr int kMaxNormWidth = 32768;

// How a norm's row is spread: `lanes` threads with `chunks` times 8 elements each.
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

constexpr int64_t kNormThreads = 2048;  // per CU: the forward pass
#ifndef NGT
#define NGT 1024
#endif
constexpr int64_t kNormGradientThreads = NGT;  // the gradient; its blocks leave a partial sum each

constexpr int64_t norm_parts(int64_t rows, int64_t width) { return norm_blocks(rows, width, kNormGradientThreads); }

// An 8-bit product's form: few rows, or tiles of 64 x 64, 128 x 128, 256 x 256.
enum ScaledForm { kScaledFew16, kScaledFew32, kScaledFew64, kScaledSmall, kScaledMiddle, kScaledLarge };

constexpr ScaledForm scaled_form(int64_t rows, int64_t n, int64_t) {
  if (rows <= 16) return kScaledFew16;
  if (rows <= 32) return kScaledFew32;
  if (rows <= 64) return kScaledFew64;
  const int64_t middle = ceil_div(rows, 128) * ceil_div(n, 128), large = ceil_div(rows, 256) * ceil_div(n, 256);
  if (middle < 205) return kScaledSmall;
  return large >= 205 ? kScaledLarge : kScaledMiddle;
}

// Bytes that the parts of a split depth take.
constexpr size_t scaled_room(int64_t, int64_t, int64_t) { return 0; }

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

// Hidden values: blocks of 16 or 32 rows of weights (8 or 16 columns of both
// projections), 16 or 32 tokens, four or eight wavefronts.
enum HiddenForm { kHiddenOne, kHiddenSmall, kHiddenWide, kHiddenRows };
// 16 / 32 rows: 4, 2, 8, 4096, 2048 33 / 36; 32, 2, 8, 4096, 1024 e 24 / 20; 64, 4, 64, 2048,
// 1024 e 61 / 49.  32 tokens where an expert has 12 on average: 64, 2, 8, 4096, 1024 44 /
// 52, but 32, 2, 8, 4096, 1024 e 26 / 20.  Eight wavefronts where CUs have one block:
// 1, 2, 8, 2048, 1024 7.2 / 7.5.
constexpr HiddenForm hidden_form(int64_t choices, int64_t experts, int64_t inner, bool gated, bool eight) {
  const int64_t wide = experts * ceil_div(inner, gated ? 16 : 32);
  if (wide < 256) return kHiddenOne;
  if (choices >= 12 * experts) return kHiddenRows;
  return wide < (eight ? 512 : 1536) ? kHiddenSmall : kHiddenWide;
}

constexpr int64_t pad4(int64_t n) { return (n + 3) / 4 * 4; }
constexpr size_t layer_hidden_bytes(int64_t tokens, int64_t top, int64_t inner) {
  return (size_t)(tokens * top * pad4(inner)) * 4;
}
constexpr size_t layer_part_bytes(int64_t tokens, int64_t top, int64_t out) {
  return layer_together(tokens, top) ? 0 : (size_t)(tokens * top * pad4(out)) * 4;
}

}  // namespace eight
}  // namespace oz
