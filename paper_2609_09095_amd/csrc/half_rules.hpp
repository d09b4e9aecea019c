// The rules by which the 16-bit products choose their tiles, from sizes alone.
// Plain C++, so that they also compile for the host's tests.  Measured on the
// whole card (256 CUs); times in us, bfloat16.
#pragma once

#include <cstddef>
#include <cstdint>

namespace oz {
namespace half {

// Tiles: large 256 x 256 (one block per CU), middle 128 x 128 (two), small 64 x 64.
enum TileSize { kSmallTile, kMiddleTile, kLargeTile };

constexpr int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Row tiles of `bm` rows that a grouped product is expected to have: every
// group's last tile is partly filled, and most groups have rows.
constexpr int64_t expected_row_tiles(int64_t rows, int64_t groups, int64_t bm) {
  const int64_t filled = groups < rows ? groups : rows;
  const int64_t t = rows / bm + groups * 3 / 5, least = ceil_div(rows, bm) > filled ? ceil_div(rows, bm) : filled;
  return t > least ? t : least;
}

// Large or middle tiles for `large` and `middle` tiles of either, by the
// measured cost of a round (all CUs busy once) per 64 depths: a large round 1.4
// if it is the only one, two rounds 3.2 whatever the second one's size, more 1.7
// each and half a round lost; a middle one 1.0 if alone, else 1.05 each and
// half a round lost.  Large / middle: rows, groups, n, k = 16384, 16, 4096, 2048
// 310 / 339; 2048, 8, 4096, 2048 47 / 54; its input gradient 75 / 51; 4096, 8,
// 4096, 2048 96 / 85; 16384, 8, 1024, 1024 56 / 48; 20000, 2, 4096, 2048 294 / 324.
constexpr TileSize large_or_middle(int64_t large, int64_t middle) {
  const double l = large / 256.0, m = middle / 512.0;
  const double cl = l <= 1 ? 1.4 : l <= 2 ? 3.2 : 1.7 * (l + 0.5);
  const double cm = m <= 1 ? 1.0 : 1.05 * (m + 0.5);
  return cl < cm ? kLargeTile : kMiddleTile;
}

// Small tiles where middle ones would fill less than four fifths of the CUs.
// Small / middle: rows, groups, n, k = 512, 8, 1024, 1024 8.5 / 11.4; 1536, 1,
// 2048, 2048 (192 middle tiles) 24 / 25; beyond (224 to 256) 3584, 2, 1024, 1024
// 18.5 / 13.9, 2048, 1, 2048, 2048 32 / 27, weights' gradient 34 / 27, 1024, 8,
// 4096, 2048 44 / 30.
constexpr int64_t kMiddleLeast = 205;
constexpr TileSize tile_of(int64_t middle, int64_t large) {
  return middle < kMiddleLeast ? kSmallTile : large_or_middle(large, middle);
}

// Large tiles beyond whole rounds that are worth a launch of their own in small
// tiles (16 each): few, so that they fill no more than a round and a half of
// those; 0: none.  2 x 4096 x 4096, a symmetric product's 272 tiles: 129 + 25 (S)
// and 139 + 27 (P), middle tiles 180 and 191.
constexpr int64_t large_tiles_over(int64_t large) {
  const int64_t over = large % 256;
  return large > 256 && over <= 48 ? over : 0;
}

// A grouped product by rows.  Middle tiles that are half empty on average have
// to fill all CUs: 512, 8, 4096, 2048 small 23.5 / middle 25.6, but 640, 8, 4096,
// 2048 29 / 27.
constexpr TileSize rows_tile(int64_t rows, int64_t groups, int64_t cols) {
  const int64_t middle = expected_row_tiles(rows, groups, 128) * ceil_div(cols, 128);
  if (rows <= 64 * groups && middle <= 256) return kSmallTile;
  return tile_of(middle, expected_row_tiles(rows, groups, 256) * ceil_div(cols, 256));
}

// The weights' gradient, whose groups differ in depth: large tiles only where
// several rounds even that out.  Large / middle, 32-bit output: 4096, 8, 4096,
// 2048 102 / 127, 16384, 16, 4096, 2048 340 / 396; 8192, 16, 2048, 1024 71 / 58,
// 20000, 2, 4096, 2048 381 / 312; small / middle: 700, 2, 512, 256 5.3 / 10,
// beyond 205 middle tiles 4096, 7, 1024, 512 14.5 / 11.5, 2048, 2, 2048, 1024 19.9
// / 16.8.
constexpr TileSize weights_tile(int64_t n, int64_t k, int64_t groups) {
  const int64_t middle = groups * ceil_div(n, 128) * ceil_div(k, 128);
  if (groups == 1) return tile_of(middle, ceil_div(n, 256) * ceil_div(k, 256));
  if (middle < kMiddleLeast) return kSmallTile;
  return groups * ceil_div(n, 256) * ceil_div(k, 256) >= 768 ? kLargeTile : kMiddleTile;
}

// Operands that cannot go to LDS by DMA take middle tiles of eight wavefronts
// (more loads in flight), and small ones sooner for the weights' gradient.
// 4999, 7, 1031, 777 small / middle: forward 48 / 40, weights' gradient 40 / 49;
// 16384, 8, 1031, 2049: weights' gradient 230 / 159.
constexpr bool masked_small(bool weights, int64_t middle_tiles) { return middle_tiles <= (weights ? 512 : 256); }

// Small tiles of such operands with four sets of wavefronts that share the depth
// (a stage waits for loads into registers), where no CU has a second tile: one
// set / four: weights' gradient of 8704, 4, 389, 263 39 / 25, input gradient of 300,
// 3, 1000, 777 16.7 / 12.8, but 700, 2, 513, 257 12 / 12, weights' gradient 9.8 /
// 10.8.  (With loads into LDS one set already takes what a CU can: 1024, 1, 512,
// 4096 22.1 / 21.2, 1024, 1, 1024, 1024 8.7 / 9.6.)
constexpr bool masked_sets(int64_t small_tiles, int64_t depth) { return small_tiles <= 256 && depth > 640; }

// Few rows per group: the weights go straight into fragments (at most 48 rows
// a group on average).  Few-row form / tiles: 256, 8, 4096, 2048 42 / 51, 384,
// 8, 2048, 2048 32 / 32, 512, 8, 4096, 2048 62 / 30.
constexpr bool few_rows(int64_t rows, int64_t groups) { return groups > 0 && rows <= 48 * groups; }

// The same for operands that cannot go to LDS by DMA: a fragment's rows then start
// anywhere in a cache line, and the tiles read them in longer pieces.  Few-row form /
// tiles: 960, 29, 1024, 1971 74 / 35, 3000, 64, 1000, 777 77 / 27, 500, 16, 3001, 3000
// 96 / 75; with at most 16 rows a group 100, 29, 1024, 1971 50 / 37, 64, 8, 2048,
// 2047 37 / 24, but short depths, many tiles or few of them 128, 8, 512, 513 9.0 /
// 10.3, 300, 64, 4000, 777 127 / 135, 250, 16, 3001, 3000 63 / 74, 16, 1, 4096, 4095
// 27 / 30.  (One or two rows a group: the tiles would be empty.)
constexpr bool few_rows_masked(int64_t rows, int64_t groups, int64_t cols, int64_t depth) {
  if (rows <= 2 * groups) return true;
  const int64_t tiles = expected_row_tiles(rows, groups, 64) * ceil_div(cols, 64);
  return rows <= 16 * groups && (depth <= 640 || tiles > 512 || tiles <= 64);
}

// Its blocks: 64 columns where that gives at least a block per CU (with 32 or,
// above 16 rows a group, 64 rows each), else 16 columns (32 above 16 rows a
// group, with 32 rows).  16 / 64 columns: 2, 8, 2048, 1024 4.0 / 6.8, 16, 1,
// 4096, 4096 10.5 / 22; 256, 64, 1024, 2048 57 / 51, 64, 8, 4096, 2048 38 / 30.
enum FewForm { kFew16, kFew32, kFew64x32, kFew64x64 };
constexpr FewForm few_form(int64_t rows, int64_t groups, int64_t cols) {
  const int64_t filled = groups < rows ? groups : rows;
  const bool many = rows > 16 * groups;
  if (filled * ceil_div(cols, 64) >= 256) return many ? kFew64x64 : kFew64x32;
  return many ? kFew32 : kFew16;
}

// How an adapter product runs: `rows - serve_rows` rows in whole tiles, the
// last serve_rows in the few-row form, which reads the weights once per 64 rows.
struct AdapterPlan {
  int serve_rows;
  int splits, serve_splits;  // parts of the depth of X A^T in either
  int base_splits;           // of X W^T in the few-row form
  size_t h_bytes, h16_bytes, factor_bytes, partial_bytes;
};

constexpr int clamp_parts(int64_t parts, int64_t most) {
  const int64_t p = parts < most ? parts : most;
  return (int)(p < 1 ? 1 : p > 8 ? 8 : p);
}

// Few-row form / tiles, eight adapters (rows, n, k, rank): 65, 4096, 4096, 16 25 /
// 60; 128, 4096, 4096, 64 53 / 54; 256, 1024, 1024, 16 12 / 17; beyond 200, 4096,
// 4096, 16 47 / 50, 512, 1024, 1024, 16 19 / 16, 512, 4096, 4096, 64 157 / 49.
constexpr int64_t kServeRows = 128, kServeOutputs = 1 << 18;

// Rows whose adapters the tiles would go through one after the other, up to 64 in
// a tile of 64 rows.  The host knows how many adapters there are, not how many the
// rows name, and the form that wins where each row chooses its own loses where rows
// come in runs.  Few-row form / tiles (rows, n, k, rank, adapters), rows of their own
// choice and in runs of 16 and 64:
//   256, 4096, 4096, 16, 16   47 / 94    47 / 41   47 / 33
//   256, 4096, 4096, 64, 64   96 / 222   92 / 46   83 / 35
//   256, 2048, 2048, 16, 16   23 / 78    23 / 29   23 / 22
//   192, 4096, 4096, 32, 32   64 / 139   61 / 42   60 / 33
//   512, 1024, 1024, 16, 32   19 / 114   19 / 24   19 / 17
//   333, 1000, 1111, 16, 16   23 / 97    23 / 33   23 / 24
//   512, 2048, 2048, 64, 32   80 / 170   77 / 36   74 / 26
// The tiles' worst loss (2 to 6 times, rows of their own choice) is the larger one up
// to rank 32; at rank 64 the few-row form's in runs is as large (2.4 and 2.9).  Beyond
// the rule 512, 4096, 4096, 16, 16 85 / 95, in runs 85 / 57.  Depths that cannot go to
// LDS by DMA: 256, 4096, 4095, 16, 16 129 / 149, in runs 126 / 57.
constexpr bool serve_many(int64_t rows, int64_t n, int64_t k, int64_t rank_pad, int64_t adapters) {
  if (rank_pad == 0) return false;
  if (rows <= 2 * kServeRows && k % 8 == 0) return 2 * adapters >= rank_pad;
  return rows <= 4 * kServeRows && adapters >= 16 && rows * n * k <= (adapters < 64 ? adapters : 64) << 26;
}

constexpr AdapterPlan adapter_plan(int64_t rows, int64_t n, int64_t k, int64_t rank_pad, int64_t adapters = 0) {
  AdapterPlan a{};
  const int64_t over = rows % 256;
  if (rows <= kServeRows || (rows <= 4 * kServeRows && rows * n <= kServeOutputs) ||
      serve_many(rows, n, k, rank_pad, adapters)) {
    a.serve_rows = (int)rows;
  } else if (over > 0 && over <= 64 && rows > 256) {
    // rows that would take large tiles a round of their own
    const int64_t with = ceil_div(rows, 256) * ceil_div(n, 256), without = rows / 256 * ceil_div(n, 256);
    if (ceil_div(with, 256) > ceil_div(without, 256)) a.serve_rows = (int)over;
  }
  const int64_t tile_rows = rows - a.serve_rows;
  // about two blocks per CU; at least 256 depths (two steps of 32 per wavefront) each
  a.base_splits = a.serve_rows > 0 ? clamp_parts(ceil_div(512, ceil_div(n, 64) * ceil_div(a.serve_rows, 64)), ceil_div(k, 256)) : 0;
  a.serve_splits = clamp_parts(ceil_div(k, 1024), 8);
  a.splits = clamp_parts(ceil_div(1024, ceil_div(tile_rows > 0 ? tile_rows : 1, 32)), ceil_div(k, tile_rows > 2048 ? 1024 : 512));
  const size_t h1 = (size_t)a.splits * tile_rows, h2 = (size_t)a.serve_splits * a.serve_rows;
  a.h_bytes = ((h1 > h2 ? h1 : h2) * rank_pad * sizeof(float) + 255) / 256 * 256;
  a.h16_bytes = ((size_t)tile_rows * 2 * rank_pad * 2 + 255) / 256 * 256;
  a.factor_bytes = ((size_t)(rank_pad > 0 ? tile_rows : 0) * sizeof(float) + 255) / 256 * 256;
  a.partial_bytes = ((size_t)a.base_splits * a.serve_rows * (ceil_div(n, 4) * 4) * sizeof(float) + 255) / 256 * 256;
  return a;
}

}  // namespace half
}  // namespace oz
