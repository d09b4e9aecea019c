// The 8-bit path's rules (eight_rules.hpp) behind a C interface, compiled with g++
// by tests/test_eight_rules.py.
#include "eight_rules.hpp"

using namespace oz::eight;

extern "C" {
int rule_norm_lanes(int64_t width) { return norm_form(width).lanes; }
int rule_norm_chunks(int64_t width) { return norm_form(width).chunks; }
int rule_norm_threads(int64_t width) { return norm_threads(norm_form(width).lanes); }
int64_t rule_norm_blocks(int64_t rows, int64_t width) { return norm_blocks(rows, width, kNormThreads); }
int64_t rule_norm_parts(int64_t rows, int64_t width) { return norm_parts(rows, width); }
int rule_scaled_form(int64_t rows, int64_t n, int64_t k) { return scaled_plan(rows, n, k).form; }
int rule_scaled_split(int64_t rows, int64_t n, int64_t k) { return scaled_plan(rows, n, k).split; }
int rule_scaled_tall(int64_t rows, int64_t n) { return scaled_tall(rows, n); }
int64_t rule_scaled_room(int64_t rows, int64_t n, int64_t k) { return (int64_t)scaled_room(rows, n, k); }
int rule_together(int64_t tokens, int64_t top) { return layer_together(tokens, top); }
int rule_share_rows(int64_t choices, int64_t experts, int64_t out) { return share_rows(choices, experts, out); }
int rule_hidden(int64_t choices, int64_t experts, int64_t inner, int gated, int eight) {
  return hidden_form(choices, experts, inner, gated != 0, eight != 0);
}
}
