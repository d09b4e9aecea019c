// The 16-bit products' rules (half_rules.hpp) behind a C interface, compiled
// with g++ by tests/half_routes.py.
#include "half_rules.hpp"

using namespace oz::half;

extern "C" {
int rule_rows_tile(int64_t rows, int64_t groups, int64_t cols) { return rows_tile(rows, groups, cols); }
int rule_weights_tile(int64_t n, int64_t k, int64_t groups) { return weights_tile(n, k, groups); }
int rule_tile_of(int64_t middle, int64_t large) { return tile_of(middle, large); }
int rule_few_rows(int64_t rows, int64_t groups) { return few_rows(rows, groups); }
int rule_few_rows_masked(int64_t rows, int64_t groups, int64_t cols, int64_t depth) {
  return few_rows_masked(rows, groups, cols, depth);
}
int rule_few_form(int64_t rows, int64_t groups, int64_t cols) { return few_form(rows, groups, cols); }
int rule_masked_small(int weights, int64_t middle) { return masked_small(weights != 0, middle); }
int64_t rule_row_tiles(int64_t rows, int64_t groups, int64_t bm) { return expected_row_tiles(rows, groups, bm); }
int64_t rule_tiles_over(int64_t large) { return large_tiles_over(large); }
int rule_masked_sets(int64_t tiles, int64_t depth) { return masked_sets(tiles, depth); }
int rule_serve_rows(int64_t rows, int64_t n, int64_t k) { return adapter_plan(rows, n, k, 16).serve_rows; }
int rule_plan_serve_rows(int64_t rows, int64_t n, int64_t k, int64_t rank_pad, int64_t adapters) {
  return adapter_plan(rows, n, k, rank_pad, adapters).serve_rows;
}
int rule_serve_many(int64_t rows, int64_t n, int64_t k, int64_t rank_pad, int64_t adapters) {
  return serve_many(rows, n, k, rank_pad, adapters);
}
int rule_serve_parts(int64_t rows, int64_t n, int64_t k) { return adapter_plan(rows, n, k, 16).base_splits; }
int rule_shrink_parts(int64_t rows, int64_t n, int64_t k) { return adapter_plan(rows, n, k, 16).splits; }
}
