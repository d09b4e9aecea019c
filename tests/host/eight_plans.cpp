// Which form an 8-bit product takes (eight_rules.hpp), behind a C interface, compiled
// with g++ by tests/eight_routes.py.
#include "eight_rules.hpp"

using namespace oz::eight;

extern "C" {
int plan_form(int64_t rows, int64_t n, int64_t k, int aligned) {
  const ScaledForm form = scaled_plan(rows, n, k).form;
  return !aligned && few_as_tiles(rows) && form < kScaledSmall ? kScaledSmall : form;
}
int plan_split(int64_t rows, int64_t n, int64_t k, int) { return scaled_plan(rows, n, k).split; }
int plan_tall(int64_t rows, int64_t n) { return scaled_tall(rows, n); }
}
