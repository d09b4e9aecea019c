// Which form an 8-bit product takes (eight_rules.hpp), behind a C interface, compiled
// with g++ by tests/eight_routes.py.
#include "eight_rules.hpp"

using namespace oz::eight;

extern "C" {
int plan_form(int64_t rows, int64_t n, int64_t k, int words) { return scaled_plan(rows, n, k, words != 0).form; }
int plan_split(int64_t rows, int64_t n, int64_t k, int words) { return scaled_plan(rows, n, k, words != 0).split; }
int plan_tall(int64_t rows, int64_t n) { return scaled_tall(rows, n); }
int64_t plan_room(int64_t rows, int64_t n, int64_t k, int words) { return (int64_t)scaled_room(rows, n, k, words != 0); }
int plan_words(int64_t a, int64_t lda, int64_t b, int64_t ldb) { return scaled_words((uintptr_t)a, lda, (uintptr_t)b, ldb); }
int plan_dma(int64_t a, int64_t lda, int64_t b, int64_t ldb) { return scaled_dma((uintptr_t)a, lda, (uintptr_t)b, ldb); }
}
