// The C entry points of the 16-bit products: argument checks and launches.
#include <hip/hip_runtime.h>

#include "half_products.hpp"
#include "ozaki25.h"

namespace {

static_assert(OZAKI25_BF16 == oz::half::kBF16 && OZAKI25_F16 == oz::half::kF16 && OZAKI25_F32 == oz::half::kF32,
              "type numbering");

bool half_type(ozaki25_dtype t) { return t == OZAKI25_BF16 || t == OZAKI25_F16; }
size_t bytes_of(ozaki25_dtype t) { return t == OZAKI25_F32 ? 4 : 2; }

// Bytes from the first to the last element of a stack of matrices.
size_t span(int64_t count, int64_t stride, int64_t rows, int64_t ld, int64_t cols, size_t elem) {
  if (count <= 0 || rows <= 0 || cols <= 0) return 0;
  return ((size_t)(count - 1) * (size_t)stride + (size_t)(rows - 1) * (size_t)ld + (size_t)cols) * elem;
}

bool overlaps(const void* p, size_t bytes, const void* q, size_t qbytes) {
  const uintptr_t a = (uintptr_t)p, b = (uintptr_t)q;
  return bytes && qbytes && a < b + qbytes && b < a + bytes;
}

bool aligned(const void* p, size_t elem) { return (uintptr_t)p % elem == 0; }

// sizes of one matrix: rows x cols with pitch ld
bool bad_matrix(int64_t rows, int64_t cols, int64_t ld) {
  return rows < 0 || cols < 0 || ld < cols || ld < 1 || ld > OZAKI25_MAX_LD;
}

bool too_large(int64_t rows, int64_t n, int64_t k, int64_t groups) {
  return rows > OZAKI25_MAX_ROWS || n > OZAKI25_MAX_WIDTH || k > OZAKI25_MAX_WIDTH || groups > OZAKI25_MAX_GROUPS;
}

ozaki25_status status_of(hipError_t e) {
  if (e == hipSuccess) return OZAKI25_SUCCESS;
  return e == hipErrorInvalidConfiguration ? OZAKI25_ERR_UNSUPPORTED : OZAKI25_ERR_HIP;
}

// the checks that the two products by rows share; W a stack of n x k
ozaki25_status check_rows(int64_t rows, int64_t n, int64_t k, int64_t groups, const void* in, int64_t ldin,
                          int64_t depth, const void* W, int64_t ldw, int64_t stride, const int32_t* ends, const void* out,
                          int64_t ldout, int64_t cols, ozaki25_dtype type) {
  if (!half_type(type) || groups < 0 || n < 0 || k < 0) return OZAKI25_ERR_INVALID_VALUE;
  if (bad_matrix(rows, depth, ldin) || bad_matrix(n, k, ldw) || bad_matrix(rows, cols, ldout))
    return OZAKI25_ERR_INVALID_VALUE;
  if (groups > 1 && stride < 0) return OZAKI25_ERR_INVALID_VALUE;
  if (too_large(rows, n, k, groups)) return OZAKI25_ERR_UNSUPPORTED;
  if (rows == 0 || cols == 0) return OZAKI25_SUCCESS;
  if (!out || !aligned(out, 2) || (groups > 0 && (!ends || !aligned(ends, 4)))) return OZAKI25_ERR_INVALID_VALUE;
  if (depth > 0 && groups > 0 && (!in || !W || !aligned(in, 2) || !aligned(W, 2))) return OZAKI25_ERR_INVALID_VALUE;
  const size_t ob = span(1, 0, rows, ldout, cols, 2);
  if (overlaps(out, ob, in, span(1, 0, rows, ldin, depth, 2)) ||
      overlaps(out, ob, W, span(groups, stride, n, ldw, k, 2)) ||
      overlaps(out, ob, ends, (size_t)groups * sizeof(int32_t)))
    return OZAKI25_ERR_INVALID_VALUE;
  return OZAKI25_SUCCESS;
}

}  // namespace

extern "C" {

ozaki25_status ozaki25_grouped_matmul(int64_t rows, int64_t n, int64_t k, int64_t groups, const void* X, int64_t ldx,
                                      const void* W, int64_t ldw, int64_t group_stride, const int32_t* ends, void* Y,
                                      int64_t ldy, ozaki25_dtype type, void* stream) {
  const ozaki25_status st =
      check_rows(rows, n, k, groups, X, ldx, k, W, ldw, group_stride, ends, Y, ldy, n, type);
  if (st != OZAKI25_SUCCESS || rows == 0 || n == 0) return st;
  const oz::half::GroupedRows g{X, ldx, W, ldw, group_stride, ends, Y, ldy, (int)rows, (int)n, (int)k, (int)groups, false};
  return status_of(oz::half::launch_grouped_rows(g, (int)type, false, (hipStream_t)stream));
}

ozaki25_status ozaki25_grouped_matmul_dx(int64_t rows, int64_t n, int64_t k, int64_t groups, const void* dY,
                                         int64_t lddy, const void* W, int64_t ldw, int64_t group_stride,
                                         const int32_t* ends, void* dX, int64_t lddx, ozaki25_dtype type,
                                         void* stream) {
  const ozaki25_status st =
      check_rows(rows, n, k, groups, dY, lddy, n, W, ldw, group_stride, ends, dX, lddx, k, type);
  if (st != OZAKI25_SUCCESS || rows == 0 || k == 0) return st;
  const oz::half::GroupedRows g{dY, lddy, W, ldw, group_stride, ends, dX, lddx, (int)rows, (int)k, (int)n, (int)groups, false};
  return status_of(oz::half::launch_grouped_rows(g, (int)type, true, (hipStream_t)stream));
}

ozaki25_status ozaki25_grouped_matmul_dw(int64_t rows, int64_t n, int64_t k, int64_t groups, const void* dY,
                                         int64_t lddy, const void* X, int64_t ldx, const int32_t* ends, void* dW,
                                         int64_t lddw, int64_t group_stride, ozaki25_dtype type, ozaki25_dtype out_type,
                                         void* stream) {
  if (!half_type(type) || (out_type != type && out_type != OZAKI25_F32) || groups < 0 || n < 0 || k < 0)
    return OZAKI25_ERR_INVALID_VALUE;
  if (bad_matrix(rows, n, lddy) || bad_matrix(rows, k, ldx) || bad_matrix(n, k, lddw))
    return OZAKI25_ERR_INVALID_VALUE;
  // the groups' gradients must not share elements
  if (groups > 1 && n > 0 && k > 0 && group_stride < (n - 1) * lddw + k) return OZAKI25_ERR_INVALID_VALUE;
  if (too_large(rows, n, k, groups)) return OZAKI25_ERR_UNSUPPORTED;
  if (groups == 0 || n == 0 || k == 0) return OZAKI25_SUCCESS;
  const size_t e = bytes_of(out_type);
  if (!dW || !aligned(dW, e) || !ends || !aligned(ends, 4)) return OZAKI25_ERR_INVALID_VALUE;
  if (rows > 0 && (!dY || !X || !aligned(dY, 2) || !aligned(X, 2))) return OZAKI25_ERR_INVALID_VALUE;
  const size_t ob = span(groups, group_stride, n, lddw, k, e);
  if (overlaps(dW, ob, dY, span(1, 0, rows, lddy, n, 2)) || overlaps(dW, ob, X, span(1, 0, rows, ldx, k, 2)) ||
      overlaps(dW, ob, ends, (size_t)groups * sizeof(int32_t)))
    return OZAKI25_ERR_INVALID_VALUE;
  const oz::half::GroupedWeights g{dY,   lddy,         X,         ldx,    ends,   dW,
                                   lddw, group_stride, (int)rows, (int)n, (int)k, (int)groups, false};
  return status_of(oz::half::launch_grouped_weights(g, (int)type, (int)out_type, (hipStream_t)stream));
}

}  // extern "C"
