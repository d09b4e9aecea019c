// What the entry points of the operators with 16- and 8-bit operands check and
// take: types, spans, overlaps, limits, workspaces.
#pragma once

#include <hip/hip_runtime.h>

#include "ozaki25.h"

namespace oz {
namespace api {

inline bool half_type(ozaki25_dtype t) { return t == OZAKI25_BF16 || t == OZAKI25_F16; }
inline size_t bytes_of(ozaki25_dtype t) { return t == OZAKI25_F32 ? 4 : 2; }

// Bytes from the first to the last element of a stack of matrices.
inline size_t span(int64_t count, int64_t stride, int64_t rows, int64_t ld, int64_t cols, size_t elem) {
  if (count <= 0 || rows <= 0 || cols <= 0) return 0;
  return ((size_t)(count - 1) * (size_t)stride + (size_t)(rows - 1) * (size_t)ld + (size_t)cols) * elem;
}

inline bool overlaps(const void* p, size_t bytes, const void* q, size_t qbytes) {
  const uintptr_t a = (uintptr_t)p, b = (uintptr_t)q;
  return bytes && qbytes && a < b + qbytes && b < a + bytes;
}

inline bool aligned(const void* p, size_t elem) { return (uintptr_t)p % elem == 0; }

// sizes of one matrix: rows x cols with pitch ld
inline bool bad_matrix(int64_t rows, int64_t cols, int64_t ld) {
  return rows < 0 || cols < 0 || ld < cols || ld < 1 || ld > OZAKI25_MAX_LD;
}

inline bool too_large(int64_t rows, int64_t n, int64_t k, int64_t groups) {
  return rows > OZAKI25_MAX_ROWS || n > OZAKI25_MAX_WIDTH || k > OZAKI25_MAX_WIDTH || groups > OZAKI25_MAX_GROUPS;
}

inline ozaki25_status status_of(hipError_t e) {
  if (e == hipSuccess) return OZAKI25_SUCCESS;
  return e == hipErrorInvalidConfiguration ? OZAKI25_ERR_UNSUPPORTED : OZAKI25_ERR_HIP;
}

constexpr size_t kAlign = 256;
inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

// A workspace of `need` bytes: the caller's, or one allocated on the stream
// and released there when this goes out of scope.
struct Room {
  char* p = nullptr;
  bool own = false;
  hipStream_t s;
  explicit Room(hipStream_t stream) : s(stream) {}
  ozaki25_status take(void* workspace, size_t bytes, size_t need) {
    if (workspace) {
      if ((uintptr_t)workspace % kAlign) return OZAKI25_ERR_INVALID_VALUE;
      if (bytes < need) return OZAKI25_ERR_WORKSPACE;
      p = (char*)workspace;
      return OZAKI25_SUCCESS;
    }
    void* q = nullptr;
    if (hipMallocAsync(&q, need, s) != hipSuccess) {
      (void)hipGetLastError();
      return OZAKI25_ERR_WORKSPACE;
    }
    p = (char*)q;
    own = true;
    return OZAKI25_SUCCESS;
  }
  ozaki25_status give(ozaki25_status st) {
    if (own) {
      own = false;
      if (hipFreeAsync(p, s) != hipSuccess && st == OZAKI25_SUCCESS) return OZAKI25_ERR_HIP;
    }
    return st;
  }
};

}  // namespace api
}  // namespace oz
