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

constexpr size_t kAlign = 256;
size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

int64_t pad8(int64_t x) { return (x + 7) / 8 * 8; }
int64_t pad16(int64_t x) { return (x + 15) / 16 * 16; }

// The padded rank of an adapter product; zero where nothing reaches the adapters.
int64_t used_rank(int64_t k, int64_t adapters, int64_t rank) { return k > 0 && adapters > 0 ? pad16(rank) : 0; }

// Workspace of the orthogonalisation: offsets from its start.
struct OrthRoom {
  size_t squares, x32, x16[2], s16, p16, d32, p32, total;
};

OrthRoom orth_room(int64_t count, int64_t m, int64_t n) {
  OrthRoom r{};
  r.total = kAlign;  // the least that a caller's workspace is
  if (oz::half::orthogonalise_in_one_launch(m, n)) return r;
  const size_t each = (size_t)(pad8(m) * pad8(n)) * count, s = (size_t)pad8(m < n ? m : n), ss = s * s * count;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off = align_up(off + bytes);
    return at;
  };
  r.squares = take((size_t)count * oz::half::orthogonalise_parts(m, n) * sizeof(double));
  r.x32 = take(each * 4);
  r.x16[0] = take(each * 2);
  r.x16[1] = take(each * 2);
  r.s16 = take(ss * 2);
  r.p16 = take(ss * 2);
  r.d32 = take(s * count * 4);
  r.p32 = take(s * count * 4);
  r.total = off;
  return r;
}

// sizes of an orthogonalisation that its kernels' 32-bit indices hold
bool orth_fits(int64_t count, int64_t m, int64_t n) {
  return count <= OZAKI25_MAX_GROUPS - 1 && m <= OZAKI25_MAX_SIDE && n <= OZAKI25_MAX_SIDE;
}

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

}  // namespace

extern "C" {

size_t ozaki25_adapter_matmul_workspace_size(int64_t rows, int64_t n, int64_t k, int64_t adapters, int64_t rank) {
  if (rows <= 0 || n <= 0 || k < 0 || adapters < 0 || rank < 0 || rank > OZAKI25_MAX_RANK ||
      too_large(rows, n, k, adapters))
    return 0;
  const oz::half::AdapterPlan a = oz::half::adapter_plan(rows, n, k, used_rank(k, adapters, rank), adapters);
  return a.h_bytes + a.h16_bytes + a.factor_bytes + a.partial_bytes;
}

ozaki25_status ozaki25_adapter_matmul(int64_t rows, int64_t n, int64_t k, int64_t adapters, int64_t rank, const void* X,
                                      int64_t ldx, const void* W, int64_t ldw, const int32_t* ids, const void* A,
                                      int64_t lda, int64_t a_stride, const void* B, int64_t ldb, int64_t b_stride,
                                      const float* scales, void* Y, int64_t ldy, ozaki25_dtype type, void* workspace,
                                      size_t workspace_bytes, void* stream) {
  if (!half_type(type) || adapters < 0 || rank < 0) return OZAKI25_ERR_INVALID_VALUE;
  if (bad_matrix(rows, k, ldx) || bad_matrix(n, k, ldw) || bad_matrix(rows, n, ldy) || bad_matrix(rank, k, lda) ||
      bad_matrix(n, rank, ldb))
    return OZAKI25_ERR_INVALID_VALUE;
  if (adapters > 1 && (a_stride < 0 || b_stride < 0)) return OZAKI25_ERR_INVALID_VALUE;
  if (too_large(rows, n, k, adapters) || rank > OZAKI25_MAX_RANK) return OZAKI25_ERR_UNSUPPORTED;
  if (rows == 0 || n == 0) return OZAKI25_SUCCESS;
  const bool any = adapters > 0 && rank > 0 && k > 0;
  if (!Y || !aligned(Y, 2) || (k > 0 && (!X || !W || !aligned(X, 2) || !aligned(W, 2)))) return OZAKI25_ERR_INVALID_VALUE;
  if (any && (!ids || !A || !B || !aligned(ids, 4) || !aligned(A, 2) || !aligned(B, 2) || !aligned(scales, 4)))
    return OZAKI25_ERR_INVALID_VALUE;
  const size_t yb = span(1, 0, rows, ldy, n, 2);
  const void* in[6] = {X, W, any ? ids : nullptr, any ? A : nullptr, any ? B : nullptr, any ? scales : nullptr};
  const size_t bytes[6] = {span(1, 0, rows, ldx, k, 2),
                           span(1, 0, n, ldw, k, 2),
                           (size_t)rows * 4,
                           span(adapters, a_stride, rank, lda, k, 2),
                           span(adapters, b_stride, n, ldb, rank, 2),
                           (size_t)adapters * 4};
  const size_t need = ozaki25_adapter_matmul_workspace_size(rows, n, k, adapters, rank);
  for (int i = 0; i < 6; ++i)
    if (in[i] && (overlaps(Y, yb, in[i], bytes[i]) || (workspace && overlaps(workspace, need, in[i], bytes[i]))))
      return OZAKI25_ERR_INVALID_VALUE;
  if (workspace && overlaps(workspace, need, Y, yb)) return OZAKI25_ERR_INVALID_VALUE;
  Room room((hipStream_t)stream);
  if (need) {
    const ozaki25_status st = room.take(workspace, workspace_bytes, need);
    if (st != OZAKI25_SUCCESS) return st;
  }
  oz::half::Adapter p{};
  p.x = X, p.ldx = ldx, p.w = W, p.ldw = ldw, p.ids = ids;
  p.a = A, p.lda = lda, p.a_stride = a_stride, p.b = B, p.ldb = ldb, p.b_stride = b_stride;
  p.scales = scales, p.y = Y, p.ldy = ldy;
  p.rows = (int)rows, p.n = (int)n, p.k = (int)k, p.adapters = any ? (int)adapters : 0, p.rank = any ? (int)rank : 0;
  p.rank_pad = (int)used_rank(k, adapters, rank), p.n_pad = (int)((n + 3) / 4 * 4);
  const oz::half::AdapterPlan plan = oz::half::adapter_plan(rows, n, k, p.rank_pad, adapters);
  return room.give(status_of(oz::half::launch_adapter(p, plan, room.p, (int)type, (hipStream_t)stream)));
}

size_t ozaki25_orthogonalise_workspace_size(int64_t count, int64_t m, int64_t n) {
  if (count <= 0 || m <= 0 || n <= 0 || !orth_fits(count, m, n)) return 0;
  return orth_room(count, m, n).total;
}

ozaki25_status ozaki25_orthogonalise(int64_t count, int64_t m, int64_t n, const void* G, int64_t ldg, int64_t g_stride,
                                     ozaki25_dtype type, void* X, int64_t ldx, int64_t x_stride, int steps, float a,
                                     float b, float c, float eps, void* workspace, size_t workspace_bytes,
                                     void* stream) {
  if ((!half_type(type) && type != OZAKI25_F32) || count < 0 || steps < 1 || steps > OZAKI25_MAX_STEPS)
    return OZAKI25_ERR_INVALID_VALUE;
  if (!(eps >= 0.0f) || !__builtin_isfinite(eps) || !__builtin_isfinite(a) || !__builtin_isfinite(b) ||
      !__builtin_isfinite(c))
    return OZAKI25_ERR_INVALID_VALUE;
  if (bad_matrix(m, n, ldg) || bad_matrix(m, n, ldx)) return OZAKI25_ERR_INVALID_VALUE;
  if (count > 1 && (g_stride < 0 || (m > 0 && n > 0 && x_stride < (m - 1) * ldx + n))) return OZAKI25_ERR_INVALID_VALUE;
  if (!orth_fits(count, m, n)) return OZAKI25_ERR_UNSUPPORTED;
  if (count == 0 || m == 0 || n == 0) return OZAKI25_SUCCESS;
  const size_t e = bytes_of(type);
  if (!G || !X || !aligned(G, e) || !aligned(X, 2)) return OZAKI25_ERR_INVALID_VALUE;
  const size_t xb = span(count, x_stride, m, ldx, n, 2), gb = span(count, g_stride, m, ldg, n, e);
  if (overlaps(X, xb, G, gb)) return OZAKI25_ERR_INVALID_VALUE;
  const OrthRoom r = orth_room(count, m, n);
  if (workspace && (overlaps(workspace, r.total, X, xb) || overlaps(workspace, r.total, G, gb)))
    return OZAKI25_ERR_INVALID_VALUE;
  Room room((hipStream_t)stream);
  if (workspace || !oz::half::orthogonalise_in_one_launch(m, n)) {
    const ozaki25_status st = room.take(workspace, workspace_bytes, r.total);
    if (st != OZAKI25_SUCCESS) return st;
  }
  oz::half::Orthogonalise o{};
  o.g = G, o.ldg = ldg, o.g_stride = g_stride;
  o.x = X, o.ldx = ldx, o.x_stride = x_stride;
  o.count = (int)count, o.m = (int)m, o.n = (int)n, o.mp = (int)pad8(m), o.np = (int)pad8(n);
  o.a = a, o.b = b, o.c = c, o.eps = eps;
  o.squares = (double*)(room.p + r.squares);
  o.x32 = (float*)(room.p + r.x32);
  o.x16[0] = room.p + r.x16[0], o.x16[1] = room.p + r.x16[1];
  o.s16 = room.p + r.s16, o.p16 = room.p + r.p16;
  o.d32 = (float*)(room.p + r.d32), o.p32 = (float*)(room.p + r.p32);
  return room.give(status_of(oz::half::launch_orthogonalise(o, (int)type, steps, (hipStream_t)stream)));
}

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
