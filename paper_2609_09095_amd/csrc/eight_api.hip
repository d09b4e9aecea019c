// The C entry points of the 8-bit path: argument checks and launches.
#include <hip/hip_runtime.h>

#include "api_checks.hpp"
#include "eight_products.hpp"
#include "half_tile.hpp"
#include "ozaki25.h"

using namespace oz::api;

namespace {

using oz::eight::ceil_div;

static_assert(OZAKI25_MAX_NORM_WIDTH == oz::eight::kMaxNormWidth && OZAKI25_MAX_LAYER_TOKENS == oz::eight::kMaxLayerTokens &&
                  OZAKI25_MAX_TOP == oz::eight::kMaxTop && OZAKI25_MAX_LAYER_EXPERTS == oz::eight::kMaxLayerExperts,
              "limits");

bool float_type(ozaki25_dtype t) { return half_type(t) || t == OZAKI25_F32; }

// Whether memory p is the same matrix as q, element for element.
bool same(const void* p, int64_t ldp, const void* q, int64_t ldq, int64_t rows) {
  return p == q && (ldp == ldq || rows <= 1);
}

// Memory that a call reads or writes.
struct Piece {
  const void* p;
  size_t bytes;
};

// Whether an output overlaps any of the others.
template <size_t N>
bool meets(Piece out, const Piece (&in)[N]) {
  for (const Piece& i : in)
    if (i.p && out.p && overlaps(out.p, out.bytes, i.p, i.bytes)) return true;
  return false;
}

// A stack of rows x cols weights: its sizes.
bool bad_stack(const ozaki25_expert_weights& w, int64_t experts, int64_t rows, int64_t cols) {
  if (bad_matrix(rows, cols, w.ld) || (experts > 1 && w.stride < 0)) return true;
  return w.scales && (bad_matrix(ceil_div(rows, 128), ceil_div(cols, 128), w.scales_ld) || (experts > 1 && w.scales_stride < 0));
}

bool bad_pointers(const ozaki25_expert_weights& w) {
  return !w.weights || !aligned(w.weights, w.scales ? 1 : 2) || !aligned(w.scales, 4);
}

Piece weights_of(const ozaki25_expert_weights& w, int64_t experts, int64_t rows, int64_t cols) {
  return {w.weights, span(experts, w.stride, rows, w.ld, cols, w.scales ? 1 : 2)};
}

Piece scales_of(const ozaki25_expert_weights& w, int64_t experts, int64_t rows, int64_t cols) {
  return {w.scales, span(experts, w.scales_stride, ceil_div(rows, 128), w.scales_ld, ceil_div(cols, 128), 4)};
}

bool bad_eps(float eps) { return !(eps >= 0.0f) || !__builtin_isfinite(eps); }

}  // namespace

extern "C" {

ozaki25_status ozaki25_rms_norm(int64_t rows, int64_t width, const void* X, int64_t ldx, const void* residual,
                                int64_t ldr, const void* weight, ozaki25_dtype type, float eps, void* H, int64_t ldh,
                                void* Y, int64_t ldy, float* scales, int64_t lds, void* stream) {
  if (!float_type(type) || bad_eps(eps) || bad_matrix(rows, width, ldx) || bad_matrix(rows, width, ldy))
    return OZAKI25_ERR_INVALID_VALUE;
  if (residual && (bad_matrix(rows, width, ldr) || bad_matrix(rows, width, ldh))) return OZAKI25_ERR_INVALID_VALUE;
  if (scales && bad_matrix(ceil_div(width, 128), rows, lds)) return OZAKI25_ERR_INVALID_VALUE;
  if (rows > OZAKI25_MAX_ROWS || width > OZAKI25_MAX_NORM_WIDTH) return OZAKI25_ERR_UNSUPPORTED;
  if (rows == 0 || width == 0) return OZAKI25_SUCCESS;
  const size_t e = bytes_of(type), ye = scales ? 1 : e;
  if (!X || !Y || !aligned(X, e) || !aligned(Y, ye) || !aligned(weight, e) || !aligned(scales, 4))
    return OZAKI25_ERR_INVALID_VALUE;
  if (residual ? !H || !aligned(residual, e) || !aligned(H, e) : H != nullptr) return OZAKI25_ERR_INVALID_VALUE;
  const Piece x{X, span(1, 0, rows, ldx, width, e)}, r{residual, span(1, 0, rows, ldr, width, e)},
      w{weight, (size_t)width * e}, h{H, span(1, 0, rows, ldh, width, e)}, y{Y, span(1, 0, rows, ldy, width, ye)},
      s{scales, span(1, 0, ceil_div(width, 128), lds, rows, 4)};
  if (meets(y, {x, r, w, h, s}) || meets(s, {x, r, w, h})) return OZAKI25_ERR_INVALID_VALUE;
  if (residual) {
    // the sum may take the place of either of its parts
    if (!same(H, ldh, X, ldx, rows) && meets(h, {x})) return OZAKI25_ERR_INVALID_VALUE;
    if (!same(H, ldh, residual, ldr, rows) && meets(h, {r})) return OZAKI25_ERR_INVALID_VALUE;
    if (meets(h, {w})) return OZAKI25_ERR_INVALID_VALUE;
  }
  const oz::eight::Norm p{X, ldx, residual, ldr, weight, eps, H, ldh, Y, ldy, scales, lds, (int)rows, (int)width};
  return status_of(oz::eight::launch_norm(p, (int)type, (hipStream_t)stream));
}

size_t ozaki25_rms_norm_backward_workspace_size(int64_t rows, int64_t width) {
  if (rows <= 0 || width <= 0 || rows > OZAKI25_MAX_ROWS || width > OZAKI25_MAX_NORM_WIDTH) return 0;
  return align_up((size_t)oz::eight::norm_parts(rows, width) * width * sizeof(float));
}

ozaki25_status ozaki25_rms_norm_backward(int64_t rows, int64_t width, const void* dY, int64_t lddy, const void* H,
                                         int64_t ldh, const void* weight, const void* dH, int64_t lddh,
                                         ozaki25_dtype type, float eps, void* dX, int64_t lddx, float* dweight,
                                         void* workspace, size_t workspace_bytes, void* stream) {
  if (!float_type(type) || bad_eps(eps) || bad_matrix(rows, width, lddy) || bad_matrix(rows, width, ldh) ||
      bad_matrix(rows, width, lddx) || (dH && bad_matrix(rows, width, lddh)))
    return OZAKI25_ERR_INVALID_VALUE;
  if (rows > OZAKI25_MAX_ROWS || width > OZAKI25_MAX_NORM_WIDTH) return OZAKI25_ERR_UNSUPPORTED;
  if (width == 0) return OZAKI25_SUCCESS;
  if (!dweight || !aligned(dweight, 4)) return OZAKI25_ERR_INVALID_VALUE;
  const size_t e = bytes_of(type);
  const Piece y{dY, span(1, 0, rows, lddy, width, e)}, h{H, span(1, 0, rows, ldh, width, e)},
      w{weight, (size_t)width * e}, d{dH, span(1, 0, rows, lddh, width, e)}, x{dX, span(1, 0, rows, lddx, width, e)},
      g{dweight, (size_t)width * 4};
  if (rows == 0) return status_of(oz::eight::launch_zeros(dweight, width, (hipStream_t)stream));
  if (!dY || !H || !dX || !aligned(dY, e) || !aligned(H, e) || !aligned(weight, e) || !aligned(dH, e) || !aligned(dX, e))
    return OZAKI25_ERR_INVALID_VALUE;
  // dX may take the place of dY or of dH
  if (!same(dX, lddx, dY, lddy, rows) && meets(x, {y})) return OZAKI25_ERR_INVALID_VALUE;
  if (dH && !same(dX, lddx, dH, lddh, rows) && meets(x, {d})) return OZAKI25_ERR_INVALID_VALUE;
  if (meets(x, {h, w, g}) || meets(g, {y, h, w, d})) return OZAKI25_ERR_INVALID_VALUE;
  const size_t need = ozaki25_rms_norm_backward_workspace_size(rows, width);
  if (workspace && meets({workspace, need}, {y, h, w, d, x, g})) return OZAKI25_ERR_INVALID_VALUE;
  Room room((hipStream_t)stream);
  const ozaki25_status st = room.take(workspace, workspace_bytes, need);
  if (st != OZAKI25_SUCCESS) return st;
  const oz::eight::NormGradient p{dY, lddy, H,  ldh,  weight,  dH,             lddh,      eps,
                                  dX, lddx, dweight, (float*)room.p, (int)rows, (int)width};
  return room.give(status_of(oz::eight::launch_norm_gradient(p, (int)type, (hipStream_t)stream)));
}

ozaki25_status ozaki25_quantise(int64_t count, int64_t rows, int64_t cols, const void* X, int64_t ldx, int64_t x_stride,
                                ozaki25_dtype type, int squares, uint8_t* Q, int64_t ldq, int64_t q_stride,
                                float* scales, uint8_t* QT, int64_t ldqt, int64_t qt_stride, float* scalesT,
                                void* stream) {
  if (!float_type(type) || count < 0 || (squares != 0 && squares != 1) || bad_matrix(rows, cols, ldx))
    return OZAKI25_ERR_INVALID_VALUE;
  if (!Q != !scales || !QT != !scalesT || (Q && bad_matrix(rows, cols, ldq)) || (QT && bad_matrix(cols, rows, ldqt)))
    return OZAKI25_ERR_INVALID_VALUE;
  if (count > 1 && x_stride < 0) return OZAKI25_ERR_INVALID_VALUE;
  if (count > OZAKI25_MAX_GROUPS - 1 || rows > OZAKI25_MAX_ROWS || cols > OZAKI25_MAX_WIDTH) return OZAKI25_ERR_UNSUPPORTED;
  if (count == 0 || rows == 0 || cols == 0) return OZAKI25_SUCCESS;
  if (count > 1 && ((Q && q_stride < (rows - 1) * ldq + cols) || (QT && qt_stride < (cols - 1) * ldqt + rows)))
    return OZAKI25_ERR_INVALID_VALUE;
  const size_t e = bytes_of(type);
  if (!X || !aligned(X, e) || (!Q && !QT) || !aligned(scales, 4) || !aligned(scalesT, 4)) return OZAKI25_ERR_INVALID_VALUE;
  const int64_t rb = ceil_div(rows, 128), cb = ceil_div(cols, 128);
  const Piece x{X, span(count, x_stride, rows, ldx, cols, e)}, q{Q, span(count, q_stride, rows, ldq, cols, 1)},
      t{QT, span(count, qt_stride, cols, ldqt, rows, 1)},
      s{scales, (size_t)(count * cb * (squares ? rb : rows)) * 4}, st{scalesT, (size_t)(count * rb * (squares ? cb : cols)) * 4};
  if (meets(q, {x, t, s, st}) || meets(t, {x, s, st}) || meets(s, {x, st}) || meets(st, {x})) return OZAKI25_ERR_INVALID_VALUE;
  const oz::eight::Quantise p{X,  ldx,  x_stride,  Q,       ldq,        q_stride,  scales,
                              QT, ldqt, qt_stride, scalesT, (int)count, (int)rows, (int)cols};
  return status_of(oz::eight::launch_quantise(p, (int)type, squares != 0, (hipStream_t)stream));
}

size_t ozaki25_scaled_matmul_workspace_size(int64_t rows, int64_t n, int64_t k) {
  if (rows <= 0 || n <= 0 || k <= 0 || too_large(rows, n, k, 0)) return 0;
  // the more of the two: where operands lie is not known here
  const size_t words = oz::eight::scaled_room(rows, n, k, true), other = oz::eight::scaled_room(rows, n, k, false);
  return align_up(words > other ? words : other);
}

ozaki25_status ozaki25_scaled_matmul(int64_t rows, int64_t n, int64_t k, const uint8_t* A, int64_t lda,
                                     const float* a_scales, int64_t ldas, const uint8_t* B, int64_t ldb,
                                     const float* b_scales, int64_t ldbs, int squares, void* Y, int64_t ldy,
                                     ozaki25_dtype out_type, void* workspace, size_t workspace_bytes, void* stream) {
  if (!float_type(out_type) || (squares != 0 && squares != 1) || n < 0 || k < 0) return OZAKI25_ERR_INVALID_VALUE;
  const int64_t kb = ceil_div(k, 128), sr = squares ? ceil_div(n, 128) : kb, sc = squares ? kb : n;
  if (bad_matrix(rows, k, lda) || bad_matrix(n, k, ldb) || bad_matrix(rows, n, ldy) || bad_matrix(kb, rows, ldas) ||
      bad_matrix(sr, sc, ldbs))
    return OZAKI25_ERR_INVALID_VALUE;
  if (too_large(rows, n, k, 0)) return OZAKI25_ERR_UNSUPPORTED;
  if (rows == 0 || n == 0) return OZAKI25_SUCCESS;
  const size_t e = bytes_of(out_type);
  if (!Y || !aligned(Y, e)) return OZAKI25_ERR_INVALID_VALUE;
  if (k > 0 && (!A || !B || !a_scales || !b_scales || !aligned(a_scales, 4) || !aligned(b_scales, 4)))
    return OZAKI25_ERR_INVALID_VALUE;
  const Piece a{A, span(1, 0, rows, lda, k, 1)}, as{a_scales, span(1, 0, kb, ldas, rows, 4)}, b{B, span(1, 0, n, ldb, k, 1)},
      bs{b_scales, span(1, 0, sr, ldbs, sc, 4)}, y{Y, span(1, 0, rows, ldy, n, e)};
  if (meets(y, {a, as, b, bs})) return OZAKI25_ERR_INVALID_VALUE;
  oz::eight::Scaled p{};
  p.a = A, p.lda = lda, p.as = a_scales, p.ldas = ldas;
  p.b = B, p.ldb = ldb, p.bs = b_scales, p.ldbs = ldbs;
  p.y = Y, p.ldy = ldy;
  p.rows = (int)rows, p.n = (int)n, p.k = (int)k;
  const size_t need = align_up(oz::eight::plan_scaled(p, (int)out_type));
  if (workspace && meets({workspace, need}, {a, as, b, bs, y})) return OZAKI25_ERR_INVALID_VALUE;
  Room room((hipStream_t)stream);
  if (need) {
    const ozaki25_status st = room.take(workspace, workspace_bytes, need);
    if (st != OZAKI25_SUCCESS) return st;
  }
  p.parts = (float*)room.p;
  return room.give(status_of(oz::eight::launch_scaled(p, squares != 0, (int)out_type, (hipStream_t)stream)));
}

size_t ozaki25_expert_layer_workspace_size(int64_t tokens, int64_t top, int64_t width, int64_t inner, int64_t out) {
  if (tokens <= 0 || top <= 0 || width <= 0 || inner <= 0 || out <= 0 || tokens > OZAKI25_MAX_LAYER_TOKENS ||
      top > OZAKI25_MAX_TOP || too_large(0, inner, width, 0) || out > OZAKI25_MAX_WIDTH)
    return 0;
  return align_up(oz::eight::layer_hidden_bytes(tokens, top, inner)) + align_up(oz::eight::layer_part_bytes(tokens, top, out));
}

ozaki25_status ozaki25_expert_layer(int64_t tokens, int64_t top, int64_t experts, int64_t width, int64_t inner,
                                    int64_t out, const void* X, int64_t ldx, const int32_t* which, const float* gates,
                                    const ozaki25_expert_weights* up, const ozaki25_expert_weights* gate,
                                    const ozaki25_expert_weights* down, void* Y, int64_t ldy, ozaki25_dtype type,
                                    void* workspace, size_t workspace_bytes, void* stream) {
  if (!half_type(type) || !up || !down || top < 0 || experts < 0 || bad_matrix(tokens, width, ldx) ||
      bad_matrix(tokens, out, ldy))
    return OZAKI25_ERR_INVALID_VALUE;
  if (bad_stack(*up, experts, inner, width) || (gate && bad_stack(*gate, experts, inner, width)) ||
      bad_stack(*down, experts, out, inner))
    return OZAKI25_ERR_INVALID_VALUE;
  // which kind the weights are, their scales say; an empty stack's may have no address
  if (experts > 0 && inner > 0 && width > 0 &&
      ((gate && !gate->scales != !up->scales) || (out > 0 && !down->scales != !up->scales)))
    return OZAKI25_ERR_INVALID_VALUE;
  if (tokens > OZAKI25_MAX_LAYER_TOKENS || top > OZAKI25_MAX_TOP || experts > OZAKI25_MAX_LAYER_EXPERTS ||
      too_large(0, inner, width, 0) || out > OZAKI25_MAX_WIDTH)
    return OZAKI25_ERR_UNSUPPORTED;
  if (tokens == 0 || out == 0) return OZAKI25_SUCCESS;
  if (!Y || !aligned(Y, 2)) return OZAKI25_ERR_INVALID_VALUE;
  const bool any = top > 0 && experts > 0 && width > 0 && inner > 0;
  if (any && (!X || !which || !gates || !aligned(X, 2) || !aligned(which, 4) || !aligned(gates, 4) || bad_pointers(*up) ||
              bad_pointers(*down) || (gate && bad_pointers(*gate))))
    return OZAKI25_ERR_INVALID_VALUE;
  const ozaki25_expert_weights none{}, *g = gate ? gate : &none;
  const Piece y{Y, span(1, 0, tokens, ldy, out, 2)};
  const Piece in[9] = {{X, span(1, 0, tokens, ldx, width, 2)},
                       {which, (size_t)(tokens * top) * 4},
                       {gates, (size_t)(tokens * top) * 4},
                       weights_of(*up, experts, inner, width),
                       scales_of(*up, experts, inner, width),
                       weights_of(*g, experts, inner, width),
                       scales_of(*g, experts, inner, width),
                       weights_of(*down, experts, out, inner),
                       scales_of(*down, experts, out, inner)};
  const size_t need = any ? ozaki25_expert_layer_workspace_size(tokens, top, width, inner, out) : 0;
  if (meets(y, in) || (workspace && (meets({workspace, need}, in) || meets({workspace, need}, {y}))))
    return OZAKI25_ERR_INVALID_VALUE;
  Room room((hipStream_t)stream);
  if (need) {
    const ozaki25_status st = room.take(workspace, workspace_bytes, need);
    if (st != OZAKI25_SUCCESS) return st;
  }
  auto stack = [](const ozaki25_expert_weights& w) {
    return oz::eight::ExpertWeights{w.weights, w.ld, w.stride, w.scales, w.scales_ld, w.scales_stride};
  };
  oz::eight::Layer p{};
  p.x = X, p.ldx = ldx, p.which = which, p.gates = gates;
  p.up = stack(*up), p.gate = stack(*g), p.down = stack(*down);
  p.y = Y, p.ldy = ldy;
  p.hidden = (float*)room.p;
  p.parts = (float*)(room.p + align_up(oz::eight::layer_hidden_bytes(tokens, top, inner)));
  p.tokens = (int)tokens, p.top = (int)top, p.experts = (int)experts;
  p.width = (int)width, p.inner = (int)inner, p.out = (int)out;
  p.inner_pad = (int)oz::eight::pad4(inner), p.out_pad = (int)oz::eight::pad4(out);
  return room.give(status_of(oz::eight::launch_layer(p, (int)type, up->scales != nullptr, (hipStream_t)stream)));
}

}  // extern "C"
