// Host interface of the 8-bit path (norm.hip, quantise.hip, scaled.hip,
// expert_layer.hip).  Arguments were checked by the entry points.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "eight_rules.hpp"

namespace oz {
namespace eight {

struct Norm {
  const void* x;  // rows x width
  int64_t ldx;
  const void* residual;  // the same, or null
  int64_t ldr;
  const void* weight;  // width, or null: 1
  float eps;
  void* h;  // X + residual, where there is one
  int64_t ldh;
  void* y;  // rows x width, of the type or e4m3
  int64_t ldy;
  float* scales;  // blocks x rows; null: y has the type
  int64_t lds;
  int rows, width;
};

struct NormGradient {
  const void* dy;  // rows x width
  int64_t lddy;
  const void* h;
  int64_t ldh;
  const void* weight;  // or null: 1
  const void* dh;      // the residual stream's gradient, or null
  int64_t lddh;
  float eps;
  void* dx;
  int64_t lddx;
  float* dw;     // width
  float* parts;  // workspace: norm_parts(rows, width) x width
  int rows, width;
};

struct Quantise {
  const void* x;  // count matrices rows x cols
  int64_t ldx, x_stride;
  uint8_t* q;  // rows x cols, or null
  int64_t ldq, q_stride;
  float* scales;
  uint8_t* qt;  // cols x rows, or null
  int64_t ldqt, qt_stride;
  float* scales_t;
  int count, rows, cols;
};

struct Scaled {
  const uint8_t* a;  // rows x k
  int64_t lda;
  const float* as;  // blocks x rows
  int64_t ldas;
  const uint8_t* b;  // n x k
  int64_t ldb;
  const float* bs;  // blocks x n, or of squares n blocks x blocks
  int64_t ldbs;
  void* y;  // rows x n
  int64_t ldy;
  float* parts;  // workspace: split x rows x n padded to 4
  int rows, n, k;
  // set by plan_scaled:
  ScaledForm form;
  int split;    // parts of the depth
  bool dma;     // tiles take A and B by DMA
  bool stream;  // y past the caches
};

// A stack of experts' weights: of the layer's type, or e4m3 with the scales of
// 128 x 128 blocks.
struct ExpertWeights {
  const void* w;
  int64_t ld, stride;
  const float* scales;  // or null
  int64_t scales_ld, scales_stride;
};

struct Layer {
  const void* x;  // tokens x width
  int64_t ldx;
  const int32_t* which;  // tokens x top
  const float* gates;
  ExpertWeights up, gate, down;  // experts x inner x width, the same (w null: none), experts x out x inner
  void* y;                       // tokens x out
  int64_t ldy;
  float* hidden;  // workspace: tokens top x inner_pad
  float* parts;   // workspace of more than kTogether choices: tokens top x out_pad
  int tokens, top, experts, width, inner, out;
  int inner_pad, out_pad;  // multiples of 4
};

hipError_t launch_layer(const Layer& p, int type, bool eight, hipStream_t s);
hipError_t launch_norm(const Norm& p, int type, hipStream_t s);
hipError_t launch_norm_gradient(const NormGradient& p, int type, hipStream_t s);
hipError_t launch_zeros(float* p, int64_t count, hipStream_t s);
hipError_t launch_quantise(const Quantise& p, int type, bool squares, hipStream_t s);
// Chooses the form; returns the bytes of workspace that it takes.
size_t plan_scaled(Scaled& p, int out);
hipError_t launch_scaled(const Scaled& p, bool squares, int out, hipStream_t s);

}  // namespace eight
}  // namespace oz
