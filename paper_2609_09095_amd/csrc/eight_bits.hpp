// Numbers in 8 bits (OCP e4m3) with a scale per block of 128: the scale of a
// block, its rounding, and loads and stores of 8 elements at any alignment.
//
//   s = max(max |x| / 448, 2^-126),  q = e4m3(x / s)
//
// 448 is the largest e4m3 number and 2^-126 the least normal FP32 number, so a
// block of zeros has a scale whose reciprocal is finite.  A NaN or infinity in a
// block makes its scale and all its bytes NaN.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "half_tile.hpp"

namespace oz {
namespace eight {

using half::kBF16;
using half::kF16;
using half::kF32;
using half::Out;
using half::v4f;
using half::v4i;

constexpr int kBlock = 128;         // elements that share a scale
constexpr float kTop = 448.0f;      // the largest e4m3 number
constexpr float kLeast = 0x1p-126f;

// |x| as bits: their order is that of the numbers, NaN above infinity
__device__ __forceinline__ uint32_t size_bits(float x) { return __builtin_bit_cast(uint32_t, x) & 0x7fffffffu; }

struct Scale {
  float s, inverse;
};

__device__ __forceinline__ Scale scale_of(uint32_t most) {
  Scale r;
  r.s = fmaxf(__builtin_bit_cast(float, most) / kTop, kLeast);
  if (most >= 0x7f800000u) r.s = __builtin_nanf("");
  r.inverse = 1.0f / r.s;
  return r;
}

// x / s, rounded as a division is: the residual of the first quotient is exact
__device__ __forceinline__ float quotient(float x, Scale s) {
  const float q = x * s.inverse;
  return __builtin_fmaf(__builtin_fmaf(-q, s.s, x), s.inverse, q);
}

// Four numbers of at most 448 (or NaN) in e4m3, the first in the lowest byte.
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// 8 elements as they are in memory
template <int TYPE>
struct Raw {
  static constexpr int Q = TYPE == kF32 ? 2 : 1;
  v4i q[Q];
};

template <int TYPE>
constexpr int kBytes = TYPE == kF32 ? 4 : 2;

// Elements p[0 .. n), zeros above them, n at most 8; nothing is read for n < 1.
template <int TYPE>
__device__ __forceinline__ Raw<TYPE> load_raw(const char* p, int n) {
  Raw<TYPE> r{};
  const auto g = (const __attribute__((address_space(1))) char*)(half::global_bytes)p;
  if (n >= 8) {
#pragma unroll
    for (int i = 0; i < Raw<TYPE>::Q; ++i)
      __builtin_memcpy(&r.q[i], (const __attribute__((address_space(1))) void*)(g + i * 16), 16);
  } else if (n > 0) {
    using E = typename Out<TYPE>::type;
    E e[8] = {};
#pragma unroll
    for (int j = 0; j < 7; ++j)
      if (j < n) e[j] = ((const __attribute__((address_space(1))) E*)g)[j];
    __builtin_memcpy(&r, e, sizeof(e));
  }
  return r;
}

template <int TYPE>
__device__ __forceinline__ void values(const Raw<TYPE>& r, float (&v)[8]) {
  using E = typename Out<TYPE>::type;
  E e[8];
  __builtin_memcpy(e, &r, sizeof(e));
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = (float)e[j];
}

// v[0 .. n) rounded to TYPE, n at most 8
template <int TYPE>
__device__ __forceinline__ Raw<TYPE> rounded(const float (&v)[8]) {
  using E = typename Out<TYPE>::type;
  E e[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) e[j] = (E)v[j];
  Raw<TYPE> r;
  __builtin_memcpy(&r, e, sizeof(e));
  return r;
}

// p[0 .. n), n at most 8; a part of 8 in pieces of 4, 2 and 1.
template <int TYPE>
__device__ __forceinline__ void store_raw(char* p, const Raw<TYPE>& r, int n) {
  const auto g = (__attribute__((address_space(1))) char*)p;
  using to = __attribute__((address_space(1))) void*;
  if (n >= 8) {
#pragma unroll
    for (int i = 0; i < Raw<TYPE>::Q; ++i) __builtin_memcpy((to)(g + i * 16), &r.q[i], 16);
  } else if (n > 0) {
    constexpr int E = kBytes<TYPE>;
    typename Out<TYPE>::type e[8];
    __builtin_memcpy(e, &r, sizeof(e));
    if (n & 4) {
      __builtin_memcpy((to)g, e, 4 * E);
#pragma unroll
      for (int j = 0; j < 3; ++j) e[j] = e[4 + j];
    }
    if (n & 2) {
      __builtin_memcpy((to)(g + (n & 4) * E), e, 2 * E);
      e[0] = e[2];
    }
    if (n & 1) __builtin_memcpy((to)(g + (n & 6) * E), e, E);
  }
}

// 8 bytes, of which n exist
__device__ __forceinline__ void store_bytes(uint8_t* p, uint2 w, int n) {
  const auto g = (__attribute__((address_space(1))) uint8_t*)p;
  if (n >= 8) {
    __builtin_memcpy((__attribute__((address_space(1))) void*)g, &w, 8);
  } else if (n > 0) {
    using to = __attribute__((address_space(1))) void*;
    uint64_t v = (uint64_t)w.y << 32 | w.x;
    if (n & 4) {
      __builtin_memcpy((to)g, &v, 4);
      v >>= 32;
    }
    if (n & 2) {
      __builtin_memcpy((to)(g + (n & 4)), &v, 2);
      v >>= 16;
    }
    if (n & 1) g[n & 6] = (uint8_t)v;
  }
}

// 16 bytes of which the upper `have` are moved down, zeros above them.
__device__ __forceinline__ v4i keep_upper_bytes(v4i v, int have) {
  const int s = 8 * (16 - have);  // bits to drop; 128: all
  const uint4 x = __builtin_bit_cast(uint4, v);
  uint64_t lo = (uint64_t)x.y << 32 | x.x, hi = (uint64_t)x.w << 32 | x.z;
  const uint64_t up = hi << 1 << (63 - (s & 63));  // hi << (64 - s), also for s = 0
  lo = s < 64 ? lo >> (s & 63) | up : hi >> (s & 63);
  hi = s < 64 ? hi >> (s & 63) : 0;
  if (s == 128) lo = 0;
  return v4i{(int)lo, (int)(lo >> 32), (int)hi, (int)(hi >> 32)};
}

// Bytes o .. o + 15 of a row of `size`, zeros past its end, at any alignment.  A
// chunk that the end cuts is read as the row's last 16 bytes; no branch around the
// load where rows have 16.
__device__ __forceinline__ v4i load16(const char* row, int64_t o, int64_t size) {
  const int64_t n = size - o;
  const int have = n < 0 ? 0 : n < 16 ? (int)n : 16;
  if (size >= 16) return keep_upper_bytes(half::load_whole(row + (have > 0 ? o - (16 - have) : 0)), have);
  uint64_t lo = 0, hi = 0;
  const auto q = (const __attribute__((address_space(1))) uint8_t*)(half::global_bytes)row;
#pragma unroll
  for (int j = 0; j < 15; ++j)
    if (j < have) {
      if (j < 8)
        lo |= (uint64_t)q[o + j] << (8 * j);
      else
        hi |= (uint64_t)q[o + j] << (8 * (j - 8));
    }
  return v4i{(int)lo, (int)(lo >> 32), (int)hi, (int)(hi >> 32)};
}

// 8 e4m3 numbers (two words) in a 16-bit type, both of which hold them exactly.
template <int TYPE>
__device__ __forceinline__ v4i widened(int lo, int hi) {
  v4i r;
  if constexpr (TYPE == kBF16) {
    typedef __bf16 v2 __attribute__((ext_vector_type(2)));
    const v2 e[4] = {
        __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true),
        __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true)};
    __builtin_memcpy(&r, e, 16);
  } else {
    typedef _Float16 v2 __attribute__((ext_vector_type(2)));
    const v2 e[4] = {
        __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false), __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true),
        __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false), __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true)};
    __builtin_memcpy(&r, e, 16);
  }
  return r;
}

// A value from the lane `ror` further round the 16 lanes of its row.
template <int ROR>
__device__ __forceinline__ uint32_t turned(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x120 + ROR, 0xf, 0xf, false);
}

__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }

// The largest of 16 neighbouring lanes, in all of them.
__device__ __forceinline__ uint32_t max16(uint32_t v) {
  v = umax(v, turned<8>(v));
  v = umax(v, turned<4>(v));
  v = umax(v, turned<2>(v));
  return umax(v, turned<1>(v));
}

// The sum of 16 neighbouring lanes, in all of them; the order is the lanes'.
__device__ __forceinline__ float sum16(float v) {
  auto add = [](float a, uint32_t b) { return a + __builtin_bit_cast(float, b); };
  v = add(v, turned<8>(__builtin_bit_cast(uint32_t, v)));
  v = add(v, turned<4>(__builtin_bit_cast(uint32_t, v)));
  v = add(v, turned<2>(__builtin_bit_cast(uint32_t, v)));
  return add(v, turned<1>(__builtin_bit_cast(uint32_t, v)));
}

}  // namespace eight
}  // namespace oz
