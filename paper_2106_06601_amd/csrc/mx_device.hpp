// Element conversions of the microscaled formats, for the kernels.
#pragma once

#include <hip/hip_runtime.h>

#include "mx.hpp"

namespace costa {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef short v2s __attribute__((ext_vector_type(2)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

// The scale byte of a block from the bits of its largest magnitude.  Integers
// order the bits as the magnitudes, NaN above infinity above the finite ones.
template <int BITS>
__device__ inline uint32_t mx_scale(uint32_t amax_bits) {
  const int e = (int)(amax_bits >> 23);
  const int s = e - (BITS == 4 ? 2 : 8);
  return e == 255 ? 255u : s > 0 ? (uint32_t)s : 0u;
}

// Scale bytes as the converting instructions take them: they read a float's
// exponent field only, so 0 is 2^-127 and 255 NaN.
__device__ inline float mx_scale_float(uint32_t s) { return __builtin_bit_cast(float, s << 23); }

// The largest of four neighbouring lanes.
__device__ inline uint32_t quad_max(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true));  // lanes 1 0 3 2
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true));  // lanes 2 3 0 1
}

__device__ inline uint32_t magnitude(float x) { return __builtin_bit_cast(uint32_t, x) & 0x7fffffffu; }

// Eight elements in the format, divided by the scale; zeros for a block of NaN.
// (Rounding to 4 bits saturates by itself; past 448 the 8-bit conversion would
// give NaN, so it is clamped first.)
template <int BITS>
__device__ inline v2u mx_encode8(const float x[8], uint32_t s) {
  const float f = mx_scale_float(s);
  v2u r = {0u, 0u};
  if (BITS == 4) {
    uint32_t d = 0;
    d = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(d, x[0], x[1], f, 0);
    d = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(d, x[2], x[3], f, 1);
    d = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(d, x[4], x[5], f, 2);
    d = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(d, x[6], x[7], f, 3);
    r.x = s == 255u ? 0u : d;
  } else {
    // s <= 246 where the block is finite: the limit is, too
    const float top = 448.0f * __builtin_bit_cast(float, s == 0u ? 1u << 22 : (s < 247u ? s : 0u) << 23);
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = fminf(fmaxf(x[i], -top), top);
    v2s d = {0, 0}, e = {0, 0};
    d = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(d, y[0], y[1], f, false);
    d = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(d, y[2], y[3], f, true);
    e = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(e, y[4], y[5], f, false);
    e = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(e, y[6], y[7], f, true);
    r.x = s == 255u ? 0u : __builtin_bit_cast(uint32_t, d);
    r.y = s == 255u ? 0u : __builtin_bit_cast(uint32_t, e);
  }
  return r;
}

// Eight stored elements as 32-bit floats.
template <int BITS>
__device__ inline void mx_decode8(v2u d, uint32_t s, float x[8]) {
  const float f = mx_scale_float(s);
  v2f p[4];
  if (BITS == 4) {
    p[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(d.x, f, 0);
    p[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(d.x, f, 1);
    p[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(d.x, f, 2);
    p[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(d.x, f, 3);
  } else {
    p[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(d.x, f, false);
    p[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(d.x, f, true);
    p[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(d.y, f, false);
    p[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(d.y, f, true);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = p[i].x;
    x[2 * i + 1] = p[i].y;
  }
}

// Eight stored elements as bfloat16 (exact, but for results below 2^-133).
template <int BITS>
__device__ inline v4u mx_decode8_bf16(v2u d, uint32_t s) {
  const float f = mx_scale_float(s);
  v2bf p[4];
  if (BITS == 4) {
    p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(d.x, f, 0);
    p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(d.x, f, 1);
    p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(d.x, f, 2);
    p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(d.x, f, 3);
  } else {
    p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(d.x, f, false);
    p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(d.x, f, true);
    p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(d.y, f, false);
    p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(d.y, f, true);
  }
  v4u r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = __builtin_bit_cast(uint32_t, p[i]);
  return r;
}

// Splits x into bfloat16 parts that sum to it: each part takes the leading 8
// bits that are left (by truncation, so that no part overflows), which leaves
// nothing of 24 bits after three and of 11 after two.  An infinity or a NaN is
// the first part alone.
template <int PARTS>
__device__ inline void bf16_parts(float x, uint16_t out[PARTS]) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x);
  const bool finite = (b & 0x7f800000u) != 0x7f800000u;
  const bool nan = (b & 0x7fffffffu) > 0x7f800000u;
  out[0] = (uint16_t)(nan ? 0x7fc0u : b >> 16);
  float r = finite ? x - __builtin_bit_cast(float, b & 0xffff0000u) : 0.0f;
#pragma unroll
  for (int i = 1; i < PARTS; ++i) {
    const uint32_t c = __builtin_bit_cast(uint32_t, r);
    out[i] = (uint16_t)(c >> 16);
    r -= __builtin_bit_cast(float, c & 0xffff0000u);
  }
}

}  // namespace costa
