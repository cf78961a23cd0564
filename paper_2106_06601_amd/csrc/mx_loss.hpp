// Shared by the kernels of the loss.
#pragma once

#include "mx_layer.hpp"
#include "mx_device.hpp"

namespace costa {

// e^x for x up to about 80: 2^(x log2 e), the product's rounding made good (by itself it costs
// |x| 2^-24 of the result).  Results below 2^-126 are 0; NaN stays.
__device__ inline float exp_of(float x) {
  x = x < -1000.0f ? -1000.0f : x;
  const float h = x * 1.44269502f, l = fmaf(x, 1.44269502f, -h) + x * 1.92596299e-8f;
  return __builtin_amdgcn_exp2f(h) * fmaf(l, 0.693147182f, 1.0f);
}

// Statistics of two sets of columns together; either may be empty (-infinity, 0).
__device__ inline LossStat join_stats(LossStat a, LossStat b) {
  const float top = fmaxf(a.top, b.top), from = top == -__builtin_inff() ? 0.0f : top;
  return LossStat{top, a.sum * exp_of(a.top - from) + b.sum * exp_of(b.top - from)};
}

}  // namespace costa
