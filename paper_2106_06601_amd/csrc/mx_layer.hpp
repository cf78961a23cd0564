// The operators around the products of a layer: what the host code and the kernels share.
#pragma once

#include "../../include/costa_layer.h"
#include "mx.hpp"

namespace costa {

// ---- norm (mx_norm.hip) ------------------------------------------------------
// A plain row-major matrix as the kernels see it; data null: not there.
struct RowsView {
  void* data;
  int64_t ld;
};
struct NormArgs {
  int64_t rows, cols;
  costa_real type, w_type;
  RowsView x, r, h, y;
  MxView q;
  const void* w;
  float* rstd;
  float eps;
  double inverse;  // 1 / cols
};
hipError_t launch_mx_norm(const NormArgs& a, hipStream_t stream);

struct NormBackArgs {
  int64_t rows, cols;
  costa_real type, w_type, dw_type;
  RowsView dy, h, dh, dx;
  const void* w;
  const float* rstd;
  void* dw;
  float* parts;  // of dw: `most` x cols
  int64_t most;
  double inverse;
};
// Parts of dw that a call has to have room for, and that it can use.
struct Parts {
  int64_t least, most;
};
Parts mx_norm_parts(int64_t rows, int64_t cols);
hipError_t launch_mx_norm_backward(const NormBackArgs& a, hipStream_t stream);

}  // namespace costa
