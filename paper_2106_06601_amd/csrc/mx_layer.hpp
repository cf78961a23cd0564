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

// ---- adapters (mx_adapters.hip) -----------------------------------------------
// Which adapter a row has and how much of it is there.
struct AdapterIndex {
  int32_t count, rank;
  const int32_t* ranks;
  const float* scales;
  const int32_t* index;
};
constexpr int kRankMax = 256;

// v (m x rank, v_ld) <- the products of x's rows with their adapters' rows of `low`, 0 where
// there are none.
struct AdapterDotsArgs {
  AdapterIndex at;
  int64_t m, k;
  costa_real type;
  RowsView x, low;
  float* v;
  int64_t v_ld;
};
hipError_t launch_mx_adapter_dots(const AdapterDotsArgs& a, hipStream_t stream);

// c <- alpha * (the sum of `splits` parts, m x n floats each) + s v low + beta c
struct AdapterAddArgs {
  AdapterIndex at;
  int64_t m, n;
  costa_real type, c_type;
  RowsView low, c;
  const float* v;
  int64_t v_ld;
  const float* parts;
  int32_t splits;
  float alpha, beta;
};
hipError_t launch_mx_adapter_add(const AdapterAddArgs& a, hipStream_t stream);

// g ((count rank) x len) <- s * sum over the rows of v^T z + beta g
struct AdapterGradArgs {
  AdapterIndex at;
  int64_t m, len;
  costa_real type, g_type;
  RowsView z, g;
  const float* v;
  int64_t v_ld;
  float beta;
  float* parts;
  int64_t most;  // parts that there is room for
};
int64_t mx_adapter_grad_parts(int64_t m, int64_t len, int32_t count, int32_t rank);
hipError_t launch_mx_adapter_grad(const AdapterGradArgs& a, hipStream_t stream);

}  // namespace costa
