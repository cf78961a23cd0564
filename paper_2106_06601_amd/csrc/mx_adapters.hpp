// Shared by the kernels of the adapters.
#pragma once

#include "mx_layer.hpp"
#include "mx_rows.hpp"

namespace costa {

__device__ inline int32_t adapter_of(const AdapterIndex& at, int64_t row) {
  const int32_t a = at.index[row];
  return a >= 0 && a < at.count ? a : -1;
}
__device__ inline int rank_of(const AdapterIndex& at, int32_t a) {
  if (a < 0) return 0;
  return at.ranks ? min(max(at.ranks[a], 0), at.rank) : at.rank;
}
__device__ inline float scale_of(const AdapterIndex& at, int32_t a) { return at.scales ? at.scales[a] : 1.0f; }

// Sums of products of parts, those of 2^-24 and less left out.
template <int PA, int PB>
__device__ inline v4f mfma_parts(const v4u* a, const v4u* b, v4f c) {
#pragma unroll
  for (int i = 0; i < PA; ++i)
#pragma unroll
    for (int j = 0; j < PB; ++j)
      if (i + j < 3) c = mfma_bf16(a[i], b[j], c);
  return c;
}

}  // namespace costa
