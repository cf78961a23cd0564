// Products of microscaled matrices on the matrix instructions.
#include <algorithm>

#include "mx_device.hpp"

namespace costa {
namespace {

// Kinds of left operands.
enum Source : int { SRC_MX4, SRC_MX8, SRC_BF16, SRC_F16, SRC_F32 };
constexpr int parts_of(int src) { return src == SRC_F32 ? 3 : src == SRC_F16 ? 2 : 1; }

struct Epilogue {
  void* c;
  int64_t rs, cs;
  int32_t type;
  float alpha, beta;
};

__device__ inline void put_c(const Epilogue& e, int64_t i, int64_t j, float acc) {
  const int64_t at = i * e.rs + j * e.cs;
  float v = e.alpha * acc;
  if (e.type == COSTA_REAL_F32) {
    float* p = static_cast<float*>(e.c) + at;
    if (e.beta != 0.0f) v += e.beta * *p;
    *p = v;
  } else if (e.type == COSTA_REAL_BF16) {
    __bf16* p = static_cast<__bf16*>(e.c) + at;
    if (e.beta != 0.0f) v += e.beta * (float)*p;
    *p = (__bf16)v;
  } else {
    _Float16* p = static_cast<_Float16*>(e.c) + at;
    if (e.beta != 0.0f) v += e.beta * (float)*p;
    *p = (_Float16)v;
  }
}

struct Args {
  int64_t m, n, k;
  MxView a, b;
  const void* real;
  int64_t a_rs, a_cs;
  Epilogue e;
};

// Eight consecutive elements of row i of the left operand from k0 on, as bfloat16 parts.
template <int SRC>
__device__ inline void load_left(const Args& p, int64_t i, int64_t k0, v4u out[parts_of(SRC)]) {
  if (SRC == SRC_MX4 || SRC == SRC_MX8) {
    constexpr int BITS = SRC == SRC_MX4 ? 4 : 8;
    v2u d = {0u, 0u};
    uint32_t s = 0;
    if (k0 < p.a.row_scales * kMxBlock) {
      const uint8_t* row = p.a.data + i * p.a.row_bytes;
      if (BITS == 4) d.x = *reinterpret_cast<const uint32_t*>(row + k0 / 2);
      else d = *reinterpret_cast<const v2u*>(row + k0);
      s = p.a.scales[i * p.a.row_scales + k0 / kMxBlock];
    }
    out[0] = mx_decode8_bf16<BITS>(d, s);
  } else {
    constexpr int P = parts_of(SRC);
    uint16_t w[8][P];
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      float x = 0.0f;
      if (k0 + q < p.k) {
        const int64_t at = i * p.a_rs + (k0 + q) * p.a_cs;
        x = SRC == SRC_BF16  ? (float)static_cast<const __bf16*>(p.real)[at]
            : SRC == SRC_F16 ? (float)static_cast<const _Float16*>(p.real)[at]
                             : static_cast<const float*>(p.real)[at];
      }
      bf16_parts<P>(x, w[q]);
    }
#pragma unroll
    for (int t = 0; t < P; ++t)
#pragma unroll
      for (int q = 0; q < 4; ++q) out[t][q] = w[2 * q][t] | (uint32_t)w[2 * q + 1][t] << 16;
  }
}

// A wave makes 16 x 16 elements of C from 32 elements of k at a time: lane l
// holds row l % 16 of either operand at k = 8 * (l / 16) .. + 7, and of the result
// rows 4 * (l / 16) .. + 3 of column l % 16.
template <int SRC, int BBITS>
__global__ __launch_bounds__(256) void product_simple(Args p, int64_t tiles_n, int64_t tiles) {
  const int lane = threadIdx.x % 64, r = lane % 16, g = lane / 16;
  for (int64_t t = (int64_t)blockIdx.x * 4 + threadIdx.x / 64; t < tiles; t += (int64_t)gridDim.x * 4) {
    const int64_t i0 = t / tiles_n * 16, j0 = t % tiles_n * 16;
    const int64_t i = min(i0 + r, p.m - 1), j = min(j0 + r, p.n - 1);
    v4f acc = {0, 0, 0, 0};
    for (int64_t k0 = 0; k0 < p.k; k0 += 32) {
      v4u a[parts_of(SRC)];
      load_left<SRC>(p, i, k0 + 8 * g, a);
      v2u d = {0u, 0u};
      const uint8_t* row = p.b.data + j * p.b.row_bytes;
      if (BBITS == 4) d.x = *reinterpret_cast<const uint32_t*>(row + k0 / 2 + 4 * g);
      else d = *reinterpret_cast<const v2u*>(row + k0 + 8 * g);
      const v8bf b =
          __builtin_bit_cast(v8bf, mx_decode8_bf16<BBITS>(d, p.b.scales[j * p.b.row_scales + k0 / kMxBlock]));
#pragma unroll
      for (int q = 0; q < parts_of(SRC); ++q)
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a[q]), b, acc, 0, 0, 0);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (i0 + 4 * g + q < p.m && j0 + r < p.n) put_c(p.e, i0 + 4 * g + q, j0 + r, acc[q]);
  }
}

template <int SRC>
hipError_t launch_source(const Args& p, hipStream_t stream) {
  const int64_t tn = (p.n + 15) / 16, tiles = (p.m + 15) / 16 * tn;
  const dim3 grid((unsigned)std::min<int64_t>((tiles + 3) / 4, 1 << 20));
  if (p.b.bits == 4) product_simple<SRC, 4><<<grid, 256, 0, stream>>>(p, tn, tiles);
  else product_simple<SRC, 8><<<grid, 256, 0, stream>>>(p, tn, tiles);
  return hipGetLastError();
}

}  // namespace

size_t mx_product_workspace(int64_t, int64_t, int64_t) { return 0; }

hipError_t launch_mx_product(const ProductArgs& a, hipStream_t stream) {
  const Args p{a.m, a.n, a.k, a.amx, a.b, a.real, a.a_rs, a.a_cs, {a.c, a.c_rs, a.c_cs, a.c_type, a.alpha, a.beta}};
  if (a.amx.bits == 4) return launch_source<SRC_MX4>(p, stream);
  if (a.amx.bits == 8) return launch_source<SRC_MX8>(p, stream);
  switch (a.a_type) {
    case COSTA_REAL_BF16: return launch_source<SRC_BF16>(p, stream);
    case COSTA_REAL_F16: return launch_source<SRC_F16>(p, stream);
    default: return launch_source<SRC_F32>(p, stream);
  }
}

}  // namespace costa
