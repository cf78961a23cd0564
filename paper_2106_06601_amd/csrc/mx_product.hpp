// Shared by the product kernels.
#pragma once

#include "mx_device.hpp"
#include "mx_plan.hpp"

namespace costa {

constexpr int bytes_of(int src) { return src == SRC_F32 ? 4 : 2; }  // of plain elements

// Where the sums go: C, or a part's place in the workspace.
struct Epilogue {
  void* c;
  int64_t rs, cs;
  int32_t type;
  int32_t vec;  // four elements of a row from a multiple of four on make one aligned store
  float alpha, beta;
};

template <typename T>
__device__ inline void put_elem(const Epilogue& e, int64_t at, float acc) {
  T* p = static_cast<T*>(e.c) + at;
  float v = e.alpha * acc;
  if (e.beta != 0.0f) v += e.beta * (float)*p;
  *p = (T)v;
}

// n (at most 4) elements of row i from column j on.
template <typename T>
__device__ inline void put_typed(const Epilogue& e, int64_t i, int64_t j, v4f acc, int n) {
  const int64_t at = i * e.rs + j * e.cs;
  if (e.vec && n == 4) {
    typedef T V __attribute__((ext_vector_type(4)));
    V* p = reinterpret_cast<V*>(static_cast<T*>(e.c) + at);
    v4f v;
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = e.alpha * acc[q];
    if (e.beta != 0.0f) {
      const V old = *p;
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] += e.beta * (float)old[q];
    }
    V out;
#pragma unroll
    for (int q = 0; q < 4; ++q) out[q] = (T)v[q];
    *p = out;
    return;
  }
#pragma unroll
  for (int q = 0; q < 4; ++q)
    if (q < n) put_elem<T>(e, at + q * e.cs, acc[q]);
}
__device__ inline void put_four(const Epilogue& e, int64_t i, int64_t j, v4f acc, int n) {
  if (n <= 0) return;
  if (e.type == COSTA_REAL_F32) put_typed<float>(e, i, j, acc, n);
  else if (e.type == COSTA_REAL_BF16) put_typed<__bf16>(e, i, j, acc, n);
  else put_typed<_Float16>(e, i, j, acc, n);
}

// A wave's accesses to shared memory take effect in their order: this keeps the
// compiler to it, between lanes that write and others that read.
__device__ inline void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Arguments of the product kernels.
struct Args {
  int64_t m, n, k;
  MxView a, b;
  const void* real;
  int64_t a_rs, a_cs;
  Epilogue e;
  int64_t part;  // elements between the parts of a split sum (0: not split)
};

// Eight consecutive elements of a line of a plain matrix.  Vector loads need no alignment.
template <int SRC>
struct Raw8 {
  uint32_t w[2 * bytes_of(SRC)];
};
// Elements k .. k + 7 of a line of len >= 8 elements that begins at `line`: the load is of
// the line's last eight where fewer are left (always one load, so that none waits for
// another), and place8 moves them into place, with zeros behind.
template <int SRC>
__device__ inline void load8(Raw8<SRC>& r, const char* line, int64_t k, int64_t len) {
  __builtin_memcpy(r.w, line + min(k, len - 8) * bytes_of(SRC), sizeof r.w);
}
template <int SRC>
__device__ inline void place8(Raw8<SRC>& r, int64_t k, int64_t len) {
  const uint32_t s = (uint32_t)max((int64_t)0, min(k - (len - 8), (int64_t)8));  // elements to drop
  if constexpr (bytes_of(SRC) == 4) {
#pragma unroll
    for (int q = 0; q < 8; ++q) r.w[q] = s >= 8 ? 0u : r.w[q];
#pragma unroll
    for (int by = 4; by > 0; by /= 2)
#pragma unroll
      for (int q = 0; q < 8; ++q) r.w[q] = (s & by) ? (q + by < 8 ? r.w[(q + by) % 8] : 0u) : r.w[q];
  } else {
    uint64_t lo = r.w[0] | (uint64_t)r.w[1] << 32, hi = r.w[2] | (uint64_t)r.w[3] << 32;
    if (s & 4) lo = hi, hi = 0;
    const uint32_t bits = 16 * (s & 3);
    if (bits) lo = lo >> bits | hi << (64 - bits), hi >>= bits;
    if (s >= 8) lo = 0, hi = 0;
    r.w[0] = (uint32_t)lo, r.w[1] = (uint32_t)(lo >> 32), r.w[2] = (uint32_t)hi, r.w[3] = (uint32_t)(hi >> 32);
  }
}

// bfloat16 parts of eight elements: each takes the leading 8 bits that are left
// (by truncation, so that none overflows), which leaves nothing of 24 bits after
// three and of 11 after two.  An infinity or a NaN is the first part alone.
template <int SRC>
__device__ inline void raw_parts(const Raw8<SRC>& r, v4u out[parts_of(SRC)]) {
  constexpr int P = parts_of(SRC);
  if constexpr (SRC == SRC_BF16) {
    out[0] = v4u{r.w[0], r.w[1], r.w[2], r.w[3]};
  } else {
    uint32_t x[8];
    bool odd = false;  // an infinity or a NaN among them
    if constexpr (SRC == SRC_F32) {
      uint32_t most = 0;
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        x[q] = r.w[q];
        most = max(most, x[q] & 0x7fffffffu);
      }
      odd = most >= 0x7f800000u;
    } else {
      typedef unsigned short v2h __attribute__((ext_vector_type(2)));
      v2h most = {0, 0};
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        most = __builtin_elementwise_max(most, __builtin_bit_cast(v2h, r.w[q] & 0x7fff7fffu));
        x[2 * q] = __builtin_bit_cast(uint32_t, (float)__builtin_bit_cast(_Float16, (uint16_t)r.w[q]));
        x[2 * q + 1] = __builtin_bit_cast(uint32_t, (float)__builtin_bit_cast(_Float16, (uint16_t)(r.w[q] >> 16)));
      }
      odd = most.x >= 0x7c00 || most.y >= 0x7c00;
    }
    uint32_t rest[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) rest[q] = x[q];
#pragma unroll
    for (int t = 0; t < P; ++t) {
#pragma unroll
      for (int q = 0; q < 4; ++q) out[t][q] = __builtin_amdgcn_perm(rest[2 * q + 1], rest[2 * q], 0x07060302u);
      if (t + 1 < P)
#pragma unroll
        for (int q = 0; q < 8; ++q)
          rest[q] = __builtin_bit_cast(
              uint32_t, __builtin_bit_cast(float, rest[q]) - __builtin_bit_cast(float, rest[q] & 0xffff0000u));
    }
    if (__any(odd)) {
      uint16_t w[8][P];
#pragma unroll
      for (int q = 0; q < 8; ++q) bf16_parts<P>(__builtin_bit_cast(float, x[q]), w[q]);
#pragma unroll
      for (int t = 0; t < P; ++t)
#pragma unroll
        for (int q = 0; q < 4; ++q) out[t][q] = w[2 * q][t] | (uint32_t)w[2 * q + 1][t] << 16;
    }
  }
}

__device__ inline v4f mfma_bf16(v4u a, v4u b, v4f c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
}

hipError_t launch_tiles_bf16(int src, const Args& p, const ProductPlan& plan, hipStream_t stream);
hipError_t launch_tiles_scaled(const Args& p, const ProductPlan& plan, hipStream_t stream);

}  // namespace costa
