// Eight elements of a row of a plain matrix at a time, for the kernels.
#pragma once

#include "mx_layer.hpp"
#include "mx_product.hpp"

namespace costa {

template <int SRC>
using Elem = typename std::conditional<SRC == SRC_F32, float,
                                       typename std::conditional<SRC == SRC_F16, _Float16, __bf16>::type>::type;

template <int SRC>
__device__ inline void raw_floats(const Raw8<SRC>& r, float x[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if constexpr (SRC == SRC_F32) x[i] = __builtin_bit_cast(float, r.w[i]);
    else if constexpr (SRC == SRC_BF16)
      x[i] = __builtin_bit_cast(float, i % 2 ? r.w[i / 2] & 0xffff0000u : r.w[i / 2] << 16);
    else x[i] = (float)__builtin_bit_cast(_Float16, (uint16_t)(r.w[i / 2] >> (i % 2 * 16)));
  }
}

// The eight elements of a line (of `len`) from c on; zeros past its end.  WIDE: the line
// has 8 or more, and the load is one, which waits for no branch (placed8() moves what it read
// into place).  I: 32 bits where a line's elements are counted in them.
template <int SRC, bool WIDE, typename I>
__device__ inline void get8(Raw8<SRC>& r, const void* line, I c, I len) {
  if constexpr (WIDE) {
    __builtin_memcpy(r.w, static_cast<const char*>(line) + (int64_t)min(c, (I)(len - 8)) * bytes_of(SRC), sizeof r.w);
  } else {
#pragma unroll
    for (int i = 0; i < (int)(sizeof r.w / 4); ++i) r.w[i] = 0;
    for (int i = 0; i < 8; ++i)
      if (c + i < len) {
        if constexpr (bytes_of(SRC) == 4) r.w[i] = static_cast<const uint32_t*>(line)[c + i];
        else r.w[i / 2] |= (uint32_t) static_cast<const uint16_t*>(line)[c + i] << (i % 2 * 16);
      }
  }
}
// Moves what get8() read at the end of a line into place: once.
template <int SRC, bool WIDE, typename I>
__device__ inline void placed8(Raw8<SRC>& r, I c, I len) {
  if (WIDE && c + 8 > len) place8<SRC>(r, c, len);
}
template <int SRC, bool WIDE, typename I>
__device__ inline void floats8(Raw8<SRC>& r, I c, I len, float x[8]) {
  placed8<SRC, WIDE>(r, c, len);
  raw_floats<SRC>(r, x);
}
template <int SRC, typename I>
__device__ inline void put8(void* line, I c, I len, const float x[8]) {
  Elem<SRC> v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (Elem<SRC>)x[i];
  Elem<SRC>* p = static_cast<Elem<SRC>*>(line) + c;
  if (c + 8 <= len) __builtin_memcpy(p, v, sizeof v);
  else
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < len) p[i] = v[i];
}

template <int SRC>
__device__ inline const void* line_of(const RowsView& v, int64_t row) {
  return static_cast<const char*>(v.data) + row * v.ld * bytes_of(SRC);
}
template <int SRC>
__device__ inline void* line_to(const RowsView& v, int64_t row) {
  return static_cast<char*>(v.data) + row * v.ld * bytes_of(SRC);
}

}  // namespace costa
