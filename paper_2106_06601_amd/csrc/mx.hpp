// Microscaled matrices: what the host code and the kernels share.
#pragma once

#include "../../include/costa_mx.h"
#include "internal.hpp"

namespace costa {

constexpr int kMxBlock = 32;  // elements that share a scale
inline int mx_pad(costa_mx_format f) { return f == COSTA_MX_E2M1 ? 256 : 128; }
inline int64_t mx_padded_cols(costa_mx_format f, int64_t cols) {
  const int64_t p = mx_pad(f);
  return (cols + p - 1) / p * p;
}
inline int64_t mx_row_bytes(costa_mx_format f, int64_t cols) {
  const int64_t pc = mx_padded_cols(f, cols);
  return f == COSTA_MX_E2M1 ? pc / 2 : pc;
}

// A microscaled matrix as the kernels see it; data null: not there.
struct MxView {
  uint8_t* data;
  uint8_t* scales;
  int64_t rows, cols;
  int64_t row_bytes, row_scales;
  int32_t bits;  // 4 or 8
};

// ---- quantise (mx_store.hip) -----------------------------------------------
// The source is taken by lines: `lines` of them, `len` elements each, elements
// of a line next to one another.  (A row-major matrix by its rows, a
// column-major one by its columns.)  `along` holds blocks that run along the
// lines, `across` blocks that run over 32 lines; either may be missing.
struct QuantArgs {
  int64_t lines, len;
  const void* src;
  int64_t ld;
  costa_real type;
  float alpha;
  MxView along, across;
};
hipError_t launch_mx_quantize(const QuantArgs& a, hipStream_t stream);

// A layout's lines and elements.  Line i lies in block line `lb`, the last with
// start[lb] <= i; then (class, local line) = (lb, i - start[lb]).  Block-cyclic
// layouts (blk > 0) have no such arrays: of the dealt dimension, index off + i is in
// block (off + i) / blk, whose process (shifted by src) is the class, and is the
// process's (off + i) / (blk * np) * blk + (off + i) % blk -th.  The same for an
// element's place in its line.  The cell (line class, place class) gives the place of
// the pointer in the call's array, the offset and the leading dimension: the element
// is at offset + local line * ld + local place.
struct MxCell {
  int64_t offset, ld;
  int64_t pointer;
};
struct MxSplits {
  const int64_t* start;  // n + 1 entries
  int32_t n;
  int32_t np, src;  // block-cyclic: processes, and the one that has block 0
  int64_t off, blk;
  int32_t narrow;  // off + i is below 2^32 - 1
};
struct MxLayoutArgs {
  MxSplits line, place;
  const MxCell* cells;  // line class * nplace + place class
  int32_t nplace;
  int32_t dealt;  // block-cyclic: a cell's pointer is at the cell's own index
};
constexpr int kMxRanksMax = 256;
struct MxPointers {
  const void* p[kMxRanksMax];
};
hipError_t launch_mx_quantize_layout(const QuantArgs& a, const MxLayoutArgs& l, const MxPointers& p,
                                     hipStream_t stream);

// ---- dequantise (mx_store.hip) -----------------------------------------------
struct DequantArgs {
  MxView q;
  void* dst;
  int64_t rs, cs;  // strides of A's rows and columns, elements; one of them is 1
  costa_real type;
  float alpha, beta;
};
hipError_t launch_mx_dequantize(const DequantArgs& a, hipStream_t stream);

// ---- products (mx_plan.hpp, mx_product.hip, mx_tiles.hip) -------------------------------------------------
// C (m x n) <- alpha * A B^T + beta * C over k; A microscaled (mx.data set) or
// plain with element (i, l) at real[i*rs + l*cs].
struct ProductArgs {
  int64_t m, n, k;
  MxView amx;
  const void* real;
  int64_t a_rs, a_cs;
  costa_real a_type;
  MxView b;
  void* c;
  int64_t c_rs, c_cs;
  costa_real c_type;
  float alpha, beta;
  float* workspace;
  size_t workspace_bytes;
};
size_t mx_product_workspace(int64_t m, int64_t n, int64_t k);
hipError_t launch_mx_product(const ProductArgs& a, hipStream_t stream);
// The sums alone (k > 0), neither scaled nor joined: `splits` parts of m x n floats in the
// workspace, which holds one at least.  Of a, alpha, beta and C are not looked at.
hipError_t launch_mx_product_parts(const ProductArgs& a, int& splits, hipStream_t stream);
size_t mx_product_parts_workspace(int64_t m, int64_t n, int64_t k);  // what it can use

// ---- entry points (mx.cpp) -------------------------------------------------------
// Frees the layout tables (called by costa_finalize); waits for the kernels that read them.
void release_mx_tables();

}  // namespace costa
