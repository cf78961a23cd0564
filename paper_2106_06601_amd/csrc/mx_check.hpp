// Argument checks of the microscaled calls.  Host code.
#pragma once

#include <climits>
#include <initializer_list>
#include <string>

#include "mx.hpp"
#include "spans.hpp"

namespace costa {

#define HIP_OR_FAIL(expr)                                                                      \
  do {                                                                                         \
    hipError_t e_ = (expr);                                                                    \
    if (e_ != hipSuccess)                                                                      \
      return fail(COSTA_ERROR_DEVICE, std::string(#expr) + ": " + hipGetErrorString(e_));      \
  } while (0)

#define CHECKED(expr)                          \
  do {                                         \
    const costa_status s_ = (expr);            \
    if (s_ != COSTA_SUCCESS) return s_;        \
  } while (0)

inline int real_size(costa_real t) {
  switch (t) {
    case COSTA_REAL_F64: return 8;
    case COSTA_REAL_F32: return 4;
    case COSTA_REAL_BF16:
    case COSTA_REAL_F16: return 2;
    default: return 0;  // not an element type
  }
}

inline costa_status check_dims(const char* what, int64_t rows, int64_t cols) {
  if (rows < 0 || cols < 0) return fail(COSTA_ERROR_INVALID_VALUE, std::string(what) + ": negative dimension");
  if (rows > INT32_MAX || cols > INT32_MAX)
    return fail(COSTA_ERROR_NOT_SUPPORTED, std::string(what) + ": dimension above 2^31-1");
  return COSTA_SUCCESS;
}

inline costa_status check_mx(const char* what, const costa_mx* q, MxView& v) {
  if (!q) return fail(COSTA_ERROR_INVALID_VALUE, std::string(what) + ": null matrix");
  if (q->format != COSTA_MX_E2M1 && q->format != COSTA_MX_E4M3)
    return fail(COSTA_ERROR_INVALID_VALUE, std::string(what) + ": unknown element format");
  CHECKED(check_dims(what, q->rows, q->cols));
  if (q->rows > 0 && q->cols > 0) {
    if (!q->data || !q->scales) return fail(COSTA_ERROR_INVALID_VALUE, std::string(what) + ": null buffer");
    if ((uintptr_t)q->data % 16 != 0 || (uintptr_t)q->scales % 16 != 0)
      return fail(COSTA_ERROR_INVALID_VALUE, std::string(what) + ": a buffer is not 16-byte aligned");
  }
  v.data = static_cast<uint8_t*>(q->data);
  v.scales = static_cast<uint8_t*>(q->scales);
  v.rows = q->rows;
  v.cols = q->cols;
  v.row_bytes = mx_row_bytes(q->format, q->cols);
  v.row_scales = mx_padded_cols(q->format, q->cols) / kMxBlock;
  v.bits = q->format == COSTA_MX_E2M1 ? 4 : 8;
  return COSTA_SUCCESS;
}

inline costa_status check_matrix(const char* what, const costa_matrix* a, bool f64) {
  if (!a) return fail(COSTA_ERROR_INVALID_VALUE, std::string(what) + ": null matrix");
  const int es = real_size(a->type);
  if (!es) return fail(COSTA_ERROR_INVALID_VALUE, std::string(what) + ": unknown element type");
  if (a->type == COSTA_REAL_F64 && !f64)
    return fail(COSTA_ERROR_NOT_SUPPORTED, std::string(what) + ": no products of 64-bit matrices");
  if (a->order != COSTA_COL_MAJOR && a->order != COSTA_ROW_MAJOR)
    return fail(COSTA_ERROR_INVALID_VALUE, std::string(what) + ": unknown order");
  CHECKED(check_dims(what, a->rows, a->cols));
  const int64_t line = a->order == COSTA_COL_MAJOR ? a->rows : a->cols;
  if (a->ld < 1 || a->ld < line)
    return fail(COSTA_ERROR_INVALID_VALUE, std::string(what) + ": leading dimension too small");
  const int64_t lines = a->order == COSTA_COL_MAJOR ? a->cols : a->rows;
  if (lines > 0 && a->ld > ((int64_t)1 << 58) / lines)  // byte offsets stay within 64 bits
    return fail(COSTA_ERROR_NOT_SUPPORTED, std::string(what) + ": leading dimension too large");
  if (a->rows > 0 && a->cols > 0) {
    if (!a->data) return fail(COSTA_ERROR_INVALID_VALUE, std::string(what) + ": null buffer");
    if ((uintptr_t)a->data % es != 0)
      return fail(COSTA_ERROR_INVALID_VALUE, std::string(what) + ": buffer not aligned to its element type");
  }
  return COSTA_SUCCESS;
}

// The memory of a matrix's elements, and of a buffer of `bytes`.
inline Span span_of(const costa_matrix& a) {
  if (a.rows == 0 || a.cols == 0) return Span{0, 0, 0, 0};
  const int64_t es = real_size(a.type), line = a.order == COSTA_COL_MAJOR ? a.rows : a.cols;
  return Span{(uintptr_t)a.data, line * es, a.ld * es, a.order == COSTA_COL_MAJOR ? a.cols : a.rows};
}
inline Span span_of(const void* p, int64_t bytes) { return Span{(uintptr_t)p, p ? bytes : 0, bytes, 1}; }
inline Span data_of(const MxView& q) { return span_of(q.data, q.rows * q.row_bytes); }
inline Span scales_of(const MxView& q) { return span_of(q.scales, q.rows * q.row_scales); }

// INVALID_VALUE where two of the buffers have a byte in common, `what` they are.
inline costa_status check_apart(const char* what, std::initializer_list<Span> one, std::initializer_list<Span> other) {
  for (const Span& x : one)
    for (const Span& y : other)
      if (spans_meet(x, y)) return fail(COSTA_ERROR_INVALID_VALUE, what);
  return COSTA_SUCCESS;
}

}  // namespace costa
