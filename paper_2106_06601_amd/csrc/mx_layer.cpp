// C ABI entry points of the operators around products (include/costa_layer.h):
// argument checks and launches.
#include <algorithm>
#include <climits>
#include <cmath>

#include "mx_check.hpp"
#include "mx_layer.hpp"

namespace costa {
namespace {

// A row-major matrix of F32, BF16 or F16.
costa_status check_rows(const char* what, const costa_matrix* a) {
  CHECKED(check_matrix(what, a, true));
  if (a->type == COSTA_REAL_F64) return fail(COSTA_ERROR_NOT_SUPPORTED, std::string(what) + ": a 64-bit matrix");
  if (a->order != COSTA_ROW_MAJOR) return fail(COSTA_ERROR_NOT_SUPPORTED, std::string(what) + ": not row-major");
  return COSTA_SUCCESS;
}
// One of `rows` x `cols` and, if it is not null, of the given type; F32 too where `wide`.
costa_status check_like(const char* what, const costa_matrix* a, int64_t rows, int64_t cols, costa_real type,
                        bool wide = false) {
  CHECKED(check_rows(what, a));
  if (a->rows != rows || a->cols != cols) return fail(COSTA_ERROR_SHAPE_MISMATCH, std::string(what) + ": not the shape asked for");
  if (a->type != type && !(wide && a->type == COSTA_REAL_F32))
    return fail(COSTA_ERROR_INVALID_VALUE, std::string(what) + ": not the type asked for");
  return COSTA_SUCCESS;
}
costa_status check_vector(const char* what, const void* p, int64_t n, size_t align) {
  if (n > 0 && !p) return fail(COSTA_ERROR_INVALID_VALUE, std::string(what) + ": null buffer");
  if ((uintptr_t)p % align != 0) return fail(COSTA_ERROR_INVALID_VALUE, std::string(what) + ": not aligned to its elements");
  return COSTA_SUCCESS;
}
costa_status check_workspace(const void* p, size_t bytes, size_t least) {
  if ((uintptr_t)p % 16 != 0) return fail(COSTA_ERROR_INVALID_VALUE, "the workspace is not 16-byte aligned");
  if (least > 0 && (!p || bytes < least))
    return fail(COSTA_ERROR_INVALID_VALUE, "the workspace has less than " + std::to_string(least) + " bytes");
  return COSTA_SUCCESS;
}

bool same(const costa_matrix* a, const costa_matrix* b) {
  return a && b && a->data == b->data && a->ld == b->ld && a->type == b->type;
}

// What a call reads and writes: no output may meet anything else, but the matrix that it may
// be (`self`).
struct Used {
  const char* what;
  Span span;
  bool out;
  const costa_matrix* self;
};
struct Uses {
  Used all[24];
  int n = 0;
  void add(const char* what, const costa_matrix* a, bool out) {
    if (a) all[n++] = Used{what, span_of(*a), out, a};
  }
  void add(const char* what, const MxView& q, bool out) {
    if (!q.data) return;
    all[n++] = Used{what, data_of(q), out, nullptr};
    all[n++] = Used{what, scales_of(q), out, nullptr};
  }
  void add(const char* what, const void* p, int64_t bytes, bool out) {
    if (p) all[n++] = Used{what, span_of(p, bytes), out, nullptr};
  }
  void workspace(const void* p, size_t bytes) {
    add("the workspace", p, (int64_t)std::min(bytes, (size_t)INT64_MAX), true);
  }
  // may: pairs of matrices that may be the same one
  costa_status check(std::initializer_list<std::pair<const costa_matrix*, const costa_matrix*>> may = {}) const {
    for (int i = 0; i < n; ++i)
      for (int j = 0; j < i; ++j) {
        if (!all[i].out && !all[j].out) continue;
        bool fine = false;
        for (const auto& m : may)
          if (same(m.first, m.second) && ((all[i].self == m.first && all[j].self == m.second) ||
                                          (all[i].self == m.second && all[j].self == m.first)))
            fine = true;
        if (!fine && spans_meet(all[i].span, all[j].span))
          return fail(COSTA_ERROR_INVALID_VALUE, std::string(all[i].what) + " overlaps " + all[j].what);
      }
    return COSTA_SUCCESS;
  }
};

RowsView rows_of(const costa_matrix* a) { return a ? RowsView{a->data, a->ld} : RowsView{nullptr, 0}; }

void give(size_t* to, size_t v) {
  if (to) *to = v;
}

}  // namespace
}  // namespace costa

using namespace costa;

extern "C" costa_status costa_mx_norm(float eps, const costa_matrix* X, const costa_matrix* W, const costa_matrix* R,
                                      const costa_matrix* H, const costa_matrix* Y, const costa_mx* Q, float* rstd,
                                      hipStream_t stream) {
  return guarded([&]() -> costa_status {
    if (!(eps >= 0x1p-126f && eps < INFINITY)) return fail(COSTA_ERROR_INVALID_VALUE, "eps is not a positive normal number");
    CHECKED(check_rows("X", X));
    const int64_t m = X->rows, n = X->cols;
    NormArgs a{};
    if (W) CHECKED(check_like("W", W, 1, n, X->type, true));
    if (R) CHECKED(check_like("R", R, m, n, X->type));
    if (H) CHECKED(check_like("H", H, m, n, X->type));
    if (Y) CHECKED(check_like("Y", Y, m, n, X->type));
    if (Q) {
      CHECKED(check_mx("Q", Q, a.q));
      if (Q->rows != m || Q->cols != n) return fail(COSTA_ERROR_SHAPE_MISMATCH, "Q is not the shape of X");
    }
    if (!H && !Y && !Q && !rstd) return fail(COSTA_ERROR_INVALID_VALUE, "no result is asked for");
    if (rstd) CHECKED(check_vector("rstd", rstd, m, 4));
    Uses u;
    u.add("X", X, false), u.add("W", W, false), u.add("R", R, false);
    u.add("H", H, true), u.add("Y", Y, true), u.add("Q", a.q, true), u.add("rstd", rstd, m * 4, true);
    CHECKED(u.check({{H, X}, {H, R}}));
    if (m == 0 || n == 0) return COSTA_SUCCESS;
    a.rows = m, a.cols = n;
    a.type = X->type, a.w_type = W ? W->type : X->type;
    a.x = rows_of(X), a.r = rows_of(R), a.h = rows_of(H), a.y = rows_of(Y);
    a.w = W ? W->data : nullptr;
    a.rstd = rstd;
    a.eps = eps;
    a.inverse = 1.0 / (double)n;
    HIP_OR_FAIL(launch_mx_norm(a, stream));
    return COSTA_SUCCESS;
  });
}

extern "C" costa_status costa_mx_norm_backward(const costa_matrix* dY, const costa_matrix* H, const costa_matrix* W,
                                               const float* rstd, const costa_matrix* dH, const costa_matrix* dX,
                                               const costa_matrix* dW, void* workspace, size_t workspace_bytes,
                                               hipStream_t stream) {
  return guarded([&]() -> costa_status {
    CHECKED(check_rows("dY", dY));
    const int64_t m = dY->rows, n = dY->cols;
    CHECKED(check_like("H", H, m, n, dY->type));
    if (W) CHECKED(check_like("W", W, 1, n, dY->type, true));
    CHECKED(check_vector("rstd", rstd, m, 4));
    if (dH) CHECKED(check_like("dH", dH, m, n, dY->type));
    CHECKED(check_like("dX", dX, m, n, dY->type));
    if (dW) CHECKED(check_like("dW", dW, 1, n, dY->type, true));
    const Parts parts = mx_norm_parts(m, n);
    CHECKED(check_workspace(workspace, workspace_bytes, dW && m > 0 ? (size_t)parts.least * n * 4 : 0));
    Uses u;
    u.add("dY", dY, false), u.add("H", H, false), u.add("W", W, false), u.add("rstd", rstd, m * 4, false);
    u.add("dH", dH, false), u.add("dX", dX, true), u.add("dW", dW, true), u.workspace(workspace, workspace_bytes);
    CHECKED(u.check({{dX, dY}, {dX, dH}}));
    if (n == 0 || (m == 0 && !dW)) return COSTA_SUCCESS;
    NormBackArgs a{};
    a.rows = m, a.cols = n;
    a.type = dY->type, a.w_type = W ? W->type : dY->type;
    a.dy = rows_of(dY), a.h = rows_of(H), a.dh = rows_of(dH), a.dx = rows_of(dX);
    a.w = W ? W->data : nullptr;
    a.rstd = rstd;
    if (dW) {
      a.dw = dW->data;
      a.dw_type = dW->type;
      a.parts = static_cast<float*>(workspace);
      a.most = (int64_t)std::min<size_t>(workspace_bytes / ((size_t)n * 4), (size_t)INT64_MAX);
    }
    a.inverse = 1.0 / (double)n;
    HIP_OR_FAIL(launch_mx_norm_backward(a, stream));
    return COSTA_SUCCESS;
  });
}

extern "C" costa_status costa_mx_norm_workspace(int64_t rows, int64_t cols, size_t* least, size_t* most) {
  return guarded([&]() -> costa_status {
    CHECKED(check_dims("X", rows, cols));
    const Parts p = mx_norm_parts(rows, cols);
    give(least, rows == 0 ? 0 : (size_t)p.least * cols * 4);
    give(most, rows == 0 ? 0 : (size_t)p.most * cols * 4);
    return COSTA_SUCCESS;
  });
}
