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

namespace costa {
namespace {

constexpr size_t kSliceBytes = (size_t)128 << 20;  // of a slice's sums: the last-level cache holds them

size_t up16(size_t v) { return (v + 15) / 16 * 16; }

// Rows of C whose sums are in the workspace at a time: all, or so many.
int64_t slice_rows(int64_t m, int64_t n) {
  const int64_t most = (int64_t)(kSliceBytes / 4) / std::max<int64_t>(n, 1) / 256 * 256;
  return std::min(m, std::max<int64_t>(most, 256));
}

// Bytes of the sums of `rows` rows, and of those with what a split sum can use.
size_t sums_bytes(int64_t rows, int64_t n) { return (size_t)rows * n * 4; }
size_t split_bytes(int64_t rows, int64_t n, int64_t k) {
  return std::max(mx_product_parts_workspace(rows, n, k), sums_bytes(rows, n));
}

// The adapters' index and, where they are given, A and B.
costa_status check_adapters(const costa_mx_adapters* p, const int32_t* index, int64_t m, AdapterIndex& at) {
  if (!p) return fail(COSTA_ERROR_INVALID_VALUE, "adapters: null");
  if (p->count < 0 || p->rank < 0) return fail(COSTA_ERROR_INVALID_VALUE, "adapters: negative count or rank");
  if (p->rank > kRankMax) return fail(COSTA_ERROR_NOT_SUPPORTED, "adapters: a rank above 256");
  if ((int64_t)p->count * p->rank > INT32_MAX) return fail(COSTA_ERROR_NOT_SUPPORTED, "adapters: more than 2^31-1 rows");
  CHECKED(check_vector("ranks", p->ranks, 0, 4));
  CHECKED(check_vector("scales", p->scales, 0, 4));
  CHECKED(check_vector("index", index, m, 4));
  at = AdapterIndex{p->count, p->rank, p->ranks, p->scales, index};
  return COSTA_SUCCESS;
}

}  // namespace
}  // namespace costa

extern "C" costa_status costa_mx_product_adapted(float alpha, const costa_matrix* X, const costa_mx* W,
                                                 const costa_mx_adapters* adapters, const int32_t* index, float beta,
                                                 const costa_matrix* C, const costa_matrix* V, void* workspace,
                                                 size_t workspace_bytes, hipStream_t stream) {
  return guarded([&]() -> costa_status {
    CHECKED(check_rows("X", X));
    const int64_t m = X->rows, k = X->cols;
    MxView w;
    CHECKED(check_mx("W", W, w));
    if (W->cols != k) return fail(COSTA_ERROR_SHAPE_MISMATCH, "X and W have different lengths to sum over");
    const int64_t n = W->rows;
    AdapterIndex at;
    CHECKED(check_adapters(adapters, index, m, at));
    const int64_t all = (int64_t)at.count * at.rank;
    CHECKED(check_like("A", adapters->A, all, k, X->type));
    CHECKED(check_like("B", adapters->B, all, n, X->type));
    CHECKED(check_rows("C", C));
    if (C->rows != m || C->cols != n) return fail(COSTA_ERROR_SHAPE_MISMATCH, "C is not the shape of X W^T");
    if (V) CHECKED(check_like("V", V, m, at.rank, COSTA_REAL_F32));
    size_t least = 0;
    CHECKED(costa_mx_adapted_workspace(m, n, k, at.rank, &least, nullptr));
    CHECKED(check_workspace(workspace, workspace_bytes, least));
    Uses u;
    u.add("X", X, false), u.add("W", w, false), u.add("A", adapters->A, false), u.add("B", adapters->B, false);
    u.add("ranks", at.ranks, (int64_t)at.count * 4, false), u.add("scales", at.scales, (int64_t)at.count * 4, false);
    u.add("index", index, m * 4, false);
    u.add("C", C, true), u.add("V", V, true), u.workspace(workspace, workspace_bytes);
    CHECKED(u.check());
    if (m == 0) return COSTA_SUCCESS;
    char* room = static_cast<char*>(workspace);
    size_t left = workspace ? workspace_bytes : 0;
    AdapterDotsArgs d{at, m, k, X->type, rows_of(X), rows_of(adapters->A), nullptr, at.rank, nullptr, 0};
    if (V) {
      d.v = static_cast<float*>(V->data), d.v_ld = V->ld;
    } else {
      d.v = reinterpret_cast<float*>(room);
      const size_t taken = up16((size_t)m * at.rank * 4);
      room += taken, left -= taken;
    }
    const bool fused = mx_adapted_fused(X->type, w.bits, m, n, k);
    void* const spread = room;
    if (fused) room += mx_spread_bytes(m, at.rank), left -= mx_spread_bytes(m, at.rank);
    if (at.rank > 0) {  // (the parts of v lie where the product's sums will)
      int64_t splits = 0;
      d.parts = reinterpret_cast<float*>(room);
      d.most = (int64_t)(left / ((size_t)m * at.rank * 4));
      HIP_OR_FAIL(launch_mx_adapter_dots(d, splits, stream));
      if (fused) HIP_OR_FAIL(launch_mx_adapter_spread(d, splits, spread, stream));
      else if (splits > 0) HIP_OR_FAIL(launch_mx_adapter_dots_join(d, splits, stream));
    }
    if (n == 0) return COSTA_SUCCESS;
    if (fused) {
      AdapterAddArgs c{};
      c.at = at;
      c.m = m, c.n = n;
      c.type = X->type, c.c_type = C->type;
      c.low = rows_of(adapters->B), c.c = rows_of(C);
      c.alpha = alpha, c.beta = beta;
      c.spread = static_cast<const v4u*>(spread);
      HIP_OR_FAIL(launch_mx_adapted_product(c, rows_of(X), k, w, stream));
      return COSTA_SUCCESS;
    }
    // slices of rows whose sums the workspace holds
    const int64_t per = k == 0 ? m : std::min<int64_t>(slice_rows(m, n), (int64_t)(left / sums_bytes(1, n)));
    for (int64_t i = 0; i < m; i += per) {
      const int64_t rows = std::min(per, m - i);
      const int64_t es = real_size(X->type);
      AdapterAddArgs c{};
      c.at = at, c.at.index += i;
      c.m = rows, c.n = n;
      c.type = X->type, c.c_type = C->type;
      c.low = rows_of(adapters->B);
      c.c = RowsView{static_cast<char*>(C->data) + i * C->ld * real_size(C->type), C->ld};
      c.v = d.v + i * d.v_ld, c.v_ld = d.v_ld;
      c.parts = reinterpret_cast<float*>(room);
      c.alpha = alpha, c.beta = beta;
      if (k > 0) {
        ProductArgs p{};
        p.m = rows, p.n = n, p.k = k;
        p.real = static_cast<const char*>(X->data) + i * X->ld * es;
        p.a_rs = X->ld, p.a_cs = 1, p.a_type = X->type;
        p.b = w;
        p.workspace = reinterpret_cast<float*>(room), p.workspace_bytes = left;
        HIP_OR_FAIL(launch_mx_product_parts(p, c.splits, stream));
      }
      HIP_OR_FAIL(launch_mx_adapter_add(c, stream));
    }
    return COSTA_SUCCESS;
  });
}

extern "C" costa_status costa_mx_adapted_workspace(int64_t m, int64_t n, int64_t k, int32_t rank, size_t* least,
                                                   size_t* most) {
  return guarded([&]() -> costa_status {
    CHECKED(check_dims("C", m, n));
    CHECKED(check_dims("X", m, k));
    if (rank < 0) return fail(COSTA_ERROR_INVALID_VALUE, "negative rank");
    if (rank > kRankMax) return fail(COSTA_ERROR_NOT_SUPPORTED, "a rank above 256");
    // what calls of these sizes do, of whatever types: spread v, or keep sums
    bool spreads = false, sums = false;
    for (const costa_real type : {COSTA_REAL_F32, COSTA_REAL_BF16, COSTA_REAL_F16})
      for (const int bits : {4, 8}) {
        const bool fused = mx_adapted_fused(type, bits, m, n, k);
        spreads |= fused;
        sums |= !fused && m > 0 && n > 0 && k > 0;
      }
    const size_t v = up16((size_t)m * rank * 4), spread = spreads ? mx_spread_bytes(m, rank) : 0;
    give(least, v + std::max(spread, sums ? sums_bytes(std::min<int64_t>(m, 256), n) : 0));
    give(most, v + spread + std::max(sums ? split_bytes(slice_rows(m, n), n, k) : 0,
                                     (size_t)m * rank * 4 * mx_adapter_dots_parts(m, k, rank)));
    return COSTA_SUCCESS;
  });
}

extern "C" costa_status costa_mx_adapter_gradient(const costa_mx_adapters* adapters, const int32_t* index,
                                                  const costa_matrix* V, const costa_matrix* Z, float beta,
                                                  const costa_matrix* G, void* workspace, size_t workspace_bytes,
                                                  hipStream_t stream) {
  return guarded([&]() -> costa_status {
    CHECKED(check_rows("Z", Z));
    const int64_t m = Z->rows, len = Z->cols;
    AdapterGradArgs a{};
    CHECKED(check_adapters(adapters, index, m, a.at));
    CHECKED(check_like("V", V, m, a.at.rank, COSTA_REAL_F32));
    const int64_t all = (int64_t)a.at.count * a.at.rank;
    CHECKED(check_rows("G", G));
    if (G->rows != all || G->cols != len) return fail(COSTA_ERROR_SHAPE_MISMATCH, "G is not the shape of the adapters' rows");
    CHECKED(check_workspace(workspace, workspace_bytes, 0));
    Uses u;
    u.add("V", V, false), u.add("Z", Z, false), u.add("index", index, m * 4, false);
    u.add("ranks", a.at.ranks, (int64_t)a.at.count * 4, false), u.add("scales", a.at.scales, (int64_t)a.at.count * 4, false);
    u.add("G", G, true), u.workspace(workspace, workspace_bytes);
    CHECKED(u.check());
    if (all == 0 || len == 0) return COSTA_SUCCESS;
    a.m = m, a.len = len;
    a.type = Z->type, a.g_type = G->type;
    a.z = rows_of(Z), a.g = rows_of(G);
    a.v = static_cast<const float*>(V->data), a.v_ld = V->ld;
    a.beta = beta;
    a.parts = static_cast<float*>(workspace);
    a.most = workspace ? (int64_t)std::min<size_t>(workspace_bytes / ((size_t)all * len * 4), 65535) : 0;
    HIP_OR_FAIL(launch_mx_adapter_grad(a, stream));
    return COSTA_SUCCESS;
  });
}

extern "C" costa_status costa_mx_adapter_gradient_workspace(int64_t m, int64_t len, int32_t count, int32_t rank,
                                                            size_t* least, size_t* most) {
  return guarded([&]() -> costa_status {
    CHECKED(check_dims("Z", m, len));
    if (count < 0 || rank < 0) return fail(COSTA_ERROR_INVALID_VALUE, "negative count or rank");
    if (rank > kRankMax) return fail(COSTA_ERROR_NOT_SUPPORTED, "a rank above 256");
    if ((int64_t)count * rank > INT32_MAX) return fail(COSTA_ERROR_NOT_SUPPORTED, "more than 2^31-1 rows");
    const int64_t parts = mx_adapter_grad_parts(m, len, count, rank);
    give(least, 0);
    give(most, parts > 1 ? (size_t)count * rank * len * 4 * parts : 0);
    return COSTA_SUCCESS;
  });
}

namespace costa {
namespace {

constexpr int64_t kPieceColumns = 256;  // pieces of the vocabulary are multiples: blocks and rows of few-bit matrices stay whole
constexpr size_t kPieceBytes = (size_t)256 << 20;  // of what a piece keeps of every row and column

int64_t chunks_of(int64_t n) { return (n + kLossChunk - 1) / kLossChunk; }

// Columns of a piece, with `bytes` of memory for `elem` bytes of each of its m x columns
// elements: whole chunks if there is room.  At least kPieceColumns (the caller has asked for as much).
int64_t piece_columns(int64_t m, int64_t n, size_t bytes, size_t elem) {
  const size_t most = bytes / ((size_t)std::max<int64_t>(m, 1) * elem);
  if (most >= (size_t)n) return n;
  const int64_t to = most >= (size_t)kLossChunk ? kLossChunk : kPieceColumns;
  return std::max<int64_t>((int64_t)most / to * to, kPieceColumns);
}
size_t piece_bytes(int64_t m, int64_t n, size_t elem) {
  return (size_t)m * (size_t)std::min<int64_t>(n, std::max<int64_t>(piece_columns(m, n, kPieceBytes, elem), kPieceColumns)) * elem;
}
size_t least_piece(int64_t m, int64_t n, size_t elem) { return (size_t)m * std::min(n, kPieceColumns) * elem; }

MxView columns_of(const MxView& q, int64_t first, int64_t n) {  // first: a multiple of 256
  MxView v = q;
  v.data += first * q.bits / 8;
  v.scales += first / kMxBlock;
  v.cols = n;
  return v;
}
MxView rows_of(const MxView& q, int64_t first, int64_t n) {
  MxView v = q;
  v.data += first * q.row_bytes;
  v.scales += first * q.row_scales;
  v.rows = n;
  return v;
}

// Chunks of columns whose statistics a call keeps: a piece of fewer columns than a chunk makes
// a chunk of its own.
int64_t chunks_kept(int64_t n, int64_t per) { return (n + per - 1) / per * chunks_of(std::min(n, per)); }

// What both calls check; `w` and the row's vectors.
costa_status check_loss(const costa_matrix* X, const costa_mx* W, const int64_t* target, MxView& w) {
  CHECKED(check_rows("X", X));
  CHECKED(check_mx("W", W, w));
  if (W->cols != X->cols) return fail(COSTA_ERROR_SHAPE_MISMATCH, "X and W have different lengths to sum over");
  return check_vector("target", target, X->rows, 8);
}

// Whether G, its types allowing it, is in bfloat16 where dW is wanted: both products take whole tiles of a piece as
// large as the most workspace holds.  Not of the piece that a call's workspace holds: results would then have
// more or fewer bits by the room that they were made in.
bool bf16_with_dw(costa_real type, int bits, int xt_bits, int64_t m, int64_t n, int64_t k) {
  const int64_t per = piece_columns(m, n, up16(piece_bytes(m, n, 4)), 2);
  return mx_loss_fused(type, bits, m, per, k) && mx_loss_dw_fused(xt_bits, m, per, k);
}

ProductArgs logits_of(const costa_matrix* X, const MxView& w, int64_t first, int64_t n, float alpha) {
  ProductArgs p{};
  p.m = X->rows, p.n = n, p.k = X->cols;
  p.real = X->data;
  p.a_rs = X->ld, p.a_cs = 1, p.a_type = X->type;
  p.b = rows_of(w, first, n);
  p.alpha = alpha;
  return p;
}

}  // namespace
}  // namespace costa

extern "C" costa_status costa_mx_loss_workspace(int64_t m, int64_t n, int64_t k, int backward, size_t* least,
                                                size_t* most) {
  return guarded([&]() -> costa_status {
    CHECKED(check_dims("logits", m, n));
    CHECKED(check_dims("X", m, k));
    if (m == 0) {
      give(least, 0), give(most, 0);
    } else if (!backward) {
      const size_t at = up16((size_t)m * 4);
      give(least, at + up16((size_t)m * chunks_kept(n, kPieceColumns) * sizeof(LossStat)) + least_piece(m, n, 4));
      const size_t sums = piece_bytes(m, n, 4);
      // (statistics of every 128 columns, where the logits stay in the tiles)
      give(most, at + std::max(up16((size_t)m * chunks_kept(n, kPieceColumns) * sizeof(LossStat)) +
                                   std::max(sums, mx_product_parts_workspace(m, std::min(n, piece_columns(m, n, sums, 4)), k)),
                               (size_t)m * ((n + 127) / 128) * sizeof(LossStat)));
    } else {
      const size_t dx = up16((size_t)m * k * 4) + up16((size_t)m * 4);  // what dX is summed in, and the factors of G's rows
      give(least, dx + up16(least_piece(m, n, 4)) + up16(least_piece(m, n, 4)));
      const size_t g = piece_bytes(m, n, 4);
      const int64_t per = piece_columns(m, n, g, 4);
      give(most, dx + up16(g) + std::max({up16(g), mx_product_parts_workspace(m, per, k), mx_product_workspace(m, k, per),
                                          mx_product_workspace(per, k, m)}));
    }
    return COSTA_SUCCESS;
  });
}

extern "C" costa_status costa_mx_loss(float alpha, const costa_matrix* X, const costa_mx* W, const int64_t* target,
                                      float* loss, float* lse, void* workspace, size_t workspace_bytes,
                                      hipStream_t stream) {
  return guarded([&]() -> costa_status {
    MxView w;
    CHECKED(check_loss(X, W, target, w));
    const int64_t m = X->rows, n = W->rows, k = X->cols;
    CHECKED(check_vector("loss", loss, m, 4));
    CHECKED(check_vector("lse", lse, m, 4));
    size_t least = 0;
    CHECKED(costa_mx_loss_workspace(m, n, k, 0, &least, nullptr));
    CHECKED(check_workspace(workspace, workspace_bytes, least));
    Uses u;
    u.add("X", X, false), u.add("W", w, false), u.add("target", target, m * 8, false);
    u.add("loss", loss, m * 4, true), u.add("lse", lse, m * 4, true), u.workspace(workspace, workspace_bytes);
    CHECKED(u.check());
    if (m == 0) return COSTA_SUCCESS;
    char* room = static_cast<char*>(workspace);
    float* const at = reinterpret_cast<float*>(room);
    room += up16((size_t)m * 4);
    LossStat* const stats = reinterpret_cast<LossStat*>(room);
    room += up16((size_t)m * chunks_kept(n, kPieceColumns) * sizeof(LossStat));
    const size_t left = workspace_bytes - (size_t)(room - static_cast<char*>(workspace));
    if (mx_loss_fused(X->type, w.bits, m, n, k)) {
      const int64_t chunks = mx_loss_tile_chunks(X->type, w.bits, m, n, k);
      if (workspace_bytes >= up16((size_t)m * 4) + (size_t)m * chunks * sizeof(LossStat)) {
        HIP_OR_FAIL(launch_mx_loss_tiles(logits_of(X, w, 0, n, alpha), target, stats, at, stream));
        HIP_OR_FAIL(launch_mx_loss_join(m, n, chunks, stats, at, target, loss, lse, stream));
        return COSTA_SUCCESS;
      }
    }
    const int64_t per = n == 0 ? 1 : piece_columns(m, n, std::min(left, piece_bytes(m, n, 4)), 4);
    int64_t chunks = 0;
    for (int64_t j = 0; j < n; j += per) {
      const int64_t cols = std::min(per, n - j);
      LogitsPart l{m, cols, j, reinterpret_cast<float*>(room), 0, alpha, target};
      if (k > 0) {
        ProductArgs p = logits_of(X, w, j, cols, alpha);
        p.workspace = reinterpret_cast<float*>(room), p.workspace_bytes = left;
        HIP_OR_FAIL(launch_mx_product_parts(p, l.splits, stream));
      }
      HIP_OR_FAIL(launch_mx_loss_stats(l, stats + chunks * m, at, stream));
      chunks += chunks_of(cols);
    }
    HIP_OR_FAIL(launch_mx_loss_join(m, n, chunks, stats, at, target, loss, lse, stream));
    return COSTA_SUCCESS;
  });
}

extern "C" costa_status costa_mx_loss_backward(float alpha, const costa_matrix* X, const costa_mx* W,
                                               const int64_t* target, const float* lse, const float* dloss,
                                               const costa_mx* WT, const costa_matrix* dX, const costa_mx* XT,
                                               float beta, const costa_matrix* dW, void* workspace,
                                               size_t workspace_bytes, hipStream_t stream) {
  return guarded([&]() -> costa_status {
    MxView w, wt{}, xt{};
    CHECKED(check_loss(X, W, target, w));
    const int64_t m = X->rows, n = W->rows, k = X->cols;
    CHECKED(check_vector("lse", lse, m, 4));
    if (dloss) CHECKED(check_vector("dloss", dloss, m, 4));
    if (!dX && !dW) return fail(COSTA_ERROR_INVALID_VALUE, "neither dX nor dW");
    if (dX) {
      CHECKED(check_rows("dX", dX));
      CHECKED(check_mx("WT", WT, wt));
      if (dX->rows != m || dX->cols != k) return fail(COSTA_ERROR_SHAPE_MISMATCH, "dX is not the shape of X");
      if (WT->rows != k || WT->cols != n) return fail(COSTA_ERROR_SHAPE_MISMATCH, "WT is not the shape of the transposed W");
    }
    if (dW) {
      CHECKED(check_rows("dW", dW));
      CHECKED(check_mx("XT", XT, xt));
      if (dW->rows != n || dW->cols != k) return fail(COSTA_ERROR_SHAPE_MISMATCH, "dW is not the shape of W");
      if (XT->rows != k || XT->cols != m) return fail(COSTA_ERROR_SHAPE_MISMATCH, "XT is not the shape of the transposed X");
    }
    size_t least = 0;
    CHECKED(costa_mx_loss_workspace(m, n, k, 1, &least, nullptr));
    CHECKED(check_workspace(workspace, workspace_bytes, least));
    Uses u;
    u.add("X", X, false), u.add("W", w, false), u.add("WT", wt, false), u.add("XT", xt, false);
    u.add("target", target, m * 8, false), u.add("lse", lse, m * 4, false), u.add("dloss", dloss, m * 4, false);
    u.add("dX", dX, true), u.add("dW", dW, true), u.workspace(workspace, workspace_bytes);
    CHECKED(u.check());
    if (k == 0) return COSTA_SUCCESS;  // no gradient has elements
    // alpha G B^^T or alpha G^T B^^T + be C, of G (gm x gn); by: a factor in device memory (null: none)
    auto product = [&](bool turned, const void* g, bool bf16, int64_t gm, int64_t gn, const MxView& b, float be, void* c,
                       int64_t ld, costa_real type, char* room, size_t bytes, const float* by) {
      ProductArgs p{};
      p.m = turned ? gn : gm, p.k = turned ? gm : gn, p.n = b.rows;
      p.real = g;
      p.a_rs = turned ? 1 : gn, p.a_cs = turned ? gn : 1;
      p.a_type = bf16 ? COSTA_REAL_BF16 : COSTA_REAL_F32;
      p.b = b;
      p.c = c, p.c_rs = ld, p.c_cs = 1, p.c_type = type;
      p.alpha = alpha, p.beta = be;
      p.workspace = reinterpret_cast<float*>(room), p.workspace_bytes = bytes;
      return p.m == 0 || p.n == 0 ? hipSuccess : by ? launch_mx_loss_dw(p, by, stream) : launch_mx_product(p, stream);
    };
    if (m == 0 || n == 0) {  // sums over nothing
      if (dX) HIP_OR_FAIL(product(false, nullptr, true, m, 0, columns_of(wt, 0, 0), 0.0f, dX->data, dX->ld, dX->type, nullptr, 0, nullptr));
      if (dW) HIP_OR_FAIL(product(true, nullptr, true, 0, n, columns_of(xt, 0, 0), beta, dW->data, dW->ld, dW->type, nullptr, 0, nullptr));
      return COSTA_SUCCESS;
    }
    char* room = static_cast<char*>(workspace);
    float* const sum = reinterpret_cast<float*>(room);  // of dX
    room += up16((size_t)m * k * 4);
    float* const factor = reinterpret_cast<float*>(room);  // of G's rows
    room += up16((size_t)m * 4);
    size_t left = workspace_bytes - up16((size_t)m * k * 4) - up16((size_t)m * 4);
    // half for G, half for the logits, where they are kept, and for what products split
    const size_t half = std::min(left / 32 * 16, up16(piece_bytes(m, n, 4)));
    const bool bf16 = (!dX || dX->type == COSTA_REAL_BF16) && (!dW || dW->type == COSTA_REAL_BF16) &&
                      (!dW || bf16_with_dw(X->type, w.bits, xt.bits, m, n, k));
    int64_t per = piece_columns(m, n, half, 2);
    bool fused = mx_loss_fused(X->type, w.bits, m, per, k);
    if (!bf16 || !fused) {
      per = piece_columns(m, n, half, 4);
      fused = mx_loss_fused(X->type, w.bits, m, per, k);
    }
    if (bf16 && dW) HIP_OR_FAIL(launch_mx_loss_scale(m, n, target, dloss, factor, stream));
    else if (bf16) HIP_OR_FAIL(launch_mx_loss_factors(logits_of(X, w, 0, n, alpha), target, lse, dloss, factor, stream));
    const float* const by = bf16 ? factor : nullptr;
    void* const g = room;
    const size_t taken = up16((size_t)m * per * (fused && bf16 ? 2 : 4));
    room += taken, left -= taken;
    const bool whole = per >= n;
    for (int64_t j = 0; j < n; j += per) {
      const int64_t cols = std::min(per, n - j);
      ProductArgs p = logits_of(X, w, j, cols, alpha);
      if (fused) {
        HIP_OR_FAIL(launch_mx_loss_grad_tiles(p, n, j, target, lse, dloss, by, g, bf16, stream));
      } else {
        p.workspace = reinterpret_cast<float*>(room), p.workspace_bytes = left;
        LogitsPart l{m, cols, j, p.workspace, 0, alpha, target};
        HIP_OR_FAIL(launch_mx_product_parts(p, l.splits, stream));
        HIP_OR_FAIL(launch_mx_loss_grad(l, n, lse, dloss, by, g, bf16, stream));
      }
      if (dX) {
        const bool direct = !bf16 && (whole || dX->type == COSTA_REAL_F32);
        HIP_OR_FAIL(product(false, g, bf16, m, cols, columns_of(wt, j, cols), j > 0 ? 1.0f : 0.0f,
                            direct ? dX->data : sum, direct ? dX->ld : k, direct ? dX->type : COSTA_REAL_F32, room, left,
                            nullptr));
      }
      if (dW)
        HIP_OR_FAIL(product(true, g, bf16, m, cols, xt, beta,
                            static_cast<char*>(dW->data) + j * dW->ld * real_size(dW->type), dW->ld, dW->type, room, left, by));
    }
    if (dX && (bf16 || (!whole && dX->type != COSTA_REAL_F32)))
      HIP_OR_FAIL(launch_mx_round(m, k, sum, by, rows_of(dX), dX->type, stream));
    return COSTA_SUCCESS;
  });
}
