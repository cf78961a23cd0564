// C ABI entry points of the microscaled matrices (include/costa_mx.h): argument
// checks, the tables of distributed layouts, launches.
#include <algorithm>
#include <climits>
#include <initializer_list>
#include <map>
#include <memory>
#include <mutex>
#include <string>
#include <vector>

#include "mx.hpp"
#include "plan.hpp"
#include "spans.hpp"

namespace costa {
namespace {

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

int real_size(costa_real t) {
  switch (t) {
    case COSTA_REAL_F64: return 8;
    case COSTA_REAL_F32: return 4;
    case COSTA_REAL_BF16:
    case COSTA_REAL_F16: return 2;
    default: return 0;  // not an element type
  }
}

costa_status check_dims(const char* what, int64_t rows, int64_t cols) {
  if (rows < 0 || cols < 0) return fail(COSTA_ERROR_INVALID_VALUE, std::string(what) + ": negative dimension");
  if (rows > INT32_MAX || cols > INT32_MAX)
    return fail(COSTA_ERROR_NOT_SUPPORTED, std::string(what) + ": dimension above 2^31-1");
  return COSTA_SUCCESS;
}

costa_status check_mx(const char* what, const costa_mx* q, MxView& v) {
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

costa_status check_matrix(const char* what, const costa_matrix* a, bool f64) {
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
Span span_of(const costa_matrix& a) {
  if (a.rows == 0 || a.cols == 0) return Span{0, 0, 0, 0};
  const int64_t es = real_size(a.type), line = a.order == COSTA_COL_MAJOR ? a.rows : a.cols;
  return Span{(uintptr_t)a.data, line * es, a.ld * es, a.order == COSTA_COL_MAJOR ? a.cols : a.rows};
}
Span span_of(const void* p, int64_t bytes) { return Span{(uintptr_t)p, p ? bytes : 0, bytes, 1}; }
Span data_of(const MxView& q) { return span_of(q.data, q.rows * q.row_bytes); }
Span scales_of(const MxView& q) { return span_of(q.scales, q.rows * q.row_scales); }

// INVALID_VALUE where two of the buffers have a byte in common, `what` they are.
costa_status check_apart(const char* what, std::initializer_list<Span> one, std::initializer_list<Span> other) {
  for (const Span& x : one)
    for (const Span& y : other)
      if (spans_meet(x, y)) return fail(COSTA_ERROR_INVALID_VALUE, what);
  return COSTA_SUCCESS;
}

// Q and QT of a rows x cols source; at least one of them.
costa_status check_outputs(int64_t rows, int64_t cols, const costa_mx* Q, const costa_mx* QT, MxView& q, MxView& qt) {
  if (!Q && !QT) return fail(COSTA_ERROR_INVALID_VALUE, "neither Q nor QT");
  q = MxView{};
  qt = MxView{};
  if (Q) {
    CHECKED(check_mx("Q", Q, q));
    if (Q->rows != rows || Q->cols != cols) return fail(COSTA_ERROR_SHAPE_MISMATCH, "Q is not the shape of B");
  }
  if (QT) {
    CHECKED(check_mx("QT", QT, qt));
    if (QT->rows != cols || QT->cols != rows)
      return fail(COSTA_ERROR_SHAPE_MISMATCH, "QT is not the shape of the transposed B");
  }
  CHECKED(check_apart("Q overlaps itself", {data_of(q)}, {scales_of(q)}));
  CHECKED(check_apart("QT overlaps itself", {data_of(qt)}, {scales_of(qt)}));
  return check_apart("Q overlaps QT", {data_of(q), scales_of(q)}, {data_of(qt), scales_of(qt)});
}

// ---------------------------------------------------------------------------
// tables of layouts
// ---------------------------------------------------------------------------
constexpr int64_t kMxCellsMax = (int64_t)1 << 22;
constexpr size_t kMxTablesMax = 64;

struct LayoutTables {
  void* dev = nullptr;
  MxLayoutArgs args{};
  std::vector<int32_t> rank;  // (HostTables::rank)
  bool captured = false;  // a graph reads them: kept until costa_finalize
  ~LayoutTables() {
    if (dev) (void)hipFree(dev);
  }
};

struct TableState {
  std::mutex mu;
  std::map<std::pair<int, uint64_t>, std::unique_ptr<LayoutTables>> tables;  // (device, layout id)
};
TableState& table_state() {
  static TableState* s = new TableState();
  return *s;
}

// The host side of a layout's tables, by its lines (columns of a column-major
// layout, rows of a row-major one): [0] lines, [1] places.
struct HostTables {
  std::vector<int64_t> start[2];
  MxSplits splits[2] = {};
  std::vector<MxCell> cells;
  std::vector<int32_t> rank;  // of each cell of a block-cyclic layout
  int32_t nplace = 0;
};

void fill_tables(const Layout& L, HostTables& h) {
  const bool col = L.order == COSTA_COL_MAJOR;
  const int row = col ? 1 : 0;  // which of the two the rows are
  if (L.block_cyclic) {
    // the local matrix of a process: classes are process rows and columns
    auto narrow = [](int64_t off, int64_t n) { return off <= (int64_t)UINT32_MAX - 1 - n ? 1 : 0; };
    h.splits[row] = MxSplits{nullptr, 0, L.prow, L.rsrc, L.r0, L.mb, narrow(L.r0, L.nrows)};
    h.splits[1 - row] = MxSplits{nullptr, 0, L.pcol, L.csrc, L.c0, L.nb, narrow(L.c0, L.ncols)};
    const int32_t nline = col ? L.pcol : L.prow;
    h.nplace = col ? L.prow : L.pcol;
    h.cells.resize((size_t)nline * h.nplace);
    h.rank.resize(h.cells.size());
    for (int32_t pr = 0; pr < L.prow; ++pr)
      for (int32_t pc = 0; pc < L.pcol; ++pc) {
        const int64_t ext = col ? L.lrows[pr] : L.lcols[pc];
        const size_t at = (size_t)(col ? pc : pr) * h.nplace + (col ? pr : pc);
        h.cells[at] = MxCell{0, L.lld ? L.lld : std::max<int64_t>(ext, 1), (int64_t)at};
        h.rank[at] = L.rank_at(pr, pc);
      }
    return;
  }
  h.start[row] = L.rsplit;
  h.start[1 - row] = L.csplit;
  const int32_t nline = col ? L.nbc : L.nbr;
  h.nplace = col ? L.nbr : L.nbc;
  h.cells.resize((size_t)nline * h.nplace);
  for (int32_t bi = 0; bi < L.nbr; ++bi)
    for (int32_t bj = 0; bj < L.nbc; ++bj) {
      const int64_t b = L.block(bi, bj);
      h.cells[(size_t)(col ? bj : bi) * h.nplace + (col ? bi : bj)] = MxCell{L.boff[b], L.bld[b], L.owner[b]};
    }
  for (int s = 0; s < 2; ++s) h.splits[s] = MxSplits{nullptr, (int32_t)h.start[s].size() - 1, 0, 0, 0, 0, 0};
}

// The device tables of a layout; uploaded on the first call.  The caller holds T.mu
// until the kernel that reads them is enqueued: a call that starts the tables over
// waits for kernels that are, not for one that is yet to be.
// `p` holds the ranks' buffers and gets them in the order that the kernel looks them up.
costa_status layout_tables(TableState& T, const Layout& L, hipStream_t stream, MxLayoutArgs& out, MxPointers& p) {
  int device = 0;
  HIP_OR_FAIL(hipGetDevice(&device));
  hipStreamCaptureStatus cs = hipStreamCaptureStatusNone;
  bool capturing = false;
  if (hipStreamIsCapturing(stream, &cs) == hipSuccess) capturing = cs == hipStreamCaptureStatusActive;
  else (void)hipGetLastError();  // the null stream, while another stream captures
  const std::pair<int, uint64_t> key(device, L.id);
  auto it = T.tables.find(key);
  if (it == T.tables.end()) {
    if (capturing)
      return fail(COSTA_ERROR_NOT_SUPPORTED, "the first quantise call of a layout uploads its tables: call it once "
                                             "before the stream captures");
    HostTables h;
    fill_tables(L, h);
    if (T.tables.size() >= kMxTablesMax) {
      HIP_OR_FAIL(hipDeviceSynchronize());
      for (auto k = T.tables.begin(); k != T.tables.end();) k = k->second->captured ? std::next(k) : T.tables.erase(k);
    }
    std::vector<unsigned char> all;
    auto put = [&](const void* p, size_t n) {
      const size_t at = all.size();
      all.resize(at + (n + 15) / 16 * 16);
      if (n) std::copy_n(static_cast<const unsigned char*>(p), n, all.data() + at);
      return at;
    };
    size_t at_start[2];
    for (int s = 0; s < 2; ++s) at_start[s] = put(h.start[s].data(), h.start[s].size() * sizeof(int64_t));
    const size_t at_cells = put(h.cells.data(), h.cells.size() * sizeof(MxCell));
    std::unique_ptr<LayoutTables> t(new LayoutTables());
    if (hipMalloc(&t->dev, all.size()) != hipSuccess) {
      (void)hipGetLastError();
      t->dev = nullptr;
      return fail(COSTA_ERROR_OUT_OF_MEMORY, "cannot allocate the layout's tables");
    }
    HIP_OR_FAIL(hipMemcpy(t->dev, all.data(), all.size(), hipMemcpyHostToDevice));
    const unsigned char* d = static_cast<const unsigned char*>(t->dev);
    for (int s = 0; s < 2; ++s)
      if (!h.start[s].empty()) h.splits[s].start = reinterpret_cast<const int64_t*>(d + at_start[s]);
    t->args = MxLayoutArgs{h.splits[0], h.splits[1], reinterpret_cast<const MxCell*>(d + at_cells), h.nplace,
                           L.block_cyclic ? 1 : 0};
    t->rank = std::move(h.rank);
    it = T.tables.emplace(key, std::move(t)).first;
  }
  if (capturing) it->second->captured = true;
  out = it->second->args;
  if (out.dealt) {  // (at most as many cells as ranks)
    const MxPointers by_rank = p;
    for (size_t c = 0; c < it->second->rank.size(); ++c) p.p[c] = by_rank.p[it->second->rank[c]];
  }
  return COSTA_SUCCESS;
}

// The part of a product's checks and arguments that both entry points share.
costa_status product_common(std::initializer_list<Span> a, int64_t m, int64_t k, const costa_mx* B, const costa_matrix* C, float alpha, float beta,
                            void* workspace, size_t workspace_bytes, ProductArgs& p) {
  CHECKED(check_mx("B", B, p.b));
  CHECKED(check_matrix("C", C, false));
  if (B->cols != k) return fail(COSTA_ERROR_SHAPE_MISMATCH, "A and B have different lengths to sum over");
  if (C->rows != m || C->cols != B->rows) return fail(COSTA_ERROR_SHAPE_MISMATCH, "C is not the shape of A B^T");
  if (workspace && (uintptr_t)workspace % 16 != 0)
    return fail(COSTA_ERROR_INVALID_VALUE, "the workspace is not 16-byte aligned");
  const Span c = span_of(*C), w = span_of(workspace, (int64_t)std::min(workspace_bytes, (size_t)INT64_MAX));
  CHECKED(check_apart("C overlaps B", {c}, {data_of(p.b), scales_of(p.b)}));
  CHECKED(check_apart("C overlaps the workspace", {c}, {w}));
  CHECKED(check_apart("B overlaps the workspace", {w}, {data_of(p.b), scales_of(p.b)}));
  CHECKED(check_apart("C overlaps A", {c}, a));
  CHECKED(check_apart("A overlaps the workspace", {w}, a));
  p.m = m;
  p.n = B->rows;
  p.k = k;
  p.c = C->data;
  p.c_rs = C->order == COSTA_ROW_MAJOR ? C->ld : 1;
  p.c_cs = C->order == COSTA_ROW_MAJOR ? 1 : C->ld;
  p.c_type = C->type;
  p.alpha = alpha;
  p.beta = beta;
  p.workspace = static_cast<float*>(workspace);
  p.workspace_bytes = workspace ? workspace_bytes : 0;
  return COSTA_SUCCESS;
}

}  // namespace

void release_mx_tables() {
  TableState& T = table_state();
  std::lock_guard<std::mutex> lock(T.mu);
  T.tables.clear();  // hipFree waits for the kernels that read them
}

}  // namespace costa

using namespace costa;

extern "C" costa_status costa_mx_sizes(costa_mx_format format, int64_t rows, int64_t cols, int64_t* data_bytes,
                                       int64_t* scale_bytes) {
  return guarded([&]() -> costa_status {
    if (!data_bytes || !scale_bytes) return fail(COSTA_ERROR_INVALID_VALUE, "null argument");
    if (format != COSTA_MX_E2M1 && format != COSTA_MX_E4M3)
      return fail(COSTA_ERROR_INVALID_VALUE, "unknown element format");
    CHECKED(check_dims("matrix", rows, cols));
    *data_bytes = rows * mx_row_bytes(format, cols);
    *scale_bytes = rows * (mx_padded_cols(format, cols) / kMxBlock);
    return COSTA_SUCCESS;
  });
}

extern "C" costa_status costa_mx_quantize(float alpha, const costa_matrix* B, const costa_mx* Q, const costa_mx* QT,
                                          hipStream_t stream) {
  return guarded([&]() -> costa_status {
    CHECKED(check_matrix("B", B, true));
    QuantArgs a{};
    MxView q, qt;
    CHECKED(check_outputs(B->rows, B->cols, Q, QT, q, qt));
    CHECKED(check_apart("B overlaps Q", {span_of(*B)}, {data_of(q), scales_of(q)}));
    CHECKED(check_apart("B overlaps QT", {span_of(*B)}, {data_of(qt), scales_of(qt)}));
    if (B->rows == 0 || B->cols == 0) return COSTA_SUCCESS;
    const bool row = B->order == COSTA_ROW_MAJOR;
    a.lines = row ? B->rows : B->cols;
    a.len = row ? B->cols : B->rows;
    a.src = B->data;
    a.ld = B->ld;
    a.type = B->type;
    a.alpha = alpha;
    a.along = row ? q : qt;
    a.across = row ? qt : q;
    HIP_OR_FAIL(launch_mx_quantize(a, stream));
    return COSTA_SUCCESS;
  });
}

extern "C" costa_status costa_mx_quantize_layout(costa_real type, float alpha, costa_layout B,
                                                 const void* const* B_local, const costa_mx* Q, const costa_mx* QT,
                                                 hipStream_t stream) {
  return guarded([&]() -> costa_status {
    const Layout* L = layout_of(B);
    if (!L) return fail(COSTA_ERROR_INVALID_VALUE, "null layout");
    const int es = real_size(type);
    if (!es) return fail(COSTA_ERROR_INVALID_VALUE, "unknown element type");
    if (!B_local) return fail(COSTA_ERROR_INVALID_VALUE, "null buffer array");
    CHECKED(check_dims("B", L->nrows, L->ncols));
    QuantArgs a{};
    MxView q, qt;
    CHECKED(check_outputs(L->nrows, L->ncols, Q, QT, q, qt));
    if (L->nranks > kMxRanksMax) return fail(COSTA_ERROR_NOT_SUPPORTED, "more than 256 ranks");
    if (!L->block_cyclic && (int64_t)L->nbr * L->nbc > kMxCellsMax)
      return fail(COSTA_ERROR_NOT_SUPPORTED, "more than 2^22 blocks");
    MxPointers p{};
    for (int32_t r = 0; r < L->nranks; ++r) {
      if (L->local_elems[r] == 0) continue;
      if (!B_local[r]) return fail(COSTA_ERROR_INVALID_VALUE, "null B buffer for a rank that holds data");
      if ((uintptr_t)B_local[r] % es != 0)
        return fail(COSTA_ERROR_INVALID_VALUE, "a B buffer is not aligned to its element type");
      p.p[r] = B_local[r];
    }
    if (L->nrows == 0 || L->ncols == 0) return COSTA_SUCCESS;
    const bool row = L->order == COSTA_ROW_MAJOR;
    a.lines = row ? L->nrows : L->ncols;
    a.len = row ? L->ncols : L->nrows;
    a.type = type;
    a.alpha = alpha;
    a.along = row ? q : qt;
    a.across = row ? qt : q;
    if (L->nbr == 1 && L->nbc == 1) {  // one block: a plain matrix
      const int32_t r = L->owner_of(0, 0);
      a.src = static_cast<const char*>(p.p[r]) + L->offset_of(0, 0) * es;
      a.ld = L->ld_of(0, 0);
      HIP_OR_FAIL(launch_mx_quantize(a, stream));
      return COSTA_SUCCESS;
    }
    MxLayoutArgs l{};
    TableState& T = table_state();
    std::lock_guard<std::mutex> lock(T.mu);
    CHECKED(layout_tables(T, *L, stream, l, p));
    HIP_OR_FAIL(launch_mx_quantize_layout(a, l, p, stream));
    return COSTA_SUCCESS;
  });
}

extern "C" costa_status costa_mx_dequantize(float alpha, const costa_mx* Q, float beta, const costa_matrix* A,
                                            hipStream_t stream) {
  return guarded([&]() -> costa_status {
    DequantArgs d{};
    CHECKED(check_mx("Q", Q, d.q));
    CHECKED(check_matrix("A", A, true));
    if (A->rows != Q->rows || A->cols != Q->cols) return fail(COSTA_ERROR_SHAPE_MISMATCH, "A is not the shape of Q");
    CHECKED(check_apart("A overlaps Q", {span_of(*A)}, {data_of(d.q), scales_of(d.q)}));
    if (A->rows == 0 || A->cols == 0) return COSTA_SUCCESS;
    d.dst = A->data;
    d.rs = A->order == COSTA_ROW_MAJOR ? A->ld : 1;
    d.cs = A->order == COSTA_ROW_MAJOR ? 1 : A->ld;
    d.type = A->type;
    d.alpha = alpha;
    d.beta = beta;
    HIP_OR_FAIL(launch_mx_dequantize(d, stream));
    return COSTA_SUCCESS;
  });
}

extern "C" costa_status costa_mx_product(float alpha, const costa_mx* A, const costa_mx* B, float beta,
                                         const costa_matrix* C, void* workspace, size_t workspace_bytes,
                                         hipStream_t stream) {
  return guarded([&]() -> costa_status {
    ProductArgs p{};
    CHECKED(check_mx("A", A, p.amx));
    CHECKED(product_common({data_of(p.amx), scales_of(p.amx)}, A->rows, A->cols, B, C, alpha, beta, workspace,
                           workspace_bytes, p));
    if (p.m == 0 || p.n == 0) return COSTA_SUCCESS;
    HIP_OR_FAIL(launch_mx_product(p, stream));
    return COSTA_SUCCESS;
  });
}

extern "C" costa_status costa_mx_product_real(float alpha, costa_op op, const costa_matrix* A, const costa_mx* B,
                                              float beta, const costa_matrix* C, void* workspace,
                                              size_t workspace_bytes, hipStream_t stream) {
  return guarded([&]() -> costa_status {
    ProductArgs p{};
    if (op != COSTA_OP_N && op != COSTA_OP_T && op != COSTA_OP_C) return fail(COSTA_ERROR_INVALID_VALUE, "unknown op");
    CHECKED(check_matrix("A", A, false));
    const bool tr = op != COSTA_OP_N;
    CHECKED(product_common({span_of(*A)}, tr ? A->cols : A->rows, tr ? A->rows : A->cols, B, C, alpha, beta, workspace,
                           workspace_bytes, p));
    if (p.m == 0 || p.n == 0) return COSTA_SUCCESS;
    const int64_t rs = A->order == COSTA_ROW_MAJOR ? A->ld : 1, cs = A->order == COSTA_ROW_MAJOR ? 1 : A->ld;
    p.real = A->data;
    p.a_rs = tr ? cs : rs;
    p.a_cs = tr ? rs : cs;
    p.a_type = A->type;
    HIP_OR_FAIL(launch_mx_product(p, stream));
    return COSTA_SUCCESS;
  });
}

extern "C" costa_status costa_mx_workspace(int64_t m, int64_t n, int64_t k, size_t* bytes) {
  return guarded([&]() -> costa_status {
    if (!bytes) return fail(COSTA_ERROR_INVALID_VALUE, "null argument");
    CHECKED(check_dims("C", m, n));
    CHECKED(check_dims("A", m, k));
    *bytes = mx_product_workspace(m, n, k);
    return COSTA_SUCCESS;
  });
}
