// The operators around the products of a layer: what the host code and the kernels share.
#pragma once

#include "../../include/costa_layer.h"
#include "mx.hpp"

namespace costa {

typedef uint32_t v4u __attribute__((ext_vector_type(4)));

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
  float* parts;  // m x rank floats each
  int64_t most;  // parts that there is room for
};
// s v as operands of the matrix instructions, three bfloat16 parts: of sixteen rows and 32 ranks, 64 lanes' 16
// bytes of each part (lane l: row l % 16, eight ranks from 8 (l / 16) on).
inline size_t mx_spread_bytes(int64_t m, int rank) { return (size_t)((m + 15) / 16) * ((rank + 31) / 32) * 3 * 1024; }
hipError_t launch_mx_adapter_spread(const AdapterDotsArgs& a, int64_t splits, void* spread, hipStream_t stream);
// Parts of v that a call can use.
int64_t mx_adapter_dots_parts(int64_t m, int64_t k, int rank);
// splits: parts of v that are left to be added (0: v is there).
hipError_t launch_mx_adapter_dots(const AdapterDotsArgs& a, int64_t& splits, hipStream_t stream);
hipError_t launch_mx_adapter_dots_join(const AdapterDotsArgs& a, int64_t splits, hipStream_t stream);

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
  const v4u* spread;
};
hipError_t launch_mx_adapter_add(const AdapterAddArgs& a, hipStream_t stream);
// The same in the product's own kernel, from x (m x k) and w, where that takes one (mx_tiles_adapted.hip).
bool mx_adapted_fused(costa_real type, int bits, int64_t m, int64_t n, int64_t k);
hipError_t launch_mx_adapted_product(const AdapterAddArgs& a, const RowsView& x, int64_t k, const MxView& w,
                                     hipStream_t stream);

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

// ---- loss (mx_loss.hip) -----------------------------------------------------------
// Largest logit and the sum of exponentials from it, of a row's columns of one chunk:
// stats[chunk * m + row].
struct LossStat {
  float top, sum;
};
constexpr int64_t kLossChunk = 2048;  // columns of a chunk where logits are in memory

// The logits of columns col0 .. col0 + n - 1: alpha * the sum of `splits` parts of m x n floats.
struct LogitsPart {
  int64_t m, n, col0;
  const float* sums;
  int32_t splits;
  float alpha;
  const int64_t* target;
};
// stats: of col0's chunk; at: the target's logits, of rows whose target is among the columns.
hipError_t launch_mx_loss_stats(const LogitsPart& p, LossStat* stats, float* at, hipStream_t stream);
// From the stats of all chunks.  n: the vocabulary.
hipError_t launch_mx_loss_join(int64_t m, int64_t n, int64_t chunks, const LossStat* stats, const float* at,
                               const int64_t* target, float* loss, float* lse, hipStream_t stream);
// g (m x p.n by rows; bfloat16 or float; apart from the sums) <- dloss (exp(logit - lse) - [target]) / factor (null: 1)
hipError_t launch_mx_loss_grad(const LogitsPart& p, int64_t vocabulary, const float* lse, const float* dloss,
                               const float* factor, void* g, bool bf16, hipStream_t stream);
// Both in the product's own kernel (mx_tiles_loss.hip), where that takes one: statistics by mx_loss_tile_chunks() chunks of
// columns; of the arguments C, beta and the workspace are not looked at.
bool mx_loss_fused(costa_real type, int bits, int64_t m, int64_t n, int64_t k);
int64_t mx_loss_tile_chunks(costa_real type, int bits, int64_t m, int64_t n, int64_t k);
hipError_t launch_mx_loss_tiles(const ProductArgs& x, const int64_t* target, LossStat* stats, float* at,
                                hipStream_t stream);
hipError_t launch_mx_loss_grad_tiles(const ProductArgs& x, int64_t vocabulary, int64_t col0, const int64_t* target,
                                     const float* lse, const float* dloss, const float* factor, void* g, bool bf16,
                                     hipStream_t stream);
// What the rows of a G in bfloat16 are divided by, and its products are multiplied by, in 32 bits: m floats.
//
// For dX alone, whose rows can each have a factor of their own: |dloss| (1 - p), p the target's probability (at least
// 2^-24 |dloss|; 1 where that is 0 or not finite, and in rows that do not count).  The target's element is then -1
// and loses nothing to its rounding, and with it goes nearly all of the error: the others' roundings are as
// large of each, but theirs are many and small.  (4096 rows of 4096 over 65536 words: dX 1.97e-3 off 64 bits with one
// factor for all rows; so 1.7e-3, which are dX's own rounding, as with a G in 32 bits.)
// (What the rounding is for: dX of 4096 rows of 4096 over 32768 words in 4 bits takes 1.9 ms, 3.5 with a G in 32 bits, whose
// three parts each cost a matrix instruction; dX and dW 2.9 and 6.4.)
hipError_t launch_mx_loss_factors(const ProductArgs& x, const int64_t* target, const float* lse, const float* dloss,
                                  float* factor, hipStream_t stream);
// For dW, which sums over the rows, the same for all: the largest |dloss| of rows that count (1 where that is 0 or
// not finite, and without dloss).  (Where all of them are equal, as in a mean, the target's element of an unsure
// row, nearly -1, loses little to its rounding; rounded as a part of 1/3686 all of them were 1.6e-3
// off, in the same direction.)
hipError_t launch_mx_loss_scale(int64_t m, int64_t n, const int64_t* target, const float* dloss, float* factor,
                                hipStream_t stream);
// The gradient of the vocabulary's weights from a G in bfloat16, with the rows' common factor out of device
// memory: C <- alpha *factor G^T B^^T + beta C, where the products' tiles take it (G m x n by rows, n rows of C).
bool mx_loss_dw_fused(int bits, int64_t m, int64_t n, int64_t k);
hipError_t launch_mx_loss_dw(const ProductArgs& a, const float* factor, hipStream_t stream);
// y <- x times its row's factor (null: x): floats, to a row-major matrix
hipError_t launch_mx_round(int64_t m, int64_t n, const float* x, const float* factor, const RowsView& y, costa_real type,
                           hipStream_t stream);

}  // namespace costa
