/*
 * costa_layer.h -- what stands around the products of a layer whose weights are
 * kept in few bits (costa_mx.h): the norm that makes a product's operand, low-rank
 * adapters beside a product, and the loss behind the last one; each with its
 * gradients.
 *
 * Conventions are those of costa_mx.h: calls are asynchronous on `stream`, on the
 * current device; every argument error is returned before anything is enqueued; the
 * caller owns every buffer; no call allocates device memory, and all of them can be
 * captured.  Plain matrices here are ROW_MAJOR (NOT_SUPPORTED else), of F32, BF16 or
 * F16; vectors of floats and integers are aligned to their elements.  No output may
 * overlap an input, another output or the workspace, but where a call says so.
 * Arithmetic is in 32 bits or more, every result rounded once to its type; no atomics:
 * the same call gives the same bits.
 *
 * Workspaces: device memory, 16-byte aligned, its contents neither needed nor kept.
 * The functions *_workspace say what a call has to have (`least`: with less it is
 * refused, INVALID_VALUE) and what it can use (`most`); either pointer may be NULL.  In
 * between, sums in 32 bits are split and ordered otherwise and a call is slower: results differ by
 * those sums' roundings, no operand is held in fewer bits.
 */
#ifndef COSTA_LAYER_H
#define COSTA_LAYER_H

#include "costa_mx.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- root-mean-square norm -------------------------------------------------
 *
 *     h = x + r                     (r: the residual; without R: h = x)
 *     s = 1 / sqrt(mean(h^2) + eps)           of each row
 *     y = h s w                               (without W: w = 1)
 *
 * H <- h, Y <- y, Q <- mx(y) (the operand of the products behind it), rstd <- s;
 * each may be NULL, not all.  X, R, H, Y: rows x cols of one type; W: 1 x cols of
 * that type or F32; rstd: `rows` floats.  h goes on in 32 bits, y is not made of the
 * rounded one; squares are summed in 64 bits (no h is too large or too small).  H may be
 * X or R itself (the same matrix: data, ld and type).  eps: at least 2^-126, finite.
 * Without columns there is no mean: nothing is written, rstd neither. */
costa_status costa_mx_norm(float eps, const costa_matrix* X, const costa_matrix* W, const costa_matrix* R,
                           const costa_matrix* H, const costa_matrix* Y, const costa_mx* Q, float* rstd,
                           hipStream_t stream);

/* The gradients, from that of y (through Q unchanged), H and rstd of costa_mx_norm():
 *
 *     u = h s,  g = dy w,  dx = s (g - u mean(g u)) + dh         (the gradient of x and of r)
 *     dw = sum over the rows of dy u
 *
 * dH (NULL: none): the gradient that reaches h past the norm.  dY, H, dH, dX: rows x cols
 * of one type; W as above, NULL: ones; dW: 1 x cols of that type or F32, NULL: not
 * wanted.  dX may be dY or dH itself.  The workspace is for dW's parts. */
costa_status costa_mx_norm_backward(const costa_matrix* dY, const costa_matrix* H, const costa_matrix* W,
                                    const float* rstd, const costa_matrix* dH, const costa_matrix* dX,
                                    const costa_matrix* dW, void* workspace, size_t workspace_bytes,
                                    hipStream_t stream);

/* Workspace of costa_mx_norm_backward() with dW (without: none). */
costa_status costa_mx_norm_workspace(int64_t rows, int64_t cols, size_t* least, size_t* most);

/* ---- low-rank adapters beside a product ------------------------------------
 * `count` adapters of up to `rank` (at most 256): rows a*rank .. of A (count*rank x k)
 * and of B (count*rank x n) are those of adapter a, both kept rank by rank: B is
 * the transpose of the usual n x rank matrix, so that the two change places in the backward
 * pass.  ranks (device memory, `count` entries; NULL: all of them `rank`): how many of its
 * rows an adapter has (taken into 0 .. rank); what stands past them has no effect.  scales (device
 * memory, `count`; NULL: 1): s below. */
typedef struct {
  int32_t count, rank;
  const costa_matrix* A;
  const costa_matrix* B;
  const int32_t* ranks;
  const float* scales;
} costa_mx_adapters;

/* C <- alpha X W^^T + s V B + beta C, row i with the adapter a = index[i]: V = X A_a^T.
 * X m x k, W n x k, C m x n; A, B of X's type; index: m entries, in any order; a row whose
 * entry is not in 0 .. count-1 has no adapter.  V (NULL: not wanted): m x rank of F32, the
 * rows' products, 0 past their adapter's rank; what the gradients below need.  An
 * infinity or a NaN of one adapter reaches its own rows alone (where an infinity may come out
 * as NaN).  beta == 0: C is not read.
 *
 * The gradient of X is this call with dY in X's place, mx(W^T) in W's, and A and B swapped;
 * its V is dY B_a^T. */
costa_status costa_mx_product_adapted(float alpha, const costa_matrix* X, const costa_mx* W,
                                      const costa_mx_adapters* adapters, const int32_t* index, float beta,
                                      const costa_matrix* C, const costa_matrix* V, void* workspace,
                                      size_t workspace_bytes, hipStream_t stream);
costa_status costa_mx_adapted_workspace(int64_t m, int64_t n, int64_t k, int32_t rank, size_t* least, size_t* most);

/* G_a <- s_a sum over the rows i of adapter a of V_i^T Z_i + beta G_a: with (V, Z) = (dY B^T, X)
 * the gradient of A, with (X A^T, dY) that of B.  V m x rank of F32, Z m x len, G (count*rank) x
 * len of any type here.  Of `adapters` A and B are not looked at (NULL allowed).  Rows past an
 * adapter's rank, and adapters without rows, get beta G (0 for beta == 0: G is not read then). */
costa_status costa_mx_adapter_gradient(const costa_mx_adapters* adapters, const int32_t* index,
                                       const costa_matrix* V, const costa_matrix* Z, float beta,
                                       const costa_matrix* G, void* workspace, size_t workspace_bytes,
                                       hipStream_t stream);
costa_status costa_mx_adapter_gradient_workspace(int64_t m, int64_t len, int32_t count, int32_t rank, size_t* least,
                                                 size_t* most);

/* ---- softmax cross entropy over a vocabulary -------------------------------
 *
 *     L = alpha X W^^T,  lse_i = log sum_j exp(L_ij),  loss_i = lse_i - L_i,target(i)
 *
 * X m x k, W n x k (n: the vocabulary), target, loss, lse: m entries.  A row whose target
 * is not in 0 .. n-1 does not count: its loss is 0.  A logit that is NaN or +infinity makes its
 * row's lse NaN.  L is not kept. */
costa_status costa_mx_loss(float alpha, const costa_matrix* X, const costa_mx* W, const int64_t* target, float* loss,
                           float* lse, void* workspace, size_t workspace_bytes, hipStream_t stream);

/* The gradients, by pieces of the vocabulary:
 *
 *     G_ij = dloss_i (exp(L_ij - lse_i) - [j = target(i)]),  0 in rows that do not count
 *     dX <- alpha G W'^          W' = WT^T, WT = mx(W^T), k x n
 *     dW <- alpha G^T X'^ + beta dW    X' = XT^T, XT = mx(X^T), k x m
 *
 * dloss (NULL: ones): m floats, the gradient that reaches each row's loss.  dX with WT and dW
 * with XT may be NULL, not both.  lse: what costa_mx_loss() gave.  Probabilities below 2^-126 are 0.  lse is one
 * float: its rounding, up to 2^-24 |lse|, is a factor exp(that) of all of a row's probabilities, and an error as large
 * of the target's element p - 1, which of a row that is sure up to about that much keeps no digit (the row's loss
 * does: it is not made from lse).
 * G is held in 32 bits, or, where dX and dW (those wanted) are BF16, in bfloat16: for dX alone a row as a part
 * of |dloss| (1 - p), p the target's probability, so that the target's element is -1 and rounds to itself; with
 * dW (where m, n and k are large enough for whole tiles of both products, whatever the workspace) as a part of
 * the largest |dloss| of rows that count.  The factors are in 32 bits and go back in before dX and dW are rounded. */
costa_status costa_mx_loss_backward(float alpha, const costa_matrix* X, const costa_mx* W, const int64_t* target,
                                    const float* lse, const float* dloss, const costa_mx* WT, const costa_matrix* dX,
                                    const costa_mx* XT, float beta, const costa_matrix* dW, void* workspace,
                                    size_t workspace_bytes, hipStream_t stream);

/* Workspace of costa_mx_loss() (backward == 0) and costa_mx_loss_backward(). */
costa_status costa_mx_loss_workspace(int64_t m, int64_t n, int64_t k, int backward, size_t* least, size_t* most);

#ifdef __cplusplus
}
#endif

#endif /* COSTA_LAYER_H */
