/*
 * costa_layer.h -- what stands around the products of a layer whose weights are
 * kept in few bits (costa_mx.h): the norm that makes a product's operand, with its
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
 * refused, INVALID_VALUE) and what it can use (`most`); either pointer may be NULL.
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
 * X or R itself (the same matrix: data, ld and type).  eps: at least 2^-126, finite. */
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

#ifdef __cplusplus
}
#endif

#endif /* COSTA_LAYER_H */
