/*
 * costa_mx.h -- matrices kept in 4 and 8 bits (microscaled floating point) and
 * the products that read them, next to the layout transform of costa.h.
 *
 * A microscaled matrix is stored by rows, every row in blocks of 32 elements
 * that share one power of two.  For a block x_0 .. x_31 of 32-bit floats, with
 * a = max |x_i| and e the exponent field of a (0 for zero and subnormals):
 *
 *     scale byte  s = max(e - emax, 0)       emax = 2 (E2M1), 8 (E4M3)
 *     element     q_i = x_i * 2^(127 - s), rounded to the nearest value of the
 *                 format (ties to the even one), past its largest value (6;
 *                 448) to that
 *     stands for  q_i * 2^(s - 127)
 *
 * A block that holds an infinity or a NaN gets the scale byte 255 and zero
 * elements: all of it stands for NaN (a finite stand-in would hide the
 * overflow).  The last block of a row may be shorter; what pads it is zero.
 *
 * Uses, for a layer Y = X W^T (X: tokens x inputs, W: outputs x inputs):
 *   forward            Y  = X W^T    costa_mx_product_real(N, X, mx(W))
 *                                    costa_mx_product(mx(X), mx(W))
 *   input's gradient   dX = dY W     costa_mx_product_real(N, dY, mx(W^T))
 *   weight's gradient  dW = dY^T X   costa_mx_product_real(T, dY, mx(X^T))
 * where mx(X^T) in 8 bits is the activation's checkpoint: the blocks run along
 * the tokens, the direction the gradient sums over.  One quantise call writes
 * mx(B) and mx(B^T).  Quantisation passes gradients through unchanged.
 * (mx(W^T) is rounded in blocks along the outputs, mx(W) in blocks along the
 * inputs: dX is the derivative of a layer with the former's weights, off that of
 * Y by what the two roundings differ by.)
 *
 * Conventions are those of costa.h: every call returns a costa_status, details
 * from costa_last_error(); calls are asynchronous on `stream`, on the current
 * device; every argument error is returned before anything is enqueued; the
 * caller owns every buffer.  No call allocates device memory, but for the first
 * quantise call of a layout (below).
 */
#ifndef COSTA_MX_H
#define COSTA_MX_H

#include "costa.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element formats of a microscaled matrix. */
typedef enum {
  COSTA_MX_E2M1 = 0, /* 4 bits: sign, 2 exponent bits, 1 mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6 */
  COSTA_MX_E4M3 = 1, /* 8 bits: sign, 4 exponent bits, 3 mantissa bits, up to 448 */
  COSTA_MX_INT32 = 0x7fffffff
} costa_mx_format;

/* Element types of the plain matrices of these calls. */
typedef enum {
  COSTA_REAL_F64 = 0, /* quantise and dequantise only */
  COSTA_REAL_F32 = 1,
  COSTA_REAL_BF16 = 2,
  COSTA_REAL_F16 = 3,
  COSTA_REAL_INT32 = 0x7fffffff
} costa_real;

/* A plain rows x cols matrix in device memory: element (i, j) is
 * data[i + j*ld] (COSTA_COL_MAJOR, ld >= rows) or data[i*ld + j]
 * (COSTA_ROW_MAJOR, ld >= cols), in elements; ld >= 1.  `data` is aligned to
 * the element size and may be NULL when the matrix has no elements. */
typedef struct {
  costa_real type;
  costa_order order;
  int64_t rows, cols, ld;
  void* data;
} costa_matrix;

/* A microscaled rows x cols matrix in device memory.  With pc = cols rounded
 * up to a multiple of 256 (E2M1) or 128 (E4M3), so that a row starts on a
 * multiple of 128 bytes:
 *   data   : rows x pc elements by rows; E2M1 two to a byte, the one of even
 *            column in the low half; columns past `cols` zero
 *   scales : rows x pc/32 scale bytes by rows; those of blocks past `cols` 0
 * Both 16-byte aligned; NULL allowed for a matrix without elements. */
typedef struct {
  costa_mx_format format;
  int64_t rows, cols;
  void* data;
  void* scales;
} costa_mx;

/* Bytes that the two buffers of a matrix must hold. */
costa_status costa_mx_sizes(costa_mx_format format, int64_t rows, int64_t cols, int64_t* data_bytes,
                            int64_t* scale_bytes);

/* Q <- mx(alpha * B) and QT <- mx(alpha * B^T), either of them or (one read of
 * B) both; the other is NULL.  Q has B's shape, QT the transposed one; their
 * formats may differ.  x = alpha * b: b rounded to a 32-bit float, then the
 * product rounded (alpha == 1: no rounding).  B, Q and QT must not overlap.
 * Errors: INVALID_VALUE for null or misaligned pointers, unknown types, a
 * leading dimension that is too small, operands that overlap, neither Q nor
 * QT; SHAPE_MISMATCH; NOT_SUPPORTED for dimensions above
 * 2^31 - 1 (as in every call here). */
costa_status costa_mx_quantize(float alpha, const costa_matrix* B, const costa_mx* Q, const costa_mx* QT,
                               hipStream_t stream);

/* The same out of the blocks of a distributed matrix: B_local[r] is the buffer
 * of rank r of layout B (as in costa_transform(); a rank that owns nothing may
 * pass NULL), its elements of type `type`.  The blocks of 32 are those of the
 * whole matrix, whatever blocks the layout cuts it into.  (That B's buffers do
 * not overlap Q and QT is not checked.)
 * The first call for a layout on a device uploads the layout's tables (device
 * memory, kept until costa_finalize(); the tables of up to 64 layouts, then all
 * of them start over but for those that captured calls read): such a call
 * synchronises, and is refused under stream capture (NOT_SUPPORTED).  NOT_SUPPORTED
 * also for layouts of more than 256 ranks or, unless block-cyclic, more than
 * 2^22 blocks. */
costa_status costa_mx_quantize_layout(costa_real type, float alpha, costa_layout B, const void* const* B_local,
                                      const costa_mx* Q, const costa_mx* QT, hipStream_t stream);

/* A <- alpha * Q^ + beta * A, Q^ the values that Q stands for, A of the same
 * shape.  In 32 bits (A of type F64: in 64), rounded once to A's type; a
 * product by alpha == 1 or beta == 1 is exact; beta == 0: A is not read.
 * A must not overlap Q. */
costa_status costa_mx_dequantize(float alpha, const costa_mx* Q, float beta, const costa_matrix* A,
                                 hipStream_t stream);

/* C <- alpha * A^ B^^T + beta * C: A m x k, B n x k, C m x n (F32, BF16 or F16;
 * F64: NOT_SUPPORTED); A^ and B^ the values that A and B stand for.  Products
 * are exact and summed in 32 bits; alpha and beta apply in 32 bits, C is rounded
 * once.  (With an 8-bit operand the values enter as bfloat16, which holds all of
 * them but those below 2^-133: blocks whose largest magnitude is under 2^-116.)
 * C must not overlap A or B, nor the workspace any of them (elements count, not what
 * lies between them: slices of one buffer may be side by side).
 * beta == 0: C is not read.  k == 0: C <- beta * C.  NOT_SUPPORTED for a C of
 * more than 2^31 - 1 of the kernels' tiles (16 TiB and more).
 * workspace: device memory for the parts of a sum that is split over several
 * workgroups (calls with few rows or columns and a long sum), 16-byte aligned,
 * workspace_bytes of it; costa_mx_workspace() says how much a call can use.
 * With less, or NULL, the sum is split less or not at all.  Its contents need not be
 * set, and are read and written by the call's kernels only. */
costa_status costa_mx_product(float alpha, const costa_mx* A, const costa_mx* B, float beta, const costa_matrix* C,
                              void* workspace, size_t workspace_bytes, hipStream_t stream);

/* C <- alpha * op(A) B^^T + beta * C with a plain A (F32, BF16 or F16): op(A) is
 * m x k, A itself k x m for op T (op C is op T).  As above; F32 elements enter the
 * product as three bfloat16 parts and F16 ones as two, which hold all of their
 * bits (F32: all but those below 2^-133), and B's values as bfloat16 (see above). */
costa_status costa_mx_product_real(float alpha, costa_op op, const costa_matrix* A, const costa_mx* B, float beta,
                                   const costa_matrix* C, void* workspace, size_t workspace_bytes,
                                   hipStream_t stream);

/* Workspace that a product of an m x k with a (transposed) n x k matrix can use. */
costa_status costa_mx_workspace(int64_t m, int64_t n, int64_t k, size_t* bytes);

#ifdef __cplusplus
}
#endif

#endif /* COSTA_MX_H */
