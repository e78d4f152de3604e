/*
 * gett_matrix.h -- matrix operators for training and serving in 4 bits.
 *
 * Beside the tensor contraction of gett.h the library carries the matrix
 * operators of a model whose products run in microscaled 4-bit floating point
 * and whose weight updates are made orthogonal before they are applied:
 *
 *   gett_mx_quantize     a float matrix -> packed 4-bit matrix (one or both
 *                        orientations in one pass)
 *   gett_mx_dequantize   the values a packed matrix stands for
 *   gett_mx_contract     C <- alpha * A * B^T + beta * C, A and B packed
 *   gett_mx_apply        the same with a float A that is quantised in the call
 *   gett_mx_linear, gett_mx_linear_grad   a linear layer of a training step
 *   gett_orthogonalize   Newton-Schulz steps on a stack of matrices
 *
 * Element types are those of gett_dtype_t and GETT_BFLOAT16 / GETT_FLOAT16.
 * A matrix argument is a device pointer to element [0, 0] with a stride per
 * row and per column in elements (both >= 1, any order; the library's other
 * entry points describe tensors the same way).
 *
 * Calls enqueue work on `stream` (a hipStream_t, NULL: the default stream)
 * and return.  Errors are statuses; nothing is thrown.  Extents that need more
 * threads than a launch has (2^32) are GETT_ERROR_NOT_SUPPORTED.  Workspaces are the
 * library's own, one per device and stream, as for gett_contract: a call that
 * needs more than the stream's workspace holds allocates, which is refused
 * with GETT_ERROR_NOT_SUPPORTED, nothing enqueued, while `stream` captures a
 * graph (run the call eagerly on that stream first).  A graph goes on using the
 * workspace of the stream it was captured on, which is left to it when a later
 * call gets a larger one; a replay has to be ordered with that stream's other
 * calls (on that stream, or by events), as calls from several streams would be
 * that share a workspace.  A workspace is kept until the process ends, at the size
 * of the largest call on its stream: 17/32 byte for each number that
 * gett_mx_apply (more than 16 rows, or more than 8 of a large product),
 * gett_mx_linear (X and W) and gett_mx_linear_grad (dY, twice) pack; for
 * gett_orthogonalize, unless one workgroup takes a whole matrix, 12 rows cols + 8
 * min(rows, cols)^2 bytes a matrix (335 MB for 4096 x 4096); and up to 64 MB
 * for each product whose sums several workgroups share.
 *
 * The packed format ("MX4").  A matrix of `rows` x `cols` is packed along its
 * columns, the direction a product sums over.  Each run of 32 neighbours
 * x_0..x_31 of one row shares the scale
 *
 *     s = 2^(floor(log2(max |x_i|)) - 2)          (2^-127 at least)
 *
 * and holds q_i = x_i / s rounded to the nearest of
 * 0, 0.5, 1, 1.5, 2, 3, 4, 6 (and their negatives), ties to the value whose
 * code is even; magnitudes above 6 become 6.  A run that holds an infinity
 * or a NaN gets the NaN scale and stands for 32 NaNs.  Columns are padded with
 * zeros to T = ceil(cols / 256) tiles of 256.
 *
 *   codes   T x rows x 128 bytes, tile after tile and in it row after row: two
 *           codes (sign, two exponent bits, one mantissa bit) a byte, the even
 *           column in the low half.
 *   scales  T x 2 x R x 4 bytes, R = rows rounded up to 16: byte
 *           ((t * 2 + b / 4) * R + row) * 4 + b % 4 is the scale of block b
 *           (columns 256 t + 32 b and 31 more) of `row`, as exponent + 127;
 *           255 is NaN.  The bytes of rows >= `rows` may hold anything.
 *
 * Both pointers are aligned to 16 bytes.  A product takes one tile of columns
 * of many rows at a time: tile after tile these are neighbours in memory (row
 * after row they would lie a power of two apart, on few memory channels), and
 * the scales of one lane's rows and blocks reach its registers in one load.
 */
#ifndef GETT_MATRIX_H
#define GETT_MATRIX_H

#include "gett.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of these operators only, values of gett_dtype_t beside
 * GETT_FLOAT32; the contraction's entry points refuse them. */
#define GETT_BFLOAT16 ((gett_dtype_t)2)
#define GETT_FLOAT16 ((gett_dtype_t)3)

/*
 * gett_mx_size -- bytes of the codes and scales of a packed rows x cols
 * matrix.  GETT_ERROR_INVALID_VALUE for a null pointer or a negative extent,
 * GETT_ERROR_NOT_SUPPORTED for rows of 2^30 or cols of 2^24 and more.
 */
gett_status_t gett_mx_size(int64_t rows, int64_t cols, uint64_t *code_bytes,
                           uint64_t *scale_bytes);

/*
 * gett_mx_quantize -- pack X, its transpose, or both, in one pass over X.
 *
 *   dtype            GETT_FLOAT32, GETT_BFLOAT16 or GETT_FLOAT16.
 *   codes, scales    X packed along its columns (gett_mx_size(rows, cols)),
 *                    or both NULL.
 *   codes_t, scales_t  X^T, a cols x rows matrix, packed along X's rows
 *                    (gett_mx_size(cols, rows)), or both NULL.
 *
 * Errors: GETT_ERROR_INVALID_VALUE (unknown dtype, negative extent, stride
 * < 1, no output, half of an output, a null or misaligned pointer, an output
 * that overlaps X or another output), GETT_ERROR_NOT_SUPPORTED (extents
 * beyond gett_mx_size's), GETT_ERROR_HIP.  An empty X enqueues nothing and its
 * pointers are not looked at.
 */
gett_status_t gett_mx_quantize(gett_dtype_t dtype, int64_t rows, int64_t cols, const void *X,
                               int64_t stride_row, int64_t stride_col, void *codes, void *scales,
                               void *codes_t, void *scales_t, void *stream);

/*
 * gett_mx_dequantize -- the values of a packed rows x cols matrix, written to
 * X in `dtype` (rounded where it cannot hold them: GETT_FLOAT16 only).
 * Strides that map two elements to one address are refused
 * (GETT_ERROR_NOT_SUPPORTED); other errors as for gett_mx_quantize.
 */
gett_status_t gett_mx_dequantize(gett_dtype_t dtype, int64_t rows, int64_t cols,
                                 const void *codes, const void *scales, void *X,
                                 int64_t stride_row, int64_t stride_col, void *stream);

/*
 * gett_mx_contract -- C[m, n] <- alpha * sum_k A[m, k] B[n, k] + beta * C[m, n].
 *
 *   codes_A, scales_A   a packed m x k matrix;
 *   codes_B, scales_B   a packed n x k matrix.
 *   dtype, C            C's element type and data.  Sums are held in 32 bits;
 *                       alpha, beta and the sum are combined in 32 bits and
 *                       rounded once.  beta == 0: C is not read; alpha == 0
 *                       or k == 0: A and B are not read.
 *
 * Repeated calls give identical results.  Errors: GETT_ERROR_INVALID_VALUE
 * (unknown dtype, negative extent, stride < 1, null or misaligned pointer, C
 * overlapping an operand), GETT_ERROR_NOT_SUPPORTED (extents beyond
 * gett_mx_size's; strides that map two elements of C to one address),
 * GETT_ERROR_HIP.
 */
gett_status_t gett_mx_contract(int64_t m, int64_t n, int64_t k, double alpha,
                               const void *codes_A, const void *scales_A, const void *codes_B,
                               const void *scales_B, double beta, gett_dtype_t dtype, void *C,
                               int64_t stride_m, int64_t stride_n, void *stream);

/*
 * gett_mx_apply -- gett_mx_contract with a float A, quantised in the call.
 *
 *   dtype_A, A, stride_am, stride_ak   an m x k matrix in 16 or 32 bits; the
 *            result is that of gett_mx_quantize and gett_mx_contract.
 *
 * For few rows (single tokens) A is quantised on its way into the product,
 * in the same launch; for more, into the stream's workspace first.
 */
gett_status_t gett_mx_apply(int64_t m, int64_t n, int64_t k, double alpha, gett_dtype_t dtype_A,
                            const void *A, int64_t stride_am, int64_t stride_ak,
                            const void *codes_B, const void *scales_B, double beta,
                            gett_dtype_t dtype, void *C, int64_t stride_m, int64_t stride_n,
                            void *stream);

/*
 * gett_mx_linear -- Y <- Q(X) Q(W)^T, both quantised in the call, for training.
 *
 *   X   m x k, W   n x k, Y   m x n in X's type.
 *   codes_xt, scales_xt   X^T packed (gett_mx_size(k, m)) as
 *   codes_wt, scales_wt   and W^T packed (gett_mx_size(k, n)): what
 *                         gett_mx_linear_grad needs, or NULL where not wanted.
 *
 * The same results as gett_mx_quantize and gett_mx_contract in fewer calls and
 * launches.  Errors as for those; outputs must not overlap one another or an
 * input.
 */
gett_status_t gett_mx_linear(int64_t m, int64_t n, int64_t k, gett_dtype_t dtype_X, const void *X,
                             int64_t stride_xm, int64_t stride_xk, gett_dtype_t dtype_W,
                             const void *W, int64_t stride_wn, int64_t stride_wk, void *Y,
                             int64_t stride_ym, int64_t stride_yn, void *codes_xt,
                             void *scales_xt, void *codes_wt, void *scales_wt, void *stream);

/*
 * gett_mx_linear_grad -- the gradients of gett_mx_linear,
 *     dX <- Q(dY) Q(W^T)^T   (m x k, in dY's type),
 *     dW <- Q(dY^T) Q(X^T)^T (n x k, in dtype_W),
 * each product's operands packed along the direction it sums over; the
 * gradient of the rounding itself is taken as one.  dX or dW may be NULL where
 * not wanted (dX needs W^T, dW needs X^T).  Errors as for gett_mx_linear.
 */
gett_status_t gett_mx_linear_grad(int64_t m, int64_t n, int64_t k, gett_dtype_t dtype_Y,
                                  const void *dY, int64_t stride_ym, int64_t stride_yn,
                                  const void *codes_xt, const void *scales_xt,
                                  const void *codes_wt, const void *scales_wt, void *dX,
                                  int64_t stride_xm, int64_t stride_xk, gett_dtype_t dtype_W,
                                  void *dW, int64_t stride_wn, int64_t stride_wk, void *stream);

/*
 * gett_orthogonalize -- O <- the Newton-Schulz iterate of G, per matrix.
 *
 *     X_0 = G / (|G|_F + eps)            |G|_F summed in 64 bits
 *     X_{i+1} = a X_i + (b S + c S^2) X_i,   S = X_i X_i^T,   i < steps
 *     O = X_steps                         (S = X^T X where rows > cols)
 *
 * The singular vectors of G stay and each singular value s moves by
 * s <- a s + b s^3 + c s^5; with (3.4445, -4.7750, 2.0315) and five steps
 * those above about 1e-3 |G|_F end between 0.7 and 1.2.
 *
 *   dtype     of G and O: GETT_FLOAT32, GETT_BFLOAT16 or GETT_FLOAT16.
 *   batch     matrices in the stack (stride_batch between them, >= 1; any
 *             value when batch is 1).  They may interleave in memory, as the
 *             column slices of a wide matrix do.
 *   a, b, c   the polynomial.  Coefficients for which a singular value may
 *             pass 3, or b s^2 + c s^4 may pass 15, within the steps
 *             are refused (GETT_ERROR_NOT_SUPPORTED): the iterates are kept
 *             in 16-bit parts that hold such values.
 *   steps     0 to 1000.
 *
 * O may be G itself (same pointer and strides); otherwise they must not
 * overlap.  Iterates are held in two 16-bit parts (22 bits) for every dtype, with
 * sums in 32 bits, and the result is rounded once.  With the usual inputs that
 * is as near the 64-bit result as iterates in 32 bits are.  The parts' grid ends at
 * 2^-36 (|X_0| is 1), and the steps magnify small singular values by a each, so
 * that the result is off by up to about 2^-37 sqrt(rows cols) a^steps in its norm
 * beside some 2^-22 of it: more than 32 bits leave where one element is 1e6 times the
 * others and more (512 x 512 and the coefficients above: 1.5e-6 to 1.8e-6 of the
 * norm, with iterates in 32 bits 2e-7 to 1e-8).  A NaN or an infinity in a
 * matrix makes that matrix NaN.  Errors: GETT_ERROR_INVALID_VALUE (unknown
 * dtype, negative extent or steps, stride < 1, eps negative or NaN, a
 * coefficient that is not finite, null or misaligned pointer, overlap),
 * GETT_ERROR_NOT_SUPPORTED (see above; rows or cols of 2^20 and more, steps
 * above 1000; strides that map two elements to one address; batch x tiles
 * beyond a launch), GETT_ERROR_HIP.
 */
gett_status_t gett_orthogonalize(gett_dtype_t dtype, int64_t batch, int64_t rows, int64_t cols,
                                 const void *G, int64_t stride_batch, int64_t stride_row,
                                 int64_t stride_col, double a, double b, double c, double eps,
                                 int steps, void *O, int64_t ostride_batch, int64_t ostride_row,
                                 int64_t ostride_col, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* GETT_MATRIX_H */
