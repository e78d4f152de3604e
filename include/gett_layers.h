/*
 * gett_layers.h -- operators of a feed-forward layer in 16 and 32 bits.
 *
 * Beside the contraction of gett.h and the 4-bit operators of gett_matrix.h the
 * library carries what surrounds a product in a layer that is trained and served
 * in 16 or 32 bits, and the same for layers that are split into experts:
 *
 *   gett_dropout                        y = x keep / (1 - p), no mask stored
 *   gett_linear, gett_linear_grad       y = residual + dropout(act(x w^T + bias))
 *   gett_route, gett_route_grad         k experts for every token, and the order
 *                                       of the chosen rows by expert
 *   gett_experts, gett_experts_grad     act(x_r w_e^T + bias_e) for each row r of
 *                                       each expert e
 *   gett_combine, gett_combine_grad     the experts' rows summed back to tokens
 *
 * Element types are GETT_FLOAT32, GETT_BFLOAT16 and GETT_FLOAT16; all tensors of
 * a call have the call's type unless said otherwise.  Sums, activations and the
 * epilogue are held in 32 bits and rounded once, at the store.  Matrices are
 * row-major with a row stride in elements (at least their columns); rows may be
 * wider apart.  Addresses need only their element's alignment: operands of a product
 * that do not lie on the 16-byte grid, in base, stride and columns, are copied into
 * the stream's workspace first, unless they are multiplied with few rows (up to 32, of
 * experts 64), which take them as they lie and may sum in another order.
 *
 * Calls enqueue work on `stream` and return; errors are statuses; workspaces are
 * the library's own, one per device and stream, as gett_matrix.h describes: a
 * call that needs more than the stream's holds allocates, which is refused with
 * GETT_ERROR_NOT_SUPPORTED while the stream captures a graph.  They hold the copies
 * above, dZ of a gradient (unless it is dY itself), the rows of the experts' X (in the
 * type) and dX (in 32 bits) where these are gathered, 4 bytes for each 8 to 64 numbers
 * whose columns are summed, and up to 64 MB for a product whose sums several workgroups
 * share; and they stay, at the size of the largest call on the stream, until the process
 * ends: a gradient of 32768 gathered rows of 2048 with n = 1536 in bf16 leaves 0.5 GB.
 * A call that needs more than there is waits for the stream.
 * Repeated calls give identical results.  Outputs must not overlap inputs or one
 * another except where it is said.
 *
 * Errors of every call: GETT_ERROR_INVALID_VALUE (unknown dtype, activation or
 * scoring, a negative extent, a stride smaller than the columns, a null or
 * misaligned pointer, an overlap, a probability outside [0, 1]),
 * GETT_ERROR_NOT_SUPPORTED (rows of 2^30 and more, columns of 2^21 and more, a
 * launch or an operand too large), GETT_ERROR_HIP, GETT_ERROR_ALLOC.  Extents of
 * zero enqueue what remains to be written; pointers of empty tensors are not
 * looked at.
 */
#ifndef GETT_LAYERS_H
#define GETT_LAYERS_H

#include "gett_matrix.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Activations: z; max(z, 0); z (1 + erf(z / sqrt 2)) / 2; z / (1 + e^-z).  Values are
 * within 2^-20 (1 + |z|) |z|, slopes within 2^-20 (1 + |z|); of infinities they are the
 * limits, of NaN NaN. */
#define GETT_ACTIVATION_NONE 0
#define GETT_ACTIVATION_RELU 1
#define GETT_ACTIVATION_GELU 2
#define GETT_ACTIVATION_SILU 3

/*
 * Dropout.  The number at (row, col) is kept where its field is at least
 * t = round(65536 p) (ties to even), and then multiplied by 65536 / (65536 - t);
 * otherwise it is zero (whatever it was).  Its field are 16 bits of the block
 *
 *     Philox4x32-10(key = seed, counter = {col / 8, row, offset, offset >> 32}),
 *
 * word (col % 8) / 2, the low half for even columns (Salmon, Moraes, Dror and
 * Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC 2011).  A call that is
 * given the same seed and offset has the same mask: the gradient makes it again.
 *
 *   p            in [0, 1]; t = 0 keeps all, t = 65536 none.
 *   seed_device  NULL, or a device pointer to the seed, read by the kernels in
 *                the place of `seed` (a captured graph draws a new mask when its
 *                value changes between replays).
 */
typedef struct {
    double p;
    uint64_t seed, offset;
    const int64_t *seed_device;
} gett_dropout_t;

/* Y <- dropout(X), rows x cols; Y may be X itself (same pointer and stride).
 * The gradient is the same call on dY. */
gett_status_t gett_dropout(gett_dtype_t dtype, int64_t rows, int64_t cols, const void *X,
                           int64_t stride_x, const gett_dropout_t *drop, void *Y, int64_t stride_y,
                           void *stream);

/*
 * gett_linear -- Y <- residual + dropout(act(X W^T + bias)).
 *
 *   X   m x k;  W  n x k;  bias  n, or NULL;  residual  m x n, or NULL (it may be Y
 *       itself, same pointer and stride).
 *   drop  NULL, or the dropout of the activation.
 *   Z   NULL, or m x n: X W^T + bias, rounded (what gett_linear_grad takes the
 *       activation's slope from).
 */
gett_status_t gett_linear(gett_dtype_t dtype, int64_t m, int64_t n, int64_t k, const void *X,
                          int64_t stride_x, const void *W, int64_t stride_w, const void *bias,
                          int activation, const gett_dropout_t *drop, const void *residual,
                          int64_t stride_r, void *Z, int64_t stride_z, void *Y, int64_t stride_y,
                          void *stream);

/*
 * gett_linear_grad -- with dZ = dropout(dY) act'(Z), rounded to the type,
 *     dX <- dZ W  (m x k),  dW <- dZ^T X  (n x k),  dbias <- the sums of dZ's columns
 *                                                   (taken before it is rounded).
 * Each output may be NULL.  Z may be NULL without an activation, W without dX, X
 * without dW.  The residual's gradient is dY itself.  The slope of the ReLU at 0
 * is 0.
 */
gett_status_t gett_linear_grad(gett_dtype_t dtype, int64_t m, int64_t n, int64_t k, const void *dY,
                               int64_t stride_dy, const void *Z, int64_t stride_z, const void *X,
                               int64_t stride_x, const void *W, int64_t stride_w, int activation,
                               const gett_dropout_t *drop, void *dX, int64_t stride_dx, void *dW,
                               int64_t stride_dw, void *dbias, void *stream);

/*
 * gett_route -- k of `experts` experts for each of `tokens` tokens.
 *
 *     s       softmax or sigmoid of the token's logits
 *     choice  s + bias; -inf where the logit is
 *     groups > 1: the experts lie in `groups` runs of experts / groups; a group
 *             counts as the sum of its two largest choices (without those of -inf),
 *             and only the experts of the `top_groups` largest groups are open
 *     index   the k open experts of largest choice, largest first; never one of
 *             choice -inf
 *     weights s at these experts; divided by their sum where `renormalize` is not
 *             0 (0 where sigmoids sum to 0 in 64 bits); times `scale`
 *
 * What is compared is held in 64 bits (without a bias and groups the logits are
 * compared themselves); ties go to the lowest index.  Where fewer than k experts
 * are open the last indices are -1 and their weights 0: such a row belongs to no
 * expert.  A NaN counts as -inf in the choice, and one among the logits makes the
 * token's weights NaN, as does a +inf under a softmax.
 *
 *   logits   tokens x experts, of type dtype.
 *   bias     experts floats, or NULL.
 *   weights (float), index (int32)   tokens x k.
 *   order    tokens k int32: the rows token * k + choice, expert after expert and
 *            within one in rising order; -1 behind the last.
 *   offsets  experts + 1 int32: where each expert's rows begin in `order`.
 *   place    tokens x k int32: where `order` has the row (-1: nowhere).
 *
 * GETT_ERROR_NOT_SUPPORTED for more than 1024 experts, k > 32, or tokens * k of
 * 2^30 and more (of the other calls with tokens, too); GETT_ERROR_INVALID_VALUE
 * where groups do not divide the experts or top_groups of them hold fewer than k.
 */
#define GETT_SCORE_SOFTMAX 0
#define GETT_SCORE_SIGMOID 1
gett_status_t gett_route(gett_dtype_t dtype, int64_t tokens, int experts, int k,
                         const void *logits, int64_t stride, int scoring, const float *bias,
                         int groups, int top_groups, int renormalize, double scale, float *weights,
                         int32_t *index, int32_t *order, int32_t *offsets, int32_t *place,
                         void *stream);

/* dlogits <- the gradient of gett_route's weights (the choice is constant), from
 * its logits, its index and dweights (float, tokens x k).  Of a token whose weights
 * are NaN all are NaN. */
gett_status_t gett_route_grad(gett_dtype_t dtype, int64_t tokens, int experts, int k,
                              const void *logits, int64_t stride, int scoring, int renormalize,
                              double scale, const int32_t *index, const float *dweights,
                              void *dlogits, int64_t stride_d, void *stream);

/*
 * gett_experts -- Y[p] <- act(X[r(p)] W_e^T + bias_e) for each place p of each expert
 * e, offsets[e] <= p < offsets[e + 1]; the rows of Y (and Z) behind the last
 * expert's are set to zero.
 *
 *   X       gather != 0: tokens x width, and r(p) = order[p] / k;
 *           gather == 0: tokens k x width, and r(p) = p.
 *   W       experts x n x width: stride_w between rows, stride_we between experts.
 *   bias    experts x n, or NULL.
 *   Y, Z    tokens k x n (Z or NULL, as for gett_linear).
 *
 * `order` and `offsets` are gett_route's for `tokens` tokens of k choices; values
 * out of range are brought into it and give rows of no meaning.
 */
gett_status_t gett_experts(gett_dtype_t dtype, int64_t tokens, int k, int experts, int64_t n,
                           int64_t width, const void *X, int64_t stride_x, int gather,
                           const void *W, int64_t stride_w, int64_t stride_we, const void *bias,
                           int activation, const int32_t *order, const int32_t *offsets, void *Z,
                           int64_t stride_z, void *Y, int64_t stride_y, void *stream);

/*
 * gett_experts_grad -- with dZ = dY act'(Z), rounded to the type,
 *     dX  <- dZ[p] W_e at p (gather == 0; zero behind the last row), or summed over
 *            each token's places in 32 bits (gather != 0)
 *     dW  <- dZ_e^T X_e, dbias <- the sums of dZ_e's columns, for each expert
 * Each output may be NULL.  dW is experts x n x width without gaps.
 */
gett_status_t gett_experts_grad(gett_dtype_t dtype, int64_t tokens, int k, int experts, int64_t n,
                                int64_t width, const void *dY, int64_t stride_dy, const void *Z,
                                int64_t stride_z, const void *X, int64_t stride_x, int gather,
                                const void *W, int64_t stride_w, int64_t stride_we, int activation,
                                const int32_t *order, const int32_t *offsets, const int32_t *place,
                                void *dX, int64_t stride_dx, void *dW, void *dbias, void *stream);

/*
 * gett_combine -- Y[t] <- residual[t] + sum_j weights[t, j] H[place[t, j]], summed in
 * rising j in 32 bits; places of -1 are left out.
 *
 *   H         tokens k x cols;  residual, Y  tokens x cols (residual or NULL; it may
 *             be Y itself).
 *   weights   tokens x k of type dtype_w (GETT_FLOAT32 or dtype).
 */
gett_status_t gett_combine(gett_dtype_t dtype, int64_t tokens, int k, int64_t cols, const void *H,
                           int64_t stride_h, gett_dtype_t dtype_w, const void *weights,
                           const int32_t *place, const void *residual, int64_t stride_r, void *Y,
                           int64_t stride_y, void *stream);

/* dH[place[t, j]] <- weights[t, j] dY[t] (zero in the rows of no place, from
 * offsets[experts] on); dweights[t, j] <- dY[t] . H[place[t, j]] in dtype_w.  Each
 * may be NULL (H is needed for dweights alone, weights for dH alone). */
gett_status_t gett_combine_grad(gett_dtype_t dtype, int64_t tokens, int k, int64_t cols,
                                const void *dY, int64_t stride_dy, const void *H, int64_t stride_h,
                                gett_dtype_t dtype_w, const void *weights, const int32_t *place,
                                int experts, const int32_t *offsets, void *dH, int64_t stride_dh,
                                void *dweights, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* GETT_LAYERS_H */
