/*
 * libones, the jobs' side - operators of a scheduled language-model job's training step on an AMD MI355X (gfx950).
 *
 * The search (ones.h) decides at which batch a job trains and describes the job by its iteration time
 * t(B,g) = a*B/g + c*log2(g) + d.  These are the parts of such an iteration: layer norm, a gated linear recurrence over the
 * steps of a sequence and the loss over a large vocabulary, whose work grows with the local batch B/g (a), and the
 * orthogonalised update of a weight matrix, whose work does not (d).
 *
 * Conventions.  Every function returns ONES_OK (0) or a negative ONES_E_* code of ones.h; nothing aborts or throws across this
 * boundary, all sizes are checked before the first launch and nothing is launched on error.  All arrays are DEVICE pointers
 * owned by the caller, on the device that is current.  Work is put on hip_stream (a hipStream_t, NULL = the default stream) and
 * the call returns at once; nothing is allocated, no call waits, and calls may be captured into a HIP graph.  A workspace is
 * scratch of one call (256-byte aligned; nothing in it outlives the call's work on the stream) of at least the bytes that the
 * function's ..._workspace_bytes gives for the same sizes, which is 0 where none is needed (or the sizes are refused).
 * Rows lie `stride` elements apart, the elements of a row one after another; outputs have no gaps.  Rows that allow wide
 * accesses (base and strides multiples of 16 bytes) are faster, all others are taken too.  Sums and states are kept in 32
 * bits; results of 16 bits are rounded once, to nearest.  Every sum has a fixed order: equal inputs give equal bits.
 * A size of zero is not an error: sums over nothing are zero.
 */
#ifndef ONES_TRAIN_H
#define ONES_TRAIN_H

#include "ones.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Types of elements. */
#define ONES_F32  0
#define ONES_F16  1
#define ONES_BF16 2

#define ONES_MAX_NORM_COLUMNS 32768       /* columns of a layer norm                                */
#define ONES_MAX_STEPS        (1 << 30)   /* steps of a sequence                                    */
#define ONES_MAX_CHANNELS     (1 << 24)   /* channels of a recurrence                               */
#define ONES_MAX_BATCH        65535       /* sequences of a recurrence                              */
#define ONES_MAX_LOSS_ROWS    (1 << 24)   /* rows of a cross entropy                                */
#define ONES_MAX_LOSS_COLUMNS 65536
#define ONES_MAX_VOCABULARY   (1 << 24)
#define ONES_MAX_UPDATE_SIDE  65536       /* rows and columns of an orthogonalised update           */

/* Layer norm over the columns of x[rows][cols], 1 <= cols <= ONES_MAX_NORM_COLUMNS:
 *   y = (x - mean) * rstd * weight + bias, mean and rstd = (variance + eps)^-1/2 per row (variance: the mean square of x - mean).
 * type: of x, y, dy, dx.  weight_type: of weight, bias and their gradients: type or ONES_F32.  weight, bias: cols
 * elements each, or NULL (1 and 0).  mean, rstd: rows floats each, written forward and read backward.  eps >= 0.
 * Backward writes dx[rows][cols] and the sums over the rows dweight (of dy * (x - mean) * rstd) and dbias (of dy); either may
 * be NULL.  Errors: ONES_E_INVALID_ARG, ONES_E_BOUNDS (cols, rows * stride), ONES_E_WORKSPACE_TOO_SMALL, ONES_E_HIP. */
int ones_layer_norm_forward(const void *x, int64_t x_stride, int64_t rows, int64_t cols, int32_t type,
                            const void *weight, const void *bias, int32_t weight_type, float eps,
                            void *y, float *mean, float *rstd, void *hip_stream);
size_t ones_layer_norm_workspace_bytes(int64_t rows, int64_t cols);
int ones_layer_norm_backward(const void *dy, int64_t dy_stride, const void *x, int64_t x_stride,
                             int64_t rows, int64_t cols, int32_t type, const void *weight, int32_t weight_type,
                             const float *mean, const float *rstd, void *dx, void *dweight, void *dbias,
                             void *d_workspace, size_t workspace_bytes, void *hip_stream);

/* Gated linear recurrence over the steps of every sequence, channel by channel:
 *   a_t = sigmoid(gate_t), h_t = a_t * h_{t-1} + (1 - a_t) * x_t, h_{-1} = state (NULL: 0).
 * gate, x, dh: [batch][steps][channels] with the strides given (a stride of 0 repeats a row); h, dgate, dx: without gaps.
 * state, last, dlast, dstate: float [batch][channels]; carry: ones_recurrence_carry_bytes, written forward (NULL: not
 * wanted) and read backward, which needs neither state nor h.  lengths: int32 [batch] or NULL; of sequence b only the first
 * lengths[b] steps (pulled into 0..steps) count: the rest is not read, h and the gradients are 0 there, last is the state behind
 * the last step that counts.  last, dstate may be NULL, dlast too (0).  batch <= ONES_MAX_BATCH, batch * channels <= 2^36.
 * ones_recurrence_step: one step of every sequence, gate and x [batch][channels] with a row stride, state updated in place.
 * Errors: ONES_E_INVALID_ARG, ONES_E_BOUNDS (a size or a stride above its limit), ONES_E_WORKSPACE_TOO_SMALL, ONES_E_HIP. */
size_t ones_recurrence_carry_bytes(int64_t batch, int64_t steps, int64_t channels);
size_t ones_recurrence_workspace_bytes(int64_t batch, int64_t steps, int64_t channels);
int ones_recurrence_forward(const void *gate, int64_t gate_batch_stride, int64_t gate_step_stride,
                            const void *x, int64_t x_batch_stride, int64_t x_step_stride,
                            int64_t batch, int64_t steps, int64_t channels, int32_t type,
                            const float *state, const int32_t *lengths, void *h, float *last, float *carry,
                            void *d_workspace, size_t workspace_bytes, void *hip_stream);
int ones_recurrence_backward(const void *dh, int64_t dh_batch_stride, int64_t dh_step_stride, const float *dlast,
                             const void *gate, int64_t gate_batch_stride, int64_t gate_step_stride,
                             const void *x, int64_t x_batch_stride, int64_t x_step_stride,
                             int64_t batch, int64_t steps, int64_t channels, int32_t type,
                             const float *carry, const int32_t *lengths, void *dgate, void *dx, float *dstate,
                             void *d_workspace, size_t workspace_bytes, void *hip_stream);
int ones_recurrence_step(const void *gate, int64_t gate_stride, const void *x, int64_t x_stride,
                         int64_t batch, int64_t channels, int32_t type, float *state, void *h, void *hip_stream);

/* Softmax cross entropy of the logits x[rows][cols] weight[vocabulary][cols]^T, which are not kept:
 *   lse_i = log sum_v exp(x_i . weight_v), loss_i = lse_i - x_i . weight_target_i.
 * type (of x, weight, dx, dweight): ONES_F16 or ONES_BF16.  target: int64 [rows]; below 0: the row is ignored (loss 0, no
 * gradient, and what x holds there does not matter); vocabulary or above: the row's loss, its dx and dweight are NaN.
 * loss, lse: float [rows].  Backward: dloss float [rows], lse as forward left it; dx[rows][cols] and dweight[vocabulary][cols]
 * are written.  It goes through the vocabulary in pieces, and through more than 2^18 rows in blocks, so that at most 128 MiB of logits'
 * gradients, rounded to type, are held at a time (in units of dloss: in fp16 dx of a row is as exact as fp16 is while the row's |dloss|
 * is above 2^-26 of the largest).
 * wide: not 0 if cols, both strides and both bases are multiples of 16 bytes and no stride is above 2^20 elements; otherwise the
 * workspace has room for copies.
 * Errors: ONES_E_INVALID_ARG, ONES_E_BOUNDS (a size above its limit, or the product of two of them above 2^36),
 * ONES_E_WORKSPACE_TOO_SMALL, ONES_E_HIP. */
size_t ones_cross_entropy_forward_workspace_bytes(int64_t rows, int64_t cols, int64_t vocabulary, int32_t wide);
size_t ones_cross_entropy_backward_workspace_bytes(int64_t rows, int64_t cols, int64_t vocabulary, int32_t wide);
int ones_cross_entropy_forward(const void *x, int64_t x_stride, const void *weight, int64_t weight_stride,
                               int64_t rows, int64_t cols, int64_t vocabulary, int32_t type, const int64_t *target,
                               float *loss, float *lse, void *d_workspace, size_t workspace_bytes, void *hip_stream);
int ones_cross_entropy_backward(const float *dloss, const void *x, int64_t x_stride, const void *weight, int64_t weight_stride,
                                int64_t rows, int64_t cols, int64_t vocabulary, int32_t type, const int64_t *target,
                                const float *lse, void *dx, void *dweight, void *d_workspace, size_t workspace_bytes,
                                void *hip_stream);

/* The orthogonalised update of `count` weight matrices [rows][cols] that lie one behind the other: momentum and Newton-Schulz products.
 *   momentum = beta * momentum + grad; u = grad + beta * momentum if nesterov, else momentum; X = u / (|u| + eps), |u| the root of
 *   the sum of squares of each matrix; `steps` times, with coefficients a, b, c: A = X X^T, X = a X + (b A + c A A) X; update = X
 * (with X^T X for rows > cols, which gives the same).  grad_type: any; momentum: float, updated in place, or NULL (u = grad);
 * update_type: ONES_F16 or ONES_BF16.  coefficients: HOST array of three, of size up to 16, that keep the singular values below 7.9
 * (they start below 1).  Products have fp16 operands for ONES_BF16, which puts the result of five steps about as far off again as its own
 * rounding does (2.4e-3 of its norm in all), and pairs of fp16 for ONES_F16, three products each, which leaves its own rounding (2e-4).
 * The workspace is enough for either.  1 <= steps <= 100, 0 <= beta <= 1, eps >= 0.  A matrix of zeros gives zeros
 * if eps > 0.  Errors: ONES_E_INVALID_ARG, ONES_E_BOUNDS (a side, count above 65535, a coefficient), ONES_E_WORKSPACE_TOO_SMALL,
 * ONES_E_HIP. */
size_t ones_orthogonal_update_workspace_bytes(int64_t count, int64_t rows, int64_t cols);
int ones_orthogonal_update(const void *grad, float *momentum, int64_t count, int64_t rows, int64_t cols, int32_t grad_type,
                           float beta, int32_t nesterov, int32_t steps, const float *coefficients, float eps,
                           void *update, int32_t update_type, void *d_workspace, size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif
