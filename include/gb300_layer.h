/*
 * gb300_layer.h -- C ABI of the operators a training step runs around its
 * projection GEMMs (gb300_gemm.h): layer norm forward and backward, 8-bit
 * activation checkpoints, and a projection's weight gradient taken from such
 * a checkpoint.  With C = A . B of gb300_gemm.h they make a pre-norm
 * projection block, y = layer_norm(x), o = y . W, and its backward pass
 * dy = do . W^T, dW = y^T . do, dx = layer_norm'(dy).
 *
 * Conventions are those of gb300_gemm.h: device pointers owned by the caller,
 * leading dimensions in elements, calls asynchronous on `stream`, status
 * codes instead of exceptions, library scratch per stream (which is what
 * limits CUDA graph capture: a captured call needs its stream's scratch to
 * have grown to that size before).  Matrices are row-major; outputs must not
 * overlap inputs unless a declaration says so.  Any sizes, pitches and (for
 * its type) aligned addresses are supported; 16-byte aligned rows are
 * fastest.  Nothing outside a matrix is read or written.  Every result is the
 * same from run to run: sums are taken in an order that the sizes fix.
 *
 * Activation checkpoint ("q8").  A rows x cols matrix is held as signed bytes
 * q (rows x cols, pitch ldq) and one byte e (rows x ceil(cols / 32), pitch
 * lde) per block of 32 consecutive values of a row:
 *
 *     value(r, c) = q(r, c) * 2^(e(r, c / 32) - 127).
 *
 * Of a block, with top its largest magnitude, E = e - 127 is the least
 * exponent >= -126 with top <= 127 * 2^E, and q = round_half_even(x / 2^E)
 * (at E = 122, the largest, limited to -63 .. 63: 64 * 2^122 is past float32).
 * A block with a NaN or an infinity is held as q = 0, e = 255, which stands
 * for NaN throughout, so that a diverged activation stays visible; e = 0 is
 * not produced (and stands for 0).  The scale is a power of two on purpose:
 * x / 2^E and q * 2^E are exact, so the checkpoint is determined bit for bit,
 * and every value it stands for is a bf16 number, so that a bf16 tensor core
 * multiplies checkpointed activations without a further rounding.  The error
 * of a value is at most 2^(E-1), which is below top / 126 for -126 < E < 122;
 * at E = -126 it is at most 2^-127 whatever top is (a value below that is held
 * as 0), at E = 122 at most 2^E.
 */
#ifndef GB300_LAYER_H
#define GB300_LAYER_H

#include "gb300_gemm.h"

#ifdef __cplusplus
extern "C" {
#endif
#if defined(__GNUC__)
#pragma GCC visibility push(default)
#endif

typedef enum {
  GEMM_TYPE_F32 = 0,
  GEMM_TYPE_BF16 = 1
} gemm_type_t;

#define GEMM_Q8_BLOCK 32 /* consecutive values of a row that share an exponent */

/*
 * Layer norm of the rows of x: with mu and var the mean and the (biased)
 * variance of a row,
 *     y = (x - mu) * rstd * gamma + beta,   rstd = 1 / sqrt(var + eps),
 * computed in float32 (the variance from the differences x - mu; a mean far
 * above the deviations costs y none of their digits) and rounded once to y's
 * type.
 *   x: rows x cols, pitch ldx, of x_type.  y: rows x cols, pitch ldy, of
 *   y_type.  gamma, beta: cols values of param_type; NULL stands for ones and
 *   zeros.  eps >= 0.
 *   mean, rstd: rows float32 values each, kept for the backward pass; either
 *   may be NULL.
 *   q, ldq, e, lde: when q and e are not NULL, the checkpoint of y (as
 *   rounded to y_type), as gemm_q8_save writes it, in the same pass.
 * rows == 0 or cols == 0 is a no-op.
 */
gemm_status_t gemm_layernorm_forward(int64_t rows, int64_t cols, const void *x, int64_t ldx, int x_type,
                                     const void *gamma, const void *beta, int param_type, float eps,
                                     void *y, int64_t ldy, int y_type, float *mean, float *rstd,
                                     int8_t *q, int64_t ldq, uint8_t *e, int64_t lde, gemm_stream_t stream);

/*
 * Gradients of that layer norm.  With xh = (x - mean) * rstd and
 * g = dy * gamma, row by row,
 *     dx = rstd * (g - avg(g) - xh * avg(g * xh)),
 * and over the rows dgamma = sum(dy * xh), dbeta = sum(dy), all in float32.
 *   x: what the forward pass read, of x_type; or NULL, and then q and e hold
 *   its checkpoint (gemm_q8_save) and x_type, ldx are ignored.  Exactly one of
 *   the two forms is given.
 *   gamma: cols values of param_type; NULL stands for ones.  mean, rstd: as
 *   the forward pass wrote them.
 *   dy: rows x cols of dy_type, pitch lddy.  dx: rows x cols of dx_type,
 *   pitch lddx; dx_type is x_type where x is given.
 *   dgamma, dbeta: cols float32 values, overwritten; either may be NULL.
 * rows == 0 writes zeros to dgamma and dbeta; cols == 0 is a no-op.
 */
gemm_status_t gemm_layernorm_backward(int64_t rows, int64_t cols, const void *x, int64_t ldx, int x_type,
                                      const int8_t *q, int64_t ldq, const uint8_t *e, int64_t lde,
                                      const void *gamma, int param_type, const float *mean, const float *rstd,
                                      const void *dy, int64_t lddy, int dy_type, void *dx, int64_t lddx,
                                      int dx_type, float *dgamma, float *dbeta, gemm_stream_t stream);

/*
 * Checkpoint of the rows x cols matrix x (pitch ldx, of x_type) into q and e,
 * and the values it stands for (exact in float32, and in bf16 too) back into
 * x.  rows == 0 or cols == 0 is a no-op.
 */
gemm_status_t gemm_q8_save(int64_t rows, int64_t cols, const void *x, int64_t ldx, int x_type,
                           int8_t *q, int64_t ldq, uint8_t *e, int64_t lde, gemm_stream_t stream);
gemm_status_t gemm_q8_restore(int64_t rows, int64_t cols, const int8_t *q, int64_t ldq, const uint8_t *e,
                              int64_t lde, void *x, int64_t ldx, int x_type, gemm_stream_t stream);

/*
 * Weight gradient of the projection Y = X . W (X: T x K, W: K x N) from X's
 * checkpoint and Y's gradient:
 *     dW = base + X^T . dY,   dW(k, n) = base(k, n) + sum_t X(t, k) * dY(t, n),
 * with the products exact and summed in float32 (the base added last), then
 * rounded once to w_type.
 *   q, e: the checkpoint of X, T x K.  dY: T x N bf16 bit patterns, pitch
 *   lddy.
 *   dW: of w_type, in W's own layout: w_layout GEMM_B_ROW_MAJOR_KxN has
 *   dW(k, n) at dW[k * ldw + n], GEMM_B_COL_MAJOR_NxK at dW[n * ldw + k].
 *   base: NULL (zero), or a gradient of the same type and layout, pitch
 *   ldbase, to which this one is added; it may be dW itself (base == dW with
 *   ldbase == ldw), which accumulates over micro-batches.
 * T == 0 leaves dW = base (zero without one); K == 0 or N == 0 is a no-op.
 * Accuracy contract, per element, with ref the exact value and
 * S = |base| + sum_t |X(t, k) * dY(t, n)|:
 *     float32 dW:  |dW - ref| <= 2^-24 |ref| + c(512) S,
 *     bf16 dW:     |dW - ref| <= 2^-8 |ref| + c(8192) S,
 *     c(L) = (min(T, L) + T / L + 32) * 2^-24
 * (and the last rounding of that error).  The tensor core adds chains of L
 * tokens, cutting what lies below 2^-25 of the larger of the running sum and
 * the products; the chains are joined in float32 with round-to-nearest.  The
 * worst inputs have one large product among many small ones; of products
 * whose signs are random a float32 dW measures within 2^-20 S.
 */
gemm_status_t gemm_q8_weight_grad(int64_t T, int64_t K, int64_t N, const int8_t *q, int64_t ldq,
                                  const uint8_t *e, int64_t lde, const uint16_t *dY, int64_t lddy,
                                  const void *base, int64_t ldbase, void *dW, int64_t ldw, int w_layout,
                                  int w_type, gemm_stream_t stream);

#if defined(__GNUC__)
#pragma GCC visibility pop
#endif
#ifdef __cplusplus
}
#endif

#endif /* GB300_LAYER_H */
