/*
 * gb300_layer.h -- C ABI of the operators a training step runs around its
 * projection GEMMs (gb300_gemm.h): layer norm forward and backward, 8-bit
 * activation checkpoints, a projection's weight gradient taken from such
 * a checkpoint, the gated feed-forward block's two projections with their gate
 * and its gradient, and dropout.  With C = A . B of gb300_gemm.h they make a
 * pre-norm projection block, y = layer_norm(x), o = y . W, and its backward
 * pass dy = do . W^T, dW = y^T . do, dx = layer_norm'(dy); and a gated
 * feed-forward block (at the end of this file).
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

/*
 * Gated feed-forward block.  Of T tokens X (T x K), with the gate and up
 * projections Wg, Wu (K x F), the down projection Wd (F x N) and an activation
 * applied element by element,
 *
 *     G = X . Wg,  U = X . Wu,  H = act(G) * U,  O = H . Wd;
 *
 * back from dO,  dH = dO . Wd^T,  dG = dH * U * act'(G),  dU = dH * act(G).
 * The calls here take the projections with the gate, and the gate's gradient
 * with or without the down projection's product (those with a product use the
 * stream's scratch where rows are not 16-byte aligned and where a last round of
 * tiles is split); the rest are GEMMs and weight gradients above.  With Wg and Wu the halves of one K x 2F matrix W, and dG
 * and dU those of a T x 2F matrix, dX is one GEMM with W^T and dW one
 * gemm_q8_weight_grad.
 */
typedef enum {
  GEMM_ACT_SILU = 0,      /* g / (1 + exp(-g)) */
  GEMM_ACT_GELU = 1,      /* g * P(g), P the normal distribution function */
  GEMM_ACT_GELU_TANH = 2, /* g * (1 + tanh(sqrt(2 / pi) * (g + 0.044715 g^3))) / 2 */
  GEMM_ACT_RELU = 3       /* max(g, 0); slope 0 at 0 */
} gemm_activation_t;

/*
 * H = act(X . Wg) * (X . Wu), all bf16 bit patterns, for one token or many.
 *   X: T x K, pitch ldx.  Wg, Wu: of w_layout, a weight's layout as in the
 *   GEMM calls: GEMM_B_ROW_MAJOR_KxN has Wg(k, f) at Wg[k * ldwg + f],
 *   GEMM_B_COL_MAJOR_NxK at Wg[f * ldwg + k].
 *   H: T x F, pitch ldh.  G, U: T x F, pitches ldg, ldu, kept for the backward
 *   pass; both or neither.
 * The sums are float32, H is taken from them unrounded, and H, G and U are
 * rounded once.  T == 0 or F == 0 is a no-op; K == 0 writes zeros.
 * Accuracy contract, per element, with g, u the exact sums, Sg, Su those of
 * the products' magnitudes and c = (K + 32) * 2^-24:
 *     |G - g| <= 2^-8 |g| + c Sg,   |U - u| <= 2^-8 |u| + c Su,
 *     |H - act(g) u| <= 2^-8 |act(g) u| + c (1.13 Sg |u| + |act(g)| Su)
 *                       + 1.13 c^2 Sg Su + 2^-18 |g u|
 * (and the last rounding of that error).  As in the weight gradient, c allows
 * for what the tensor core cuts of its additions, worst for one large product
 * among many small ones; of products whose signs are random the sums measure
 * within 2^-20 Sg.  1.13 is the activations' largest slope.  Infinite or NaN
 * sums give what the formulas give in float32: act of -infinity is NaN, except
 * of relu.
 */
gemm_status_t gemm_gated_forward(int64_t T, int64_t K, int64_t F, const uint16_t *X, int64_t ldx,
                                 const uint16_t *Wg, int64_t ldwg, const uint16_t *Wu, int64_t ldwu, int w_layout,
                                 int activation, uint16_t *H, int64_t ldh, uint16_t *G, int64_t ldg, uint16_t *U,
                                 int64_t ldu, gemm_stream_t stream);

/*
 * The gate's gradient from dH: dG = dH * U * act'(G), dU = dH * act(G), in
 * float32, each rounded once to bf16.
 *   dH, G, U: T x F bf16, pitches lddh, ldg, ldu.  dG, dU: T x F bf16, pitches
 *   lddg, lddu; dG may be G and dU may be U (the same address and pitch).
 *   q, ldq, e, lde: when q and e are not NULL, the checkpoint of the float32
 *   values act(G) * U, as gemm_q8_save writes it: H for the down projection's
 *   weight gradient, dWd = H^T . dO, without H having been kept.
 * act and act' are off by at most 2^-18 |G| and 2^-18 before the products.
 * T == 0 or F == 0 is a no-op.
 */
gemm_status_t gemm_gated_backward(int64_t T, int64_t F, const uint16_t *dH, int64_t lddh, const uint16_t *G,
                                  int64_t ldg, const uint16_t *U, int64_t ldu, int activation, uint16_t *dG,
                                  int64_t lddg, uint16_t *dU, int64_t lddu, int8_t *q, int64_t ldq, uint8_t *e,
                                  int64_t lde, gemm_stream_t stream);

/*
 * The same with dH = dO . Wd^T taken in the same kernel, in float32 and not
 * rounded in between; dH is off by at most (N + 32) * 2^-24 of its products'
 * magnitudes' sum.
 *   dO: T x N bf16, pitch lddo.  Wd: the down projection, O = H . Wd, of
 *   w_layout: GEMM_B_ROW_MAJOR_KxN has Wd(f, n) at Wd[f * ldwd + n],
 *   GEMM_B_COL_MAJOR_NxK at Wd[n * ldwd + f].
 * N == 0 takes dH as zero.
 */
gemm_status_t gemm_gated_down_backward(int64_t T, int64_t N, int64_t F, const uint16_t *dO, int64_t lddo,
                                       const uint16_t *Wd, int64_t ldwd, int w_layout, const uint16_t *G, int64_t ldg,
                                       const uint16_t *U, int64_t ldu, int activation, uint16_t *dG, int64_t lddg,
                                       uint16_t *dU, int64_t lddu, int8_t *q, int64_t ldq, uint8_t *e, int64_t lde,
                                       gemm_stream_t stream);

/*
 * Dropout, into a residual stream if asked, and its gradient:
 *     y = residual + keep * x / (1 - P),    dx = keep * dy / (1 - P),
 * in float32, rounded once.  What is kept is a function of (seed, the call's
 * step, row, column) alone -- not of types, pitches or the launch -- so that
 * the backward pass finds it again and no mask is stored.
 *   p: 0 .. 1, taken as the nearest multiple P of 1 / 65536 (ties to even);
 *   P = 1 keeps nothing.  A value that is not kept contributes 0 whatever it
 *   is, a NaN included.
 *   seed: the generator's key.  The call's step is `step`, plus *step_device
 *   where that is not NULL: 8 bytes of device memory (8-byte aligned) read
 *   when the kernel runs, so that a captured graph draws anew at each launch
 *   if something on its stream counts the word up between them.  The two add
 *   modulo 2^64.
 *   x: rows x cols of x_type, pitch ldx.  residual: rows x cols of y_type,
 *   pitch ldr, or NULL (zero).  y: rows x cols of y_type, pitch ldy; it may be
 *   the residual, or x where the types are the same (the same address and
 *   pitch).  dy, dx: of dy_type, dx_type; dx may be dy likewise.  The residual's
 *   gradient is dy itself.
 * rows == 0 or cols == 0 is a no-op.
 * The generator is Philox4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel
 * random numbers: as easy as 1, 2, 3", 2011) with key (low, high word of seed)
 * and counter (column / 8, row, low, high word of the step): bits 16 i .. 16 i
 * + 15 of its 128 are the number of the value in column 8 * (column / 8) + i,
 * which is kept where that number is at least 65536 P.
 */
gemm_status_t gemm_dropout_forward(int64_t rows, int64_t cols, const void *x, int64_t ldx, int x_type,
                                   const void *residual, int64_t ldr, void *y, int64_t ldy, int y_type, float p,
                                   uint64_t seed, uint64_t step, const uint64_t *step_device, gemm_stream_t stream);
gemm_status_t gemm_dropout_backward(int64_t rows, int64_t cols, const void *dy, int64_t lddy, int dy_type, void *dx,
                                    int64_t lddx, int dx_type, float p, uint64_t seed, uint64_t step,
                                    const uint64_t *step_device, gemm_stream_t stream);

#if defined(__GNUC__)
#pragma GCC visibility pop
#endif
#ifdef __cplusplus
}
#endif

#endif /* GB300_LAYER_H */
