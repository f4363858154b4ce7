/*
 * lqsgd_block.h -- C ABI of what stands around the linear layers of lqsgd_linear.h in a block, for MI355X (gfx950): the root-mean-square
 * norm with the residual's addition and its backward pass, rows kept in 8 bits with a scale each, the linear layer on such rows, and
 * dropout whose mask is never stored.  Calls take a context of lqsgd_linear.h; everything said there about types, strides, streams,
 * graphs, determinism and errors holds here.
 *
 *   rms norm            h = x + residual;  rstd = 1 / sqrt(mean over the features of h^2 + eps);  y = h rstd gain
 *   its backward        v = dy gain;  dx = rstd (v - h^ rstd^2 mean(v h^)) + dh;  dgain = sum over samples of dy h^ rstd
 *   8-bit linear layer  y = act(s_x s_w (sum of q_x q_w) + bias) + residual
 *   dropout             y = keep x / (1 - p) + residual
 *
 * 8-bit rows
 *   A tensor's row v is kept as integers and one scale s: s = max|v| (1 / 127), at least 2^-126, and a value's code is v (1 / s) rounded
 *   to the nearest integer, ties to even, with 1 / 127, 1 / s and both products rounded to fp32: |v - q s| <= (1/2 + 2^-16) s.  A row that holds a NaN or an
 *   infinity has a scale of NaN and codes of 0.  As the weight of a linear layer that is a scale an output feature, as its input a
 *   scale a sample.
 *     codes  : int8, samples x lqsgd_checkpoint_stride(features), 16-byte aligned; the codes behind the last feature are 0
 *     scales : float, samples
 *
 * Dropout's mask
 *   Each value has 16 bits of Philox 4x32 with 10 rounds (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2, 3",
 *   2011), of counter (feature / 8, sample, offset's low 32 bits, its high 32 bits) and key (seed's low 32 bits, its high 32 bits): value 2 k + h of
 *   a feature's eight has half h (0: the low one) of word k.  With t = p 65536 rounded to the nearest integer (ties to even) a value stays where its
 *   16 bits are t or more, times 65536 / (65536 - t); elsewhere it is 0, whatever x holds there.  The mask depends on seed, offset and
 *   the place in the tensor alone: not on types, strides or alignment.  The gradient of x is the same call on dy, without the residual.
 */
#ifndef LQSGD_BLOCK_H
#define LQSGD_BLOCK_H

#include <stdint.h>

#include "lqsgd_linear.h"

#ifdef __cplusplus
extern "C" {
#endif

#define LQSGD_INT8_MAX_COLS 131040    /* whatever the codes are, as many products add up within 32 bits */

/* x (samples x features, of `type`) into 8-bit rows, and back.  Errors of these and of the calls below: those of lqsgd_checkpoint_save. */
int lqsgd_rows_save(lqsgd_linear* ctx, int32_t type, int64_t samples, int32_t features, const void* x, int64_t ldx, int8_t* codes,
                    float* scales);
int lqsgd_rows_load(lqsgd_linear* ctx, int32_t type, int64_t samples, int32_t features, const int8_t* codes, const float* scales, void* x,
                    int64_t ldx);

/* The norm.  residual (samples x features) may be NULL: h is x then.  gain (features) may be NULL: ones.  What is wanted of
 *   h       x + residual, rounded to `type` before the norm is taken of it; needs a residual; may be x or the residual itself
 *           (same pointer, same ld)
 *   y       the norm
 *   rstd    float, samples: what the backward pass needs
 *   y_codes, y_exponents   a checkpoint of y as it was rounded to `type` (the bits that lqsgd_checkpoint_save of y gives)
 *   q_codes, q_scales      8-bit rows of h gain, the scales multiplied by rstd: those of y, without y's rounding
 * is not NULL; one of the last four at least.  eps: 0 or more, finite.  Squares are added up in fp64, where none overflows or is lost.
 * Where rstd is no normal fp32 number (mean h^2 + eps below 2^-252 or above 2^252), y and the 8-bit rows are made of h 2^k and rstd 2^-k, 2^k the power of
 * two below rstd (2^-126 to 2^126), and so are the 8-bit rows where |h gain| stays below 2^-119 and rstd is above 1, or h gain leaves fp32's
 * range and rstd is below 1: no digit of a small row is lost, and no large one overflows.  rstd itself is rounded to fp32; it is infinite up
 * to a mean of 2^-256, and the gradients that the backward pass makes with it are not finite.  A row of zeros with eps = 0 is NaN, as the
 * formula has it. */
int lqsgd_rms_norm(lqsgd_linear* ctx, int32_t type, int64_t samples, int32_t features, double eps, const void* x, int64_t ldx,
                   const void* residual, int64_t ldr, const void* gain, void* h, int64_t ldh, void* y, int64_t ldy, float* rstd,
                   int8_t* y_codes, uint8_t* y_exponents, int8_t* q_codes, float* q_scales);

/* The gradients of dy, and of dh, which came to h past the norm (NULL: nothing did): dx is the gradient of x and of the residual alike.  h^ is
 * given as a tensor (h) or as a checkpoint (h_codes, h_exponents; h NULL).  rstd is the forward pass's.  dx and dgain may be NULL (not
 * wanted), not both; dx may be dy or dh itself (same pointer, same ld).  dgain: float, features; accumulate != 0 adds to what it holds.  Sums are
 * fp32. */
int lqsgd_rms_norm_backward(lqsgd_linear* ctx, int32_t type, int64_t samples, int32_t features, const void* dy, int64_t lddy,
                            const void* h, int64_t ldh, const int8_t* h_codes, const uint8_t* h_exponents, const float* rstd,
                            const void* gain, const void* dh, int64_t lddh, void* dx, int64_t lddx, float* dgain, int32_t accumulate);

/* The linear layer on 8-bit rows: x samples x cols, w rows x cols, y (samples x rows), bias (rows) and residual of `type`; bias and residual
 * may be NULL, y may be the residual itself.  The sum of q_x q_w is exact, s_x s_w is rounded to fp32, the rest is fp32 and y is
 * rounded once.  ESHAPE also for more than LQSGD_INT8_MAX_COLS cols. */
int lqsgd_int8_forward(lqsgd_linear* ctx, int32_t type, int32_t act, int64_t samples, int32_t rows, int32_t cols, const int8_t* x_codes,
                       const float* x_scales, const int8_t* w_codes, const float* w_scales, const void* bias, const void* residual,
                       int64_t ldr, void* y, int64_t ldy);

/* p: 0 to 1.  residual may be NULL; y may be x or the residual itself (same pointer, same ld).  y_codes, y_exponents: NULL, or a checkpoint
 * of y as it was rounded.  more_offset: NULL, or device memory whose 64 bits are added to `offset` when the call runs, so that replays of a
 * graph have masks of their own (8-byte aligned). */
int lqsgd_dropout(lqsgd_linear* ctx, int32_t type, int64_t samples, int32_t features, double p, uint64_t seed, uint64_t offset,
                  const uint64_t* more_offset, const void* x, int64_t ldx, const void* residual, int64_t ldr, void* y, int64_t ldy,
                  int8_t* y_codes, uint8_t* y_exponents);

#ifdef __cplusplus
}
#endif
#endif /* LQSGD_BLOCK_H */
