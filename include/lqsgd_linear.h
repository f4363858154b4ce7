/*
 * lqsgd_linear.h -- C ABI of the linear layer whose gradients the compressor of lqsgd.h takes, for MI355X (gfx950).
 *
 * x is samples x cols, w is rows x cols (a layer of lqsgd.h: rows = output features, cols = input features), y is samples x rows:
 *
 *   forward              z = x w^T + bias;   y = act(z) + residual            (z and y may be kept in 8 bits beside y)
 *   activation backward  dz = dy act'(z^);   dbias = sum over samples of dy act'(z^)
 *   weight gradient      dw = dz^T x^        (rows x cols, fp32 or bfloat16: a gradient tensor of lqsgd_step)
 *   input gradient       dx = dz w
 *
 * where z^ and x^ are what 8-bit checkpoints of z and x stand for.
 *
 * Checkpoints
 *   A checkpoint keeps a samples x features tensor in 8 bits and a 32nd of a byte per value.  Each sample's features go in groups
 *   of 32 (the last group may be shorter); a group shares a power of two 2^e and a value v is kept as the integer code
 *   q = v / 2^e rounded to nearest, ties to even, -127 <= q <= 127; it stands for q 2^e.  e is the smallest integer for which the
 *   group's largest magnitude is below 127.5 * 2^e, held to -126..121 (LQSGD_TYPE_F16: -24..9), so that every q 2^e is a number of
 *   the type it was saved from and reading a checkpoint back rounds nothing: |v - q 2^e| <= 2^e / 2, except where the upper bound
 *   of e takes effect (up to 2^e there; a z beyond half's range is kept as 127 2^9).  A group that holds a NaN or an infinity is kept as NaN in all its values.
 *     codes      : int8, samples x lqsgd_checkpoint_stride(features), 16-byte aligned; the codes behind the last feature are 0
 *     exponents  : uint8, samples x lqsgd_checkpoint_stride(features) / 32: e + 127, or 255 for NaN
 *
 * Conventions (those of lqsgd.h, and)
 *   - Tensors are row-major device memory; ld* is the distance between rows in elements, at least the row's length; elements of a
 *     row are contiguous.  Any alignment that the type itself needs will do; rows that start at multiples of 16 bytes are faster.
 *   - LQSGD_TYPE_F32, _BF16 or _F16 is the type of x, w, bias, residual, y, dy, dz and dx of one call.  Products are accumulated in
 *     fp32, bias, activation, residual and sums are fp32, and each output is rounded once (to nearest even).
 *   - samples may be 0: nothing is written then, except that sums over no samples are 0.
 *   - Outputs must not overlap inputs or each other, with two exceptions: y may be the residual itself and dz may be dy itself (same
 *     pointer, same ld).  An output that starts where an input or another output does is refused otherwise (EINVAL; checkpoints' codes and
 *     exponents are inputs and outputs too); an overlap of another kind is not looked for.
 *   - Results are the same bits from run to run: nothing is added in an order that depends on timing.
 *   - NaN and infinities go the way of the formulas, with two exceptions.  LQSGD_TYPE_F32 products are made from operands split
 *     into three bfloat16 terms: an infinite operand may make the outputs it reaches NaN instead of infinite, and operands are taken
 *     to multiples of 2^-133 (magnitudes below 2^-109 lose their last bits).  A checkpoint reads back as above.
 *   - A call only enqueues kernels on the context's stream; it neither allocates nor waits.  It may be captured into a HIP graph, whose
 *     replays use the context's workspace like the call itself: order replays, on whatever stream they run, with one another and with
 *     the context's other calls.  Work that is to run side by side takes a context each (two users of one workspace at a time add up
 *     each other's sums).  A context has to live as long as the graphs that hold calls of it are replayed.
 */
#ifndef LQSGD_LINEAR_H
#define LQSGD_LINEAR_H

#include <stdint.h>

#include "lqsgd.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct lqsgd_linear lqsgd_linear;

#define LQSGD_TYPE_F32 0
#define LQSGD_TYPE_BF16 1
#define LQSGD_TYPE_F16 2

#define LQSGD_ACT_NONE 0
#define LQSGD_ACT_RELU 1   /* max(z, 0); slope 1 for z > 0, else 0     */
#define LQSGD_ACT_GELU 2   /* z Phi(z), Phi the normal distribution's  */
#define LQSGD_ACT_SILU 3   /* z / (1 + exp(-z))                        */

#define LQSGD_LINEAR_MAX_FEATURES (1 << 20)  /* rows, cols              */
#define LQSGD_LINEAR_MAX_STRIDE (1 << 21)    /* ld*, in elements        */
#define LQSGD_LINEAR_MAX_SAMPLES (1 << 30)       /* and an output of forward, input_grad or weight_grad that is longer than 2^36
                                                     values may be refused (ESHAPE) */

/* A context on the current HIP device: the stream its calls run on (a hipStream_t, NULL = the default stream) and 64 MiB of
 * workspace, which the calls share: work of one context is ordered by its stream, replays of graphs by the caller.  Not thread-safe.
 * Errors: EINVAL, ENOMEM, EHIP. */
int lqsgd_linear_create(void* hip_stream, lqsgd_linear** out);
/* Waits for the stream and frees everything, also what graphs of its calls would use; NULL is accepted. */
int lqsgd_linear_destroy(lqsgd_linear* ctx);
/* Waits for the context's stream. */
int lqsgd_linear_synchronize(lqsgd_linear* ctx);
/* Text for the most recent error on ctx (NULL: of a failed lqsgd_linear_create, or of a call without a context). */
const char* lqsgd_linear_last_error(const lqsgd_linear* ctx);

/* Bytes of codes that one sample of `features` takes: features rounded up to a multiple of 32; or a negative status. */
int64_t lqsgd_checkpoint_stride(int32_t features);

/* x (samples x features, of `type`) into a checkpoint, and back; loading into a type other than the one it was saved from rounds
 * to nearest.  Errors of these and of the calls below: EINVAL (NULL, unknown type or activation, pointers that are not aligned to
 * their type, codes not aligned to 16 bytes, an output at the address of an input or another output), ESHAPE (sizes or strides out of range), EHIP. */
int lqsgd_checkpoint_save(lqsgd_linear* ctx, int32_t type, int64_t samples, int32_t features, const void* x, int64_t ldx,
                          int8_t* codes, uint8_t* exponents);
int lqsgd_checkpoint_load(lqsgd_linear* ctx, int32_t type, int64_t samples, int32_t features, const int8_t* codes,
                          const uint8_t* exponents, void* x, int64_t ldx);

/* y = act(x w^T + bias) + residual.  bias (rows) and residual (samples x rows) may be NULL.  z_codes / z_exponents: NULL, or a
 * checkpoint (samples x rows) that receives z in fp32, before the activation; y_codes / y_exponents: the same for y as it was
 * rounded to `type` (the bits that lqsgd_checkpoint_save of y gives): the next layer's x^. */
int lqsgd_linear_forward(lqsgd_linear* ctx, int32_t type, int32_t act, int64_t samples, int32_t rows, int32_t cols, const void* x,
                         int64_t ldx, const void* w, int64_t ldw, const void* bias, const void* residual, int64_t ldr, void* y,
                         int64_t ldy, int8_t* z_codes, uint8_t* z_exponents, int8_t* y_codes, uint8_t* y_exponents);

/* dz = dy act'(z^) (NULL: not wanted) and dbias = its sum over the samples, in fp32 from values not yet rounded (NULL: not wanted);
 * accumulate != 0 adds to what dbias holds.  With LQSGD_ACT_NONE the checkpoint is not read and may be NULL.  A NaN in z^ makes dz
 * NaN for every activation that reads it. */
int lqsgd_linear_activation_backward(lqsgd_linear* ctx, int32_t type, int32_t act, int64_t samples, int32_t rows, const void* dy,
                                     int64_t lddy, const int8_t* z_codes, const uint8_t* z_exponents, void* dz, int64_t lddz,
                                     float* dbias, int32_t accumulate);

/* dx = dz w. */
int lqsgd_linear_input_grad(lqsgd_linear* ctx, int32_t type, int64_t samples, int32_t rows, int32_t cols, const void* dz, int64_t lddz,
                            const void* w, int64_t ldw, void* dx, int64_t lddx);

/* dw = dz^T x^, x^ a checkpoint of samples x cols saved from a tensor of `type` (one of another type is rounded to it);
 * grad_type: LQSGD_TYPE_F32, or LQSGD_TYPE_BF16 (what a compressor with LQSGD_FLAG_BF16_GRADIENTS takes).  accumulate != 0 adds
 * to what dw holds, in fp32 before the rounding. */
int lqsgd_linear_weight_grad(lqsgd_linear* ctx, int32_t type, int64_t samples, int32_t rows, int32_t cols, const void* dz, int64_t lddz,
                             const int8_t* x_codes, const uint8_t* x_exponents, int32_t grad_type, void* dw, int64_t lddw,
                             int32_t accumulate);

#ifdef __cplusplus
}
#endif
#endif /* LQSGD_LINEAR_H */
