// C ABI of what stands around the linear layer: argument checks and launches.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "lqsgd_block.h"
#include "lqsgd_block_kernels.h"
#include "lqsgd_linear_context.h"

using namespace lqsgd::linear;

namespace {

constexpr const char kBadRows[] = "8-bit rows need both of their pointers, codes aligned to 16 bytes and scales to 4";

bool rows_ok(const void* codes, const void* scales, bool optional) {
  if (!codes || !scales) return optional && !codes && !scales;
  return aligned(codes, 16) && aligned(scales, 4);
}

}  // namespace

extern "C" {

int lqsgd_rows_save(lqsgd_linear* c, int32_t type, int64_t samples, int32_t features, const void* x, int64_t ldx, int8_t* codes, float* scales) {
  if (!c) return fail(nullptr, LQSGD_EINVAL, kNull);
  if (!known_type(type)) return fail(c, LQSGD_EINVAL, kBadType);
  if (!samples_ok(samples) || !features_ok(features) || !stride_ok(ldx, features)) return fail(c, LQSGD_ESHAPE, kBadSize);
  if (samples == 0) return LQSGD_OK;
  if (!x) return fail(c, LQSGD_EINVAL, kNull);
  if (!aligned(x, size_of(type))) return fail(c, LQSGD_EINVAL, kBadAlign);
  if (!rows_ok(codes, scales, false)) return fail(c, LQSGD_EINVAL, kBadRows);
  if (lies_over({codes, scales}, {x})) return fail(c, LQSGD_EINVAL, kOver);
  return done(c, launch_rows_save(type, samples, features, x, ldx, Rows{codes, scales}, c->stream), "lqsgd_rows_save");
}

int lqsgd_rows_load(lqsgd_linear* c, int32_t type, int64_t samples, int32_t features, const int8_t* codes, const float* scales, void* x,
                    int64_t ldx) {
  if (!c) return fail(nullptr, LQSGD_EINVAL, kNull);
  if (!known_type(type)) return fail(c, LQSGD_EINVAL, kBadType);
  if (!samples_ok(samples) || !features_ok(features) || !stride_ok(ldx, features)) return fail(c, LQSGD_ESHAPE, kBadSize);
  if (samples == 0) return LQSGD_OK;
  if (!x) return fail(c, LQSGD_EINVAL, kNull);
  if (!aligned(x, size_of(type))) return fail(c, LQSGD_EINVAL, kBadAlign);
  if (!rows_ok(codes, scales, false)) return fail(c, LQSGD_EINVAL, kBadRows);
  if (lies_over({x}, {codes, scales})) return fail(c, LQSGD_EINVAL, kOver);
  const Rows rows{const_cast<int8_t*>(codes), const_cast<float*>(scales)};
  return done(c, launch_rows_load(type, samples, features, rows, x, ldx, c->stream), "lqsgd_rows_load");
}

int lqsgd_rms_norm(lqsgd_linear* c, int32_t type, int64_t samples, int32_t features, double eps, const void* x, int64_t ldx,
                   const void* residual, int64_t ldr, const void* gain, void* h, int64_t ldh, void* y, int64_t ldy, float* rstd,
                   int8_t* y_codes, uint8_t* y_exponents, int8_t* q_codes, float* q_scales) {
  if (!c) return fail(nullptr, LQSGD_EINVAL, kNull);
  if (!known_type(type)) return fail(c, LQSGD_EINVAL, kBadType);
  if (!samples_ok(samples) || !features_ok(features) || !stride_ok(ldx, features) || (residual && !stride_ok(ldr, features)) ||
      (h && !stride_ok(ldh, features)) || (y && !stride_ok(ldy, features)))
    return fail(c, LQSGD_ESHAPE, kBadSize);
  if (!(eps >= 0.0) || !std::isfinite(eps)) return fail(c, LQSGD_EINVAL, "eps has to be 0 or more, and finite");
  if (h && !residual) return fail(c, LQSGD_EINVAL, "h is wanted without a residual: it is x");
  if (samples == 0) return LQSGD_OK;
  if (!x) return fail(c, LQSGD_EINVAL, kNull);
  if (!y && !rstd && !y_codes && !q_codes) return fail(c, LQSGD_EINVAL, "neither y nor rstd, a checkpoint or 8-bit rows of y are wanted");
  const uintptr_t s = size_of(type);
  if (!aligned(x, s) || !aligned(residual, s) || !aligned(gain, s) || !aligned(h, s) || !aligned(y, s) || !aligned(rstd, 4))
    return fail(c, LQSGD_EINVAL, kBadAlign);
  if (!codes_ok(y_codes, y_exponents, true)) return fail(c, LQSGD_EINVAL, kBadCodes);
  if (!rows_ok(q_codes, q_scales, true)) return fail(c, LQSGD_EINVAL, kBadRows);
  if (lies_over({h, y, rstd, y_codes, y_exponents, q_codes, q_scales}, {gain}) ||
      lies_over({y, rstd, y_codes, y_exponents, q_codes, q_scales}, {x, residual}))
    return fail(c, LQSGD_EINVAL, kOver);
  if (h && ((h == x && ldh != ldx) || (h == residual && ldh != ldr)))
    return fail(c, LQSGD_EINVAL, "h is x or the residual, with another stride");
  NormArgs a{};
  a.samples = samples; a.features = features; a.eps = eps;
  a.x = x; a.ldx = ldx; a.residual = residual; a.ldr = ldr; a.gain = gain;
  a.h = h; a.ldh = ldh; a.y = y; a.ldy = ldy; a.rstd = rstd;
  a.kept = Codes{y_codes, y_exponents}; a.rows = Rows{q_codes, q_scales};
  return done(c, launch_rms_norm(type, a, c->stream), "lqsgd_rms_norm");
}

int lqsgd_rms_norm_backward(lqsgd_linear* c, int32_t type, int64_t samples, int32_t features, const void* dy, int64_t lddy, const void* h,
                            int64_t ldh, const int8_t* h_codes, const uint8_t* h_exponents, const float* rstd, const void* gain,
                            const void* dh, int64_t lddh, void* dx, int64_t lddx, float* dgain, int32_t accumulate) {
  if (!c) return fail(nullptr, LQSGD_EINVAL, kNull);
  if (!known_type(type)) return fail(c, LQSGD_EINVAL, kBadType);
  if (!samples_ok(samples) || !features_ok(features) || !stride_ok(lddy, features) || (h && !stride_ok(ldh, features)) ||
      (dh && !stride_ok(lddh, features)) || (dx && !stride_ok(lddx, features)))
    return fail(c, LQSGD_ESHAPE, kBadSize);
  if (!dx && !dgain) return fail(c, LQSGD_EINVAL, "neither dx nor dgain is wanted");
  const uintptr_t s = size_of(type);
  if (!aligned(dy, s) || !aligned(h, s) || !aligned(rstd, 4) || !aligned(gain, s) || !aligned(dh, s) || !aligned(dx, s) || !aligned(dgain, 4))
    return fail(c, LQSGD_EINVAL, kBadAlign);
  if (samples > 0) {
    if (!dy || !rstd) return fail(c, LQSGD_EINVAL, kNull);
    if (!h == !h_codes) return fail(c, LQSGD_EINVAL, "h is given as a tensor or as a checkpoint");
    if (!codes_ok(h_codes, h_exponents, true)) return fail(c, LQSGD_EINVAL, kBadCodes);
    if (lies_over({dx, dgain}, {h, h_codes, h_exponents, rstd, gain}) || lies_over({dgain}, {dy, dh})) return fail(c, LQSGD_EINVAL, kOver);
    if (dx && ((dx == dy && lddx != lddy) || (dx == dh && lddx != lddh)))
      return fail(c, LQSGD_EINVAL, "dx is dy or dh, with another stride");
  }
  if (samples == 0 && (!dgain || accumulate)) return LQSGD_OK;
  NormBackwardArgs a{};
  a.samples = samples; a.features = features;
  a.dy = dy; a.lddy = lddy; a.h = h; a.ldh = ldh;
  a.held = Codes{const_cast<int8_t*>(h_codes), const_cast<uint8_t*>(h_exponents)};
  a.rstd = rstd; a.gain = gain; a.dh = dh; a.lddh = lddh; a.dx = dx; a.lddx = lddx;
  a.dgain = dgain; a.accumulate = accumulate != 0; a.workspace = c->workspace; a.arrived = c->arrived;
  return done(c, launch_rms_norm_backward(type, a, c->stream), "lqsgd_rms_norm_backward");
}

int lqsgd_int8_forward(lqsgd_linear* c, int32_t type, int32_t act, int64_t samples, int32_t rows, int32_t cols, const int8_t* x_codes,
                       const float* x_scales, const int8_t* w_codes, const float* w_scales, const void* bias, const void* residual,
                       int64_t ldr, void* y, int64_t ldy) {
  if (!c) return fail(nullptr, LQSGD_EINVAL, kNull);
  if (!known_type(type) || act < LQSGD_ACT_NONE || act > LQSGD_ACT_SILU) return fail(c, LQSGD_EINVAL, kBadType);
  if (!samples_ok(samples) || !features_ok(rows) || !features_ok(cols) || cols > LQSGD_INT8_MAX_COLS || !stride_ok(ldy, rows) ||
      (residual && !stride_ok(ldr, rows)) || !output_ok(rows, samples))
    return fail(c, LQSGD_ESHAPE, kBadSize);
  if (samples == 0) return LQSGD_OK;
  if (!y) return fail(c, LQSGD_EINVAL, kNull);
  const uintptr_t s = size_of(type);
  if (!aligned(bias, s) || !aligned(residual, s) || !aligned(y, s)) return fail(c, LQSGD_EINVAL, kBadAlign);
  if (!rows_ok(x_codes, x_scales, false) || !rows_ok(w_codes, w_scales, false)) return fail(c, LQSGD_EINVAL, kBadRows);
  if (lies_over({y}, {x_codes, x_scales, w_codes, w_scales, bias})) return fail(c, LQSGD_EINVAL, kOver);
  if (residual == y && ldr != ldy) return fail(c, LQSGD_EINVAL, "y is the residual, with another stride");
  Int8Args a{};
  a.ni = rows; a.nj = samples; a.stride = (cols + kGroup - 1) / kGroup * kGroup;
  a.a = w_codes; a.scales_a = w_scales; a.b = x_codes; a.scales_b = x_scales;
  a.bias = bias; a.residual = residual; a.ldr = ldr; a.act = act;
  a.out = y; a.ldo = ldy; a.workspace = c->workspace; a.arrived = c->arrived;
  return done(c, launch_int8_product(type, a, c->stream), "lqsgd_int8_forward");
}

int lqsgd_dropout(lqsgd_linear* c, int32_t type, int64_t samples, int32_t features, double p, uint64_t seed, uint64_t offset,
                  const uint64_t* more_offset, const void* x, int64_t ldx, const void* residual, int64_t ldr, void* y, int64_t ldy,
                  int8_t* y_codes, uint8_t* y_exponents) {
  if (!c) return fail(nullptr, LQSGD_EINVAL, kNull);
  if (!known_type(type)) return fail(c, LQSGD_EINVAL, kBadType);
  if (!(p >= 0.0 && p <= 1.0)) return fail(c, LQSGD_EINVAL, "p has to be from 0 to 1");
  if (!samples_ok(samples) || !features_ok(features) || !stride_ok(ldx, features) || !stride_ok(ldy, features) ||
      (residual && !stride_ok(ldr, features)))
    return fail(c, LQSGD_ESHAPE, kBadSize);
  if (samples == 0) return LQSGD_OK;
  if (!x || !y) return fail(c, LQSGD_EINVAL, kNull);
  const uintptr_t s = size_of(type);
  if (!aligned(x, s) || !aligned(residual, s) || !aligned(y, s) || !aligned(more_offset, 8)) return fail(c, LQSGD_EINVAL, kBadAlign);
  if (!codes_ok(y_codes, y_exponents, true)) return fail(c, LQSGD_EINVAL, kBadCodes);
  if (lies_over({y, y_codes, y_exponents}, {more_offset}) || lies_over({y_codes, y_exponents}, {x, residual}))
    return fail(c, LQSGD_EINVAL, kOver);
  if ((y == x && ldy != ldx) || (y == residual && ldy != ldr)) return fail(c, LQSGD_EINVAL, "y is x or the residual, with another stride");
  DropoutArgs a{};
  a.samples = samples; a.features = features;
  a.least = (uint32_t)std::rint(p * 65536.0);
  a.factor = a.least < 65536u ? 65536.f / (float)(65536u - a.least) : 0.f;
  a.seed = seed; a.offset = offset; a.more_offset = more_offset;
  a.x = x; a.ldx = ldx; a.residual = residual; a.ldr = ldr; a.y = y; a.ldy = ldy; a.kept = Codes{y_codes, y_exponents};
  return done(c, launch_dropout(type, a, c->stream), "lqsgd_dropout");
}

}  // extern "C"
