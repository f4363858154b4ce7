// C ABI of the linear layer: argument checks and launches.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <cstdio>
#include <new>
#include <string>

#include "lqsgd_linear_context.h"

using namespace lqsgd::linear;

namespace lqsgd {
namespace linear {
namespace {
thread_local std::string g_error;
}  // namespace

int fail(lqsgd_linear* c, int code, const char* msg) {
  try {
    (c ? c->err : g_error) = msg;
  } catch (...) {      // no memory for the text: the status says what it can
  }
  return code;
}

int done(lqsgd_linear* c, hipError_t e, const char* what) {
  if (e == hipSuccess) return LQSGD_OK;
  (void)hipGetLastError();                         // a later call does not report it again
  char buf[256];
  std::snprintf(buf, sizeof buf, "%s: %s", what, hipGetErrorString(e));
  return fail(c, LQSGD_EHIP, buf);
}

}  // namespace linear
}  // namespace lqsgd

extern "C" {

int lqsgd_linear_create(void* hip_stream, lqsgd_linear** out) {
  if (!out) return fail(nullptr, LQSGD_EINVAL, kNull);
  *out = nullptr;
  lqsgd_linear* c = new (std::nothrow) lqsgd_linear;
  if (!c) return fail(nullptr, LQSGD_ENOMEM, "out of host memory");
  c->stream = static_cast<hipStream_t>(hip_stream);
  hipError_t e = hipMalloc(&c->workspace, kWorkspaceBytes + kTiles * sizeof(int) + kSlopeFloats * sizeof(float));
  if (e != hipSuccess) {
    delete c;
    const int rc = done(nullptr, e, "hipMalloc of the workspace");
    return e == hipErrorOutOfMemory ? LQSGD_ENOMEM : rc;
  }
  c->arrived = reinterpret_cast<int*>(static_cast<char*>(c->workspace) + kWorkspaceBytes);
  c->slopes = reinterpret_cast<float*>(c->arrived + kTiles);
  e = launch_prepare(c->slopes, c->arrived, c->stream);
  if (e != hipSuccess) {
    (void)hipFree(c->workspace);
    delete c;
    return done(nullptr, e, "preparing the workspace");
  }
  *out = c;
  return LQSGD_OK;
}

int lqsgd_linear_destroy(lqsgd_linear* c) {
  if (!c) return LQSGD_OK;
  hipError_t e = hipStreamSynchronize(c->stream);
  hipError_t f = hipFree(c->workspace);
  delete c;
  return done(nullptr, e != hipSuccess ? e : f, "lqsgd_linear_destroy");
}

int lqsgd_linear_synchronize(lqsgd_linear* c) {
  if (!c) return fail(nullptr, LQSGD_EINVAL, kNull);
  return done(c, hipStreamSynchronize(c->stream), "hipStreamSynchronize");
}

const char* lqsgd_linear_last_error(const lqsgd_linear* c) { return c ? c->err.c_str() : g_error.c_str(); }

int64_t lqsgd_checkpoint_stride(int32_t features) {
  if (!features_ok(features)) return LQSGD_ESHAPE;
  return ((int64_t)features + kGroup - 1) / kGroup * kGroup;
}

int lqsgd_checkpoint_save(lqsgd_linear* c, int32_t type, int64_t samples, int32_t features, const void* x, int64_t ldx, int8_t* codes,
                          uint8_t* exponents) {
  if (!c) return fail(nullptr, LQSGD_EINVAL, kNull);
  if (!known_type(type)) return fail(c, LQSGD_EINVAL, kBadType);
  if (!samples_ok(samples) || !features_ok(features) || !stride_ok(ldx, features)) return fail(c, LQSGD_ESHAPE, kBadSize);
  if (samples == 0) return LQSGD_OK;
  if (!x) return fail(c, LQSGD_EINVAL, kNull);
  if (!aligned(x, size_of(type))) return fail(c, LQSGD_EINVAL, kBadAlign);
  if (!codes_ok(codes, exponents, false)) return fail(c, LQSGD_EINVAL, kBadCodes);
  if (lies_over({codes, exponents}, {x})) return fail(c, LQSGD_EINVAL, kOver);
  return done(c, launch_checkpoint_save(type, samples, features, x, ldx, Codes{codes, exponents}, c->stream), "lqsgd_checkpoint_save");
}

int lqsgd_checkpoint_load(lqsgd_linear* c, int32_t type, int64_t samples, int32_t features, const int8_t* codes, const uint8_t* exponents,
                          void* x, int64_t ldx) {
  if (!c) return fail(nullptr, LQSGD_EINVAL, kNull);
  if (!known_type(type)) return fail(c, LQSGD_EINVAL, kBadType);
  if (!samples_ok(samples) || !features_ok(features) || !stride_ok(ldx, features)) return fail(c, LQSGD_ESHAPE, kBadSize);
  if (samples == 0) return LQSGD_OK;
  if (!x) return fail(c, LQSGD_EINVAL, kNull);
  if (!aligned(x, size_of(type))) return fail(c, LQSGD_EINVAL, kBadAlign);
  if (!codes_ok(codes, exponents, false)) return fail(c, LQSGD_EINVAL, kBadCodes);
  if (lies_over({x}, {codes, exponents})) return fail(c, LQSGD_EINVAL, kOver);
  const Codes held{const_cast<int8_t*>(codes), const_cast<uint8_t*>(exponents)};
  return done(c, launch_checkpoint_load(type, samples, features, held, x, ldx, c->stream), "lqsgd_checkpoint_load");
}

int lqsgd_linear_forward(lqsgd_linear* c, int32_t type, int32_t act, int64_t samples, int32_t rows, int32_t cols, const void* x, int64_t ldx,
                         const void* w, int64_t ldw, const void* bias, const void* residual, int64_t ldr, void* y, int64_t ldy,
                         int8_t* z_codes, uint8_t* z_exponents, int8_t* y_codes, uint8_t* y_exponents) {
  if (!c) return fail(nullptr, LQSGD_EINVAL, kNull);
  if (!known_type(type) || act < LQSGD_ACT_NONE || act > LQSGD_ACT_SILU) return fail(c, LQSGD_EINVAL, kBadType);
  if (!samples_ok(samples) || !features_ok(rows) || !features_ok(cols) || !stride_ok(ldx, cols) || !stride_ok(ldw, cols) ||
      !stride_ok(ldy, rows) || (residual && !stride_ok(ldr, rows)))
    return fail(c, LQSGD_ESHAPE, kBadSize);
  if (!output_ok(rows, samples)) return fail(c, LQSGD_ESHAPE, kBadSize);
  if (samples == 0) return LQSGD_OK;
  if (!x || !w || !y) return fail(c, LQSGD_EINVAL, kNull);
  const uintptr_t s = size_of(type);
  if (!aligned(x, s) || !aligned(w, s) || !aligned(bias, s) || !aligned(residual, s) || !aligned(y, s)) return fail(c, LQSGD_EINVAL, kBadAlign);
  if (!codes_ok(z_codes, z_exponents, true) || !codes_ok(y_codes, y_exponents, true)) return fail(c, LQSGD_EINVAL, kBadCodes);
  if (lies_over({y, z_codes, z_exponents, y_codes, y_exponents}, {x, w, bias}) ||
      lies_over({z_codes, z_exponents, y_codes, y_exponents}, {residual}))
    return fail(c, LQSGD_EINVAL, kOver);
  if (residual == y && ldr != ldy) return fail(c, LQSGD_EINVAL, "y is the residual, with another stride");
  ProductArgs a{};
  a.ni = rows; a.nj = samples; a.depth = cols;
  a.a = w; a.lda = ldw; a.b = x; a.ldb = ldx;
  a.bias = bias; a.residual = residual; a.ldr = ldr; a.act = act;
  a.z = Codes{z_codes, z_exponents}; a.y = Codes{y_codes, y_exponents};
  a.out = y; a.ldo = ldy; a.workspace = c->workspace; a.arrived = c->arrived;
  return done(c, launch_product(kForward, type, a, c->stream), "lqsgd_linear_forward");
}

int lqsgd_linear_activation_backward(lqsgd_linear* c, int32_t type, int32_t act, int64_t samples, int32_t rows, const void* dy, int64_t lddy,
                                     const int8_t* z_codes, const uint8_t* z_exponents, void* dz, int64_t lddz, float* dbias,
                                     int32_t accumulate) {
  if (!c) return fail(nullptr, LQSGD_EINVAL, kNull);
  if (!known_type(type) || act < LQSGD_ACT_NONE || act > LQSGD_ACT_SILU) return fail(c, LQSGD_EINVAL, kBadType);
  if (!samples_ok(samples) || !features_ok(rows) || !stride_ok(lddy, rows) || (dz && !stride_ok(lddz, rows)))
    return fail(c, LQSGD_ESHAPE, kBadSize);
  if (!dz && !dbias) return fail(c, LQSGD_EINVAL, "neither dz nor dbias is wanted");
  if (samples > 0) {
    if (!dy) return fail(c, LQSGD_EINVAL, kNull);
    if (!codes_ok(z_codes, z_exponents, act == LQSGD_ACT_NONE)) return fail(c, LQSGD_EINVAL, kBadCodes);
  }
  if (!aligned(dy, size_of(type)) || !aligned(dz, size_of(type)) || !aligned(dbias, 4)) return fail(c, LQSGD_EINVAL, kBadAlign);
  if (samples > 0) {
    const bool reads_z = act != LQSGD_ACT_NONE;
    if (lies_over({dz, dbias}, {reads_z ? z_codes : nullptr, reads_z ? z_exponents : nullptr}) || lies_over({dbias}, {dy}))
      return fail(c, LQSGD_EINVAL, kOver);
  }
  if (dz == dy && dz && lddz != lddy) return fail(c, LQSGD_EINVAL, "dz is dy, with another stride");
  if (samples == 0 && !dbias) return LQSGD_OK;
  const Codes held{const_cast<int8_t*>(z_codes), const_cast<uint8_t*>(z_exponents)};
  return done(c, launch_activation_backward(type, act, samples, rows, dy, lddy, held, dz, lddz, dbias, accumulate != 0, c->workspace, c->slopes, c->stream),
              "lqsgd_linear_activation_backward");
}

int lqsgd_linear_input_grad(lqsgd_linear* c, int32_t type, int64_t samples, int32_t rows, int32_t cols, const void* dz, int64_t lddz,
                            const void* w, int64_t ldw, void* dx, int64_t lddx) {
  if (!c) return fail(nullptr, LQSGD_EINVAL, kNull);
  if (!known_type(type)) return fail(c, LQSGD_EINVAL, kBadType);
  if (!samples_ok(samples) || !features_ok(rows) || !features_ok(cols) || !stride_ok(lddz, rows) || !stride_ok(ldw, cols) ||
      !stride_ok(lddx, cols))
    return fail(c, LQSGD_ESHAPE, kBadSize);
  if (!output_ok(cols, samples)) return fail(c, LQSGD_ESHAPE, kBadSize);
  if (samples == 0) return LQSGD_OK;
  if (!dz || !w || !dx) return fail(c, LQSGD_EINVAL, kNull);
  const uintptr_t s = size_of(type);
  if (!aligned(dz, s) || !aligned(w, s) || !aligned(dx, s)) return fail(c, LQSGD_EINVAL, kBadAlign);
  if (lies_over({dx}, {dz, w})) return fail(c, LQSGD_EINVAL, kOver);
  ProductArgs a{};
  a.ni = cols; a.nj = samples; a.depth = rows;
  a.a = w; a.lda = ldw; a.b = dz; a.ldb = lddz;
  a.out = dx; a.ldo = lddx; a.workspace = c->workspace; a.arrived = c->arrived;
  return done(c, launch_product(kInputGrad, type, a, c->stream), "lqsgd_linear_input_grad");
}

int lqsgd_linear_weight_grad(lqsgd_linear* c, int32_t type, int64_t samples, int32_t rows, int32_t cols, const void* dz, int64_t lddz,
                             const int8_t* x_codes, const uint8_t* x_exponents, int32_t grad_type, void* dw, int64_t lddw,
                             int32_t accumulate) {
  if (!c) return fail(nullptr, LQSGD_EINVAL, kNull);
  if (!known_type(type) || (grad_type != LQSGD_TYPE_F32 && grad_type != LQSGD_TYPE_BF16)) return fail(c, LQSGD_EINVAL, kBadType);
  if (!samples_ok(samples) || !features_ok(rows) || !features_ok(cols) || !stride_ok(lddz, rows) || !stride_ok(lddw, cols))
    return fail(c, LQSGD_ESHAPE, kBadSize);
  if (!output_ok(cols, rows)) return fail(c, LQSGD_ESHAPE, kBadSize);
  if (!dw || (samples > 0 && !dz)) return fail(c, LQSGD_EINVAL, kNull);
  if (samples > 0 && !codes_ok(x_codes, x_exponents, false)) return fail(c, LQSGD_EINVAL, kBadCodes);
  if (!aligned(dz, size_of(type)) || !aligned(dw, size_of(grad_type))) return fail(c, LQSGD_EINVAL, kBadAlign);
  if (lies_over({dw}, {dz, x_codes, x_exponents})) return fail(c, LQSGD_EINVAL, kOver);
  if (samples == 0 && accumulate) return LQSGD_OK;
  ProductArgs a{};
  a.ni = cols; a.nj = rows; a.depth = samples;
  a.held = Codes{const_cast<int8_t*>(x_codes), const_cast<uint8_t*>(x_exponents)};
  a.b = dz; a.ldb = lddz;
  a.out = dw; a.ldo = lddw; a.out_type = grad_type; a.accumulate = accumulate != 0; a.workspace = c->workspace; a.arrived = c->arrived;
  return done(c, launch_product(kWeightGrad, type, a, c->stream), "lqsgd_linear_weight_grad");
}

}  // extern "C"
