// The context of the linear layer and of its neighbours, and the argument checks that their entry points share.  Host only.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <initializer_list>
#include <string>

#include "lqsgd_linear.h"
#include "lqsgd_linear_kernels.h"

struct lqsgd_linear {
  hipStream_t stream = nullptr;
  void* workspace = nullptr;
  int* arrived = nullptr;     // behind it
  float* slopes = nullptr;    // behind those
  std::string err;
};

namespace lqsgd {
namespace linear {

// Keep the text of an error on c (NULL: the thread's) and give the status back.
int fail(lqsgd_linear* c, int code, const char* msg);
int done(lqsgd_linear* c, hipError_t e, const char* what);

inline bool known_type(int32_t t) { return t == LQSGD_TYPE_F32 || t == LQSGD_TYPE_BF16 || t == LQSGD_TYPE_F16; }
inline uintptr_t size_of(int32_t t) { return t == LQSGD_TYPE_F32 ? 4 : 2; }
inline bool aligned(const void* p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
inline bool features_ok(int32_t n) { return n >= 1 && n <= LQSGD_LINEAR_MAX_FEATURES; }
inline bool samples_ok(int64_t n) { return n >= 0 && n <= LQSGD_LINEAR_MAX_SAMPLES; }
// An output of ni x nj values that the kernels of 128 x 128 tiles can be launched for (of any shape up to 2^36 values): as many threads
// as one launch has.
inline bool output_ok(int64_t ni, int64_t nj) { return ((ni + 127) / 128) * ((nj + 127) / 128) * 256 < int64_t(1) << 32; }
inline bool stride_ok(int64_t ld, int32_t n) { return ld >= n && ld <= LQSGD_LINEAR_MAX_STRIDE; }
// A checkpoint's two pointers: both or neither (neither only if it is optional).
inline bool codes_ok(const void* codes, const void* exponents, bool optional) {
  if (!codes || !exponents) return optional && !codes && !exponents;
  return aligned(codes, 16);
}

// Whether an output starts where an input or another output does (NULL: not there).
inline bool lies_over(std::initializer_list<const void*> outputs, std::initializer_list<const void*> inputs) {
  for (auto o = outputs.begin(); o != outputs.end(); ++o) {
    if (!*o) continue;
    for (const void* i : inputs)
      if (*o == i) return true;
    for (auto p = o + 1; p != outputs.end(); ++p)
      if (*o == *p) return true;
  }
  return false;
}

inline constexpr const char kNull[] = "a pointer that is needed is NULL";
inline constexpr const char kBadType[] = "unknown type or activation";
inline constexpr const char kBadSize[] = "samples, features or a stride out of range";
inline constexpr const char kBadAlign[] = "a pointer is not aligned to its type";
inline constexpr const char kOver[] = "an output lies over an input or another output";
inline constexpr const char kBadCodes[] = "a checkpoint needs both of its pointers, and codes aligned to 16 bytes";

}  // namespace linear
}  // namespace lqsgd
