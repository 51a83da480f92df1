// Argument checks that the operator calls of the C boundary share.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <string>

#include "common.h"

namespace ckpt {

// a device buffer of elements of `size` bytes (a power of two); the message is put
// together only for a bad one
inline void need_ptr(const void *p, const char *fn, const char *arg, uintptr_t size = 1) {
  if (p && !(reinterpret_cast<uintptr_t>(p) & (size - 1))) return;
  const std::string what = std::string(fn) + "(" + arg + ")";
  if (!p) fail(CKPT_E_INVALID, what + ": null pointer");
  fail(CKPT_E_INVALID, what + ": misaligned address");
}

[[noreturn]] inline void refuse(int code, const char *fn, const char *what) { fail(code, std::string(fn) + what); }

inline void launched(const char *fn) {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) fail(CKPT_E_HIP, std::string(fn) + ": " + hipGetErrorString(e));
}

// a * b, both positive, below 2^62; -1 past it
inline int64_t product(int64_t a, int64_t b) {
  return a > (int64_t(1) << 62) / b ? -1 : a * b;
}

}  // namespace ckpt
