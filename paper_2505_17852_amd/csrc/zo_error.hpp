// The thread-local description of the last failure, shared by the C ABI's sources.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdarg>
#include <cstdint>
#include <cstdio>

#include "../../include/zo.h"

namespace zo {

inline thread_local char g_err[512] = "";

int fail(int code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
inline int fail(int code, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  std::vsnprintf(g_err, sizeof g_err, fmt, ap);
  va_end(ap);
  return code;
}

inline int ok() {
  g_err[0] = '\0';
  return ZO_OK;
}

inline int device_status(hipError_t e, const char* what) {
  if (e == hipSuccess) return ok();
  return fail(ZO_EDEVICE, "%s: %s", what, hipGetErrorString(e));
}

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

}  // namespace zo
