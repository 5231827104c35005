// Status and message helpers shared by the C ABI's sources.
#pragma once

#include <hip/hip_runtime_api.h>

#include <cstdarg>
#include <cstddef>
#include <cstdint>
#include <cstdio>

#include "../../include/hs_merge.h"

namespace hs {

inline thread_local char g_err[512];   // hs_last_error()'s message

inline hs_status fail(hs_status s, const char *fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_err, sizeof(g_err), fmt, ap);
  va_end(ap);
  return s;
}

inline hs_status ok() {
  g_err[0] = 0;
  return HS_OK;
}

inline bool aligned(const void *p, size_t a) { return ((uintptr_t)p % a) == 0; }

inline hs_status device_status(hipError_t e, const char *what) {
  if (e == hipSuccess) return ok();
  return fail(HS_ERR_DEVICE, "%s: %s", what, hipGetErrorString(e));
}

}  // namespace hs
