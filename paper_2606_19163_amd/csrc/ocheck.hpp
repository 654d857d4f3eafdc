// Checks of host arguments shared by the operators' C entries (ops.cpp,
// rowops.cpp).
#pragma once

#include <cstdarg>
#include <cstdio>

#include "error.hpp"
#include "okernels.hpp"

namespace pulse {

inline pulse_status ofail(pulse_status s, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  return set_last_error(s, buf);
}

#define OCHK(expr)                    \
  do {                                \
    pulse_status s_ = (expr);         \
    if (s_ != PULSE_OK) return s_;    \
  } while (0)

inline pulse_status launched(hipError_t e, const char* what) {
  return e == hipSuccess ? PULSE_OK
                         : ofail(PULSE_E_HIP, "%s failed: %s", what, hipGetErrorString(e));
}

inline bool aligned(const void* p, uintptr_t n) {
  return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0;
}

constexpr int MAX_TOKENS = 1 << 24;
constexpr int64_t MAX_EXTENT = INT64_C(1) << 47;

inline pulse_status check_ws(const void* ws, size_t have, size_t need) {
  if (need == 0) return PULSE_OK;
  if (!ws) return ofail(PULSE_E_INVALID_ARG, "workspace is NULL");
  if (!aligned(ws, 256)) return ofail(PULSE_E_INVALID_ARG, "workspace is not 256-byte aligned");
  if (have < need)
    return ofail(PULSE_E_INVALID_ARG, "workspace has %zu bytes, needs %zu", have, need);
  return PULSE_OK;
}

}  // namespace pulse
