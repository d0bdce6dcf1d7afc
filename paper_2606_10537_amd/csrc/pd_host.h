// Host-side helpers shared by the files that hold entry points: status and error
// message, argument checks, workspace arithmetic.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <string>

#include "pd.h"

namespace pd_host {

// The calling thread's message of its last error.
inline std::string& last_error() {
  static thread_local std::string s;
  return s;
}

inline pd_status fail(pd_status s, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  last_error() = buf;
  return s;
}

inline pd_status ok() {
  last_error().clear();
  return PD_OK;
}

constexpr size_t kAlign = 256;

inline size_t round_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
inline int cdiv(long long a, long long b) { return (int)((a + b - 1) / b); }

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

inline pd_status check_ws(void* ws, size_t have, size_t need) {
  if (need == 0) return PD_OK;
  if (!ws) return fail(PD_ERR_WORKSPACE, "workspace is NULL but %zu bytes are needed", need);
  if (!aligned16(ws)) return fail(PD_ERR_MISALIGNED, "workspace is not 16-byte aligned");
  if (have < need) return fail(PD_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", have, need);
  return PD_OK;
}

#define PD_REQUIRE_PTR(p)                                               \
  do {                                                                  \
    if (!(p)) return fail(PD_ERR_NULL_PTR, "pointer '%s' is NULL", #p); \
    if (!aligned16(p)) return fail(PD_ERR_MISALIGNED, "pointer '%s' is not 16-byte aligned", #p); \
  } while (0)

#define PD_RETURN_IF(st)          \
  do {                            \
    pd_status _s = (st);          \
    if (_s != PD_OK) return _s;   \
  } while (0)

inline pd_status hip_status(hipError_t e, const char* what) {
  if (e == hipSuccess) return ok();
  return fail(PD_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

}  // namespace pd_host
