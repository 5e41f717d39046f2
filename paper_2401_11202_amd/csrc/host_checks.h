// What the host files of the operators beside the nests share: error messages,
// and the checks of workspaces and matrices.
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstdlib>
#include <string>

#include "../../include/partir.h"

namespace partir {

void set_last_error(const std::string& msg);   // the C ABI's thread-local message

constexpr size_t kWsAlign = 256;
constexpr int64_t kMaxLd = (int64_t)1 << 24, kMaxSize = (int64_t)1 << 30;

inline int fail(int status, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  set_last_error(std::string(partir_status_string(status)) + ": " + buf);
  return status;
}

inline size_t align_up(size_t x) { return (x + kWsAlign - 1) / kWsAlign * kWsAlign; }
inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline bool aligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

// Runs the body of an entry point; what it throws becomes a status.
template <typename F>
int guarded(F body) {
  try {
    return body();
  } catch (...) {
    try {
      return fail(PARTIR_E_HIP, "the host ran out of memory");
    } catch (...) {
      return PARTIR_E_HIP;
    }
  }
}

inline int check_ws(size_t need, const void* ws, size_t ws_bytes) {
  if (ws_bytes < need) return fail(PARTIR_E_WORKSPACE, "workspace of %zu bytes, need %zu", ws_bytes, need);
  if (need && !ws) return fail(PARTIR_E_NULL, "workspace pointer is NULL");
  if (need && !aligned(ws, 16)) return fail(PARTIR_E_LAYOUT, "workspace not 16-byte aligned");
  return PARTIR_OK;
}

// Clears an older error of the runtime before the first launch of a call.
inline int begin_launches() {
  const char* force = getenv("PARTIR_FAIL_LAUNCH");
  if (force && force[0] == '1') return fail(PARTIR_E_HIP, "launch failure forced by PARTIR_FAIL_LAUNCH");
  (void)hipGetLastError();
  return PARTIR_OK;
}

inline int launched(hipError_t e, const char* what) {
  return e == hipSuccess ? PARTIR_OK : fail(PARTIR_E_HIP, "launch of %s failed: %s", what, hipGetErrorString(e));
}

// A row-major matrix of `cols` values a row: its leading dim and alignment.
inline int check_matrix(const char* name, const void* p, int64_t rows, int64_t cols, int64_t ld, int es) {
  if (rows == 0 || cols == 0) return PARTIR_OK;
  if (!p) return fail(PARTIR_E_NULL, "%s must be non-NULL", name);
  if (!aligned(p, 16)) return fail(PARTIR_E_LAYOUT, "%s must be 16-byte aligned", name);
  if (ld < cols || (ld * es) % 16)
    return fail(PARTIR_E_LAYOUT, "%s: leading dim %lld must be at least %lld and a multiple of 16 bytes", name,
                (long long)ld, (long long)cols);
  if (ld > kMaxLd) return fail(PARTIR_E_SHAPE, "%s: leading dim %lld above 2^24", name, (long long)ld);
  return PARTIR_OK;
}

}  // namespace partir
