// What the host files of the operators beside the nests share: error messages,
// and the checks of workspaces and matrices.
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstdlib>
#include <initializer_list>
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

struct Matrix {
  const char* name;
  const void* p;
  int64_t rows, cols, ld;
  int es;
  int64_t bytes() const { return rows && cols ? ((rows - 1) * ld + cols) * es : 0; }
};

inline int check(const Matrix& m) { return check_matrix(m.name, m.p, m.rows, m.cols, m.ld, m.es); }

// Whether two matrices share a byte.  Column blocks of one array lie between one
// another's rows: with one pitch it is told row for row.
inline bool overlap(const Matrix& a, const Matrix& b) {
  const int64_t na = a.bytes(), nb = b.bytes();
  if (!na || !nb || !a.p || !b.p) return false;
  const int64_t d = (int64_t)((uintptr_t)b.p - (uintptr_t)a.p);
  if (d >= na || -d >= nb) return false;
  const int64_t pitch = a.ld * a.es;
  if (pitch != b.ld * b.es || a.rows == 1 || b.rows == 1) return true;
  // a's row r and b's row r + k are d + k pitch apart
  for (int64_t k = -d / pitch - 1; k <= -d / pitch + 1; ++k)
    if (k > -a.rows && k < b.rows && d + k * pitch < a.cols * a.es && -(d + k * pitch) < b.cols * b.es) return true;
  return false;
}

inline bool same(const Matrix& a, const Matrix& b) { return a.p == b.p && a.es == b.es && (a.ld == b.ld || a.rows <= 1); }

// Output o is `in`, or apart from it; and apart from every other matrix.
inline int check_apart(const Matrix& o, const Matrix* in, std::initializer_list<const Matrix*> others) {
  if (in && overlap(o, *in) && !same(o, *in))
    return fail(PARTIR_E_LAYOUT, "%s must be %s, with its type and leading dim, or apart from it", o.name, in->name);
  for (const Matrix* m : others)
    if (m->p && overlap(o, *m)) return fail(PARTIR_E_LAYOUT, "%s overlaps %s", o.name, m->name);
  return PARTIR_OK;
}

}  // namespace partir
