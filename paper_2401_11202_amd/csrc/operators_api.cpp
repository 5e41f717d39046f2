// Host side of the operators around the loop nests: rotary positions, the
// norms of queries and keys, cross attention, the global norm of gradients.
// As in partir_api.cpp a call validates its arguments, plans its launches and
// enqueues them on the caller's stream; nothing is enqueued before every
// argument has passed, and no exception leaves an entry point.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <string>
#include <vector>

#include "../../include/partir.h"
#include "operators.h"

namespace partir {

void set_last_error(const std::string& msg);   // the C ABI's thread-local message

namespace {

constexpr size_t kWsAlign = 256;
constexpr int64_t kMaxLd = (int64_t)1 << 24, kMaxSize = (int64_t)1 << 30;

int fail(int status, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  set_last_error(std::string(partir_status_string(status)) + ": " + buf);
  return status;
}

size_t align_up(size_t x) { return (x + kWsAlign - 1) / kWsAlign * kWsAlign; }
int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
bool aligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

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

int check_ws(size_t need, const void* ws, size_t ws_bytes) {
  if (ws_bytes < need) return fail(PARTIR_E_WORKSPACE, "workspace of %zu bytes, need %zu", ws_bytes, need);
  if (need && !ws) return fail(PARTIR_E_NULL, "workspace pointer is NULL");
  if (need && !aligned(ws, 16)) return fail(PARTIR_E_LAYOUT, "workspace not 16-byte aligned");
  return PARTIR_OK;
}

// Clears an older error of the runtime before the first launch of a call.
int begin_launches() {
  const char* force = getenv("PARTIR_FAIL_LAUNCH");
  if (force && force[0] == '1') return fail(PARTIR_E_HIP, "launch failure forced by PARTIR_FAIL_LAUNCH");
  (void)hipGetLastError();
  return PARTIR_OK;
}

int launched(hipError_t e, const char* what) {
  return e == hipSuccess ? PARTIR_OK : fail(PARTIR_E_HIP, "launch of %s failed: %s", what, hipGetErrorString(e));
}

// A row-major matrix of `cols` values a row: its leading dim and alignment.
int check_matrix(const char* name, const void* p, int64_t rows, int64_t cols, int64_t ld, int es) {
  if (rows == 0 || cols == 0) return PARTIR_OK;
  if (!p) return fail(PARTIR_E_NULL, "%s must be non-NULL", name);
  if (!aligned(p, 16)) return fail(PARTIR_E_LAYOUT, "%s must be 16-byte aligned", name);
  if (ld < cols || (ld * es) % 16)
    return fail(PARTIR_E_LAYOUT, "%s: leading dim %lld must be at least %lld and a multiple of 16 bytes", name,
                (long long)ld, (long long)cols);
  if (ld > kMaxLd) return fail(PARTIR_E_SHAPE, "%s: leading dim %lld above 2^24", name, (long long)ld);
  return PARTIR_OK;
}

// ---------------------------------------------------------------------------
// rotary positions and per-head norms
// ---------------------------------------------------------------------------
int validate_rotary(const RotaryParams& p, int dtype) {
  if (dtype != PARTIR_F32 && dtype != PARTIR_BF16) return fail(PARTIR_E_DTYPE, "dtype %d", dtype);
  const int es = dtype == PARTIR_BF16 ? 2 : 4;
  if (p.T < 0 || p.T > kMaxSize) return fail(PARTIR_E_SHAPE, "T = %lld", (long long)p.T);
  if (p.dh < 8 || p.dh > 256 || p.dh % 8)
    return fail(PARTIR_E_SHAPE, "d_head = %d must be a multiple of 8 up to 256", p.dh);
  if (p.rd < 0 || p.rd > p.dh || p.rd % 2)
    return fail(PARTIR_E_SHAPE, "rotary_dim = %d must be even and at most d_head = %d", p.rd, p.dh);
  if (p.H[0] < 0 || p.H[1] < 0 || (int64_t)p.H[0] * p.dh > kMaxLd || (int64_t)p.H[1] * p.dh > kMaxLd)
    return fail(PARTIR_E_SHAPE, "head counts %d and %d", p.H[0], p.H[1]);
  if (!p.pos && p.T > 0 && p.S < 1) return fail(PARTIR_E_SHAPE, "S = %lld: without positions S is at least 1", (long long)p.S);
  if (!std::isfinite(p.magnitude)) return fail(PARTIR_E_UNSUPPORTED, "magnitude must be finite");
  if (p.T > 0 && p.rd > 0 && !p.freqs) return fail(PARTIR_E_NULL, "freqs must be non-NULL");
  if (!aligned(p.freqs, 8)) return fail(PARTIR_E_LAYOUT, "freqs must be 8-byte aligned");
  if (!aligned(p.pos, p.pos64 ? 8 : 4)) return fail(PARTIR_E_LAYOUT, "positions must be aligned to their type");
  const char* names[3][2] = {{"Q", "K"}, {"dQ", "dK"}, {"the output of Q", "the output of K"}};
  for (int i = 0; i < 2; ++i) {
    const int64_t cols = (int64_t)p.H[i] * p.dh;
    int st = check_matrix(names[0][i], p.x[i], p.T, cols, p.ldx[i], es);
    if (!st && p.lddy[i] >= 0) st = check_matrix(names[1][i], p.dy[i], p.T, cols, p.lddy[i], es);
    if (!st) st = check_matrix(names[2][i], p.y[i], p.T, cols, p.ldy[i], es);
    if (st) return st;
    if (!aligned(p.g[i], 16)) return fail(PARTIR_E_LAYOUT, "gains must be 16-byte aligned");
  }
  return PARTIR_OK;
}

int check_eps(float eps) {
  return eps >= 0.0f && std::isfinite(eps) ? PARTIR_OK : fail(PARTIR_E_UNSUPPORTED, "eps must be finite and not negative");
}

int run_rotary(RotaryParams& p, int dtype, int interleaved, bool norm, void* stream) {
  if (int st = validate_rotary(p, dtype)) return st;
  if (p.T == 0 || p.H[0] + p.H[1] == 0) return PARTIR_OK;
  rotary_choice(p, dtype == PARTIR_BF16, false);
  if (int st = begin_launches()) return st;
  return launched(launch_rotary(p, dtype == PARTIR_BF16, interleaved != 0, norm, (hipStream_t)stream),
                  norm ? "qk_norm_rotary" : "rotary");
}

RotaryParams rotary_args(const void* Q, const void* K, void* Qo, void* Ko, const double* freqs, const void* positions,
                         int positions64, int64_t T, int64_t S, int64_t Hq, int64_t Hk, int64_t dh, int64_t rd,
                         int64_t ldq, int64_t ldk, int64_t ldqo, int64_t ldko, float magnitude) {
  auto to_int = [](int64_t v) { return v < -1 || v > kMaxLd ? -1 : (int)v; };   // refused by the checks
  RotaryParams p{};
  p.x[0] = Q; p.x[1] = K; p.y[0] = Qo; p.y[1] = Ko;
  p.freqs = freqs; p.pos = positions; p.pos64 = positions64 != 0;
  p.ldx[0] = ldq; p.ldx[1] = ldk; p.ldy[0] = ldqo; p.ldy[1] = ldko;
  p.lddy[0] = p.lddy[1] = -1;   // no cotangents
  p.T = T; p.S = S;
  p.H[0] = to_int(Hq); p.H[1] = to_int(Hk); p.dh = to_int(dh); p.rd = to_int(rd);
  p.magnitude = magnitude;
  p.sign = 1.0f;
  return p;
}

// What the backward pass's workspace holds: a partial gain gradient for both
// tensors from each workgroup, at most kRotaryMaxBwdGrid of them.
size_t qk_norm_backward_ws(const RotaryParams& p) {
  if (p.T <= 0 || p.H[0] + p.H[1] <= 0) return 0;
  return align_up((size_t)p.grid * 2 * p.dh * sizeof(float));
}

// ---------------------------------------------------------------------------
// global norm of gradients
// ---------------------------------------------------------------------------
int validate_grads(const void* const* in, void* const* out, const int64_t* numel, const int* dtypes, int n) {
  if (n < 0 || n > (1 << 24)) return fail(PARTIR_E_SHAPE, "%d tensors", n);
  if (n > 0 && (!in || !numel || !dtypes)) return fail(PARTIR_E_NULL, "tensors, numel and dtypes must be non-NULL");
  int64_t total = 0;
  for (int i = 0; i < n; ++i) {
    if (dtypes[i] != PARTIR_F32 && dtypes[i] != PARTIR_BF16) return fail(PARTIR_E_DTYPE, "tensor %d: dtype %d", i, dtypes[i]);
    if (numel[i] < 0 || numel[i] > ((int64_t)1 << 40)) return fail(PARTIR_E_SHAPE, "tensor %d: %lld elements", i, (long long)numel[i]);
    total += numel[i];
    if (numel[i] == 0) continue;
    const uintptr_t es = dtypes[i] == PARTIR_BF16 ? 2 : 4;
    if (!in[i] || (out && !out[i])) return fail(PARTIR_E_NULL, "tensor %d must be non-NULL", i);
    if (!aligned(in[i], es) || (out && !aligned(out[i], es)))
      return fail(PARTIR_E_LAYOUT, "tensor %d must be aligned to its type", i);
  }
  if (total > ((int64_t)1 << 44)) return fail(PARTIR_E_SHAPE, "more than 2^44 elements");
  return PARTIR_OK;
}

struct Span {
  uintptr_t lo, hi;
  int i;
};

// Every written range is apart from every other and from every read range but
// its own input's, which it is or is apart from: a value scaled twice, or
// scaled before it is read, would depend on timing.
int check_apart(const void* const* in, void* const* out, const int64_t* numel, const int* dtypes, int n) {
  std::vector<Span> w, r;
  w.reserve(n);
  auto span = [&](const void* p, int i) {
    const uintptr_t lo = (uintptr_t)p;
    return Span{lo, lo + (uintptr_t)numel[i] * (dtypes[i] == PARTIR_BF16 ? 2 : 4), i};
  };
  for (int i = 0; i < n; ++i) {
    if (numel[i] == 0) continue;
    w.push_back(span(out[i], i));
    if (in[i] != out[i]) r.push_back(span(in[i], i));
  }
  auto before = [](const Span& a, const Span& b) { return a.lo < b.lo; };
  if (!std::is_sorted(w.begin(), w.end(), before)) std::sort(w.begin(), w.end(), before);
  if (!std::is_sorted(r.begin(), r.end(), before)) std::sort(r.begin(), r.end(), before);
  for (size_t k = 1; k < w.size(); ++k)
    if (w[k].lo < w[k - 1].hi)
      return fail(PARTIR_E_LAYOUT, "tensors %d and %d overlap", std::min(w[k].i, w[k - 1].i), std::max(w[k].i, w[k - 1].i));
  // inputs may overlap one another: the last end among those before counts
  size_t k = 0;
  for (const Span& s : r) {
    while (k < w.size() && w[k].hi <= s.lo) ++k;
    if (k < w.size() && w[k].lo < s.hi)
      return fail(PARTIR_E_LAYOUT, "the output of tensor %d overlaps the input of tensor %d", w[k].i, s.i);
  }
  return PARTIR_OK;
}

// The tensors in tables of up to kGradTensors (empty ones left out), and the
// workgroups that each table's launch takes.
struct GradLaunch {
  GradTable t;
  int workgroups;
};
void grad_launches(const void* const* in, void* const* out, const int64_t* numel, const int* dtypes, int n,
                   std::vector<GradLaunch>& all) {
  for (int i = 0; i < n;) {
    all.emplace_back();
    GradTable& t = all.back().t;
    t.n = 0;
    t.chunk0[0] = 0;
    for (; i < n && t.n < kGradTensors; ++i) {
      if (numel[i] == 0) continue;
      t.in[t.n] = in[i];
      t.out[t.n] = out ? out[i] : nullptr;
      t.numel[t.n] = numel[i];
      t.bf16[t.n] = dtypes[i] == PARTIR_BF16;
      t.chunk0[t.n + 1] = t.chunk0[t.n] + cdiv(numel[i], kGradChunkBytes / (t.bf16[t.n] ? 2 : 4));
      ++t.n;
    }
    if (t.n == 0) {
      all.pop_back();
      continue;
    }
    all.back().workgroups = (int)std::min<int64_t>(t.chunk0[t.n], kGradMaxWorkgroups);
  }
}

// Workspace: a float64 partial for each workgroup of each table, at most.
size_t grad_ws(int n) { return n <= 0 ? 0 : align_up((size_t)cdiv(n, kGradTensors) * kGradMaxWorkgroups * sizeof(double)); }

int run_grads(const void* const* in, void* const* out, const int64_t* numel, const int* dtypes, int n, bool clip,
              double max_norm, float* norm, void* ws, size_t ws_bytes, void* stream) {
  if (int st = validate_grads(in, out, numel, dtypes, n)) return st;
  if (clip && !(max_norm >= 0.0)) return fail(PARTIR_E_UNSUPPORTED, "max_norm must not be negative or NaN");
  if (!norm) return fail(PARTIR_E_NULL, "norm must be non-NULL");
  if (!aligned(norm, 4)) return fail(PARTIR_E_LAYOUT, "norm must be 4-byte aligned");
  if (int st = check_ws(grad_ws(n), ws, ws_bytes)) return st;
  if (clip)
    if (int st = check_apart(in, out, numel, dtypes, n)) return st;
  std::vector<GradLaunch> all;
  all.reserve((size_t)cdiv(n, kGradTensors));
  grad_launches(in, out, numel, dtypes, n, all);
  if (int st = begin_launches()) return st;
  hipStream_t s = (hipStream_t)stream;
  double* partial = (double*)ws;
  int parts = 0;
  for (const GradLaunch& l : all) {
    if (int st = launched(launch_grad_sumsq(l.t, partial + parts, l.workgroups, s), "grad_sumsq")) return st;
    parts += l.workgroups;
  }
  if (!clip || all.empty()) return launched(launch_grad_norm(partial, parts, norm, s), "grad_norm");
  for (size_t i = 0; i < all.size(); ++i)
    if (int st = launched(launch_grad_scale(all[i].t, partial, parts, max_norm, i == 0 ? norm : nullptr,
                                            all[i].workgroups, s), "grad_scale"))
      return st;
  return PARTIR_OK;
}

}  // namespace
}  // namespace partir

using namespace partir;

extern "C" {

// ---- rotary -------------------------------------------------------------------
int partir_rotary_frequencies(int64_t rotary_dim, double base, int scaling, double factor, int64_t original_length,
                              double slow_turns, double fast_turns, double* freqs) {
  return guarded([&]() -> int {
    if (rotary_dim < 0 || rotary_dim > 256 || rotary_dim % 2)
      return fail(PARTIR_E_SHAPE, "rotary_dim = %lld must be even and at most 256", (long long)rotary_dim);
    if (rotary_dim > 0 && !freqs) return fail(PARTIR_E_NULL, "freqs must be non-NULL");
    if (!(base > 1.0) || !std::isfinite(base)) return fail(PARTIR_E_UNSUPPORTED, "base must be finite and above 1");
    if (scaling < PARTIR_ROTARY_PLAIN || scaling > PARTIR_ROTARY_PARTS) return fail(PARTIR_E_UNSUPPORTED, "scaling %d", scaling);
    if (scaling != PARTIR_ROTARY_PLAIN && (!(factor >= 1.0) || !std::isfinite(factor)))
      return fail(PARTIR_E_UNSUPPORTED, "factor must be finite and at least 1");
    if (scaling == PARTIR_ROTARY_BASE && rotary_dim == 2)
      return fail(PARTIR_E_UNSUPPORTED, "a single pair does not depend on the base");
    if (scaling == PARTIR_ROTARY_PARTS && (original_length < 1 || !(slow_turns < fast_turns) || !std::isfinite(slow_turns) ||
                                           !std::isfinite(fast_turns)))
      return fail(PARTIR_E_UNSUPPORTED, "scaling by parts needs original_length >= 1 and slow_turns < fast_turns");
    const double rd = (double)rotary_dim;
    if (scaling == PARTIR_ROTARY_BASE) base *= std::pow(factor, rd / (rd - 2.0));
    for (int64_t i = 0; i < rotary_dim / 2; ++i) {
      double f = std::pow(base, -2.0 * (double)i / rd);
      if (scaling == PARTIR_ROTARY_LINEAR) f /= factor;
      if (scaling == PARTIR_ROTARY_PARTS) {
        const double turns = (double)original_length * f / 6.283185307179586477;
        const double keep = std::min(1.0, std::max(0.0, (turns - slow_turns) / (fast_turns - slow_turns)));
        f = f * keep + f / factor * (1.0 - keep);
      }
      freqs[i] = f;
    }
    return PARTIR_OK;
  });
}

int partir_rotary(const void* Q, const void* K, void* Qo, void* Ko, const double* freqs, const void* positions,
                  int positions64, int64_t T, int64_t S, int64_t n_heads, int64_t n_kv_heads, int64_t d_head,
                  int64_t rotary_dim, int64_t ldq, int64_t ldk, int64_t ldqo, int64_t ldko, int dtype, int interleaved,
                  int inverse, float magnitude, void* stream) {
  return guarded([&]() -> int {
    RotaryParams p = rotary_args(Q, K, Qo, Ko, freqs, positions, positions64, T, S, n_heads, n_kv_heads, d_head,
                                 rotary_dim, ldq, ldk, ldqo, ldko, magnitude);
    if (inverse) p.sign = -1.0f;
    return run_rotary(p, dtype, interleaved, false, stream);
  });
}

int partir_qk_norm_rotary(const void* Q, const void* K, const float* gq, const float* gk, void* Qo, void* Ko,
                          const double* freqs, const void* positions, int positions64, int64_t T, int64_t S,
                          int64_t n_heads, int64_t n_kv_heads, int64_t d_head, int64_t rotary_dim, int64_t ldq,
                          int64_t ldk, int64_t ldqo, int64_t ldko, int dtype, int interleaved, float magnitude, float eps,
                          void* stream) {
  return guarded([&]() -> int {
    RotaryParams p = rotary_args(Q, K, Qo, Ko, freqs, positions, positions64, T, S, n_heads, n_kv_heads, d_head,
                                 rotary_dim, ldq, ldk, ldqo, ldko, magnitude);
    p.g[0] = gq; p.g[1] = gk;
    p.eps = eps;
    if (int st = check_eps(eps)) return st;
    return run_rotary(p, dtype, interleaved, true, stream);
  });
}

size_t partir_qk_norm_rotary_backward_workspace(int64_t T, int64_t n_heads, int64_t n_kv_heads, int64_t d_head,
                                                int64_t rotary_dim, int dtype) {
  RotaryParams p = rotary_args(nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, 0, 0, 1, n_heads, n_kv_heads, d_head,
                               rotary_dim, 0, 0, 0, 0, 1.0f);
  const int st = guarded([&]() -> int {
    if (int bad = validate_rotary(p, dtype)) return bad;   // T = 0: sizes alone
    if (T < 0 || T > kMaxSize) return fail(PARTIR_E_SHAPE, "T = %lld", (long long)T);
    return PARTIR_OK;
  });
  if (st) return (size_t)-1;
  p.T = T;
  rotary_choice(p, dtype == PARTIR_BF16, true);
  return qk_norm_backward_ws(p);
}

int partir_qk_norm_rotary_backward(const void* Q, const void* K, const void* dQo, const void* dKo, const float* gq,
                                   const float* gk, void* dQ, void* dK, float* dgq, float* dgk, const double* freqs,
                                   const void* positions, int positions64, int64_t T, int64_t S, int64_t n_heads,
                                   int64_t n_kv_heads, int64_t d_head, int64_t rotary_dim, int64_t ldq, int64_t ldk,
                                   int64_t lddqo, int64_t lddko, int64_t lddq, int64_t lddk, int dtype, int interleaved,
                                   float magnitude, float eps, void* ws, size_t ws_bytes, void* stream) {
  return guarded([&]() -> int {
    RotaryParams p = rotary_args(Q, K, dQ, dK, freqs, positions, positions64, T, S, n_heads, n_kv_heads, d_head,
                                 rotary_dim, ldq, ldk, lddq, lddk, magnitude);
    p.dy[0] = dQo; p.dy[1] = dKo;
    p.lddy[0] = std::max<int64_t>(lddqo, 0); p.lddy[1] = std::max<int64_t>(lddko, 0);
    p.g[0] = gq; p.g[1] = gk;
    p.eps = eps;
    p.sign = -1.0f;
    if (int st = check_eps(eps)) return st;
    if (int st = validate_rotary(p, dtype)) return st;
    if (!aligned(dgq, 4) || !aligned(dgk, 4)) return fail(PARTIR_E_LAYOUT, "gain gradients must be 4-byte aligned");
    const bool empty = p.T == 0 || p.H[0] + p.H[1] == 0;
    if (!empty) {
      rotary_choice(p, dtype == PARTIR_BF16, true);
      if (int st = check_ws(qk_norm_backward_ws(p), ws, ws_bytes)) return st;
      p.dgpart = (float*)ws;
    }
    if (empty && !dgq && !dgk) return PARTIR_OK;
    if (int st = begin_launches()) return st;
    hipStream_t s = (hipStream_t)stream;
    if (!empty)
      if (int st = launched(launch_qk_norm_backward(p, dtype == PARTIR_BF16, interleaved != 0, s), "qk_norm_backward")) return st;
    if (!dgq && !dgk) return PARTIR_OK;
    return launched(launch_gain_reduce(p.dgpart, empty ? 0 : p.grid, p.dh, dgq, dgk, s), "gain_reduce");
  });
}

// ---- global norm of gradients ----------------------------------------------------
size_t partir_grad_norm_workspace(int n) { return n < 0 || n > (1 << 24) ? (size_t)-1 : grad_ws(n); }

int partir_grad_norm(const void* const* tensors, const int64_t* numel, const int* dtypes, int n, float* norm, void* ws,
                     size_t ws_bytes, void* stream) {
  return guarded([&]() -> int { return run_grads(tensors, nullptr, numel, dtypes, n, false, 0.0, norm, ws, ws_bytes, stream); });
}

int partir_clip_grad_norm(const void* const* tensors, void* const* out, const int64_t* numel, const int* dtypes, int n,
                          double max_norm, float* norm, void* ws, size_t ws_bytes, void* stream) {
  return guarded([&]() -> int {
    if (n > 0 && !out) return fail(PARTIR_E_NULL, "out must be non-NULL (the tensors themselves to scale in place)");
    return run_grads(tensors, out, numel, dtypes, n, true, max_norm, norm, ws, ws_bytes, stream);
  });
}

}  // extern "C"
