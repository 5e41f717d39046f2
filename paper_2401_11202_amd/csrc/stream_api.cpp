// Host side of the operators on the residual stream: dropout, and the join of a
// block's output with the stream.  As in operators_api.cpp a call validates its
// arguments, plans its launches and enqueues them on the caller's stream.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "host_checks.h"
#include "operators.h"

namespace partir {
namespace {

int dtype_size(int dtype) { return dtype == PARTIR_BF16 ? 2 : 4; }
bool is_dtype(int dtype) { return dtype == PARTIR_F32 || dtype == PARTIR_BF16; }

// p, seed and row0 of a call as the kernels take them.  Nothing is dropped
// without a seed.
int resolve_dropout(Dropout& d, double p, const uint64_t* seed, int64_t row0, int64_t T) {
  if (!(p >= 0.0 && p <= 1.0)) return fail(PARTIR_E_UNSUPPORTED, "p must be within 0..1");
  if (!seed && p != 0.0) return fail(PARTIR_E_NULL, "seed must be non-NULL where p is not 0");
  if (!aligned(seed, 8)) return fail(PARTIR_E_LAYOUT, "seed must be 8-byte aligned");
  if (row0 < 0 || row0 > ((int64_t)1 << 32) - T) return fail(PARTIR_E_SHAPE, "row0 = %lld: rows are numbered below 2^32", (long long)row0);
  d.kept = (uint32_t)std::floor((1.0 - p) * 65536.0 + 0.5);
  d.seed = d.kept == 65536 ? nullptr : seed;
  d.row0 = (uint32_t)row0;
  d.factor = d.kept ? 65536.0f / (float)d.kept : 0.0f;
  return PARTIR_OK;
}

// ---------------------------------------------------------------------------
// join with the residual stream
// ---------------------------------------------------------------------------
constexpr int64_t kMaxJoin = 16384;   // columns: 16 waves of two times 8 columns a lane

struct JoinArgs {
  int64_t T, D, gate_rows, ldgate, row0;
  int x_dtype, y_dtype, post;
  const float *g_post, *g_pre, *gate;
  float scale, eps;
  double p;
  const uint64_t* seed;
};

int validate_join(const JoinArgs& a) {
  if (a.T < 0 || a.T > kMaxSize) return fail(PARTIR_E_SHAPE, "T = %lld", (long long)a.T);
  if (a.D < 0 || a.D > kMaxJoin || a.D % 8)
    return fail(PARTIR_E_SHAPE, "D = %lld must be a multiple of 8 up to %lld", (long long)a.D, (long long)kMaxJoin);
  if (!is_dtype(a.x_dtype) || !is_dtype(a.y_dtype)) return fail(PARTIR_E_DTYPE, "dtypes %d and %d", a.x_dtype, a.y_dtype);
  if (a.gate && a.gate_rows < 1) return fail(PARTIR_E_SHAPE, "gate_rows = %lld", (long long)a.gate_rows);
  return PARTIR_OK;
}

// Rows of the stream that take one row of the gate.  More than T are T: gate_rows may be
// any count, and sums with it would pass 64 bits.
int64_t gate_span(const JoinArgs& a) { return std::min(a.gate_rows, std::max<int64_t>(a.T, 1)); }
int64_t gate_groups(const JoinArgs& a) { return a.gate && a.T ? cdiv(a.T, gate_span(a)) : 0; }

Matrix gate_matrix(const JoinArgs& a) { return {"gate", a.gate, gate_groups(a), a.D, a.ldgate, 4}; }

// The parameters that forward and backward share.
int fill_join(JoinParams& p, const JoinArgs& a) {
  if (int st = validate_join(a)) return st;
  if (!std::isfinite(a.scale)) return fail(PARTIR_E_UNSUPPORTED, "scale must be finite");
  if (!(a.eps >= 0.0f && std::isfinite(a.eps))) return fail(PARTIR_E_UNSUPPORTED, "eps must be finite and not negative");
  if (a.g_post && !a.post) return fail(PARTIR_E_UNSUPPORTED, "g_post without the block's norm");
  if (!aligned(a.g_post, 16) || !aligned(a.g_pre, 16)) return fail(PARTIR_E_LAYOUT, "gains must be 16-byte aligned");
  if (int st = check(gate_matrix(a))) return st;
  if (int st = resolve_dropout(p.drop, a.p, a.seed, a.row0, a.T)) return st;
  p.g_post = a.g_post; p.g_pre = a.g_pre; p.gate = a.gate;
  p.ldgate = a.ldgate;
  p.gate_rows = a.gate ? gate_span(a) : std::max<int64_t>(a.T, 1);
  p.T = a.T; p.D = (int)a.D; p.post = a.post != 0;
  p.scale = a.scale * p.drop.factor;
  p.eps = a.eps;
  return PARTIR_OK;
}

// Partial column sums of the gradients, with room for all three: the workspace
// depends on the sizes only.
size_t join_bwd_ws(const JoinParams& p) { return align_up((size_t)3 * p.workers * p.D * sizeof(float)); }

}  // namespace
}  // namespace partir

using namespace partir;

extern "C" {

int partir_dropout(const void* X, const void* R, void* Y, int64_t T, int64_t D, int64_t ldx, int64_t ldr, int64_t ldy,
                   int x_dtype, int y_dtype, double p, const uint64_t* seed, int64_t row0, void* stream) {
  return guarded([&]() -> int {
    if (T < 0 || T > kMaxSize || D < 0 || D > kMaxLd) return fail(PARTIR_E_SHAPE, "T = %lld, D = %lld", (long long)T, (long long)D);
    if (!is_dtype(x_dtype) || !is_dtype(y_dtype)) return fail(PARTIR_E_DTYPE, "dtypes %d and %d", x_dtype, y_dtype);
    DropoutParams q{};
    if (int st = resolve_dropout(q.drop, p, seed, row0, T)) return st;
    if (!seed) return fail(PARTIR_E_NULL, "seed must be non-NULL");
    q.drop.seed = seed;
    const Matrix x{"X", X, T, D, ldx, dtype_size(x_dtype)}, y{"Y", Y, T, D, ldy, dtype_size(y_dtype)};
    const Matrix r{"R", R, R ? T : 0, D, ldr, dtype_size(y_dtype)};
    for (const Matrix* m : {&x, &r, &y})
      if (int st = check(*m)) return st;
    if (T == 0 || D == 0) return PARTIR_OK;
    const Matrix sd{"seed", seed, 1, 2, 2, 8};
    if (int st = check_apart(y, &x, {&sd})) return st;
    if (int st = check_apart(y, &r, {})) return st;
    q.cols8 = (int)cdiv(D, 8);
    // workgroups of 256 threads for 1024 groups of columns, fewer than 2^32 threads in all
    if (cdiv(T * q.cols8, 1024) >= (int64_t)1 << 24) return fail(PARTIR_E_SHAPE, "2^32 threads of a launch or more");
    q.x = X; q.r = R; q.y = Y;
    q.ldx = ldx; q.ldr = ldr; q.ldy = ldy;
    q.T = T; q.D = (int)D;
    q.by_cols8 = Div::by((uint32_t)q.cols8);
    if (int st = begin_launches()) return st;
    return launched(launch_dropout(q, x_dtype == PARTIR_BF16, y_dtype == PARTIR_BF16, (hipStream_t)stream), "dropout");
  });
}

int partir_residual_norm(const void* X, const void* Y, const float* g_post, const float* gate, const float* g_pre, void* H,
                         void* N, int64_t T, int64_t D, int64_t gate_rows, int64_t ldx, int64_t ldy, int64_t ldgate,
                         int64_t ldh, int64_t ldn, int x_dtype, int y_dtype, int post_norm, float scale, double p,
                         const uint64_t* seed, int64_t row0, float eps, void* stream) {
  return guarded([&]() -> int {
    JoinParams q{};
    const JoinArgs a{T, D, gate_rows, ldgate, row0, x_dtype, y_dtype, post_norm, g_post, g_pre, gate, scale, eps, p, seed};
    if (int st = fill_join(q, a)) return st;
    const int ex = dtype_size(x_dtype), ey = dtype_size(y_dtype);
    const Matrix x{"X", X, T, D, ldx, ex}, y{"Y", Y, T, D, ldy, ey}, h{"H", H, T, D, ldh, ex}, n{"N", N, N ? T : 0, D, ldn, ey};
    for (const Matrix* m : {&x, &y, &h, &n})
      if (int st = check(*m)) return st;
    if (T == 0 || D == 0) return PARTIR_OK;
    if (g_pre && !N) return fail(PARTIR_E_UNSUPPORTED, "g_pre without N");
    const Matrix g = gate_matrix(a), gp{"g_post", g_post, 1, D, D, 4}, gn{"g_pre", g_pre, 1, D, D, 4}, sd{"seed", seed, 1, 2, 2, 8};
    if (int st = check_apart(h, &x, {&y, &n, &g, &gp, &gn, &sd})) return st;
    if (int st = check_apart(n, &y, {&x, &g, &gp, &gn, &sd})) return st;
    q.x = X; q.y = Y; q.h = H; q.n = N;
    q.ldx = ldx; q.ldy = ldy; q.ldh = ldh; q.ldn = ldn;
    join_choice(q, false);
    if (int st = begin_launches()) return st;
    return launched(launch_join(q, x_dtype == PARTIR_BF16, y_dtype == PARTIR_BF16, (hipStream_t)stream), "residual_norm");
  });
}

size_t partir_residual_norm_backward_workspace(int64_t T, int64_t D, int64_t gate_rows) {
  JoinArgs a{T, D, gate_rows, 0, 0, PARTIR_F32, PARTIR_F32, 0, nullptr, nullptr, nullptr, 1.0f, 0.0f, 0.0, nullptr};
  if (guarded([&]() -> int {
        if (int st = validate_join(a)) return st;
        return gate_rows < 0 ? fail(PARTIR_E_SHAPE, "gate_rows = %lld", (long long)gate_rows) : PARTIR_OK;
      }))
    return (size_t)-1;
  if (T == 0 || D == 0) return 0;
  JoinParams p{};
  p.T = T; p.D = (int)D;
  p.gate_rows = gate_rows ? gate_rows : T;
  join_choice(p, true);
  return join_bwd_ws(p);
}

int partir_residual_norm_backward(const void* X, const void* Y, const void* dH, const void* dN, const float* g_post,
                                  const float* gate, const float* g_pre, void* dX, void* dY, float* dg_post, float* dgate,
                                  float* dg_pre, int64_t T, int64_t D, int64_t gate_rows, int64_t ldx, int64_t ldy,
                                  int64_t lddh, int64_t lddn, int64_t ldgate, int64_t lddx, int64_t lddy, int x_dtype,
                                  int y_dtype, int post_norm, float scale, double p, const uint64_t* seed, int64_t row0,
                                  float eps, void* ws, size_t ws_bytes, void* stream) {
  return guarded([&]() -> int {
    JoinParams q{};
    const JoinArgs a{T, D, gate_rows, ldgate, row0, x_dtype, y_dtype, post_norm, g_post, g_pre, gate, scale, eps, p, seed};
    if (int st = fill_join(q, a)) return st;
    const int ex = dtype_size(x_dtype), ey = dtype_size(y_dtype);
    const Matrix x{"X", X, dN ? T : 0, D, ldx, ex}, y{"Y", Y, T, D, ldy, ey}, dh{"dH", dH, dH ? T : 0, D, lddh, ex};
    const Matrix dn{"dN", dN, dN ? T : 0, D, lddn, ey}, dx{"dX", dX, T, D, lddx, ex}, dy{"dY", dY, T, D, lddy, ey};
    for (const Matrix* m : {&x, &y, &dh, &dn, &dx, &dy})
      if (int st = check(*m)) return st;
    if (T > 0 && D > 0 && !dH && !dN) return fail(PARTIR_E_NULL, "dH or dN must be non-NULL");
    // gains of 1 have no gradient; without columns all of these may be NULL
    if (dg_post && !g_post) return fail(PARTIR_E_UNSUPPORTED, "dg_post without g_post");
    if (dg_pre && !g_pre) return fail(PARTIR_E_UNSUPPORTED, "dg_pre without g_pre");
    if (dgate && !gate) return fail(PARTIR_E_UNSUPPORTED, "dgate without a gate");
    if (g_pre && !dN && T > 0) return fail(PARTIR_E_UNSUPPORTED, "g_pre without dN");
    for (const float* g : {dg_post, dgate, dg_pre})
      if (!aligned(g, 16)) return fail(PARTIR_E_LAYOUT, "gradients of gains and gates must be 16-byte aligned");
    if (D == 0) return PARTIR_OK;
    const int64_t groups = gate_groups(a);
    const Matrix g = gate_matrix(a), gp{"g_post", g_post, 1, D, D, 4}, gn{"g_pre", g_pre, 1, D, D, 4}, sd{"seed", seed, 1, 2, 2, 8};
    const Matrix o1{"dg_post", dg_post, 1, D, D, 4}, o2{"dgate", dgate, groups, D, D, 4}, o3{"dg_pre", dg_pre, 1, D, D, 4};
    if (int st = check_apart(dx, &dh, {&x, &y, &dn, &dy, &g, &gp, &gn, &sd, &o1, &o2, &o3})) return st;
    if (int st = check_apart(dy, &dn, {&x, &y, &dh, &g, &gp, &gn, &sd, &o1, &o2, &o3})) return st;
    if (int st = check_apart(o1, nullptr, {&x, &y, &dh, &dn, &g, &gp, &gn, &sd, &o2, &o3})) return st;
    if (int st = check_apart(o2, nullptr, {&x, &y, &dh, &dn, &g, &gp, &gn, &sd, &o3})) return st;
    if (int st = check_apart(o3, nullptr, {&x, &y, &dh, &dn, &g, &gp, &gn, &sd})) return st;
    hipStream_t s = (hipStream_t)stream;
    JoinSums sums{};
    sums.D = (int)D;
    auto add = [&](const float* part, float* out, int64_t outs, int64_t parts) {
      sums.part[sums.n] = part;
      sums.out[sums.n] = out;
      sums.outs[sums.n] = outs;
      sums.parts[sums.n++] = parts;
    };
    if (T == 0) {                        // empty sums
      if (dg_post) add(nullptr, dg_post, 1, 0);
      if (dg_pre) add(nullptr, dg_pre, 1, 0);
      if (!sums.n) return PARTIR_OK;
      if (int st = begin_launches()) return st;
      return launched(launch_join_reduce(sums, s), "residual_norm.sums");
    }
    join_choice(q, true);
    if (int st = check_ws(join_bwd_ws(q), ws, ws_bytes)) return st;
    q.x = X; q.y = Y; q.dh = dH; q.dn = dN; q.dx = dX; q.dy = dY;
    q.ldx = ldx; q.ldy = ldy; q.lddh = lddh; q.lddn = lddn; q.lddx = lddx; q.lddy = lddy;
    float* part = (float*)ws;
    const int64_t n = q.workers * D;
    if (dg_post) {
      q.part_post = part;
      add(q.part_post, dg_post, 1, q.workers);
    }
    if (dg_pre) {
      q.part_pre = part + n;
      add(q.part_pre, dg_pre, 1, q.workers);
    }
    if (dgate && q.chunks == 0) {
      q.dgate_rows = dgate;
    } else if (dgate) {
      q.part_gate = part + 2 * n;
      add(q.part_gate, dgate, groups, q.chunks);
    }
    if (int st = begin_launches()) return st;
    if (int st = launched(launch_join_backward(q, x_dtype == PARTIR_BF16, y_dtype == PARTIR_BF16, s), "residual_norm_backward"))
      return st;
    return sums.n ? launched(launch_join_reduce(sums, s), "residual_norm.sums") : PARTIR_OK;
  });
}

}  // extern "C"
