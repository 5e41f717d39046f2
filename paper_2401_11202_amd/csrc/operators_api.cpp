// Host side of the operators around the loop nests: rotary positions, the
// norms of queries and keys, cross attention, masked attention, the global norm of
// gradients.
// As in partir_api.cpp a call validates its arguments, plans its launches and
// enqueues them on the caller's stream; nothing is enqueued before every
// argument has passed, and no exception leaves an entry point.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <vector>

#include "host_checks.h"
#include "operators.h"

namespace partir {
namespace {

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
  if (p.T == 0) return PARTIR_OK;
  for (int i = 0; i < 2; ++i) {
    if (p.H[i] == 0) continue;
    // in place means row for row; the other tensor's rows are read at other times
    if ((p.y[i] == p.x[i] && p.T > 1 && p.ldy[i] != p.ldx[i]) ||
        (p.lddy[i] >= 0 && p.y[i] == p.dy[i] && p.T > 1 && p.ldy[i] != p.lddy[i]))
      return fail(PARTIR_E_LAYOUT, "an output in its input's place needs its leading dim");
    const int o = 1 - i;
    if (p.H[o] > 0 && (p.y[i] == p.x[o] || p.y[i] == p.y[o] || (p.lddy[o] >= 0 && p.y[i] == p.dy[o])))
      return fail(PARTIR_E_LAYOUT, "the queries' and the keys' tensors share an output");
  }
  return PARTIR_OK;
}

int check_eps(float eps) {
  return eps >= 0.0f && std::isfinite(eps) ? PARTIR_OK : fail(PARTIR_E_UNSUPPORTED, "eps must be finite and not negative");
}

int run_rotary(RotaryParams& p, int dtype, int interleaved, bool norm, void* stream) {
  if (int st = validate_rotary(p, dtype)) return st;
  if (p.T == 0 || p.H[0] + p.H[1] == 0) return PARTIR_OK;
  rotary_choice(p, dtype == PARTIR_BF16, norm ? ROTARY_NORM : ROTARY);
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
// tensors from each workgroup.
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
int check_spans_apart(const void* const* in, void* const* out, const int64_t* numel, const int* dtypes, int n, const float* norm) {
  std::vector<Span> w, r;
  w.reserve(n + 1);
  auto span = [&](const void* p, int i) {
    const uintptr_t lo = (uintptr_t)p;
    return Span{lo, lo + (uintptr_t)numel[i] * (dtypes[i] == PARTIR_BF16 ? 2 : 4), i};
  };
  for (int i = 0; i < n; ++i) {
    if (numel[i] == 0) continue;
    w.push_back(span(out[i], i));
    if (in[i] != out[i]) r.push_back(span(in[i], i));
  }
  w.push_back(Span{(uintptr_t)norm, (uintptr_t)(norm + 1), n});
  auto before = [](const Span& a, const Span& b) { return a.lo < b.lo; };
  if (!std::is_sorted(w.begin(), w.end(), before)) std::sort(w.begin(), w.end(), before);
  if (!std::is_sorted(r.begin(), r.end(), before)) std::sort(r.begin(), r.end(), before);
  for (size_t k = 1; k < w.size(); ++k)
    if (w[k].lo < w[k - 1].hi)
      return fail(PARTIR_E_LAYOUT, "tensors %d and %d overlap (%d: norm)", std::min(w[k].i, w[k - 1].i),
                  std::max(w[k].i, w[k - 1].i), n);
  // inputs may overlap one another: the last end among those before counts
  size_t k = 0;
  for (const Span& s : r) {
    while (k < w.size() && w[k].hi <= s.lo) ++k;
    if (k < w.size() && w[k].lo < s.hi)
      return fail(PARTIR_E_LAYOUT, "the output of tensor %d (%d: norm) overlaps the input of tensor %d", w[k].i, n, s.i);
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
      const bool bf16 = dtypes[i] == PARTIR_BF16;
      t.size[t.n] = (uint64_t)numel[i] + (bf16 ? kGradBf16 : 0);
      t.chunk0[t.n + 1] = t.chunk0[t.n] + (uint32_t)cdiv(numel[i], kGradChunkBytes / (bf16 ? 2 : 4));
      ++t.n;
    }
    if (t.n == 0) {
      all.pop_back();
      continue;
    }
    all.back().workgroups = (int)std::min<int64_t>(t.chunk0[t.n], kGradMaxWorkgroups);
  }
}

// Workspace: a float64 partial for each workgroup of each table, at most, and
// what those are added to where they are many.
size_t grad_ws(int n) {
  if (n <= 0) return 0;
  const size_t parts = (size_t)cdiv(n, kGradTensors) * kGradMaxWorkgroups;
  return align_up((parts + (parts > kGradDirect ? kGradFolded : 0)) * sizeof(double));
}

int run_grads(const void* const* in, void* const* out, const int64_t* numel, const int* dtypes, int n, bool clip,
              double max_norm, float* norm, void* ws, size_t ws_bytes, void* stream) {
  if (int st = validate_grads(in, out, numel, dtypes, n)) return st;
  if (clip && !(max_norm >= 0.0)) return fail(PARTIR_E_UNSUPPORTED, "max_norm must not be negative or NaN");
  if (!norm) return fail(PARTIR_E_NULL, "norm must be non-NULL");
  if (!aligned(norm, 4)) return fail(PARTIR_E_LAYOUT, "norm must be 4-byte aligned");
  if (int st = check_ws(grad_ws(n), ws, ws_bytes)) return st;
  if (clip)
    if (int st = check_spans_apart(in, out, numel, dtypes, n, norm)) return st;
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
  // Every workgroup of a scaling launch adds the partial sums for itself, which
  // saves a launch; but those reads grow with the square of their count, so many
  // are added to a few first (tensors of 64 values, clipped, replayed: 2000 in 107
  // us without and 105 with this launch, 16000 in 1474 and 689).
  if (parts > kGradDirect) {
    if (int st = launched(launch_grad_fold(partial, parts, partial + parts, s), "grad_fold")) return st;
    partial += parts;
    parts = kGradFolded;
  }
  if (!clip || all.empty()) return launched(launch_grad_norm(partial, parts, norm, s), "grad_norm");
  for (size_t i = 0; i < all.size(); ++i)
    if (int st = launched(launch_grad_scale(all[i].t, partial, parts, max_norm, i == 0 ? norm : nullptr,
                                            all[i].workgroups, s), "grad_scale"))
      return st;
  return PARTIR_OK;
}

// ---------------------------------------------------------------------------
// attention to another sequence
// ---------------------------------------------------------------------------
struct CrossSizes {
  int64_t B, Sq, Sk, Hq, Hk, dh;
};

int validate_cross(const CrossSizes& z) {
  if (z.B < 0 || z.Sq < 0 || z.Sk < 0 || z.B > kMaxSize || z.Sq > kMaxSize || z.Sk > kMaxSize)
    return fail(PARTIR_E_SHAPE, "B = %lld, Sq = %lld, Sk = %lld", (long long)z.B, (long long)z.Sq, (long long)z.Sk);
  if (z.dh != 128) return fail(PARTIR_E_SHAPE, "d_head = %lld, only 128 is provided", (long long)z.dh);
  if (z.Hq < 1 || z.Hk < 1 || z.Hq * z.dh > kMaxLd || z.Hk > z.Hq)
    return fail(PARTIR_E_SHAPE, "n_heads = %lld, n_kv_heads = %lld", (long long)z.Hq, (long long)z.Hk);
  if (z.Hq % z.Hk)
    return fail(PARTIR_E_DIVISIBILITY, "n_kv_heads = %lld does not divide n_heads = %lld", (long long)z.Hk, (long long)z.Hq);
  const int64_t G = z.Hq / z.Hk;
  if (z.Sq * G > kMaxSize || z.B * z.Sq > kMaxSize || z.B * z.Sk > kMaxSize)
    return fail(PARTIR_E_SHAPE, "more than 2^30 query rows of a key head, queries or keys");
  // A launch is a grid of fewer than 2^32 threads: 256 for 128 query rows of a key
  // head, 512 for 256 keys.  Parts, at most 64 (256 in the gradients of attention to
  // another sequence), are asked for only below one workgroup a CU; in the gradients of
  // masked attention below 1024 workgroups (masked_parts: where the longest outlasts
  // all of them on 512 places, with half of its steps on average at the least).
  if (z.B * z.Hk * std::max(cdiv(z.Sq * G, 128), 2 * cdiv(z.Sk, 256)) >= ((int64_t)1 << 24) || z.B * z.Sq * z.Hq > ((int64_t)1 << 33))
    return fail(PARTIR_E_SHAPE, "more than 2^32 threads of a launch");
  return PARTIR_OK;
}

int check_lens(const void* lens) {
  return aligned(lens, 4) ? PARTIR_OK : fail(PARTIR_E_LAYOUT, "k_lens must be 4-byte aligned");
}

// scale <= 0 selects 1 / sqrt(d_head)
int resolve_scale(float& scale, int64_t dh) {
  if (std::isnan(scale)) return fail(PARTIR_E_UNSUPPORTED, "scale is NaN");
  if (scale <= 0.0f) scale = 1.0f / std::sqrt((float)dh);
  if (scale < 1e-30f || scale > 1e30f) return fail(PARTIR_E_UNSUPPORTED, "scale outside 1e-30 .. 1e30");
  return PARTIR_OK;
}

constexpr float kLog2e = 1.4426950408889634f;

struct CrossPlan {
  CrossChoice c;
  size_t o_bytes = 0, ml_bytes = 0;
  size_t ws() const { return o_bytes + ml_bytes; }
};
CrossPlan plan_cross(const CrossSizes& z) {
  CrossPlan p;
  p.c = cross_choice(z.B, z.Sq, z.Sk, z.Hq, z.Hk);
  if (p.c.nsplit > 1) {
    const size_t rows = (size_t)p.c.nsplit * z.B * z.Sq * z.Hq;
    p.o_bytes = align_up(rows * z.dh * 4);
    p.ml_bytes = align_up(rows * 8);
  }
  return p;
}

int run_cross(const void* Q, const void* K, const void* V, void* O, float* lse, const CrossSizes& z, int64_t ldq, int64_t ldk,
              int64_t ldv, int64_t ldo, const int32_t* lens, float scale, void* ws, size_t ws_bytes, void* stream) {
  if (int st = validate_cross(z)) return st;
  if (int st = resolve_scale(scale, z.dh)) return st;
  const int64_t Tq = z.B * z.Sq, Tk = z.B * z.Sk;
  if (int st = check_matrix("Q", Q, Tq, z.Hq * z.dh, ldq, 2)) return st;
  if (int st = check_matrix("K", K, Tq ? Tk : 0, z.Hk * z.dh, ldk, 2)) return st;
  if (int st = check_matrix("V", V, Tq ? Tk : 0, z.Hk * z.dh, ldv, 2)) return st;
  if (int st = check_matrix("O", O, Tq, z.Hq * z.dh, ldo, 2)) return st;
  if (int st = check_lens(lens)) return st;
  if (!aligned(lse, 4)) return fail(PARTIR_E_LAYOUT, "lse must be 4-byte aligned");
  if (Tq == 0) return PARTIR_OK;
  // a workgroup holds its rows of Q before it stores those of O, but others read K and V
  if ((Tk > 0 && (O == K || O == V)) || (O == Q && Tq > 1 && ldo != ldq))
    return fail(PARTIR_E_LAYOUT, "O must be Q, with its leading dim, or apart from the inputs");
  const CrossPlan plan = plan_cross(z);
  if (int st = check_ws(plan.ws(), ws, ws_bytes)) return st;
  CrossParams p{};
  p.Q = (const uint16_t*)Q; p.K = (const uint16_t*)K; p.V = (const uint16_t*)V; p.O = (uint16_t*)O;
  p.lse = lse; p.lens = lens;
  p.ldq = ldq; p.ldk = ldk; p.ldv = ldv; p.ldo = ldo;
  p.B = (int)z.B; p.Sq = (int)z.Sq; p.Sk = (int)z.Sk; p.Hq = (int)z.Hq; p.Hk = (int)z.Hk; p.G = (int)(z.Hq / z.Hk);
  p.scale_log2 = scale * kLog2e;
  p.nsplit = plan.c.nsplit;
  p.by_g = Div::by(p.G);
  p.by_hk = Div::by(p.Hk);
  p.by_nbh = Div::by((uint32_t)(z.B * z.Hk));
  p.by_nqb = Div::by((uint32_t)cdiv((int64_t)p.G * z.Sq, 32 * plan.c.qw));
  p.by_split = Div::by(p.nsplit);
  if (p.nsplit > 1) {
    p.Opart = (float*)ws;
    p.MLpart = (float2*)((char*)ws + plan.o_bytes);
  }
  if (int st = begin_launches()) return st;
  if (int st = launched(launch_cross_attention(p, plan.c, (hipStream_t)stream), "cross_attention")) return st;
  if (p.nsplit == 1) return PARTIR_OK;
  return launched(launch_cross_combine(p, (hipStream_t)stream), "cross_combine");
}

struct CrossBwdPlan {
  CrossBwdChoice c{};
  size_t d_bytes = 0, q_bytes = 0, k_bytes = 0;   // k_bytes: of dK's and of dV's partials each
  size_t ws() const { return d_bytes + q_bytes + 2 * k_bytes; }
};
CrossBwdPlan plan_cross_bwd(const CrossSizes& z) {
  CrossBwdPlan p;
  p.c = cross_bwd_choice(z.B, z.Sq, z.Sk, z.Hq, z.Hk);
  if (!p.c.one_pass) p.d_bytes = align_up((size_t)z.B * z.Sq * z.Hq * 4);
  if (p.c.q_parts > 1) p.q_bytes = align_up((size_t)p.c.q_parts * z.B * z.Sq * z.Hq * z.dh * 4);
  if (p.c.k_parts > 1) p.k_bytes = align_up((size_t)p.c.k_parts * z.B * z.Sk * z.Hk * z.dh * 4);
  return p;
}

PartSum part_sum(int n, int parts, int64_t rows, int64_t cols) {
  PartSum r{};
  r.n = n; r.parts = parts; r.rows = rows; r.cols = (int)cols;
  r.by_cols4 = Div::by((uint32_t)(cols / 4));
  return r;
}

// ---------------------------------------------------------------------------
// masked attention
// ---------------------------------------------------------------------------
constexpr int kFormCap = 2, kFormBias = 4;   // bits of a kernel's form

// The checks of a mask, and what the kernels take of it.
int resolve_mask(MaskArgs& m, int& form, const partir_attention_mask* mask, const CrossSizes& z, float scale) {
  if (!mask) return fail(PARTIR_E_NULL, "mask must be non-NULL");
  if (!(mask->cap == 0.0f || (mask->cap >= 0.0009765625f && mask->cap <= 1024.0f)))
    return fail(PARTIR_E_UNSUPPORTED, "cap must be 0 or within 2^-10 .. 2^10");
  if (mask->prefix_lens && !mask->causal) return fail(PARTIR_E_UNSUPPORTED, "prefix_lens without causal");
  const bool pairs = z.B * z.Sq > 0 && z.B * z.Sk > 0;   // else one of the arrays is empty, and NULL perhaps
  if (pairs && !mask->q_docs != !mask->k_docs) return fail(PARTIR_E_NULL, "q_docs and k_docs must be given together");
  const struct { const char* name; const void* p; } all[] = {
      {"slopes", mask->slopes}, {"k_lens", mask->k_lens}, {"q_lens", mask->q_lens}, {"q_starts", mask->q_starts},
      {"prefix_lens", mask->prefix_lens}, {"q_docs", mask->q_docs}, {"k_docs", mask->k_docs}};
  for (const auto& a : all)
    if (!aligned(a.p, 4)) return fail(PARTIR_E_LAYOUT, "%s must be 4-byte aligned", a.name);
  m.q_lens = mask->q_lens; m.q_starts = mask->q_starts; m.prefix = mask->prefix_lens;
  if (pairs) {
    m.q_docs = mask->q_docs;
    m.k_docs = mask->k_docs;
  }
  m.slopes = mask->slopes;
  m.causal = mask->causal != 0;
  form = (mask->cap > 0.0f ? kFormCap : 0) | (mask->slopes ? kFormBias : 0);
  if (mask->cap > 0.0f) {
    m.cap_log2 = mask->cap * kLog2e;
    m.cap_rate = 2.0f * scale * kLog2e / mask->cap;
    if (!(m.cap_rate > 1e-30f && m.cap_rate < 1e30f)) return fail(PARTIR_E_UNSUPPORTED, "scale / cap outside 1e-30 .. 1e30");
    // tanh x = x (c0 + c1 x^2 + ..) up to x = 5 / 8, in powers of q k; with a scale / cap
    // whose ninth power float32 does not hold the other form takes all
    const double c[5] = {0.9999998917, -0.3333194271, 0.133043797, -0.05181591168, 0.01504335657};
    const double x = (double)scale / mask->cap, a = (double)mask->cap * 1.4426950408889634;
    m.cap_small = x > 0x1p-12 && x < 0x1p4 ? (float)(0.625 / x) : -1.0f;
    for (int i = 0; i < 5; ++i) m.cap_c[i] = m.cap_small > 0.0f ? (float)(a * c[i] * std::pow(x, 2 * i + 1)) : 0.0f;
  }
  return PARTIR_OK;
}

// An output is apart from the mask's arrays: a length that changed during a launch
// would send a workgroup's waves different ways.
int check_mask_apart(const Matrix& out, const partir_attention_mask& m, const CrossSizes& z) {
  const auto ints = [&](const char* name, const void* p, int64_t n) { return Matrix{name, p, p ? 1 : 0, n, n, 4}; };
  const Matrix slopes = ints("slopes", m.slopes, z.Hq), k = ints("k_lens", m.k_lens, z.B), q = ints("q_lens", m.q_lens, z.B);
  const Matrix at = ints("q_starts", m.q_starts, z.B), pre = ints("prefix_lens", m.prefix_lens, z.B);
  const Matrix qd = ints("q_docs", m.q_docs, z.B * z.Sq), kd = ints("k_docs", m.k_docs, z.B * z.Sk);
  return check_apart(out, nullptr, {&slopes, &k, &q, &at, &pre, &qd, &kd});
}

// The intervals of documents, at the front of the workspace.
struct DocPlan {
  int q_blocks = 0;
  size_t row_bytes = 0, block_bytes = 0, id_bytes = 0;
  size_t ws() const { return row_bytes + block_bytes + id_bytes; }
};
DocPlan plan_docs(const CrossSizes& z, const partir_attention_mask& mask) {
  DocPlan d;
  if (!mask.k_docs || z.B * z.Sq == 0 || z.B * z.Sk == 0) return d;
  d.q_blocks = (int)cdiv(z.Sq, 64);
  d.row_bytes = align_up((size_t)z.B * z.Sq * 8);
  d.block_bytes = align_up((size_t)z.B * d.q_blocks * 8);
  d.id_bytes = align_up((size_t)z.B * 4);
  return d;
}

int run_doc_rows(MaskArgs& m, const DocPlan& d, const CrossSizes& z, const int32_t* k_lens, void* ws, hipStream_t s) {
  if (!d.ws()) return PARTIR_OK;
  DocRows t{};
  t.q_docs = m.q_docs; t.k_docs = m.k_docs; t.q_lens = m.q_lens; t.k_lens = k_lens;
  t.rows = (int2*)ws;
  t.blocks = (int2*)((char*)ws + d.row_bytes);
  t.by_id = (int32_t*)((char*)ws + d.row_bytes + d.block_bytes);
  t.B = (int)z.B; t.Sq = (int)z.Sq; t.Sk = (int)z.Sk; t.q_blocks = d.q_blocks;
  m.rows = t.rows; m.blocks = t.blocks; m.by_id = t.by_id; m.q_blocks = d.q_blocks;
  return launched(launch_doc_rows(t, s), "doc_rows");
}

// What forward and backward kernels share of their parameters.
template <typename P>
void fill_sizes(P& p, const CrossSizes& z) {
  p.B = (int)z.B; p.Sq = (int)z.Sq; p.Sk = (int)z.Sk; p.Hq = (int)z.Hq; p.Hk = (int)z.Hk; p.G = (int)(z.Hq / z.Hk);
  p.by_g = Div::by(p.G);
  p.by_hk = Div::by(p.Hk);
  p.by_nbh = Div::by((uint32_t)(z.B * z.Hk));
}

int run_masked(const void* Q, const void* K, const void* V, void* O, float* lse, bool train, const CrossSizes& z, int64_t ldq,
               int64_t ldk, int64_t ldv, int64_t ldo, const partir_attention_mask* mask, float scale, void* ws, size_t ws_bytes,
               void* stream) {
  if (int st = validate_cross(z)) return st;
  if (int st = resolve_scale(scale, z.dh)) return st;
  MaskedParams p{};
  int form = 0;
  if (int st = resolve_mask(p.mask, form, mask, z, scale)) return st;
  const int64_t Tq = z.B * z.Sq, Tk = z.B * z.Sk;
  const Matrix q{"Q", Q, Tq, z.Hq * z.dh, ldq, 2}, k{"K", K, Tq ? Tk : 0, z.Hk * z.dh, ldk, 2};
  const Matrix v{"V", V, Tq ? Tk : 0, z.Hk * z.dh, ldv, 2}, o{"O", O, Tq, z.Hq * z.dh, ldo, 2};
  const Matrix l{"lse", lse, lse ? Tq : 0, z.Hq, z.Hq, 4};
  for (const Matrix* m : {&q, &k, &v, &o})
    if (int st = check(*m)) return st;
  if (train && Tq > 0 && !lse) return fail(PARTIR_E_NULL, "lse must be non-NULL");
  if (!aligned(lse, 4)) return fail(PARTIR_E_LAYOUT, "lse must be 4-byte aligned");
  if (Tq == 0) return PARTIR_OK;
  if (int st = check_apart(o, &q, {&k, &v, &l})) return st;   // a workgroup holds its rows of Q before it stores those of O
  if (int st = check_apart(l, nullptr, {&q, &k, &v})) return st;
  for (const Matrix* out : {&o, &l})
    if (int st = check_mask_apart(*out, *mask, z)) return st;
  const CrossPlan plan = plan_cross(z);
  const DocPlan docs = plan_docs(z, *mask);
  if (int st = check_ws(docs.ws() + plan.ws(), ws, ws_bytes)) return st;
  p.Q = (const uint16_t*)Q; p.K = (const uint16_t*)K; p.V = (const uint16_t*)V; p.O = (uint16_t*)O;
  p.lse = lse; p.lens = mask->k_lens;
  p.ldq = ldq; p.ldk = ldk; p.ldv = ldv; p.ldo = ldo;
  fill_sizes(p, z);
  p.scale_log2 = scale * kLog2e;
  p.nsplit = plan.c.nsplit;
  p.by_nqb = Div::by((uint32_t)cdiv((int64_t)p.G * z.Sq, 32 * plan.c.qw));
  p.by_split = Div::by(p.nsplit);
  if (p.nsplit > 1) {
    p.Opart = (float*)((char*)ws + docs.ws());
    p.MLpart = (float2*)((char*)ws + docs.ws() + plan.o_bytes);
  }
  if (int st = begin_launches()) return st;
  hipStream_t s = (hipStream_t)stream;
  if (int st = run_doc_rows(p.mask, docs, z, mask->k_lens, ws, s)) return st;
  if (int st = launched(launch_masked_attention(p, form, plan.c, s), "masked_attention")) return st;
  return p.nsplit == 1 ? PARTIR_OK : launched(launch_masked_combine(p, s), "masked_combine");
}

CrossBwdPlan plan_masked_bwd(const CrossSizes& z, const partir_attention_mask& mask) {
  CrossBwdPlan p;
  p.c = masked_bwd_choice(z.B, z.Sq, z.Sk, z.Hq, z.Hk, mask.causal != 0);
  if (!p.c.one_pass) p.d_bytes = align_up((size_t)p.c.q_parts * z.B * z.Sq * z.Hq * 4);
  if (p.c.q_parts > 1) p.q_bytes = align_up((size_t)p.c.q_parts * z.B * z.Sq * z.Hq * z.dh * 4);
  if (p.c.k_parts > 1) p.k_bytes = align_up((size_t)p.c.k_parts * z.B * z.Sk * z.Hk * z.dh * 4);
  return p;
}

void fill_info(partir_plan_info* info, int shards, int launches, size_t ws, double flops) {
  info->n_virtual_shards = shards;
  info->n_tile_loops = 1;                       // the heads
  info->n_sum_loops = info->n_sum_splitk = shards > 1;
  info->n_launches = launches;
  info->reserved = 0;
  info->workspace_bytes = ws;
  info->flops = flops;
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
  rotary_choice(p, dtype == PARTIR_BF16, ROTARY_NORM_BWD);
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
    if (dgq && dgq == dgk) return fail(PARTIR_E_LAYOUT, "dgq must not be dgk");
    const bool empty = p.T == 0 || p.H[0] + p.H[1] == 0;
    if (!empty) {
      rotary_choice(p, dtype == PARTIR_BF16, ROTARY_NORM_BWD);
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

// ---- attention to another sequence ------------------------------------------------
size_t partir_cross_attention_workspace(int64_t B, int64_t Sq, int64_t Sk, int64_t n_heads, int64_t n_kv_heads,
                                        int64_t d_head) {
  const CrossSizes z{B, Sq, Sk, n_heads, n_kv_heads, d_head};
  if (guarded([&]() -> int { return validate_cross(z); })) return (size_t)-1;
  return plan_cross(z).ws();
}

int partir_plan_cross_attention(int64_t B, int64_t Sq, int64_t Sk, int64_t n_heads, int64_t n_kv_heads, int64_t d_head,
                                partir_plan_info* info) {
  return guarded([&]() -> int {
    const CrossSizes z{B, Sq, Sk, n_heads, n_kv_heads, d_head};
    if (int st = validate_cross(z)) return st;
    if (!info) return fail(PARTIR_E_NULL, "info must be non-NULL");
    const CrossPlan p = plan_cross(z);
    fill_info(info, p.c.nsplit, B * Sq == 0 ? 0 : p.c.nsplit > 1 ? 2 : 1, p.ws(),
              4.0 * (double)B * (double)Sq * (double)Sk * (double)(n_heads * d_head));
    return PARTIR_OK;
  });
}

int partir_cross_attention(const void* Q, const void* K, const void* V, void* O, int64_t B, int64_t Sq, int64_t Sk,
                           int64_t n_heads, int64_t n_kv_heads, int64_t d_head, int64_t ldq, int64_t ldk, int64_t ldv,
                           int64_t ldo, const int32_t* k_lens, float scale, void* ws, size_t ws_bytes, void* stream) {
  return guarded([&]() -> int {
    return run_cross(Q, K, V, O, nullptr, {B, Sq, Sk, n_heads, n_kv_heads, d_head}, ldq, ldk, ldv, ldo, k_lens, scale, ws,
                     ws_bytes, stream);
  });
}

int partir_cross_attention_train(const void* Q, const void* K, const void* V, void* O, float* lse, int64_t B, int64_t Sq,
                                 int64_t Sk, int64_t n_heads, int64_t n_kv_heads, int64_t d_head, int64_t ldq, int64_t ldk,
                                 int64_t ldv, int64_t ldo, const int32_t* k_lens, float scale, void* ws, size_t ws_bytes,
                                 void* stream) {
  return guarded([&]() -> int {
    if (B > 0 && Sq > 0 && !lse) return fail(PARTIR_E_NULL, "lse must be non-NULL");
    return run_cross(Q, K, V, O, lse, {B, Sq, Sk, n_heads, n_kv_heads, d_head}, ldq, ldk, ldv, ldo, k_lens, scale, ws,
                     ws_bytes, stream);
  });
}

size_t partir_cross_attention_backward_workspace(int64_t B, int64_t Sq, int64_t Sk, int64_t n_heads, int64_t n_kv_heads,
                                                 int64_t d_head) {
  const CrossSizes z{B, Sq, Sk, n_heads, n_kv_heads, d_head};
  if (guarded([&]() -> int { return validate_cross(z); })) return (size_t)-1;
  return plan_cross_bwd(z).ws();
}

int partir_plan_cross_attention_backward(int64_t B, int64_t Sq, int64_t Sk, int64_t n_heads, int64_t n_kv_heads,
                                         int64_t d_head, partir_plan_info* info) {
  return guarded([&]() -> int {
    const CrossSizes z{B, Sq, Sk, n_heads, n_kv_heads, d_head};
    if (int st = validate_cross(z)) return st;
    if (!info) return fail(PARTIR_E_NULL, "info must be non-NULL");
    const CrossBwdPlan p = plan_cross_bwd(z);
    int launches = 0;
    if (p.c.one_pass)
      launches = B ? 1 + (p.c.k_parts > 1) : 0;
    else
      launches = (B * Sq ? 1 + (p.c.q_parts > 1) : 0) + (B * Sk ? 1 + (p.c.k_parts > 1) : 0);
    fill_info(info, std::max(p.c.q_parts, p.c.k_parts), launches, p.ws(),
              10.0 * (double)B * (double)Sq * (double)Sk * (double)(n_heads * d_head));
    return PARTIR_OK;
  });
}

int partir_cross_attention_backward(const void* Q, const void* K, const void* V, const void* O, const void* dO,
                                    const float* lse, void* dQ, void* dK, void* dV, int64_t B, int64_t Sq, int64_t Sk,
                                    int64_t n_heads, int64_t n_kv_heads, int64_t d_head, int64_t ldq, int64_t ldk,
                                    int64_t ldv, int64_t ldo, int64_t lddo, int64_t lddq, int64_t lddk, int64_t lddv,
                                    const int32_t* k_lens, float scale, void* ws, size_t ws_bytes, void* stream) {
  return guarded([&]() -> int {
    const CrossSizes z{B, Sq, Sk, n_heads, n_kv_heads, d_head};
    if (int st = validate_cross(z)) return st;
    if (int st = resolve_scale(scale, d_head)) return st;
    const int64_t Tq = B * Sq, Tk = B * Sk, cq = n_heads * d_head, ck = n_kv_heads * d_head;
    const struct { const char* name; const void* p; int64_t rows, cols, ld; } all[] = {
        {"Q", Q, Tq, cq, ldq}, {"K", K, Tk, ck, ldk}, {"V", V, Tk, ck, ldv}, {"O", O, Tq, cq, ldo}, {"dO", dO, Tq, cq, lddo},
        {"dQ", dQ, Tq, cq, lddq}, {"dK", dK, Tk, ck, lddk}, {"dV", dV, Tk, ck, lddv}};
    for (const auto& m : all)
      if (int st = check_matrix(m.name, m.p, m.rows, m.cols, m.ld, 2)) return st;
    for (int o = 5; o < 8; ++o)
      for (int i = 0; i < 8; ++i)
        if (i != o && all[o].rows * all[i].rows > 0 && all[o].p == all[i].p)
          return fail(PARTIR_E_LAYOUT, "%s must not be %s", all[o].name, all[i].name);
    if (int st = check_lens(k_lens)) return st;
    if (Tq > 0 && !lse) return fail(PARTIR_E_NULL, "lse must be non-NULL");
    if (!aligned(lse, 4)) return fail(PARTIR_E_LAYOUT, "lse must be 4-byte aligned");
    if (Tq == 0 && Tk == 0) return PARTIR_OK;
    const CrossBwdPlan plan = plan_cross_bwd(z);
    if (int st = check_ws(plan.ws(), ws, ws_bytes)) return st;
    CrossBwdParams p{};
    p.Q = (const uint16_t*)Q; p.K = (const uint16_t*)K; p.V = (const uint16_t*)V; p.O = (const uint16_t*)O;
    p.dO = (const uint16_t*)dO; p.lse = lse; p.lens = k_lens;
    p.dQ = (uint16_t*)dQ; p.dK = (uint16_t*)dK; p.dV = (uint16_t*)dV;
    char* base = (char*)ws;
    p.Dstat = (float*)base;
    p.dQpart = (float*)(base + plan.d_bytes);
    p.dKpart = (float*)(base + plan.d_bytes + plan.q_bytes);
    p.dVpart = (float*)(base + plan.d_bytes + plan.q_bytes + plan.k_bytes);
    p.ldq = ldq; p.ldk = ldk; p.ldv = ldv; p.ldo = ldo; p.ldg = lddo; p.lddq = lddq; p.lddk = lddk; p.lddv = lddv;
    p.B = (int)B; p.Sq = (int)Sq; p.Sk = (int)Sk; p.Hq = (int)n_heads; p.Hk = (int)n_kv_heads; p.G = (int)(n_heads / n_kv_heads);
    p.q_parts = plan.c.q_parts; p.k_parts = plan.c.k_parts;
    p.by_g = Div::by(p.G);
    p.by_hk = Div::by(p.Hk);
    p.by_nbh = Div::by((uint32_t)(B * n_kv_heads));
    p.by_nqb = Div::by((uint32_t)std::max<int64_t>(cdiv((int64_t)p.G * Sq, 128), 1));
    p.by_q_parts = Div::by(p.q_parts);
    p.by_k_parts = Div::by(p.k_parts);
    p.scale = scale;
    p.scale_log2 = scale * kLog2e;
    if (int st = begin_launches()) return st;
    hipStream_t s = (hipStream_t)stream;
    if (plan.c.one_pass) {   // so there are keys
      if (int st = launched(launch_cross_backward(p, CROSS_ALL, s), "cross_bwd")) return st;
    } else {
      if (Tq > 0) {
        if (int st = launched(launch_cross_backward(p, CROSS_DQ, s), "cross_bwd_dq")) return st;
        if (p.q_parts > 1) {
          PartSum r = part_sum(1, p.q_parts, Tq, cq);
          r.part[0] = p.dQpart; r.out[0] = p.dQ; r.ld[0] = lddq;
          if (int st = launched(launch_part_sum(r, s), "cross_bwd_dq.sum")) return st;
        }
      }
      if (Tk == 0) return PARTIR_OK;
      if (int st = launched(launch_cross_backward(p, CROSS_DKV, s), "cross_bwd_dkv")) return st;
    }
    if (p.k_parts == 1) return PARTIR_OK;
    PartSum r = part_sum(2, p.k_parts, Tk, ck);
    r.part[0] = p.dKpart; r.out[0] = p.dK; r.ld[0] = lddk;
    r.part[1] = p.dVpart; r.out[1] = p.dV; r.ld[1] = lddv;
    return launched(launch_part_sum(r, s), "cross_bwd_dkv.sum");
  });
}

// ---- masked attention ---------------------------------------------------------------
size_t partir_masked_attention_workspace(int64_t B, int64_t Sq, int64_t Sk, int64_t n_heads, int64_t n_kv_heads,
                                         int64_t d_head, const partir_attention_mask* mask) {
  const CrossSizes z{B, Sq, Sk, n_heads, n_kv_heads, d_head};
  if (guarded([&]() -> int {
        if (!mask) return fail(PARTIR_E_NULL, "mask must be non-NULL");
        return validate_cross(z);
      }))
    return (size_t)-1;
  return B * Sq ? plan_docs(z, *mask).ws() + plan_cross(z).ws() : 0;
}

int partir_plan_masked_attention(int64_t B, int64_t Sq, int64_t Sk, int64_t n_heads, int64_t n_kv_heads, int64_t d_head,
                                 const partir_attention_mask* mask, partir_plan_info* info) {
  return guarded([&]() -> int {
    const CrossSizes z{B, Sq, Sk, n_heads, n_kv_heads, d_head};
    if (int st = validate_cross(z)) return st;
    if (!mask || !info) return fail(PARTIR_E_NULL, "mask and info must be non-NULL");
    const CrossPlan p = plan_cross(z);
    const size_t docs = plan_docs(z, *mask).ws();
    const bool any = B * Sq > 0;
    fill_info(info, p.c.nsplit, any ? (docs > 0) + 1 + (p.c.nsplit > 1) : 0, any ? docs + p.ws() : 0,
              4.0 * (double)B * (double)Sq * (double)Sk * (double)(n_heads * d_head));
    return PARTIR_OK;
  });
}

int partir_masked_attention(const void* Q, const void* K, const void* V, void* O, int64_t B, int64_t Sq, int64_t Sk,
                            int64_t n_heads, int64_t n_kv_heads, int64_t d_head, int64_t ldq, int64_t ldk, int64_t ldv,
                            int64_t ldo, const partir_attention_mask* mask, float scale, void* ws, size_t ws_bytes,
                            void* stream) {
  return guarded([&]() -> int {
    return run_masked(Q, K, V, O, nullptr, false, {B, Sq, Sk, n_heads, n_kv_heads, d_head}, ldq, ldk, ldv, ldo, mask, scale,
                      ws, ws_bytes, stream);
  });
}

int partir_masked_attention_train(const void* Q, const void* K, const void* V, void* O, float* lse, int64_t B, int64_t Sq,
                                  int64_t Sk, int64_t n_heads, int64_t n_kv_heads, int64_t d_head, int64_t ldq, int64_t ldk,
                                  int64_t ldv, int64_t ldo, const partir_attention_mask* mask, float scale, void* ws,
                                  size_t ws_bytes, void* stream) {
  return guarded([&]() -> int {
    return run_masked(Q, K, V, O, lse, true, {B, Sq, Sk, n_heads, n_kv_heads, d_head}, ldq, ldk, ldv, ldo, mask, scale, ws,
                      ws_bytes, stream);
  });
}

size_t partir_masked_attention_backward_workspace(int64_t B, int64_t Sq, int64_t Sk, int64_t n_heads, int64_t n_kv_heads,
                                                  int64_t d_head, const partir_attention_mask* mask) {
  const CrossSizes z{B, Sq, Sk, n_heads, n_kv_heads, d_head};
  if (guarded([&]() -> int {
        if (!mask) return fail(PARTIR_E_NULL, "mask must be non-NULL");
        return validate_cross(z);
      }))
    return (size_t)-1;
  return B * (Sq + Sk) ? plan_docs(z, *mask).ws() + plan_masked_bwd(z, *mask).ws() : 0;
}

int partir_plan_masked_attention_backward(int64_t B, int64_t Sq, int64_t Sk, int64_t n_heads, int64_t n_kv_heads,
                                          int64_t d_head, const partir_attention_mask* mask, partir_plan_info* info) {
  return guarded([&]() -> int {
    const CrossSizes z{B, Sq, Sk, n_heads, n_kv_heads, d_head};
    if (int st = validate_cross(z)) return st;
    if (!mask || !info) return fail(PARTIR_E_NULL, "mask and info must be non-NULL");
    const CrossBwdPlan p = plan_masked_bwd(z, *mask);
    const size_t docs = plan_docs(z, *mask).ws();
    const int launches = (docs > 0) + (B * Sq && !p.c.one_pass ? 1 + (p.c.q_parts > 1) : 0) +
                         (B * Sk ? 1 + (p.c.k_parts > 1) : 0);
    fill_info(info, std::max(p.c.q_parts, p.c.k_parts), launches, B * (Sq + Sk) ? docs + p.ws() : 0,
              10.0 * (double)B * (double)Sq * (double)Sk * (double)(n_heads * d_head));
    return PARTIR_OK;
  });
}

int partir_masked_attention_backward(const void* Q, const void* K, const void* V, const void* O, const void* dO,
                                     const float* lse, void* dQ, void* dK, void* dV, int64_t B, int64_t Sq, int64_t Sk,
                                     int64_t n_heads, int64_t n_kv_heads, int64_t d_head, int64_t ldq, int64_t ldk,
                                     int64_t ldv, int64_t ldo, int64_t lddo, int64_t lddq, int64_t lddk, int64_t lddv,
                                     const partir_attention_mask* mask, float scale, void* ws, size_t ws_bytes, void* stream) {
  return guarded([&]() -> int {
    const CrossSizes z{B, Sq, Sk, n_heads, n_kv_heads, d_head};
    if (int st = validate_cross(z)) return st;
    if (int st = resolve_scale(scale, d_head)) return st;
    MaskedBwdParams p{};
    int form = 0;
    if (int st = resolve_mask(p.mask, form, mask, z, scale)) return st;
    const int64_t Tq = B * Sq, Tk = B * Sk, cq = n_heads * d_head, ck = n_kv_heads * d_head;
    const Matrix q{"Q", Q, Tq, cq, ldq, 2}, k{"K", K, Tk, ck, ldk, 2}, v{"V", V, Tk, ck, ldv, 2}, o{"O", O, Tq, cq, ldo, 2};
    const Matrix g{"dO", dO, Tq, cq, lddo, 2}, l{"lse", lse, Tq, n_heads, n_heads, 4};
    const Matrix dq{"dQ", dQ, Tq, cq, lddq, 2}, dk{"dK", dK, Tk, ck, lddk, 2}, dv{"dV", dV, Tk, ck, lddv, 2};
    for (const Matrix* m : {&q, &k, &v, &o, &g, &dq, &dk, &dv})
      if (int st = check(*m)) return st;
    if (int st = check_apart(dq, nullptr, {&q, &k, &v, &o, &g, &l, &dk, &dv})) return st;
    if (int st = check_apart(dk, nullptr, {&q, &k, &v, &o, &g, &l, &dv})) return st;
    if (int st = check_apart(dv, nullptr, {&q, &k, &v, &o, &g, &l})) return st;
    for (const Matrix* out : {&dq, &dk, &dv})
      if (int st = check_mask_apart(*out, *mask, z)) return st;
    if (Tq > 0 && !lse) return fail(PARTIR_E_NULL, "lse must be non-NULL");
    if (!aligned(lse, 4)) return fail(PARTIR_E_LAYOUT, "lse must be 4-byte aligned");
    if (Tq == 0 && Tk == 0) return PARTIR_OK;
    const CrossBwdPlan plan = plan_masked_bwd(z, *mask);
    const DocPlan docs = plan_docs(z, *mask);
    if (int st = check_ws(docs.ws() + plan.ws(), ws, ws_bytes)) return st;
    p.Q = (const uint16_t*)Q; p.K = (const uint16_t*)K; p.V = (const uint16_t*)V; p.O = (const uint16_t*)O;
    p.dO = (const uint16_t*)dO; p.lse = lse; p.lens = mask->k_lens;
    p.dQ = (uint16_t*)dQ; p.dK = (uint16_t*)dK; p.dV = (uint16_t*)dV;
    char* base = (char*)ws + docs.ws();
    p.Dstat = (float*)base;
    p.dQpart = (float*)(base + plan.d_bytes);
    p.dKpart = (float*)(base + plan.d_bytes + plan.q_bytes);
    p.dVpart = (float*)(base + plan.d_bytes + plan.q_bytes + plan.k_bytes);
    p.ldq = ldq; p.ldk = ldk; p.ldv = ldv; p.ldo = ldo; p.ldg = lddo; p.lddq = lddq; p.lddk = lddk; p.lddv = lddv;
    fill_sizes(p, z);
    p.q_parts = plan.c.q_parts; p.k_parts = plan.c.k_parts;
    p.by_nqb = Div::by((uint32_t)std::max<int64_t>(cdiv((int64_t)p.G * Sq, 128), 1));
    p.by_q_parts = Div::by(p.q_parts);
    p.by_k_parts = Div::by(p.k_parts);
    p.scale = scale;
    p.scale_log2 = scale * kLog2e;
    if (int st = begin_launches()) return st;
    hipStream_t s = (hipStream_t)stream;
    if (int st = run_doc_rows(p.mask, docs, z, mask->k_lens, ws, s)) return st;
    if (Tq > 0 && !plan.c.one_pass) {
      if (int st = launched(launch_masked_backward(p, form, CROSS_DQ, s), "masked_bwd_dq")) return st;
      if (p.q_parts > 1) {
        PartSum r = part_sum(1, p.q_parts, Tq, cq);
        r.part[0] = p.dQpart; r.out[0] = p.dQ; r.ld[0] = lddq;
        if (int st = launched(launch_part_sum(r, s), "masked_bwd_dq.sum")) return st;
      }
    }
    if (Tk == 0) return PARTIR_OK;
    if (int st = launched(launch_masked_backward(p, form, plan.c.one_pass ? CROSS_ALL : CROSS_DKV, s), "masked_bwd")) return st;
    if (p.k_parts == 1) return PARTIR_OK;
    PartSum r = part_sum(2, p.k_parts, Tk, ck);
    r.part[0] = p.dKpart; r.out[0] = p.dK; r.ld[0] = lddk;
    r.part[1] = p.dVpart; r.out[1] = p.dV; r.ld[1] = lddv;
    return launched(launch_part_sum(r, s), "masked_bwd.sum");
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
