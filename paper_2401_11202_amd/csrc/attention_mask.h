// Which keys a query of the masked attention sees, and how its scores are
// changed: what the forward and the gradient kernels share.
//
// F, the form of a kernel: 0 attention to another sequence (every key below the
// sequence's length), else kMasked, with kCap and kBias as the call has them.
//
// A query sees the keys of an interval [lo, lim): position p = q_start + s sees
//   j < min(k_len, causal ? max(p + 1, prefix) : k_len),
// and where there are documents those of its own, a run of keys that a launch
// before has found (doc_rows_kernel).  So masks are two comparisons, which a block
// of keys needs only where it crosses an end of a row's interval; blocks outside of
// every row's are not read.  Documents that lie in pieces have no interval: their
// sequence's keys are compared by number (by_id).
#pragma once
#include "attention_tiles.h"
#include "operators.h"

namespace partir {

constexpr int kMasked = 1, kCap = 2, kBias = 4;
constexpr int kNowhere = 2147483647;   // lo of a row that sees no key
constexpr float kLog2e = 1.4426950408889634f;

// What the forward and gradient kernels of form F take.
template <int F>
struct FormParams {
  typedef MaskedParams fwd;
  typedef MaskedBwdParams bwd;
};
template <>
struct FormParams<0> {
  typedef CrossParams fwd;
  typedef CrossBwdParams bwd;
};

__device__ __forceinline__ int clamp_len(const int32_t* lens, int b, int most) {
  return lens ? min(max(lens[b], 0), most) : most;
}

// A sequence's numbers.
struct SeqMask {
  int klen, qlen, start, prefix, causal;
  template <typename P>
  __device__ __forceinline__ SeqMask(const P& p, int b) {
    klen = clamp_len(p.lens, b, p.Sk);
    qlen = clamp_len(p.mask.q_lens, b, p.Sq);
    start = p.mask.q_starts ? min(max(p.mask.q_starts[b], -(1 << 29)), 1 << 29) : p.Sk - p.Sq;
    prefix = p.mask.prefix ? min(max(p.mask.prefix[b], 0), klen) : 0;
    causal = p.mask.causal;
  }
  // end of what query s may see, documents aside; it does not fall with s
  __device__ __forceinline__ int lim(int s) const {
    return causal ? min(max(start + s + 1, prefix), klen) : klen;   // s < 2^30
  }
};

// The keys [begin, end) that queries s0 .. s1 (below q_len) of a sequence may see,
// from a multiple of 64 on.
template <typename P>
__device__ __forceinline__ int2 key_range(const P& p, const SeqMask& m, int b, int s0, int s1) {
  int lo = 0, hi = m.lim(s1);
  if (p.mask.rows) {
    const int2* blocks = p.mask.blocks + (int64_t)b * p.mask.q_blocks;
    int from = kNowhere, to = 0;
    for (int i = s0 >> 6; i <= s1 >> 6; ++i) {
      const int2 e = blocks[i];
      from = min(from, e.x);
      to = max(to, e.y);
    }
    lo = from == kNowhere ? 0 : from & ~63;
    hi = min(hi, to);
  }
  return make_int2(lo, max(lo, hi));
}

// A lane's row of a wave's 32 (lane & 31), and what they have in common.
struct RowMask {
  int lo, lim;               // this lane's row sees [lo, lim); none: [kNowhere, 0)
  int lo0, lo1, lim0, lim1;  // least and largest of the wave's
  int pos;                   // the row's position
  template <typename P>
  __device__ __forceinline__ RowMask(const P& p, const SeqMask& m, int64_t tq, int s)
      : RowMask(m, p.mask.rows != nullptr, p.mask.rows ? p.mask.rows[tq] : make_int2(0, 0), s) {}
  // e: where there are documents, the keys of the row's
  __device__ __forceinline__ RowMask(const SeqMask& m, bool docs, int2 e, int s) {
    pos = m.start + s;
    lo = 0;
    lim = s < m.qlen ? m.lim(s) : 0;
    if (!docs) {             // the rows ascend, and so do their limits
      if (lim <= 0) lo = kNowhere;
      lo0 = 0;
      lo1 = __builtin_amdgcn_readlane(lo, 0);
      lim0 = __builtin_amdgcn_readlane(lim, 0);
      lim1 = __builtin_amdgcn_readlane(lim, 31);
      return;
    }
    lo = e.x;
    lim = min(lim, e.y);
    if (lim <= lo) {
      lo = kNowhere;
      lim = 0;
    }
    int a = lo, b = lo, c = lim, d = lim;
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) {
      a = min(a, __shfl_xor(a, o));
      b = max(b, __shfl_xor(b, o));
      c = min(c, __shfl_xor(c, o));
      d = max(d, __shfl_xor(d, o));
    }
    lo0 = __builtin_amdgcn_readfirstlane(a);
    lo1 = __builtin_amdgcn_readfirstlane(b);
    lim0 = __builtin_amdgcn_readfirstlane(c);
    lim1 = __builtin_amdgcn_readfirstlane(d);
  }
  // whether no row of the wave sees any of n keys from key0 on; and whether all rows see all of them
  __device__ __forceinline__ bool none(int key0, int n) const { return key0 >= lim1 || key0 + n <= lo0; }
  __device__ __forceinline__ bool all(int key0, int n) const { return key0 >= lo1 && key0 + n <= lim0; }
};

// Score s = q k, in units of log2: z = cap tanh(scale s / cap) log2 e with
// tanh x = 1 - 2 / (1 + e^(2x)); r = 1 / (1 + e^(2x)) gives its derivative too,
// 1 - tanh^2 = 4 (r - r^2).  z is off by 2^-20 of the cap at most (the roundings of
// exp2, of the sum and of the reciprocal, each of numbers up to 1), which for caps up
// to 1024, the most that a call takes, stays below a weight's rounding to bf16.
// z = a - 2 cap log2 e r for a = cap log2 e, or less what the caller subtracts anyway.
__device__ __forceinline__ float cap_r(float s, float rate) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(s * rate));
}
// Where no score of a wave's block is above 5 / 8 of the cap, the forward kernel takes
// an odd polynomial of degree 9 for tanh (interpolated at Chebyshev's points, off by
// 1.2e-7 in float32): six instructions, where exp2 and the reciprocal, at a quarter of
// the others' rate, make the other form's five as long as eleven (2 x 4096 tokens, 32 / 8
// heads: 400 -> 377 us).  The gradients keep the other form: a branch between their
// products costs them more (dK and dV 728 -> 961 us).
__device__ __forceinline__ float cap_small(float s, const MaskArgs& m) {
  const float u = s * s;
  float p = __builtin_fmaf(u, m.cap_c[4], m.cap_c[3]);
  p = __builtin_fmaf(u, p, m.cap_c[2]);
  p = __builtin_fmaf(u, p, m.cap_c[1]);
  p = __builtin_fmaf(u, p, m.cap_c[0]);
  return s * p;
}

// The weights P = 2^(z - lse) of a row, and with a cap a quarter of its derivative,
// from its scores: the gradients' kernels that hold a row on a lane.
template <int F>
struct RowWeights {
  float c, lse, top, slope;   // scale log2 e, the row's lse, cap log2 e - lse, slope log2 e
  bool by_id;
  // 32 keys from key0 on; element v is key 8 (v / 4) + 4 h + v % 4
  __device__ __forceinline__ void operator()(const MaskedBwdParams& p, const RowMask& mask, int b, int64_t tq, int h, int key0,
                                             f32x16& s, f32x16& sl) const {
    if constexpr ((F & (kCap | kBias)) == 0) {
#pragma unroll
      for (int v = 0; v < 16; ++v) s[v] = __builtin_fmaf(s[v], c, -lse);
    } else {
      const float far = (float)(mask.pos - key0 - 4 * h);
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        if constexpr ((F & kCap) != 0) {
          const float r = cap_r(s[v], p.mask.cap_rate);
          s[v] = __builtin_fmaf(-2.0f * p.mask.cap_log2, r, top);
          sl[v] = __builtin_fmaf(-r, r, r);
        } else {
          s[v] = __builtin_fmaf(s[v], c, -lse);
        }
        if constexpr ((F & kBias) != 0)
          s[v] = __builtin_fmaf(-slope, __builtin_fabsf(far - (float)(8 * (v >> 2) + (v & 3))), s[v]);
      }
    }
#pragma unroll
    for (int v = 0; v < 16; ++v) s[v] = __builtin_amdgcn_exp2f(s[v]);
    if (by_id || !mask.all(key0, 32)) {
      const uint32_t lo = (uint32_t)(mask.lo - key0 - 4 * h), len = (uint32_t)max(mask.lim - mask.lo, 0);
#pragma unroll
      for (int v = 0; v < 16; ++v)
        if ((uint32_t)(8 * (v >> 2) + (v & 3)) - lo >= len) s[v] = 0.0f;
      if (by_id) {
        const int32_t* ids = p.mask.k_docs + (int64_t)b * p.Sk;
        const int doc = p.mask.q_docs[tq];
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (ids[min(key0 + 8 * (v >> 2) + 4 * h + (v & 3), p.Sk - 1)] != doc) s[v] = 0.0f;
      }
    }
  }
};

}  // namespace partir
