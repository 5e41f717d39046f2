// Which keys a query of the masked attention sees, and how its scores are
// changed: what the forward and the gradient kernels share.
//
// F, the form of a kernel: 0 attention to another sequence (every key below the
// sequence's length), else kMasked, with kCap and kBias as the call has them.
//
// Position p = q_start + s of query s of a sequence, key j.  It sees
//   j < lim = min(k_len, causal ? max(p + 1, prefix) : k_len)
// of its own document.  lim does not fall from a row to the next, so that a tile's
// first row tells whether a block of keys needs the comparison at all, and its last
// row whether the block is seen.  Documents are arbitrary numbers: a table of the
// least and largest of every 64 positions tells which blocks can hold a row's;
// where documents are contiguous, as in packed rows, that leaves the blocks that do.
#pragma once
#include "attention_tiles.h"
#include "operators.h"

namespace partir {

constexpr int kMasked = 1, kCap = 2, kBias = 4;

// What a kernel of form F takes.
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
  __device__ __forceinline__ int lim(int s) const {
    return causal ? min(max(start + s + 1, prefix), klen) : klen;   // s < 2^30
  }
};

struct IntRange {
  int lo, hi;
};

// The least and largest document of positions [s0, s1] of a sequence, by its table.
__device__ __forceinline__ IntRange doc_span(const int2* table, int s0, int s1) {
  IntRange r = {2147483647, -2147483647 - 1};
  for (int i = s0 >> 6; i <= s1 >> 6; ++i) {
    const int2 e = table[i];
    r.lo = min(r.lo, e.x);
    r.hi = max(r.hi, e.y);
  }
  return r;
}

// The positions [lo, hi) within [from, to) (from a multiple of 64) whose blocks may
// hold a document of `docs`; {from, from} if none does.  Every lane of the wave.
__device__ __forceinline__ IntRange doc_range(const int2* table, IntRange docs, int from, int to, int lane) {
  int lo = -1, hi = -1;
  for (int i0 = from >> 6; 64 * i0 < to; i0 += 64) {
    const int i = i0 + lane;
    bool in = 64 * i < to;
    if (in) {
      const int2 e = table[i];
      in = e.x <= docs.hi && e.y >= docs.lo;
    }
    const uint64_t any = __builtin_amdgcn_ballot_w64(in);
    if (any) {
      if (lo < 0) lo = i0 + __builtin_ctzll(any);
      hi = i0 + 63 - __builtin_clzll(any);
    }
  }
  if (lo < 0) return {from, from};
  return {64 * lo, min(to, 64 * hi + 64)};
}

// A run [lo, hi) of positions within [from, to) whose blocks hold document `doc`
// alone: the first such run.
__device__ __forceinline__ IntRange doc_run(const int2* table, int doc, int from, int to, int lane) {
  int lo = -1;
  for (int i0 = from >> 6; 64 * i0 < to; i0 += 64) {
    const int i = i0 + lane;
    bool full = 64 * i < to;
    if (full) {
      const int2 e = table[i];
      full = e.x == doc && e.y == doc;
    }
    uint64_t yes = __builtin_amdgcn_ballot_w64(full);
    if (lo < 0) {
      if (!yes) continue;
      lo = i0 + __builtin_ctzll(yes);
      yes |= ((uint64_t)1 << (lo - i0)) - 1;   // those before it do not end the run
    }
    if (~yes) return {64 * lo, 64 * (i0 + __builtin_ctzll(~yes))};
  }
  return lo < 0 ? IntRange{0, 0} : IntRange{64 * lo, to};
}

// Score s = q k, in units of log2: z = cap tanh(scale s / cap) log2 e with
// tanh x = 1 - 2 / (1 + e^(2x)); r = 1 / (1 + e^(2x)) gives its derivative too,
// 1 - tanh^2 = 4 r (1 - r).  z is off by 2^-20 of the cap at most (the roundings of
// exp2, of the sum and of the reciprocal, each of numbers up to 1), which for caps up
// to 1024, the most that a call takes, stays below a weight's rounding to bf16.
struct Capped {
  float z, slope;
};
__device__ __forceinline__ Capped capped(float s, float rate, float cap_log2) {
  const float r = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(s * rate));
  return {__builtin_fmaf(-2.0f * cap_log2, r, cap_log2), 4.0f * r * (1.0f - r)};
}

}  // namespace partir
