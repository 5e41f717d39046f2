// Gradients of masked attention, d_head = 128, bf16.
//
// With t = tanh(scale q k / cap), z the changed score in log2 units, P = 2^(z - lse):
//     D  = rowsum(P * dP)             dV = P^T dO        dP = dO V^T
//     dS = P * (dP - D) * (1 - t^2)   dQ = scale dS K    dK = scale dS^T Q
// (without a cap the last factor is 1; the bias has no gradient).  Up to 128 keys one
// pass (attention_one_pass.h); above, two, each with one writer of a gradient and a
// fixed order of its sums, no atomics:
//  * dq: workgroup = 128 of the G Sq query rows of a (sequence, key head), 4 waves x
//    32, keys in tiles of 64; S^T = K Q^T and dP^T = V dO^T put one row on a lane,
//    dQ^T += K^T dS^T.
//  * dkv: workgroup = 128 keys of a (sequence, key head), 4 waves x 32, rows in tiles of
//    32; S = Q K^T and dP = dO V^T put one key on a lane, dV^T += dO^T P, dK^T += Q^T dS.
// Both take the range of the other axis that their rows or keys may see, and a wave
// passes blocks of 32 in which it sees nothing.
//
// D.  rowsum(dO * O) has the rounding of O to bf16, which with few keys is of the size
// of the other errors.  The dq pass starts from it, and adds the sum over its keys of
// P (dP - D), which is what it was off by (the weights sum to 1), so that dkv takes D
// with float32's error; where a wave's rows see 256 keys at most, some blocks' time
// more give the dq pass itself that D, as the sum of P dP over that of P.  (Error of dQ
// at 4 x 2048 tokens of documents of 400 on average, of its size: 2.45e-3, and 2.69e-3
// with rowsum(dO * O) alone.)
//
// What bounds it.  Many rows: matrix and vector units, two waves a SIMD, behind one
// another's time in part only.  2 x 4096 tokens, 32 / 8 heads, causal, capped: dq 447 to
// 482 us (0.41 TFLOP, 0.9 PFLOP/s; matrix units busy 45 % of the time, vector units 62),
// dkv 640 to 671 (0.55 TFLOP, 0.84 PFLOP/s; 37 and 50 %), 26 for the sum of two parts.
// Causal without a cap: 410 and 639 (0.96 TFLOP, 0.92 PFLOP/s), with a bias 409 and
// 657; without a mask, for twice the pairs, 743 and 1092 us
// (attention to another sequence 727 and 992, whose dkv pass holds 256 keys).
// Documents of 400 tokens on average, 4 x 2048, 32 heads: 157 and 167 us, with 640 and
// 576 MB read and written (4.1 and 3.5 TB/s) in chains of few tiles.  3 x 333 tokens,
// 12 / 4 heads, bias: 23 and 19, one workgroup's chain.
#include <algorithm>
#include <type_traits>

#include "attention_one_pass.h"

namespace partir {
namespace {

constexpr int kFew = 256;

template <int F>
__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(2, 2)))
void masked_bwd_dq_kernel(MaskedBwdParams p) {
  __shared__ __attribute__((aligned(1024))) char smem[2 * 2 * TILE];
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = lane >> 5, col = lane & 31;

  int qb, bh, part = 0;
  if (p.q_parts == 1 && (p.by_nbh.d & 7) == 0 && !p.mask.rows) {
    // An XCD takes one (sequence, key head) after the other, whose K and V stay in its L2.
    // With documents a row block sees few keys, and all heads of a row block together
    // read whole rows of Q, K, V, O and dO (4 x 2048 tokens, 32 heads, documents of 400 on
    // average: 171 -> 157 us).
    const int j = blockIdx.x >> 3, n = p.by_nqb.quot(j);
    bh = n * 8 + (blockIdx.x & 7);
    qb = p.by_nqb.rem(j, n);
  } else {
    const int rest = p.by_nbh.quot(blockIdx.x);
    bh = p.by_nbh.rem(blockIdx.x, rest);
    qb = p.by_q_parts.quot(rest);
    part = p.by_q_parts.rem(rest, qb);
  }
  qb = (int)p.by_nqb.d - 1 - qb;       // the longest rows of a causal mask first
  const int b = p.by_hk.quot(bh), kvh = p.by_hk.rem(bh, b);
  const SeqMask m(p, b);
  const int R = p.G * p.Sq, last = max(p.G * m.qlen - 1, 0);   // the last row that is read: those behind it repeat it
  const int r0 = qb * 128, i = r0 + 32 * w + col;
  const int ic = min(i, last), sq = p.by_g.quot(ic);
  const int64_t tq = (int64_t)b * p.Sq + sq;
  const int head = kvh * p.G + p.by_g.rem(ic, sq);

  // Q and dO of this lane's row (B operands), and a first D = rowsum(dO * O)
  bf16x8 qf[8], gf[8];
  float dsum = 0.0f;
  {
    const uint16_t* qrow = p.Q + tq * p.ldq + head * DH + 8 * h;
    const uint16_t* grow = p.dO + tq * p.ldg + head * DH + 8 * h;
    const uint16_t* orow = p.O + tq * p.ldo + head * DH + 8 * h;
#pragma unroll
    for (int ds = 0; ds < 8; ++ds) {
      qf[ds] = *(const bf16x8*)(qrow + 16 * ds);
      gf[ds] = *(const bf16x8*)(grow + 16 * ds);
      const bf16x8 of = *(const bf16x8*)(orow + 16 * ds);
#pragma unroll
      for (int e = 0; e < 8; ++e) dsum += (float)gf[ds][e] * (float)of[e];
    }
  }
  float lse = p.lse[tq * p.Hq + head];
  // a row without keys, or behind the last: its weights are 2^-inf
  const bool live = lse != -__builtin_inff() && i <= last && m.qlen > 0;
  if (!live) lse = __builtin_inff();
  float slope = 0.0f;
  if constexpr ((F & kBias) != 0) slope = p.mask.slopes[head] * kLog2e;
  const RowMask mask(p, m, tq, sq);
  const int2 keys = r0 <= last && m.qlen > 0 ? key_range(p, m, b, p.by_g.quot(r0), p.by_g.quot(min(r0 + 127, last))) : make_int2(0, 0);
  CrossRange range = cross_range(keys.y - keys.x, p.by_q_parts, part);
  range.begin += keys.x;
  range.end += keys.x;
  const bool by_id = p.mask.rows && p.mask.by_id[b];
  TileTr tr;
  tr.init(lane);
  const RowWeights<F> row{p.scale_log2, lse, p.mask.cap_log2 - lse, slope, by_id};
  auto weights = [&](f32x16& s, f32x16& sl, int key0) { row(p, mask, b, tq, h, key0, s, sl); };
  // Waves whose rows lie within 256 keys (kFew) take D from the weights themselves,
  // in tiles that the workgroup loads for all of them.
  const bool few = mask.lim1 - mask.lo0 <= kFew;
  int* const spans = (int*)smem;
  if (lane == 0) {
    spans[2 * w] = few ? mask.lo0 & ~(TR - 1) : kNowhere;
    spans[2 * w + 1] = few ? mask.lim1 : 0;
  }
  __syncthreads();
  int few0 = kNowhere, few1 = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    few0 = min(few0, spans[2 * k]);
    few1 = max(few1, spans[2 * k + 1]);
  }
  __syncthreads();
  const int nkb = (range.end - range.begin + TR - 1) / TR;
  // keys from `key` on into a stage; those behind the range's end are of rows without weight
  auto gload = [&](int key, int buf) {
    char* t = smem + buf * 2 * TILE;
    const int64_t tk = (int64_t)b * p.Sk + key;
    const int rows = min(TR, m.klen - key);
    tile_load<TR, 4>(p.K + tk * p.ldk + kvh * DH, p.ldk, rows, t, w, lane);
    tile_load<TR, 4>(p.V + tk * p.ldv + kvh * DH, p.ldv, rows, t + TILE, w, lane);
  };
  float psum = 0.0f;
  if (few0 < few1) {
    if (few) dsum = 0.0f;
    int buf = (few1 - few0 + TR - 1) / TR & 1;       // so that the first tile of the loop below is in stage 0
    gload(few0, buf);
    for (int key = few0; key < few1; key += TR, buf ^= 1) {
      WAIT_VMCNT(0);
      __syncthreads();
      if (key + TR < few1)
        gload(key + TR, buf ^ 1);
      else if (nkb > 0)
        gload(range.begin, 0);
      if (!few) continue;
      const char* ks = smem + buf * 2 * TILE;
#pragma unroll 1
      for (int t = 0; t < 2; ++t) {
        if (mask.none(key + 32 * t, 32)) continue;
        f32x16 s, dp, sl;
        zero(s);
        zero(dp);
#pragma unroll
        for (int ds = 0; ds < 8; ++ds) {
          s = mfma(tile_rows(ks, 32 * t, col, h, ds), qf[ds], s);
          dp = mfma(tile_rows(ks + TILE, 32 * t, col, h, ds), gf[ds], dp);
        }
        weights(s, sl, key + 32 * t);
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          dsum = __builtin_fmaf(s[v], dp[v], dsum);
          psum += s[v];
        }
      }
    }
  } else if (nkb > 0) {
    gload(range.begin, 0);
  }
  float Dq = dsum + __shfl_xor(dsum, 32);
  if (few) {   // over the sum of the weights, which is 1 up to the error of z: what all weights are off by leaves dP - D alone
    psum += __shfl_xor(psum, 32);
    Dq = psum > 0.0f ? Dq / psum : 0.0f;
  }

  f32x16 dq[4], nD;   // dP starts at -D: its first product reads it, where a subtraction would follow
#pragma unroll
  for (int d = 0; d < 4; ++d) zero(dq[d]);
#pragma unroll
  for (int v = 0; v < 16; ++v) nD[v] = -Dq;
  float off = 0.0f;   // sum of P (dP - D)
  auto iter = [&](int kb, auto stage) {
    constexpr int cur = decltype(stage)::value;
    if (kb + 1 < nkb) gload(range.begin + (kb + 1) * TR, cur ^ 1);
    const char* ks = smem + cur * 2 * TILE;
    const char* vs = ks + TILE;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int key0 = range.begin + kb * TR + 32 * t;
      if (mask.none(key0, 32)) continue;
      f32x16 s, dp = nD, sl;
      zero(s);
#pragma unroll
      for (int ds = 0; ds < 8; ++ds) {
        s = mfma(tile_rows(ks, 32 * t, col, h, ds), qf[ds], s);
        dp = mfma(tile_rows(vs, 32 * t, col, h, ds), gf[ds], dp);
      }
      weights(s, sl, key0);
      bf16x8 dsf[2];
      __builtin_amdgcn_s_setprio(1);   // in front of the other wave's scores (capped 505 -> 482 us)
#pragma unroll
      for (int v = 0; v < 16; v += 2) {
        float x = s[v] * dp[v], y = s[v + 1] * dp[v + 1];
        off += x + y;
        if constexpr ((F & kCap) != 0) {
          x *= sl[v];
          y *= sl[v + 1];
        }
        put2(dsf[v >> 3], v & 7, x, y);
      }
#pragma unroll
      for (int uu = 0; uu < 2; ++uu)
#pragma unroll
        for (int d = 0; d < 4; ++d) dq[d] = mfma(tr.read(ks, 2 * t + uu, d), dsf[uu], dq[d]);
      __builtin_amdgcn_s_setprio(0);
    }
    WAIT_VMCNT(0);
    __syncthreads();
  };
  WAIT_VMCNT(0);
  __syncthreads();
  for (int kb = 0; kb < nkb; kb += 2) {
    iter(kb, std::integral_constant<int, 0>{});
    if (kb + 1 < nkb) iter(kb + 1, std::integral_constant<int, 1>{});
  }
  off += __shfl_xor(off, 32);
  const int io = min(i, R - 1), so = p.by_g.quot(io);
  const int64_t tqo = (int64_t)b * p.Sq + so;
  const int ho = kvh * p.G + p.by_g.rem(io, so);
  if (h == 0 && i < R)
    p.Dstat[((int64_t)part * p.B * p.Sq + tqo) * p.Hq + ho] = live ? (part == 0 ? Dq + off : off) : 0.0f;
  if (!live) {   // whatever Q, dO and O hold there
#pragma unroll
    for (int d = 0; d < 4; ++d) zero(dq[d]);
  }
  const int rows = R - qb * 128 - 32 * w;
  const float f = (F & kCap) != 0 ? 4.0f * p.scale : p.scale;
  if (p.q_parts > 1)
    store(smem, w, p.dQpart, (((int64_t)part * p.B * p.Sq + tqo) * p.Hq + ho) * DH, rows, dq, f, lane);
  else
    store(smem, w, p.dQ, tqo * p.lddq + ho * DH, rows, dq, f, lane);
}

constexpr int KW = 128;   // keys of a dkv workgroup
constexpr int QT = 32;    // rows of its tiles

template <bool EVEN, int F>
__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(2, 2)))
void masked_bwd_dkv_kernel(MaskedBwdParams p) {
  constexpr int NS = 2, NSTAT = 6, STAGE = 2 * QT * ROWB;        // stages; numbers of a row
  constexpr int VT = NS * STAGE, STAT = VT + KW * ROWB;          // Q and dO tiles, V, the rows' numbers
  // one object: with several, the compiler tells them apart, takes every tile
  // read for one of the tiles being loaded and waits for those
  __shared__ __attribute__((aligned(1024))) char smem[STAT + NS * NSTAT * QT * 4];
  static_assert(4 * row_area<4, __bf16>() <= STAT && 4 * row_area<2, float>() <= STAT, "the end goes through the stages and V");
  enum { LSE, NEG_D, LO, LIM, POS, SLOPE };
  auto stat = [&](int buf, int which, int row) { return smem + STAT + ((buf * NSTAT + which) * QT + row) * 4; };
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = lane >> 5, col = lane & 31;

  const int rest = p.by_nbh.quot(blockIdx.x), bh = p.by_nbh.rem(blockIdx.x, rest);
  const int kblk = p.by_k_parts.quot(rest), part = p.by_k_parts.rem(rest, kblk);
  const int b = p.by_hk.quot(bh), kvh = p.by_hk.rem(bh, b);
  const SeqMask m(p, b);
  const int R = p.G * m.qlen;                                    // rows behind it are not read
  const int k0 = kblk * KW, kw = k0 + 32 * w, kj = kw + col;
  const int64_t tk = (int64_t)b * p.Sk + kj;

  f32x16 dk[4], dv[4];
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    zero(dk[d]);
    zero(dv[d]);
  }
  int first = 0, tiles = k0 < m.klen ? (R + QT - 1) / QT : 0;    // the tiles whose rows may see the workgroup's keys
  if (m.causal && k0 >= m.prefix) first = (int)max((int64_t)0, min((int64_t)k0 - m.start, (int64_t)m.qlen)) * p.G / QT;
  if (p.mask.rows && tiles > 0) {
    const int2* blocks = p.mask.blocks + (int64_t)b * p.mask.q_blocks;
    int lo = -1, hi = -1;
    for (int i0 = 0; 64 * i0 < m.qlen; i0 += 64) {               // every wave for itself
      bool in = 64 * (i0 + lane) < m.qlen;
      if (in) {
        const int2 e = blocks[i0 + lane];
        in = e.x < k0 + KW && e.y > k0;
      }
      const uint64_t any = __builtin_amdgcn_ballot_w64(in);
      if (any) {
        if (lo < 0) lo = i0 + __builtin_ctzll(any);
        hi = i0 + 63 - __builtin_clzll(any);
      }
    }
    first = max(first, lo < 0 ? tiles : 64 * lo * p.G / QT);
    if (hi >= 0) tiles = min(tiles, (int)(((int64_t)64 * (hi + 1) * p.G + QT - 1) / QT));
  }
  first = min(first, tiles);
  // From the last rows down, the parts in turn: under a causal mask the workgroups of a
  // key head end at different rows, but start at the same, and find them in the L2 (2 x
  // 4096 tokens, 32 / 8 heads, capped: 686 -> 671 us; upwards, in contiguous parts, 2.1
  // GB came from behind the L2).
  const int it0 = tiles - 1 - part, step = p.k_parts;
  if (it0 >= first) {                                               // workgroup-uniform
    tile_load<KW, 4>(p.V + ((int64_t)b * p.Sk + k0) * p.ldv + kvh * DH, p.ldv, min(KW, m.klen - k0), smem + VT, w, lane);
    bf16x8 kf[8];
    {
      const uint16_t* krow = p.K + ((int64_t)b * p.Sk + min(kj, m.klen - 1)) * p.ldk + kvh * DH + 8 * h;
#pragma unroll
      for (int ds = 0; ds < 8; ++ds) kf[ds] = *(const bf16x8*)(krow + 16 * ds);
    }
    const bool by_id = p.mask.rows && p.mask.by_id[b];
    const RowTiles<EVEN, 4, QT> rt(p, b, kvh, R, w, lane);
    const float c = p.scale_log2, inv_c = 1.0f / p.scale_log2;
    const int which = 2 * w + h;       // the number that this half of a wave provides, a lane its row's
    float st = 0.0f;
    // nothing looks at the loaded number before sstore: a use here would wait for the tile
    auto gload = [&](int it, int buf) {
      const int i = min(it * QT + col, R - 1), sq = p.by_g.quot(i), head = kvh * p.G + p.by_g.rem(i, sq);
      const int64_t tq = (int64_t)b * p.Sq + sq, at = tq * p.Hq + head;
      if (which == LSE) st = p.lse[at];
      if (which == NEG_D) {
        st = p.Dstat[at];
        for (int q = 1; q < p.q_parts; ++q) st += p.Dstat[q * ((int64_t)p.B * p.Sq * p.Hq) + at];
      }
      if (p.mask.rows) {
        if (which == LO) st = __builtin_bit_cast(float, p.mask.rows[tq].x);
        if (which == LIM) st = __builtin_bit_cast(float, p.mask.rows[tq].y);
      }
      if constexpr ((F & kBias) != 0) {
        if (which == SLOPE) st = p.mask.slopes[head];
      }
      rt.load(it, smem + buf * STAGE);
    };
    auto sstore = [&](int it, int buf) {
      const int i = it * QT + col, sq = p.by_g.quot(min(i, R - 1));
      float x = st;
      if (which == LSE) {   // a missing row, or one without keys: P = 2^-inf
        x = i < R && x != -__builtin_inff() ? x : __builtin_inff();
        x = (F & kCap) != 0 ? p.mask.cap_log2 - x : -x * inv_c;
      }
      if (which == NEG_D) x = i < R ? -x : 0.0f;
      if (which == LO && !p.mask.rows) x = 0.0f;
      if (which == LIM) {
        int lim = m.lim(sq);
        if (p.mask.rows) lim = min(lim, __builtin_bit_cast(int, x));
        x = __builtin_bit_cast(float, i < R ? lim : 0);
      }
      if (which == POS) x = (float)(m.start + sq - k0);   // from the first key on: exact where it matters
      if (which == SLOPE) x *= kLog2e;
      if (which < NSTAT) lds_write(stat(buf, which, col), x);
    };
    TileTr tr;
    tr.init(lane);
    gload(it0, 0);
    sstore(it0, 0);
    // The stage is a number, not a constant: copies of the body would each keep their
    // addresses in registers.  (Eight waves with three stages and three copies read 45
    // of them back from memory a tile.)
    int cur = 0, vt = VT + 32 * w * ROWB;
#pragma unroll 1
    for (int it = it0; it >= first; it -= step) {
      asm volatile("" : "+s"(vt));     // V's addresses are formed here
      __builtin_amdgcn_sched_barrier(0);
      WAIT_VMCNT(0);
      lds_barrier();                   // everyone's tile has landed, and everyone is done with the stage loaded next
      if (it - step >= first) gload(it - step, cur ^ 1);
      __builtin_amdgcn_sched_barrier(0);
      const char* qs = smem + cur * STAGE;
      const char* gs = qs + QT * ROWB;
      // which of the rows see the wave's keys, by the lanes of both halves alike
      const int lo = lds_read<int>(stat(cur, LO, col)), lim = lds_read<int>(stat(cur, LIM, col));
      if (__builtin_amdgcn_ballot_w64(lo < kw + 32 && lim > kw && lim > lo) != 0) {
        auto row4 = [&](int which, int q) { return lds_read<f32x4>(stat(cur, which, 8 * q + 4 * h)); };
        f32x16 s, dp;
        if constexpr ((F & kCap) != 0) {
          zero(s);
        } else {                       // the accumulators start at -lse / c, and at -D
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const f32x4 x = row4(LSE, q);
#pragma unroll
            for (int j = 0; j < 4; ++j) s[4 * q + j] = x[j];
          }
        }
#pragma unroll
        for (int ds = 0; ds < 8; ++ds) s = mfma(tile_rows(qs, 0, col, h, ds), kf[ds], s);
        f32x16 sl;                     // a quarter of the cap's derivative
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          if constexpr ((F & kCap) != 0) {
            const f32x4 top = row4(LSE, q);   // cap log2 e - lse
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float r = cap_r(s[4 * q + j], p.mask.cap_rate);
              s[4 * q + j] = __builtin_fmaf(-2.0f * p.mask.cap_log2, r, top[j]);
              sl[4 * q + j] = __builtin_fmaf(-r, r, r);
            }
          } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) s[4 * q + j] *= c;
          }
          if constexpr ((F & kBias) != 0) {
            const f32x4 at = row4(POS, q), slope = row4(SLOPE, q);
#pragma unroll
            for (int j = 0; j < 4; ++j)
              s[4 * q + j] = __builtin_fmaf(-slope[j], __builtin_fabsf(at[j] - (float)(kj - k0)), s[4 * q + j]);
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) s[4 * q + j] = __builtin_amdgcn_exp2f(s[4 * q + j]);
        }
        if (by_id || __builtin_amdgcn_ballot_w64(lo > kw || lim < kw + 32) != 0) {   // some row does not see some key
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const f32x4 lo4 = row4(LO, q), lim4 = row4(LIM, q);
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (kj < __builtin_bit_cast(int, (float)lo4[j]) || kj >= __builtin_bit_cast(int, (float)lim4[j])) s[4 * q + j] = 0.0f;
          }
          if (by_id) {
            const int doc = p.mask.k_docs[(int64_t)b * p.Sk + min(kj, m.klen - 1)];
#pragma unroll
            for (int v = 0; v < 16; ++v) {
              const int i = min(it * QT + 8 * (v >> 2) + 4 * h + (v & 3), R - 1);
              if (p.mask.q_docs[(int64_t)b * p.Sq + p.by_g.quot(i)] != doc) s[v] = 0.0f;
            }
          }
        }
        bf16x8 pf[2];
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int v = 0; v < 16; v += 2) {
          put2(pf[v >> 3], v & 7, s[v], s[v + 1]);
          if constexpr ((F & kCap) != 0) {
            s[v] *= sl[v];
            s[v + 1] *= sl[v + 1];
          }
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f32x4 x = row4(NEG_D, q);
#pragma unroll
          for (int j = 0; j < 4; ++j) dp[4 * q + j] = x[j];
        }
#pragma unroll
        for (int ds = 0; ds < 8; ++ds) dp = mfma(tile_rows(gs, 0, col, h, ds), tile_rows(smem + vt, 0, col, h, ds), dp);
#pragma unroll
        for (int uu = 0; uu < 2; ++uu)
#pragma unroll
          for (int d = 0; d < 4; ++d) dv[d] = mfma(tr.read(gs, uu, d), pf[uu], dv[d]);
#pragma unroll
        for (int v = 0; v < 16; v += 2) put2(pf[v >> 3], v & 7, s[v] * dp[v], s[v + 1] * dp[v + 1]);
#pragma unroll
        for (int uu = 0; uu < 2; ++uu)
#pragma unroll
          for (int d = 0; d < 4; ++d) dk[d] = mfma(tr.read(qs, uu, d), pf[uu], dk[d]);
        __builtin_amdgcn_s_setprio(0);
      }
      __builtin_amdgcn_sched_barrier(0);
      if (it - step >= first) sstore(it - step, cur ^ 1);
      cur ^= 1;
    }
    __syncthreads();                   // the tiles' memory takes the rows
    if (kj >= m.klen) {   // a lane's key is its own column: what its sums hold goes nowhere else
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        zero(dk[d]);
        zero(dv[d]);
      }
    }
  }
  const int rows = p.Sk - kw;
  const float f = (F & kCap) != 0 ? 4.0f * p.scale : p.scale;    // a quarter of the cap's derivative is in dS
  if (p.k_parts > 1) {
    const int64_t at = (((int64_t)part * p.B * p.Sk + tk) * p.Hk + kvh) * DH;
    store(smem, w, p.dKpart, at, rows, dk, f, lane);
    store(smem, w, p.dVpart, at, rows, dv, 1.0f, lane);
  } else {
    store(smem, w, p.dK, tk * p.lddk + kvh * DH, rows, dk, f, lane);
    store(smem, w, p.dV, tk * p.lddv + kvh * DH, rows, dv, 1.0f, lane);
  }
}

constexpr int64_t kCUs = 256;

template <int F>
void launch_form(const MaskedBwdParams& p, CrossBwdPass pass, hipStream_t s) {
  const int64_t nbh = (int64_t)p.B * p.Hk;
  if (pass == CROSS_ALL) {
    const dim3 grid((unsigned)(nbh * p.k_parts));
    if (16 % p.G == 0)
      hipLaunchKernelGGL((attention_one_pass_kernel<true, F>), grid, dim3(2 * NT), 0, s, p);
    else
      hipLaunchKernelGGL((attention_one_pass_kernel<false, F>), grid, dim3(2 * NT), 0, s, p);
  } else if (pass == CROSS_DQ) {
    const int64_t blocks = ((int64_t)p.G * p.Sq + 127) / 128;
    hipLaunchKernelGGL((masked_bwd_dq_kernel<F>), dim3((unsigned)(blocks * nbh * p.q_parts)), dim3(NT), 0, s, p);
  } else {
    const int64_t blocks = ((int64_t)p.Sk + KW - 1) / KW;
    const dim3 grid((unsigned)(blocks * nbh * p.k_parts));
    if (16 % p.G == 0)
      hipLaunchKernelGGL((masked_bwd_dkv_kernel<true, F>), grid, dim3(NT), 0, s, p);
    else
      hipLaunchKernelGGL((masked_bwd_dkv_kernel<false, F>), grid, dim3(NT), 0, s, p);
  }
}

}  // namespace

// Parts of an axis whose `grid` workgroups take up to `steps` steps each, and `share`
// of those on average: the longest workgroup, or all of them on the chip's two a compute
// unit, whichever lasts longer; from two parts on a launch that adds them (5 us) and
// part_us for the float32 rows of each, written and read.  Documents are not looked at:
// their chains are shorter than `steps`, and parts are cost alone where they are short
// (1 x 8192 tokens, 8 heads, documents of 256: 58 and 48 us in two parts each, and 13
// and 25 for their sums).
static int masked_parts(int64_t grid, int64_t steps, double share, double step_us, double part_us) {
  if (grid <= 0 || steps <= 0) return 1;
  const double all = (double)grid * (double)steps * share / (2.0 * kCUs);
  int best = 1;
  double least = std::max((double)steps, all) * step_us;
  for (int64_t n = 2; n <= 64 && n <= steps; n *= 2) {
    const double us = std::max((double)((steps + n - 1) / n), all) * step_us + 5.0 + (double)n * part_us;
    if (us < least) {
      least = us;
      best = (int)n;
    }
  }
  return best;
}

CrossBwdChoice masked_bwd_choice(int64_t B, int64_t Sq, int64_t Sk, int64_t Hq, int64_t Hk, bool causal) {
  const int64_t R = Hq / Hk * Sq, rows = (R + QT - 1) / QT, keys = (Sk + TR - 1) / TR;
  // a causal mask leaves half of the pairs where the queries are as many as the keys
  const double share = causal && Sk > 0 ? 1.0 - 0.5 * (double)std::min(Sq, Sk) / (double)Sk : 1.0;
  // As cross_bwd_choice says, whose tiles these are: 1000 rows of a part cost 0.15 us
  // (k_us: of two matrices); a tile of 64 keys takes a workgroup 1.45 us in dq, one of 32
  // rows half of 3 us in dkv, one of 64 rows 2.8 us in the one pass.
  const double q_us = 1.5e-4 * (double)(B * Sq * Hq), k_us = 2 * 1.5e-4 * (double)(B * Sk * Hk);
  // One pass, as of attention to another sequence.  Forward and gradients of 4 x 51
  // tokens, 8 heads, replayed from a graph: 15.7 us, 24.6 with two passes; 2 x 128, 8 / 2
  // heads: 23.3, 36.9.
  if (Sq > 0 && Sk > 0 && Sk <= 128) {
    const int64_t tiles = (R + TR - 1) / TR, grid = B * Hk;
    return {true, 1, best_parts(grid > 0 ? std::min(kCUs / grid, tiles) : 1, tiles, 2.8, k_us)};
  }
  return {false, masked_parts(B * Hk * ((R + 127) / 128), keys, share, 1.45, q_us),
          masked_parts(B * Hk * ((Sk + KW - 1) / KW), rows, share, 1.5, k_us)};
}

hipError_t launch_masked_backward(const MaskedBwdParams& p, int form, CrossBwdPass pass, hipStream_t s) {
  switch (form & (kCap | kBias)) {
    case 0: launch_form<kMasked>(p, pass, s); break;
    case kCap: launch_form<kMasked | kCap>(p, pass, s); break;
    case kBias: launch_form<kMasked | kBias>(p, pass, s); break;
    default: launch_form<kMasked | kCap | kBias>(p, pass, s);
  }
  return hipGetLastError();
}

}  // namespace partir
