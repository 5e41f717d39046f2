// The gradient kernels of attention to another sequence (form 0) and of masked
// attention; cross_attention_bwd.hip and masked_attention_bwd.hip say what bounds
// them.
#pragma once
#include <type_traits>

#include "attention_mask.h"

namespace partir {
namespace {

constexpr int NT = 256;
constexpr int TR = 64;                 // rows of a streamed tile
constexpr int TILE = TR * ROWB;

// The 64-row tiles of the G Sq query rows of a (sequence, key head), Q and dO
// side by side: row i is position i / G of head i mod G.  Addresses ascend with
// the rows, so a descriptor that ends with the tile's last row makes those
// behind it zeros.  Where G divides 16, a lane's rows lie at one offset from a
// tile's first position and a fixed step apart; else each is divided by G (8 %
// of dkv's time).
template <bool EVEN, int WAVES = 4>
struct RowTiles {
  const uint16_t *q, *g;
  int64_t ldq, ldg;
  Div by_g;
  int R, w, lane;
  uint32_t oq, og, chunk;
  __device__ __forceinline__ RowTiles(const CrossBwdParams& p, int b, int kvh, int rows, int w_, int lane_)
      : q(p.Q + (int64_t)b * p.Sq * p.ldq + kvh * p.G * DH), g(p.dO + (int64_t)b * p.Sq * p.ldg + kvh * p.G * DH), ldq(p.ldq),
        ldg(p.ldg), by_g(p.by_g), R(rows), w(w_), lane(lane_) {
    const int l4 = lane >> 4, r = 4 * w + l4, s = by_g.quot(r);
    chunk = ((lane & 15) ^ (l4 << 2) ^ (w & 3)) << 4;   // row 4 WAVES j + r sits at the same chunk for every j
    const uint32_t in = (uint32_t)by_g.rem(r, s) * ROWB + chunk;
    oq = (uint32_t)s * (uint32_t)(ldq * 2) + in;
    og = (uint32_t)s * (uint32_t)(ldg * 2) + in;
  }
  __device__ __forceinline__ void load(int it, char* tile) const {
    const int i0 = it * TR, s0 = by_g.quot(i0), last = min(i0 + TR, R) - 1, sl = by_g.quot(last);
    const uint32_t tail = (uint32_t)by_g.rem(last, sl) * ROWB + ROWB;
    const __amdgpu_buffer_rsrc_t rq = make_rsrc(q + s0 * ldq, (uint32_t)((sl - s0) * ldq * 2) + tail);
    const __amdgpu_buffer_rsrc_t rg = make_rsrc(g + s0 * ldg, (uint32_t)((sl - s0) * ldg * 2) + tail);
    auto put = [&](int j, uint32_t a, uint32_t b) {
      char* const t = tile + (WAVES * j + w) * 1024;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rq, (lds_void*)t, 16, a, 0, 0, 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rg, (lds_void*)(t + TILE), 16, b, 0, 0, 0);
    };
    if constexpr (EVEN) {
      const uint32_t n = by_g.quot(4 * WAVES), sq = n * (uint32_t)(ldq * 2), sg = n * (uint32_t)(ldg * 2);
#pragma unroll
      for (int j = 0; j < TR / (4 * WAVES); ++j) put(j, oq + j * sq, og + j * sg);
    } else {
#pragma unroll
      for (int j = 0; j < TR / (4 * WAVES); ++j) {
        const int i = i0 + 4 * (WAVES * j + w) + (lane >> 4), s = by_g.quot(i);
        const uint32_t in = (uint32_t)by_g.rem(i, s) * ROWB + chunk;
        put(j, (uint32_t)(s - s0) * (uint32_t)(ldq * 2) + in, (uint32_t)(s - s0) * (uint32_t)(ldg * 2) + in);
      }
    }
  }
};

// A wave's 32 rows of 128 results times f, through its share of the tiles'
// memory (free behind the loops' last barrier), as bf16 or as float32 parts.
__device__ __forceinline__ void store(char* smem, int w, uint16_t* out, int64_t off, int rows, const f32x16* a, float f, int lane) {
  store_rows<4>(smem + w * row_area<4, __bf16>(), (__bf16*)out, off, rows, a, f, lane);
}
__device__ __forceinline__ void store(char* smem, int w, float* out, int64_t off, int rows, const f32x16* a, float f, int lane) {
  char* const area = smem + w * row_area<2, float>();
  store_rows<2>(area, out, off, rows, a, f, lane);
  store_rows<2>(area, out, off + 64, rows, a + 2, f, lane);
}

template <int F>
__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(2, 2)))
void cross_bwd_dq_kernel(typename FormParams<F>::bwd p) {
  __shared__ __attribute__((aligned(1024))) char smem[2 * 2 * TILE];
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = lane >> 5, col = lane & 31;

  const int R = p.G * p.Sq;
  int qb, bh, part = 0;
  if (p.q_parts == 1 && (p.by_nbh.d & 7) == 0) {
    // as in the forward pass an XCD takes one (sequence, key head) after the other,
    // whose K and V stay in its L2 (four at a time in its 4 MiB: 818 MB read and
    // 700 us at 4 x 4096 queries over 2048 keys, 32 / 8 heads; 535 MB and 640 us so)
    const int j = blockIdx.x >> 3, n = p.by_nqb.quot(j);
    bh = n * 8 + (blockIdx.x & 7);
    qb = p.by_nqb.rem(j, n);
  } else {
    const int rest = p.by_nbh.quot(blockIdx.x);
    bh = p.by_nbh.rem(blockIdx.x, rest);
    qb = p.by_q_parts.quot(rest);
    part = p.by_q_parts.rem(rest, qb);
  }
  if constexpr (F != 0) qb = (int)p.by_nqb.d - 1 - qb;   // the longest rows of a causal mask first
  const int b = p.by_hk.quot(bh), kvh = p.by_hk.rem(bh, b);
  const int i = qb * 128 + 32 * w + col;
  int last = R - 1;                    // the last row that is read: those behind it repeat it
  if constexpr (F != 0) last = max(p.G * clamp_len(p.mask.q_lens, b, p.Sq) - 1, 0);
  const int ic = min(i, last), sq = p.by_g.quot(ic);
  const int64_t tq = (int64_t)b * p.Sq + sq;
  const int head = kvh * p.G + p.by_g.rem(ic, sq);

  // Q and dO of this lane's row (B operands), D = rowsum(dO * O)
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
  const int len = clamp_len(p.lens, b, p.Sk);
  CrossRange range;
  int lim = 0, lim0 = 0, lim1 = 0, pos = 0, doc = 0;   // as in the forward kernel
  IntRange full = {0, 2147483647};
  float slope = 0.0f;
  if constexpr (F == 0) {
    range = cross_range(len, p.by_q_parts, part);
  } else {
    const SeqMask m(p, b);
    pos = m.start + sq;
    lim = m.lim(sq);
    lim0 = __builtin_amdgcn_readlane(lim, 0);
    lim1 = __builtin_amdgcn_readlane(lim, 31);
    const int r0 = min(qb * 128, last), r1 = min(qb * 128 + 127, last);
    const int s0 = p.by_g.quot(r0), s1 = p.by_g.quot(r1);
    IntRange keys = {0, max(m.qlen > 0 && qb * 128 <= last ? m.lim(s1) : 0, 0)};
    if (p.mask.k_docs) {
      const int2* table = p.mask.k_table + (int64_t)b * p.mask.k_blocks;
      doc = p.mask.q_docs[tq];
      keys = doc_range(table, doc_span(p.mask.q_table + (int64_t)b * p.mask.q_blocks, s0, s1), 0, keys.hi, lane);
      const int first = __builtin_amdgcn_readfirstlane(doc);
      full = __builtin_amdgcn_ballot_w64(doc != first) == 0 ? doc_run(table, first, keys.lo, keys.hi, lane) : IntRange{0, 0};
    }
    range = cross_range(keys.hi - keys.lo, p.by_q_parts, part);
    range.begin += keys.lo;
    range.end += keys.lo;
    if constexpr ((F & kBias) != 0) slope = p.mask.slopes[head] * 1.4426950408889634f;
    // a row without keys, or behind the last: its weights are 0
    if (lse == -__builtin_inff() || i > last || m.qlen == 0) lse = __builtin_inff();
  }
  TileTr tr;
  tr.init(lane);
  const float c = p.scale_log2;
  if (F == 0 && len <= 256) {
    // With few keys O's rounding to bf16 would be of the size of the others in
    // D: up to four tiles more give it as sum_j P_j dP_j.  (The error of dQ at 129
    // keys, in roundings of the result alone: 1.51 from O, 1.45 so.)
    dsum = 0.0f;
    for (int key = 0; key < len; key += TR) {
      const int64_t tk = (int64_t)b * p.Sk + key;
      tile_load<TR, 4>(p.K + tk * p.ldk + kvh * DH, p.ldk, min(TR, len - key), smem, w, lane);
      tile_load<TR, 4>(p.V + tk * p.ldv + kvh * DH, p.ldv, min(TR, len - key), smem + TILE, w, lane);
      WAIT_VMCNT(0);
      __syncthreads();
      for (int t = 0; t < 2; ++t) {
        f32x16 s, dp;
        zero(s);
        zero(dp);
#pragma unroll
        for (int ds = 0; ds < 8; ++ds) {
          s = mfma(tile_rows(smem, 32 * t, col, h, ds), qf[ds], s);
          dp = mfma(tile_rows(smem + TILE, 32 * t, col, h, ds), gf[ds], dp);
        }
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (key + 32 * t + 8 * (v >> 2) + 4 * h + (v & 3) < len)
            dsum += __builtin_amdgcn_exp2f(__builtin_fmaf(s[v], c, -lse)) * dp[v];
      }
      __syncthreads();
    }
  }
  const float Dq = dsum + __shfl_xor(dsum, 32);
  if (part == 0 && h == 0 && i <= last) p.Dstat[tq * p.Hq + head] = Dq;

  const uint16_t* kbase = p.K + ((int64_t)b * p.Sk + range.begin) * p.ldk + kvh * DH;
  const uint16_t* vbase = p.V + ((int64_t)b * p.Sk + range.begin) * p.ldv + kvh * DH;
  const int nkeys = range.end - range.begin, nkb = (nkeys + TR - 1) / TR;
  auto gload = [&](int kb, int buf) {
    char* t = smem + buf * 2 * TILE;
    const int rows = min(TR, nkeys - kb * TR);
    tile_load<TR, 4>(kbase + (int64_t)kb * TR * p.ldk, p.ldk, rows, t, w, lane);
    tile_load<TR, 4>(vbase + (int64_t)kb * TR * p.ldv, p.ldv, rows, t + TILE, w, lane);
  };
  f32x16 dq[4], nD;   // dP starts at -D: its first product reads it, where a subtraction would follow
#pragma unroll
  for (int d = 0; d < 4; ++d) zero(dq[d]);
#pragma unroll
  for (int v = 0; v < 16; ++v) nD[v] = -Dq;
  auto iter = [&](int kb, auto stage) {
    constexpr int cur = decltype(stage)::value;
    if (kb + 1 < nkb) gload(kb + 1, cur ^ 1);
    const char* ks = smem + cur * 2 * TILE;
    const char* vs = ks + TILE;
    int left = nkeys - kb * TR;
    const int key0 = range.begin + kb * TR;
    if (F == 0 || key0 < lim1) {   // else no row of the wave sees the block
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      f32x16 s, dp = nD;
      zero(s);
#pragma unroll
      for (int ds = 0; ds < 8; ++ds) {
        s = mfma(tile_rows(ks, 32 * t, col, h, ds), qf[ds], s);
        dp = mfma(tile_rows(vs, 32 * t, col, h, ds), gf[ds], dp);
      }
      float pr[16];
      if constexpr ((F & (kCap | kBias)) == 0) {
#pragma unroll
        for (int v = 0; v < 16; ++v) pr[v] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[v], c, -lse));
      } else {
        const float far = (float)(pos - key0 - 32 * t - 4 * h);
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          Capped z = {s[v] * c, 1.0f};
          if constexpr ((F & kCap) != 0) z = capped(s[v], p.mask.cap_rate, p.mask.cap_log2);
          if constexpr ((F & kBias) != 0)
            z.z = __builtin_fmaf(-slope, __builtin_fabsf(far - (float)(8 * (v >> 2) + (v & 3))), z.z);
          pr[v] = __builtin_amdgcn_exp2f(z.z - lse) * z.slope;   // P times the cap's derivative
        }
      }
      if constexpr (F != 0) {
        if (key0 < full.lo || key0 + TR > full.hi) {   // a border of documents
          const int32_t* ids = p.mask.k_docs + (int64_t)b * p.Sk;
#pragma unroll
          for (int v = 0; v < 16; ++v)
            if (ids[min(key0 + 32 * t + 8 * (v >> 2) + 4 * h + (v & 3), p.Sk - 1)] != doc) pr[v] = 0.0f;
        }
        if (key0 + 32 * t + 32 > lim0) left = min(left, lim - key0);
        if (key0 + 32 * t + 32 > lim0 || left < 32 * t + 32) {
#pragma unroll
          for (int v = 0; v < 16; ++v)
            if (32 * t + 8 * (v >> 2) + 4 * h + (v & 3) >= left) pr[v] = 0.0f;
        }
      } else if (left < 32 * t + 32) {   // keys past the end
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (32 * t + 8 * (v >> 2) + 4 * h + (v & 3) >= left) pr[v] = 0.0f;
      }
      bf16x8 dsf[2];
#pragma unroll
      for (int v = 0; v < 16; v += 2)
        put2(dsf[v >> 3], v & 7, pr[v] * dp[v], pr[v + 1] * dp[v + 1]);
#pragma unroll
      for (int uu = 0; uu < 2; ++uu)
#pragma unroll
        for (int d = 0; d < 4; ++d) dq[d] = mfma(tr.read(ks, 2 * t + uu, d), dsf[uu], dq[d]);
    }
    }
    WAIT_VMCNT(0);
    __syncthreads();
  };
  if (nkb > 0) gload(0, 0);
  WAIT_VMCNT(0);
  __syncthreads();
  for (int kb = 0; kb < nkb; kb += 2) {
    iter(kb, std::integral_constant<int, 0>{});
    if (kb + 1 < nkb) iter(kb + 1, std::integral_constant<int, 1>{});
  }
  const int rows = R - qb * 128 - 32 * w;
  int64_t tqo = tq;
  int ho = head;
  if constexpr (F != 0) {
    const int io = min(i, R - 1), so = p.by_g.quot(io);
    tqo = (int64_t)b * p.Sq + so;
    ho = kvh * p.G + p.by_g.rem(io, so);
    if (lse == __builtin_inff()) {   // whatever Q, dO and O hold there
#pragma unroll
      for (int d = 0; d < 4; ++d) zero(dq[d]);
    }
  }
  if (p.q_parts > 1)
    store(smem, w, p.dQpart, (((int64_t)part * p.B * p.Sq + tqo) * p.Hq + ho) * DH, rows, dq, p.scale, lane);
  else
    store(smem, w, p.dQ, tqo * p.lddq + ho * DH, rows, dq, p.scale, lane);
}

// dK and dV: eight waves of 32 keys, K as an operand in registers, V in LDS (both
// as registers would leave one wave a SIMD); rows in tiles of 64.  Per 32 rows a
// wave forms S and P, dP, dV^T += dO^T P, then dS and dK^T += Q^T dS.  One pass for
// both gradients forms S, P and dP once, 4 products where a pass for each takes
// 5, and three quarters of their time at the size above.  Two scheduling barriers keep phases
// apart where the compiler would otherwise hold the operands of several at once;
// one at every phase costs their overlap (24 % more).  Eight registers (nine
// without EVEN) are spilled still, addresses of the tiles' loads and of the
// statistics, of which a tile reads four or five back.
template <bool EVEN, int F>
__global__ __launch_bounds__(2 * NT, 2) void cross_bwd_dkv_kernel(typename FormParams<F>::bwd p) {
  constexpr int STAGES = 0, VT = 2 * 2 * TILE, STAT = VT + 256 * ROWB;
  // one object: with several, the compiler tells them apart, takes every tile
  // read for one of the tiles being loaded and waits for those
  constexpr int NSTAT = F == 0 ? 2 : 6;   // numbers of a row
  __shared__ __attribute__((aligned(1024))) char smem[STAT + 2 * NSTAT * TR * 4];
  static_assert(8 * row_area<4, __bf16>() <= STAT && 8 * row_area<2, float>() <= STAT, "the end goes through the stages and V");
  // [stage][..][row]: -lse / c (lse where scores are capped), -D; masked: document, lim, position, slope
  float (*const stat)[NSTAT][TR] = (float (*)[NSTAT][TR])(smem + STAT);
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = lane >> 5, col = lane & 31;

  const int rest = p.by_nbh.quot(blockIdx.x), bh = p.by_nbh.rem(blockIdx.x, rest);
  const int kblk = p.by_k_parts.quot(rest), part = p.by_k_parts.rem(rest, kblk);
  const int b = p.by_hk.quot(bh), kvh = p.by_hk.rem(bh, b);
  const int len = clamp_len(p.lens, b, p.Sk);
  int R = p.G * p.Sq;
  if constexpr (F != 0) R = p.G * clamp_len(p.mask.q_lens, b, p.Sq);   // rows behind it are not read
  const int k0 = kblk * 256, kw = k0 + 32 * w;       // the workgroup's first key, the wave's
  const int kj = kw + col;                           // this lane's
  const int64_t tk = (int64_t)b * p.Sk + kj;

  f32x16 dk[4], dv[4];
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    zero(dk[d]);
    zero(dv[d]);
  }
  // workgroup-uniform: keys behind len_b get zeros
  if (k0 < len) {
#pragma unroll
    for (int half = 0; half < 2; ++half) {   // 256 rows of 2^24 values are more than a descriptor spans
      const int64_t t0 = (int64_t)b * p.Sk + k0 + 128 * half;
      tile_load<128, 8>(p.V + t0 * p.ldv + kvh * DH, p.ldv, min(128, len - k0 - 128 * half), smem + VT + 128 * half * ROWB, w,
                        lane);
    }
    bf16x8 kf[8];
    {
      const uint16_t* krow = p.K + ((int64_t)b * p.Sk + min(kj, len - 1)) * p.ldk + kvh * DH + 8 * h;
#pragma unroll
      for (int ds = 0; ds < 8; ++ds) kf[ds] = *(const bf16x8*)(krow + 16 * ds);
    }
    int first = 0, tiles = (R + TR - 1) / TR;   // the tiles whose rows may see the workgroup's keys
    int kdoc = 0, kdoc0 = 0;
    IntRange kspan = {0, 0};
    bool one_doc = true;                        // the wave's keys are of document kdoc0
    if constexpr (F != 0) {
      const SeqMask m(p, b);
      if (m.causal && k0 >= m.prefix) first = min(tiles, (int)max((int64_t)0, min((int64_t)k0 - m.start, (int64_t)p.Sq)) * p.G / TR);
      if (p.mask.k_docs) {
        const int2* table = p.mask.k_table + (int64_t)b * p.mask.k_blocks;
        const IntRange s = doc_range(p.mask.q_table + (int64_t)b * p.mask.q_blocks, doc_span(table, k0, min(k0 + 255, len - 1)), 0,
                                     m.qlen, lane);
        first = max(first, s.lo * p.G / TR);
        tiles = max(first, min(tiles, (s.hi * p.G + TR - 1) / TR));
        const int32_t* ids = p.mask.k_docs + (int64_t)b * p.Sk;
        kdoc = ids[min(kj, len - 1)];
        kdoc0 = __builtin_amdgcn_readfirstlane(kdoc);
        one_doc = __builtin_amdgcn_ballot_w64(kdoc != kdoc0) == 0;
        kspan = doc_span(table, min(kw, len - 1), min(kw + 31, len - 1));
      }
    }
    const int per = p.by_k_parts.quot(tiles - first + p.k_parts - 1);
    const int it0 = min(tiles, first + part * per), it1 = min(tiles, it0 + per);
    const RowTiles<EVEN, 8> rt(p, b, kvh, R, w, lane);
    const float inv_c = 1.0f / p.scale_log2;
    float st_l = 0.0f, st_d = 0.0f;
    auto gload = [&](int it, int buf) {
      rt.load(it, smem + STAGES + buf * 2 * TILE);
      if constexpr (F != 0) {
        // a wave loads one of a tile's numbers, a lane its row's
        const int i = min(it * TR + lane, R - 1), sq = p.by_g.quot(i), head = kvh * p.G + p.by_g.rem(i, sq);
        const int64_t tq = (int64_t)b * p.Sq + sq;
        if (w == 0) st_l = p.lse[tq * p.Hq + head];
        if (w == 1) st_l = p.Dstat[tq * p.Hq + head];
        if (w == 2 && p.mask.k_docs) st_l = __builtin_bit_cast(float, p.mask.q_docs[tq]);
        if constexpr ((F & kBias) != 0) {
          if (w == 5) st_l = p.mask.slopes[head];
        }
      } else if (tid < TR) {
        // nothing looks at the loaded values before sstore: a use here would wait
        // for the tiles' loads too
        const int i = min(it * TR + tid, R - 1), sq = p.by_g.quot(i);
        const int64_t at = ((int64_t)b * p.Sq + sq) * p.Hq + kvh * p.G + p.by_g.rem(i, sq);
        st_l = p.lse[at];
        st_d = p.Dstat[at];
      }
    };
    auto sstore = [&](int it, int buf) {
      if constexpr (F != 0) {
        const int i = it * TR + lane, sq = p.by_g.quot(min(i, R - 1));
        const SeqMask m(p, b);
        float x = st_l;
        if (w == 0) {   // a missing row, or one without keys: P = 2^-inf
          x = i < R && x != -__builtin_inff() ? x : __builtin_inff();
          if constexpr ((F & kCap) == 0) x = -x * inv_c;
        }
        if (w == 1) x = i < R ? -x : 0.0f;
        if (w == 3) x = __builtin_bit_cast(float, m.lim(sq));
        if (w == 4) x = (float)(m.start + sq);
        if (w == 5) x *= 1.4426950408889634f;
        if (w < NSTAT) lds_write((char*)&stat[buf][w][lane], x);
      } else if (tid < TR) {
        const bool row = it * TR + tid < R;   // a missing row: P = 2^-inf
        lds_write((char*)&stat[buf][0][tid], row ? -st_l * inv_c : -__builtin_inff());
        lds_write((char*)&stat[buf][1][tid], row ? -st_d : 0.0f);
      }
    };
    TileTr tr;
    tr.init(lane);
    const float c = p.scale_log2;
    auto iter = [&](int it, auto stage) {
      constexpr int cur = decltype(stage)::value;
      if (it + 1 < it1) gload(it + 1, cur ^ 1);
      const char* qs = smem + STAGES + cur * 2 * TILE;
      const char* gs = qs + TILE;
      bool work = kw < len, need_doc = false;   // wave-uniform
      int lim0 = 0;
      if constexpr (F != 0) {
        lim0 = __builtin_amdgcn_readfirstlane(lds_read<int>((const char*)&stat[cur][3][0]));
        work &= kw < __builtin_amdgcn_readfirstlane(lds_read<int>((const char*)&stat[cur][3][min(TR, R - it * TR) - 1]));
        if (p.mask.k_docs) {
          const int id = lds_read<int>((const char*)&stat[cur][2][lane]);
          work &= __builtin_amdgcn_ballot_w64(id >= kspan.lo && id <= kspan.hi) != 0;
          need_doc = !one_doc || __builtin_amdgcn_ballot_w64(id != kdoc0) != 0;
        }
      }
      if (work) {
#pragma unroll 1
        for (int t = 0; t < 2; ++t) {
          // the accumulators start at -lse / c and -D of their rows
          auto start = [&](f32x16& x, int which) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const f32x4 v = lds_read<f32x4>((const char*)&stat[cur][which][32 * t + 8 * q + 4 * h]);
#pragma unroll
              for (int j = 0; j < 4; ++j) x[4 * q + j] = v[j];
            }
          };
          f32x16 s;
          if constexpr ((F & kCap) != 0)
            zero(s);
          else
            start(s, 0);
#pragma unroll
          for (int ds = 0; ds < 8; ++ds) s = mfma(tile_rows(qs, 32 * t, col, h, ds), kf[ds], s);
          __builtin_amdgcn_sched_barrier(0);
          bf16x8 pf[2];
          if constexpr (F == 0) {
#pragma unroll
            for (int v = 0; v < 16; v += 2) {
              s[v] = __builtin_amdgcn_exp2f(s[v] * c);
              s[v + 1] = __builtin_amdgcn_exp2f(s[v + 1] * c);
              put2(pf[v >> 3], v & 7, s[v], s[v + 1]);
            }
          } else {
            const bool need_lim = kw + 32 > lim0;
            auto row4 = [&](int which, int q) { return lds_read<f32x4>((const char*)&stat[cur][which][32 * t + 8 * q + 4 * h]); };
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              f32x4 z, slope4 = {1.0f, 1.0f, 1.0f, 1.0f};
              if constexpr ((F & kCap) != 0) {
                const f32x4 lse = row4(0, q);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                  const Capped x = capped(s[4 * q + j], p.mask.cap_rate, p.mask.cap_log2);
                  z[j] = x.z - lse[j];
                  slope4[j] = x.slope;
                }
              } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) z[j] = s[4 * q + j] * c;
              }
              if constexpr ((F & kBias) != 0) {
                const f32x4 at = row4(4, q), sl = row4(5, q);
#pragma unroll
                for (int j = 0; j < 4; ++j) z[j] = __builtin_fmaf(-sl[j], __builtin_fabsf(at[j] - (float)kj), z[j]);
              }
              if (need_lim) {
                const f32x4 lim = row4(3, q);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                  if (kj >= __builtin_bit_cast(int, (float)lim[j])) z[j] = -__builtin_inff();
              }
              if (need_doc) {
                const f32x4 id = row4(2, q);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                  if (kdoc != __builtin_bit_cast(int, (float)id[j])) z[j] = -__builtin_inff();
              }
#pragma unroll
              for (int j = 0; j < 4; ++j) z[j] = __builtin_amdgcn_exp2f(z[j]);
              put2(pf[q >> 1], 4 * (q & 1), z[0], z[1]);
              put2(pf[q >> 1], 4 * (q & 1) + 2, z[2], z[3]);
#pragma unroll
              for (int j = 0; j < 4; ++j) s[4 * q + j] = (F & kCap) != 0 ? z[j] * slope4[j] : z[j];
            }
          }
          f32x16 dp;
          start(dp, 1);
#pragma unroll
          for (int ds = 0; ds < 8; ++ds)
            dp = mfma(tile_rows(gs, 32 * t, col, h, ds), tile_rows(smem + VT, 32 * w, col, h, ds), dp);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int uu = 0; uu < 2; ++uu)
#pragma unroll
            for (int d = 0; d < 4; ++d) dv[d] = mfma(tr.read(gs, 2 * t + uu, d), pf[uu], dv[d]);
#pragma unroll
          for (int v = 0; v < 16; v += 2) put2(pf[v >> 3], v & 7, s[v] * dp[v], s[v + 1] * dp[v + 1]);
#pragma unroll
          for (int uu = 0; uu < 2; ++uu)
#pragma unroll
            for (int d = 0; d < 4; ++d) dk[d] = mfma(tr.read(qs, 2 * t + uu, d), pf[uu], dk[d]);
        }
      }
      if (it + 1 < it1) sstore(it + 1, cur ^ 1);
      WAIT_VMCNT(0);
      __syncthreads();
    };
    if (it0 < it1) {
      gload(it0, 0);
      sstore(it0, 0);
    }
    WAIT_VMCNT(0);
    __syncthreads();
    for (int it = it0; it < it1; it += 2) {
      iter(it, std::integral_constant<int, 0>{});
      if (it + 1 < it1) iter(it + 1, std::integral_constant<int, 1>{});
    }
    if (kj >= len) {   // a lane's key is its own column: what its sums hold goes nowhere else
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        zero(dk[d]);
        zero(dv[d]);
      }
    }
  }
  const int rows = p.Sk - kw;
  if (p.k_parts > 1) {
    const int64_t at = (((int64_t)part * p.B * p.Sk + tk) * p.Hk + kvh) * DH;
    store(smem, w, p.dKpart, at, rows, dk, p.scale, lane);
    store(smem, w, p.dVpart, at, rows, dv, 1.0f, lane);
  } else {
    store(smem, w, p.dK, tk * p.lddk + kvh * DH, rows, dk, p.scale, lane);
    store(smem, w, p.dV, tk * p.lddv + kvh * DH, rows, dv, 1.0f, lane);
  }
}

}  // namespace
}  // namespace partir
