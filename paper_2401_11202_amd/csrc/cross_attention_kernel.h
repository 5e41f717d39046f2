// The forward kernel of attention to another sequence (form 0) and of masked
// attention; cross_attention.hip and masked_attention.hip say what bounds them.
//
// A workgroup takes 32 QW rows of the G Sq query rows of one (sequence, key
// head); its QW x KG waves hold 32 rows each, and the KG key groups take every
// KG-th block of BKV keys through a ring of LDS stages of their own.  A
// wave computes
//     S^T[BKV keys x 32 rows] = K_blk Q^T      (v_mfma_f32_32x32x16_bf16)
// so that a lane owns one row: maximum and sum of the running softmax are lane
// registers, and exp2(S^T - m), rounded to bf16 (within 2^-8 of its value, as
// the weights of partir_attention), is the B operand of
//     O^T[128 x 32 rows] += V_blk^T P^T
// with V^T from transposed LDS reads.  Where rows are few the matrix units wait
// for K and V, and what that rounding leaves is a second operand (the weights
// are within 2^-16 then), so that O's error is its own rounding: 1.66e-3 of its
// size, 2.34e-3 with one (64 x 8192 keys, 363 us either way; the smallest calls
// take 0.2 to 0.6 us more).  Sums and O are float32; groups and key parts join by
// (m, l, O) (+) (m', l', O'), in a fixed order.
#pragma once
#include <type_traits>

#include "attention_mask.h"

namespace partir {
namespace {

// The running maximum before the first key: below every finite score, and a
// finite number, so that 2^(kNoMax - kNoMax) is 1.
constexpr float kNoMax = -3.0e38f;

template <int QW, int KG, int BKV, int NS, int OCC, int F>
__global__ __launch_bounds__(64 * QW * KG, OCC) void cross_attention_kernel(typename FormParams<F>::fwd p) {
  constexpr int NSUB = BKV / 32;
  constexpr int LPB = 2 * BKV / (4 * QW);                       // tile loads of a wave per block, K and V
  constexpr int T_BYTES = BKV * ROWB, STAGE = 2 * T_BYTES;      // K tile, then V tile
  constexpr int ND = 4 / KG, PER = QW * 64;                     // 32-wide blocks of O that a key group finishes
  constexpr int MERGE = KG * (KG - 1) * ND * PER * 64, ML = KG * PER * 8;
  static_assert(KG * NS * STAGE >= MERGE + ML && KG * NS * STAGE >= QW * KG * row_area<ND, __bf16>() &&
                (KG == 1 || KG * NS * STAGE >= QW * KG * row_area<ND, float>()), "the stages are reused");
  __shared__ __attribute__((aligned(1024))) char smem[KG * NS * STAGE];

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int w = wave % QW, kg = wave / QW;
  const int h = lane >> 5, col = lane & 31;

  int qb, bh, split = 0;
  bool by_head = p.nsplit == 1 && (p.by_nbh.d & 7) == 0;
  // with documents a row block sees few keys, and all heads of a row block together
  // read whole rows (4 x 2048 tokens, 32 heads, documents of 400 on average: 108 -> 93 us)
  if constexpr (F != 0) by_head = by_head && !p.mask.rows;
  if (by_head) {
    // Workgroup i runs on XCD i mod 8: an XCD takes one (sequence, key head)
    // after the other, whose K and V stay in its L2.
    const int j = blockIdx.x >> 3, n = p.by_nqb.quot(j);
    bh = n * 8 + (blockIdx.x & 7);
    qb = p.by_nqb.rem(j, n);
  } else {
    const int r = p.by_nbh.quot(blockIdx.x);
    bh = p.by_nbh.rem(blockIdx.x, r);
    qb = p.by_split.quot(r);
    split = p.by_split.rem(r, qb);
  }
  if constexpr (F != 0) qb = (int)p.by_nqb.d - 1 - qb;   // the longest rows of a causal mask first
  const int b = p.by_hk.quot(bh), kvh = p.by_hk.rem(bh, b);

  // this lane's row: queries (B operand of S^T) in registers
  const int i = qb * 32 * QW + 32 * w + col;
  const int R = p.G * p.Sq;
  int last = R - 1;                    // the last row that is read: those behind it repeat it
  if constexpr (F != 0) last = max(p.G * clamp_len(p.mask.q_lens, b, p.Sq) - 1, 0);
  const int ic = min(i, last), sq = p.by_g.quot(ic);
  const int64_t tq = (int64_t)b * p.Sq + sq;
  const int head = kvh * p.G + p.by_g.rem(ic, sq);
  bf16x8 qf[8];
  {
    const uint16_t* qrow = p.Q + tq * p.ldq + head * DH + 8 * h;
#pragma unroll
    for (int ds = 0; ds < 8; ++ds) qf[ds] = *(const bf16x8*)(qrow + 16 * ds);
  }
  CrossRange range;
  if constexpr (F == 0) {
    range = cross_range(clamp_len(p.lens, b, p.Sk), p.by_split, split);
    if (p.nsplit > 1 && split >= range.parts) return;   // the combine does not read it
  }
  const auto mask = [&] {
    if constexpr (F == 0)
      return 0;
    else {
      const SeqMask m(p, b);
      const int r0 = qb * 32 * QW, r1 = min(r0 + 32 * QW - 1, last);   // the workgroup's rows
      const int2 keys = r0 <= last && m.qlen > 0 ? key_range(p, m, b, p.by_g.quot(r0), p.by_g.quot(r1)) : make_int2(0, 0);
      range = cross_range(keys.y - keys.x, p.by_split, split);
      range.begin += keys.x;
      range.end += keys.x;
      return RowMask(p, m, tq, sq);
    }
  }();
  float slope = 0.0f;
  if constexpr ((F & kBias) != 0) slope = p.mask.slopes[head] * 1.4426950408889634f;

  const uint16_t* kbase = p.K + (int64_t)b * p.Sk * p.ldk + kvh * DH;
  const uint16_t* vbase = p.V + (int64_t)b * p.Sk * p.ldv + kvh * DH;
  char* const stages = smem + kg * NS * STAGE;
  // K or V of key block kb of the part into a stage; the addresses are 64-bit, so
  // a part may hold any number of bytes
  auto kload = [&](int kb, int buf) {
    const int64_t k0 = range.begin + (int64_t)kb * BKV;
    tile_load<BKV, QW>(kbase + k0 * p.ldk, p.ldk, (int)min((int64_t)BKV, range.end - k0), stages + buf * STAGE, w, lane);
  };
  auto vload = [&](int kb, int buf) {
    const int64_t k0 = range.begin + (int64_t)kb * BKV;
    tile_load<BKV, QW>(vbase + k0 * p.ldv, p.ldv, (int)min((int64_t)BKV, range.end - k0), stages + buf * STAGE + T_BYTES, w,
                       lane);
  };

  f32x16 oacc[4];
#pragma unroll
  for (int d = 0; d < 4; ++d) zero(oacc[d]);
  float m_run = kNoMax, l_run = 0.0f;
  TileTr tr;
  tr.init(lane);
  const int nkb = (range.end - range.begin + BKV - 1) / BKV;
  const float sl2 = (F & (kCap | kBias)) != 0 ? 1.0f : p.scale_log2;   // the changed scores are in log2 units

  // Rings of NS stages for K and for V: loads run ahead, and blocks behind the
  // last are loaded too (no row of them is read: zeros), which keeps the counts
  // of loads in flight constant.  Where a wave has its stages to itself (QW = 1)
  // nothing but its own loads is waited for, and a stage is loaded anew as soon
  // as its products are done; else a barrier a block says that everyone's loads
  // have landed and that the stage loaded next is done with.
  constexpr bool ALONE = QW == 1;
  static_assert(!ALONE || NS == 2, "two blocks in flight");
#pragma unroll
  for (int n = 0; n < NS - !ALONE; ++n) {
    kload(n * KG + kg, n);
    vload(n * KG + kg, n);
  }
  auto block = [&](auto stage_c, int kb) {
    constexpr int cur = decltype(stage_c)::value;
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (ALONE) {
      WAIT_VMCNT(3 * LPB / 2);             // after this K: its V, the next K and V
      asm volatile("" ::: "memory");
    } else {
      WAIT_VMCNT(LPB * (NS - 2));
      asm volatile("s_barrier" ::: "memory");
    }
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (!ALONE) {
      kload(kb + KG * (NS - 1), (cur + NS - 1) % NS);
      vload(kb + KG * (NS - 1), (cur + NS - 1) % NS);
    }
    if (!ALONE && KG > 1 && kb >= nkb) return;
    const int key0 = range.begin + kb * BKV;
    if constexpr (F != 0 && !ALONE) {
      if (mask.none(key0, BKV)) return;
    }
    const char* ks = stages + cur * STAGE;
    const char* vs = ks + T_BYTES;
    __builtin_amdgcn_s_setprio(1);
    f32x16 sacc[NSUB];
#pragma unroll
    for (int t = 0; t < NSUB; ++t) {
      zero(sacc[t]);
#pragma unroll
      for (int ds = 0; ds < 8; ++ds) sacc[t] = mfma(tile_rows(ks, 32 * t, col, h, ds), qf[ds], sacc[t]);
    }
    __builtin_amdgcn_s_setprio(0);
    if constexpr (ALONE) {
      __builtin_amdgcn_sched_barrier(0);   // the products hold what they read of the stage
      WAIT_LGKMCNT(0);
      asm volatile("" ::: "memory");
      kload(kb + KG * NS, cur);
      __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr ((F & kCap) != 0) {
      float big = 0.0f;   // a NaN stays one in either form
#pragma unroll
      for (int t = 0; t < NSUB; ++t)
#pragma unroll
        for (int v = 0; v < 16; ++v) big = fmaxf(big, __builtin_fabsf(sacc[t][v]));
      if (__builtin_amdgcn_ballot_w64(big > p.mask.cap_small) == 0) {
#pragma unroll
        for (int t = 0; t < NSUB; ++t)
#pragma unroll
          for (int v = 0; v < 16; ++v) sacc[t][v] = cap_small(sacc[t][v], p.mask);
      } else {
#pragma unroll
        for (int t = 0; t < NSUB; ++t)
#pragma unroll
          for (int v = 0; v < 16; ++v)
            sacc[t][v] = __builtin_fmaf(-2.0f * p.mask.cap_log2, cap_r(sacc[t][v], p.mask.cap_rate), p.mask.cap_log2);
      }
    }
    if constexpr ((F & kBias) != 0) {
      const float far = (float)(mask.pos - key0 - 4 * h);
#pragma unroll
      for (int t = 0; t < NSUB; ++t)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          if constexpr ((F & kCap) == 0) sacc[t][v] *= p.scale_log2;
          sacc[t][v] = __builtin_fmaf(-slope, __builtin_fabsf(far - (float)(32 * t + 8 * (v >> 2) + (v & 3))), sacc[t][v]);
        }
    }
    const int left = range.end - key0;   // keys from this block on
    if constexpr (F != 0) {
      if (!mask.all(key0, BKV)) {
        // [lo, lim) of the row, in keys from this lane's first of the block on
        const uint32_t lo = (uint32_t)(mask.lo - key0 - 4 * h), len = (uint32_t)max(mask.lim - mask.lo, 0);
#pragma unroll
        for (int t = 0; t < NSUB; ++t)
#pragma unroll
          for (int v = 0; v < 16; ++v)
            if ((uint32_t)(32 * t + 8 * (v >> 2) + (v & 3)) - lo >= len) sacc[t][v] = -__builtin_inff();
      }
      if (p.mask.rows && p.mask.by_id[b]) {
        const int32_t* ids = p.mask.k_docs + (int64_t)b * p.Sk;
        const int doc = p.mask.q_docs[tq];
#pragma unroll
        for (int t = 0; t < NSUB; ++t)
#pragma unroll
          for (int v = 0; v < 16; ++v)
            if (ids[min(key0 + 32 * t + 8 * (v >> 2) + 4 * h + (v & 3), p.Sk - 1)] != doc) sacc[t][v] = -__builtin_inff();
      }
    } else if (left < BKV) {
#pragma unroll
      for (int t = 0; t < NSUB; ++t)
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (32 * t + 8 * (v >> 2) + 4 * h + (v & 3) >= left) sacc[t][v] = -__builtin_inff();
    }
    float lsum = 0.0f;
    bf16x8 pf[2 * NSUB], pl[2 * NSUB];   // the weights in bf16, and what is left of them (few rows)
    f32x16 ef[NSUB];                     // the weights (few rows)
    auto weights = [&]() {
      lsum = 0.0f;
#pragma unroll
      for (int t = 0; t < NSUB; ++t)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[t][v], sl2, -m_run));
          lsum += e;
          if constexpr (ALONE)
            ef[t][v] = e;
          else
            pf[2 * t + (v >> 3)][v & 7] = (__bf16)e;
        }
    };
    // m moves only where the block's maximum is more than 8 (log2 units)
    // above it: weights stay below 2^8, exact range in float32 and bf16, and
    // O is rescaled in few blocks.  A lane whose weights sum to at most 2^8
    // has none above, so the maximum is taken only where some lane's sum is
    // larger (or inf / NaN, as on the first block, where m is kNoMax).
    weights();
    if (__builtin_amdgcn_ballot_w64(!(lsum <= 256.0f)) != 0) {
      float mloc = -__builtin_inff();
#pragma unroll
      for (int t = 0; t < NSUB; ++t)
#pragma unroll
        for (int v = 0; v < 16; ++v) mloc = fmaxf(mloc, sacc[t][v]);
      mloc = fmaxf(mloc, __shfl_xor(mloc, 32));   // the partner lane holds the row's other keys
      const float m_blk = mloc * sl2;
      const bool move = m_blk > m_run + 8.0f;
      if (__builtin_amdgcn_ballot_w64(move) != 0) {
        const float m_new = move ? m_blk : m_run;
        const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
        l_run *= alpha;
#pragma unroll
        for (int d = 0; d < 4; ++d) oacc[d] *= alpha;
        m_run = m_new;
        weights();
      }
    }
    l_run += lsum;
    if constexpr (ALONE) {
#pragma unroll
      for (int t = 0; t < NSUB; ++t)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const __bf16 hi = (__bf16)ef[t][v];
          pf[2 * t + (v >> 3)][v & 7] = hi;
          pl[2 * t + (v >> 3)][v & 7] = (__bf16)(ef[t][v] - (float)hi);
        }
      __builtin_amdgcn_sched_barrier(0);
      WAIT_VMCNT(3 * LPB / 2);             // after this V: the next K and V, the K after
      asm volatile("" ::: "memory");
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int u = 0; u < BKV / 16; ++u)
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        const bf16x8 v = tr.read(vs, u, d);
        oacc[d] = mfma(v, pf[u], oacc[d]);
        if constexpr (ALONE) oacc[d] = mfma(v, pl[u], oacc[d]);
      }
    if constexpr (ALONE) {
      __builtin_amdgcn_sched_barrier(0);
      WAIT_LGKMCNT(0);
      asm volatile("" ::: "memory");
      vload(kb + KG * NS, cur);
    }
  };
  // NS blocks a trip, so that a block's stage is a constant and folds into the
  // reads' offsets.  With barriers the trip count is the workgroup's, not the
  // group's.
  for (int kb = 0; kb < nkb; kb += NS * KG) {
    if (!ALONE || kb + kg < nkb) block(std::integral_constant<int, 0>{}, kb + kg);
    if (ALONE ? kb + KG + kg < nkb : kb + KG < nkb) block(std::integral_constant<int, 1>{}, kb + KG + kg);
    if constexpr (NS > 2) {
      if (kb + 2 * KG < nkb) block(std::integral_constant<int, 2>{}, kb + 2 * KG + kg);
    }
  }
  WAIT_VMCNT(0);   // no LDS write is in flight behind the loop
  __syncthreads();

  float l_tot = l_run + __shfl_xor(l_run, 32);
  if constexpr (KG > 1) {
    // The groups' (m, l, O) together, in order.  Group g finishes the ND blocks
    // of O from g ND on: it hands the others theirs and takes what they hold of
    // its own.
    auto box = [&](int to, int from, int d) {   // from != to
      return (f32x4*)(smem + (((to * (KG - 1) + (from < to ? from : from - 1)) * ND + d) * PER + w * 64 + lane) * 16);
    };
    constexpr int STEP = KG * (KG - 1) * ND * PER;   // between the four quarters of a block
    float2* const ml = (float2*)(smem + MERGE) + w * 64 + lane;
    ml[kg * PER] = make_float2(m_run, l_tot);
#pragma unroll
    for (int g = 0; g < KG; ++g)
      if (g != kg) {
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            box(g, kg, d)[q * STEP] = f32x4{oacc[g * ND + d][4 * q + 0], oacc[g * ND + d][4 * q + 1],
                                            oacc[g * ND + d][4 * q + 2], oacc[g * ND + d][4 * q + 3]};
      }
    __syncthreads();
    float2 st[KG];
    m_run = kNoMax;
#pragma unroll
    for (int g = 0; g < KG; ++g) {
      st[g] = ml[g * PER];
      m_run = fmaxf(m_run, st[g].x);   // a group without keys holds (kNoMax, 0, 0)
    }
    f32x16 own[ND];
#pragma unroll
    for (int g = 0; g < KG; ++g)       // this group's own blocks (a constant index for every g)
      if (g == kg) {
#pragma unroll
        for (int d = 0; d < ND; ++d) own[d] = oacc[g * ND + d];
      }
    f32x16 sum[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d) zero(sum[d]);
    l_tot = 0.0f;
#pragma unroll
    for (int g = 0; g < KG; ++g) {
      const float a = __builtin_amdgcn_exp2f(st[g].x - m_run);
      l_tot += a * st[g].y;
#pragma unroll
      for (int d = 0; d < ND; ++d) {
        f32x16 v = own[d];
        if (g != kg) {
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const f32x4 x = box(kg, g, d)[q * STEP];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[4 * q + e] = x[e];
          }
        }
        sum[d] += a * v;
      }
    }
#pragma unroll
    for (int d = 0; d < ND; ++d) oacc[d] = sum[d];
    __syncthreads();   // the boxes are read: their memory takes the rows
  }
  const int row0 = qb * 32 * QW + 32 * w;        // this wave's first row
  bool seen = nkb > 0;                           // whether this lane's row has keys
  int64_t tqo = tq;                              // where it is stored
  int ho = head;
  if constexpr (F != 0) {
    const int io = min(i, R - 1), so = p.by_g.quot(io);
    tqo = (int64_t)b * p.Sq + so;
    ho = kvh * p.G + p.by_g.rem(io, so);
    // rows behind the last get what a row without keys gets: 0, and a log-sum-exp of -inf
    if (i > last || clamp_len(p.mask.q_lens, b, p.Sq) == 0) l_tot = 0.0f;
    seen = l_tot != 0.0f;
    if (!seen) {
#pragma unroll
      for (int d = 0; d < ND; ++d) zero(oacc[d]);
    }
  }
  const int64_t row = tqo * p.Hq + ho;
  if (p.nsplit > 1) {
    if constexpr (KG > 1) {   // cross_choice takes parts with several key groups only
      const int64_t at = (int64_t)split * p.B * p.Sq * p.Hq + row;
      store_rows<ND>(smem + wave * row_area<ND, float>(), p.Opart, at * DH + kg * ND * 32, R - row0, oacc, 1.0f, lane);
      if (kg == 0 && h == 0 && i < R) p.MLpart[at] = make_float2(m_run, l_tot);
    }
    return;
  }
  if (p.lse && kg == 0 && h == 0 && i < R) p.lse[row] = seen ? m_run + __builtin_amdgcn_logf(l_tot) : -__builtin_inff();
  // O times 1 / l of its row (the lane's own)
  store_rows<ND>(smem + wave * row_area<ND, __bf16>(), (__bf16*)p.O, tqo * p.ldo + ho * DH + kg * ND * 32, R - row0, oacc,
                 seen ? 1.0f / l_tot : 0.0f, lane);
}

}  // namespace
}  // namespace partir
