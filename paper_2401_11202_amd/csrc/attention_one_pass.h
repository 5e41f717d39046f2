// All gradients of attention to short sequences in one launch: of attention to
// another sequence (form 0) and of masked attention.
#pragma once
#include <type_traits>

#include "attention_mask.h"
#include "attention_row_tiles.h"

namespace partir {
namespace {

// What a kernel of form F knows of a sequence.
struct NoSeq {
  __device__ __forceinline__ NoSeq(const CrossBwdParams&, int) {}
};
template <int F>
struct FormSeq {
  typedef SeqMask type;
};
template <>
struct FormSeq<0> {
  typedef NoSeq type;
};

// All three gradients in one pass where a sequence has at most 128 keys: S and
// dP are formed once (5 products instead of 8), and D = sum_j P_j dP_j comes
// from the weights themselves, so that O is not read and its rounding to bf16,
// which with few keys is of the size of the other roundings, stays out.
// Workgroup = the keys of a (sequence, key head) and a part of its query rows,
// in tiles of 64; eight waves, two row halves x four groups of 32 keys, with K
// and V as operands in registers.  Per tile
//   a wave forms S^T = K Q^T and dP^T = V dO^T of its keys and rows (a lane owns a
//     row), and leaves P and its share of D in LDS;
//   with D, dS goes to LDS too, and dV^T += dO^T P over all rows, for its keys and
//     half of the columns (the row half is the column half here);
//   then dK^T += Q^T dS likewise, and 32 columns of dQ^T = K^T dS^T of its rows over
//     all keys.
// Three barriers a tile, the next one's loads in flight across them.  Two waves
// a SIMD, one workgroup a CU.  (With the rows of S on the lanes' registers
// instead, four waves of 32 keys and D from sums over lanes, 350 registers and
// one wave a SIMD, it took 35 us for 2 x 4096 queries, 77 keys and 8 heads; 25 so.)
//
// F is the form (attention_mask.h).  In the masked ones the tiles end with the last
// valid row, a wave without a visible pair of its keys and rows leaves zeros, and the
// workgroups share out the rows behind the last tile, whose dQ is 0.
template <bool EVEN, int F>
__global__ __launch_bounds__(2 * NT, 2) void attention_one_pass_kernel(typename FormParams<F>::bwd p) {
  // Two stages of Q and dO first: offsets below 64 KiB fold into the LDS
  // instructions, so that both share their address registers.
  constexpr int STAGES = 0, KT = 2 * 2 * TILE;       // K
  constexpr int EP = KT + 128 * ROWB;                // P and dS of a tile, [64 rows][128 keys] as tiles
  constexpr int ES = EP + TILE;
  constexpr int DSUM = ES + TILE;                    // [key group][row]: shares of D
  constexpr int PSUM = DSUM + 4 * TR * 4;            // and of the sum of the weights
  constexpr int ROWS = PSUM + (F != 0 ? 4 * TR * 4 : 0);   // the waves' row areas
  __shared__ __attribute__((aligned(1024))) char smem[ROWS + 8 * row_area<1, __bf16>()];
  static_assert(8 * row_area<2, float>() <= EP, "the end goes through the stages and K");
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = lane >> 5, col = lane & 31;
  const int half = w & 1, kg = w >> 1;

  const int part = p.by_nbh.quot(blockIdx.x), bh = p.by_nbh.rem(blockIdx.x, part);
  const int b = p.by_hk.quot(bh), kvh = p.by_hk.rem(bh, b);
  const typename FormSeq<F>::type m(p, b);
  const int all = p.G * p.Sq;
  int R = all, len;                                  // rows that are read, and keys
  if constexpr (F != 0) {
    R = p.G * m.qlen;
    len = m.klen;
  } else {
    len = clamp_len(p.lens, b, p.Sk);
  }
  const int tiles = (R + TR - 1) / TR, per = p.by_k_parts.quot(tiles + p.k_parts - 1);
  const int it0 = min(tiles, part * per), it1 = min(tiles, it0 + per);

  // K for good, V through the first stage (rows behind len are zeros)
  const int64_t tk0 = (int64_t)b * p.Sk;
  tile_load<128, 8>(p.K + tk0 * p.ldk + kvh * DH, p.ldk, len, smem + KT, w, lane);
  tile_load<128, 8>(p.V + tk0 * p.ldv + kvh * DH, p.ldv, len, smem + STAGES, w, lane);
  const RowTiles<EVEN, 8> rt(p, b, kvh, R, w, lane);
  TileTr tr;
  tr.init(lane);
  WAIT_VMCNT(0);
  __syncthreads();
  bf16x8 vf[8];
#pragma unroll
  for (int ds = 0; ds < 8; ++ds) vf[ds] = tile_rows(smem + STAGES, 32 * kg, col, h, ds);
  __syncthreads();

  const float c = p.scale_log2;
  float lse_next = 0.0f, slope_next = 0.0f;
  int2 docs_next = make_int2(0, 0);
  bool by_id = false;
  if constexpr (F != 0) by_id = p.mask.rows && p.mask.by_id[b];
  // tile `it` into a stage, and the numbers of this lane's row of it
  auto gload = [&](int it, int buf) {
    rt.load(it, smem + STAGES + buf * 2 * TILE);
    const int i = min(it * TR + 32 * half + col, R - 1), sq = p.by_g.quot(i), head = kvh * p.G + p.by_g.rem(i, sq);
    const int64_t tq = (int64_t)b * p.Sq + sq;
    lse_next = p.lse[tq * p.Hq + head];
    if constexpr (F != 0) {
      if (p.mask.rows) docs_next = p.mask.rows[tq];
      if constexpr ((F & kBias) != 0) slope_next = p.mask.slopes[head];
    }
  };
  const float f = (F & kCap) != 0 ? 4.0f * p.scale : p.scale;
  f32x16 dk[2], dv[2];
#pragma unroll
  for (int d = 0; d < 2; ++d) {
    zero(dk[d]);
    zero(dv[d]);
  }
  const int erow = 32 * half + col;                  // this lane's row of P and dS
  auto iter = [&](int it, auto stage) {
    const int cur = stage;
    int kt = KT, ep = EP, es = ES;
    if constexpr (F != 0) asm volatile("" : "+s"(kt), "+s"(ep), "+s"(es));   // their addresses are formed here, for want of room to keep them
    __builtin_amdgcn_sched_barrier(0);
    WAIT_VMCNT(0);                                   // the tile and lse have landed
    lds_barrier();
    const int row = it * TR + erow;
    float lse = row < R ? lse_next : __builtin_inff();         // a missing row: P = 0
    const float slope = slope_next * kLog2e;
    const int2 docs = docs_next;
    if (it + 1 < it1) gload(it + 1, cur ^ 1);
    const char* qs = smem + STAGES + cur * 2 * TILE;
    const char* gs = qs + TILE;
    f32x16 s, dp, sl;                                // sl: a quarter of the cap's derivative
    zero(s);
    zero(dp);
    auto products = [&]() {
#pragma unroll
      for (int ds = 0; ds < 8; ++ds) {
        s = mfma(tile_rows(smem + kt, 32 * kg, col, h, ds), tile_rows(qs, 32 * half, col, h, ds), s);
        dp = mfma(vf[ds], tile_rows(gs, 32 * half, col, h, ds), dp);
      }
    };
    // element v: key 32 kg + 8 (v / 4) + 4 h + v % 4
    if constexpr (F != 0) {
      if (lse == -__builtin_inff()) lse = __builtin_inff();    // a row without keys
      const int sq = p.by_g.quot(min(row, R - 1));
      const RowMask mask(m, p.mask.rows != nullptr, docs, sq);
      zero(sl);
      if (!mask.none(32 * kg, 32)) {
        products();
        const RowWeights<F> weights{c, lse, p.mask.cap_log2 - lse, slope, by_id};
        weights(p, mask, b, (int64_t)b * p.Sq + sq, h, 32 * kg, s, sl);
      }
    } else {
      products();
#pragma unroll
      for (int v = 0; v < 16; ++v) s[v] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[v], c, -lse));
      if (len < 32 * kg + 32) {
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (32 * kg + 8 * (v >> 2) + 4 * h + (v & 3) >= len) s[v] = 0.0f;
      }
    }
    float d = 0.0f;
#pragma unroll
    for (int v = 0; v < 16; ++v) d = __builtin_fmaf(s[v], dp[v], d);
    d += __shfl_xor(d, 32);
    if constexpr (F != 0) {
      float sum = 0.0f;
#pragma unroll
      for (int v = 0; v < 16; ++v) sum += s[v];
      sum += __shfl_xor(sum, 32);
      if (h == 0) lds_write(smem + PSUM + (kg * TR + erow) * 4, sum);
    }
    auto put = [&](char* e, f32x16 x) {   // four consecutive keys a lane and write
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const bf16x4 o = {(__bf16)x[4 * q + 0], (__bf16)x[4 * q + 1], (__bf16)x[4 * q + 2], (__bf16)x[4 * q + 3]};
        lds_write(e + tile_off(erow, 64 * kg + 16 * q + 8 * h), o);
      }
    };
    put(smem + ep, s);
    if (h == 0) lds_write(smem + DSUM + (kg * TR + erow) * 4, d);
    if constexpr ((F & kCap) != 0) {                 // P with the cap's derivative, for dS
#pragma unroll
      for (int v = 0; v < 16; ++v) s[v] *= sl[v];
    }
    if constexpr (F != 0) __builtin_amdgcn_sched_barrier(0);
    lds_barrier();
    float D = 0.0f;
#pragma unroll
    for (int g = 0; g < 4; ++g) D += lds_read<float>(smem + DSUM + (g * TR + erow) * 4);
    if constexpr (F != 0) {   // over the sum of the weights, which is 1 up to the error of z
      float sum = 0.0f;
#pragma unroll
      for (int g = 0; g < 4; ++g) sum += lds_read<float>(smem + PSUM + (g * TR + erow) * 4);
      D = sum > 0.0f ? D / sum : 0.0f;
    }
#pragma unroll
    for (int v = 0; v < 16; ++v) dp[v] = s[v] * (dp[v] - D);
    put(smem + es, dp);
    if constexpr (F != 0) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const bf16x8 pf = tr.read(smem + ep, u, kg);
#pragma unroll
      for (int e = 0; e < 2; ++e) dv[e] = mfma(tr.read(gs, u, 2 * half + e), pf, dv[e]);
    }
    lds_barrier();
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const bf16x8 df = tr.read(smem + es, u, kg);
#pragma unroll
      for (int e = 0; e < 2; ++e) dk[e] = mfma(tr.read(qs, u, 2 * half + e), df, dk[e]);
    }
    f32x16 dq;
    zero(dq);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      // keys 16 u + 4 h.. and 16 u + 8 + 4 h.. of this lane's row, the order of the transposed reads
      const lds_i16x4_t lo = lds_read<lds_i16x4_t>(smem + es + tile_off(erow, 32 * u + 8 * h));
      const lds_i16x4_t hi = lds_read<lds_i16x4_t>(smem + es + tile_off(erow, 32 * u + 16 + 8 * h));
      dq = mfma(tr.read(smem + kt, u, kg),
                __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7)), dq);
    }
    // a row of dO that is not finite, times weights of 0
    if (F != 0 ? lse == __builtin_inff() : len == 0) zero(dq);
    const int rc = min(row, all - 1), sq = p.by_g.quot(rc);
    store_rows<1>(smem + ROWS + w * row_area<1, __bf16>(), (__bf16*)p.dQ,
                  ((int64_t)b * p.Sq + sq) * p.lddq + (kvh * p.G + p.by_g.rem(rc, sq)) * DH + 32 * kg, all - it * TR - 32 * half,
                  &dq, f, lane);
  };
  if (it0 < it1) gload(it0, 0);
  if constexpr (F != 0) {                            // one copy of the body: two would keep more addresses than there is room for
    int cur = 0;
#pragma unroll 1
    for (int it = it0; it < it1; ++it, cur ^= 1) iter(it, cur);
  } else {
    for (int it = it0; it < it1; it += 2) {
      iter(it, std::integral_constant<int, 0>{});
      if (it + 1 < it1) iter(it + 1, std::integral_constant<int, 1>{});
    }
  }
  if constexpr (F != 0) {                            // rows of dQ behind the last tile: 4 a wave and step
    const int n = p.k_parts * 32;
    for (int i = tiles * TR + part * 32 + 4 * w + (lane >> 4); i < all; i += n) {
      const int sq = p.by_g.quot(i);
      *(bf16x8*)(p.dQ + ((int64_t)b * p.Sq + sq) * p.lddq + (kvh * p.G + p.by_g.rem(i, sq)) * DH + 8 * (lane & 15)) = bf16x8{};
    }
  }
  __syncthreads();
  // 32 keys x 64 columns of dK and dV.  Keys behind len met P = 0 only, but times
  // rows of Q and dO that need not be finite.
  const int kj = 32 * kg + col, rows = p.Sk - 32 * kg;
  if (kj >= len) {
#pragma unroll
    for (int d = 0; d < 2; ++d) {
      zero(dk[d]);
      zero(dv[d]);
    }
  }
  const int64_t tk = tk0 + kj;
  char* const area = smem + w * row_area<2, float>();
  if (p.k_parts > 1) {
    const int64_t at = (((int64_t)part * p.B * p.Sk + tk) * p.Hk + kvh) * DH + 64 * half;
    store_rows<2>(area, p.dKpart, at, rows, dk, f, lane);
    store_rows<2>(area, p.dVpart, at, rows, dv, 1.0f, lane);
  } else {
    store_rows<2>(area, (__bf16*)p.dK, tk * p.lddk + kvh * DH + 64 * half, rows, dk, f, lane);
    store_rows<2>(area, (__bf16*)p.dV, tk * p.lddv + kvh * DH + 64 * half, rows, dv, 1.0f, lane);
  }
}

}  // namespace
}  // namespace partir
