// Gradients of attention to another sequence, d_head = 128, bf16.
//
// With P = 2^(c S - lse) (c = scale log2 e, lse the forward's base-2
// log-sum-exp; P = 0 for keys at and behind len_b):
//     D  = rowsum(dO * O)             dV = P^T dO        dP = dO V^T
//     dS = P * (dP - D)               dQ = scale dS K    dK = scale dS^T Q
// Up to 128 keys a sequence, one pass (cross_bwd_one_pass_kernel).  Above, each
// pass holds one axis of the scores in registers and streams the other
// through LDS, so that a gradient has one writer and a fixed order (no
// atomics), the G query heads of a key head included:
//  * dq: workgroup = 128 of the G Sq query rows of a (sequence, key head), 4
//    waves x 32, keys in tiles of 64; S^T = K Q^T and dP^T = V dO^T put one row
//    on a lane, dQ^T += K^T dS^T.  It also writes D.
//  * dkv: workgroup = 256 keys of a (sequence, key head), 8 waves x 32; its G Sq
//    query rows in tiles of 64; S = Q K^T and dP = dO V^T put one key on a lane,
//    dV^T += dO^T P, dK^T += Q^T dS.
// Where the axis that is held is short (few queries in dq, few keys in dkv) the
// streamed one is shared out over parts, whose float32 results an ordered
// reduction adds.  P and dS are rounded to bf16 for their products
// (within 2^-8 of their value), sums are float32.
//
// Rows and keys past their end are zero rows of the tiles; P is set to 0 for
// keys behind len_b in dq, and the statistics of missing rows make P 0 in dkv.
// Keys behind len_b get zero gradients.
//
// What bounds them is the matrix units with exp2 and the conversions beside them.
// 4 x 4096 queries over up to 2048 keys (80 % of them valid), 32 / 8 heads: dq 3
// products, 0.66 TFLOP, 610 us; dkv 4 products, 0.88 TFLOP, 830 us.  The matrix
// units are busy 58 and 49 % of the time; in dkv on three quarters of the compute
// units only, as a workgroup behind its sequence's end has nothing to do.
#include <algorithm>
#include <type_traits>

#include "attention_tiles.h"
#include "operators.h"

namespace partir {
namespace {

constexpr int NT = 256;
constexpr int TR = 64;                 // rows of a streamed tile
constexpr int TILE = TR * ROWB;

__device__ __forceinline__ int key_count(const CrossBwdParams& p, int b) {
  return p.lens ? min(max(p.lens[b], 0), p.Sk) : p.Sk;
}

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
  __device__ __forceinline__ RowTiles(const CrossBwdParams& p, int b, int kvh, int w_, int lane_)
      : q(p.Q + (int64_t)b * p.Sq * p.ldq + kvh * p.G * DH), g(p.dO + (int64_t)b * p.Sq * p.ldg + kvh * p.G * DH), ldq(p.ldq),
        ldg(p.ldg), by_g(p.by_g), R(p.G * p.Sq), w(w_), lane(lane_) {
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

__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(2, 2)))
void cross_bwd_dq_kernel(CrossBwdParams p) {
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
  const int b = p.by_hk.quot(bh), kvh = p.by_hk.rem(bh, b);
  const int i = qb * 128 + 32 * w + col;
  const int ic = min(i, R - 1), sq = p.by_g.quot(ic);
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
  const float lse = p.lse[tq * p.Hq + head];
  const int len = key_count(p, b);
  const CrossRange range = cross_range(len, p.by_q_parts, part);
  TileTr tr;
  tr.init(lane);
  const float c = p.scale_log2;
  if (len <= 256) {
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
#pragma unroll 1
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
  if (part == 0 && h == 0 && i < R) p.Dstat[tq * p.Hq + head] = Dq;

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
    const int left = nkeys - kb * TR;
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
#pragma unroll
      for (int v = 0; v < 16; ++v) pr[v] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[v], c, -lse));
      if (left < 32 * t + 32) {   // keys past the end
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
  if (p.q_parts > 1)
    store(smem, w, p.dQpart, (((int64_t)part * p.B * p.Sq + tq) * p.Hq + head) * DH, rows, dq, p.scale, lane);
  else
    store(smem, w, p.dQ, tq * p.lddq + head * DH, rows, dq, p.scale, lane);
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
template <bool EVEN>
__global__ __launch_bounds__(2 * NT, 2) void cross_bwd_dkv_kernel(CrossBwdParams p) {
  constexpr int STAGES = 0, VT = 2 * 2 * TILE, STAT = VT + 256 * ROWB;
  // one object: with several, the compiler tells them apart, takes every tile
  // read for one of the tiles being loaded and waits for those
  __shared__ __attribute__((aligned(1024))) char smem[STAT + 2 * 2 * TR * 4];
  static_assert(8 * row_area<4, __bf16>() <= STAT && 8 * row_area<2, float>() <= STAT, "the end goes through the stages and V");
  float (*const stat)[2][TR] = (float (*)[2][TR])(smem + STAT);   // [stage][-lse / c, -D][row]
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = lane >> 5, col = lane & 31;

  const int rest = p.by_nbh.quot(blockIdx.x), bh = p.by_nbh.rem(blockIdx.x, rest);
  const int kblk = p.by_k_parts.quot(rest), part = p.by_k_parts.rem(rest, kblk);
  const int b = p.by_hk.quot(bh), kvh = p.by_hk.rem(bh, b);
  const int len = key_count(p, b), R = p.G * p.Sq;
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
    const int tiles = (R + TR - 1) / TR, per = p.by_k_parts.quot(tiles + p.k_parts - 1);
    const int it0 = min(tiles, part * per), it1 = min(tiles, it0 + per);
    const RowTiles<EVEN, 8> rt(p, b, kvh, w, lane);
    const float inv_c = 1.0f / p.scale_log2;
    float st_l = 0.0f, st_d = 0.0f;
    auto gload = [&](int it, int buf) {
      rt.load(it, smem + STAGES + buf * 2 * TILE);
      if (tid < TR) {
        // nothing looks at the loaded values before sstore: a use here would wait
        // for the tiles' loads too
        const int i = min(it * TR + tid, R - 1), sq = p.by_g.quot(i);
        const int64_t at = ((int64_t)b * p.Sq + sq) * p.Hq + kvh * p.G + p.by_g.rem(i, sq);
        st_l = p.lse[at];
        st_d = p.Dstat[at];
      }
    };
    auto sstore = [&](int it, int buf) {
      if (tid < TR) {
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
      if (kw < len) {   // wave-uniform
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
          start(s, 0);
#pragma unroll
          for (int ds = 0; ds < 8; ++ds) s = mfma(tile_rows(qs, 32 * t, col, h, ds), kf[ds], s);
          __builtin_amdgcn_sched_barrier(0);
          bf16x8 pf[2];
#pragma unroll
          for (int v = 0; v < 16; v += 2) {
            s[v] = __builtin_amdgcn_exp2f(s[v] * c);
            s[v + 1] = __builtin_amdgcn_exp2f(s[v + 1] * c);
            put2(pf[v >> 3], v & 7, s[v], s[v + 1]);
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
template <bool EVEN>
__global__ __launch_bounds__(2 * NT, 2) void cross_bwd_one_pass_kernel(CrossBwdParams p) {
  // Two stages of Q and dO first: offsets below 64 KiB fold into the LDS
  // instructions, so that both share their address registers.
  constexpr int STAGES = 0, KT = 2 * 2 * TILE;       // K
  constexpr int EP = KT + 128 * ROWB;                // P and dS of a tile, [64 rows][128 keys] as tiles
  constexpr int ES = EP + TILE;
  constexpr int DSUM = ES + TILE;                    // [key group][row]: shares of D
  constexpr int ROWS = DSUM + 4 * TR * 4;            // the waves' row areas
  __shared__ __attribute__((aligned(1024))) char smem[ROWS + 8 * row_area<1, __bf16>()];
  static_assert(8 * row_area<2, float>() <= EP, "the end goes through the stages and K");
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = lane >> 5, col = lane & 31;
  const int half = w & 1, kg = w >> 1;

  const int part = p.by_nbh.quot(blockIdx.x), bh = p.by_nbh.rem(blockIdx.x, part);
  const int b = p.by_hk.quot(bh), kvh = p.by_hk.rem(bh, b);
  const int R = p.G * p.Sq, tiles = (R + TR - 1) / TR, per = p.by_k_parts.quot(tiles + p.k_parts - 1);
  const int it0 = min(tiles, part * per), it1 = min(tiles, it0 + per);
  const int len = key_count(p, b);

  // K for good, V through the first stage (rows behind len are zeros)
  const int64_t tk0 = (int64_t)b * p.Sk;
  tile_load<128, 8>(p.K + tk0 * p.ldk + kvh * DH, p.ldk, len, smem + KT, w, lane);
  tile_load<128, 8>(p.V + tk0 * p.ldv + kvh * DH, p.ldv, len, smem + STAGES, w, lane);
  const RowTiles<EVEN, 8> rt(p, b, kvh, w, lane);
  TileTr tr;
  tr.init(lane);
  WAIT_VMCNT(0);
  __syncthreads();
  bf16x8 vf[8];
#pragma unroll
  for (int ds = 0; ds < 8; ++ds) vf[ds] = tile_rows(smem + STAGES, 32 * kg, col, h, ds);
  __syncthreads();

  const float c = p.scale_log2;
  float lse_next = 0.0f;
  // tile `it` into a stage, and the log-sum-exp of this lane's row of it
  auto gload = [&](int it, int buf) {
    rt.load(it, smem + STAGES + buf * 2 * TILE);
    const int i = min(it * TR + 32 * half + col, R - 1), sq = p.by_g.quot(i);
    lse_next = p.lse[((int64_t)b * p.Sq + sq) * p.Hq + kvh * p.G + p.by_g.rem(i, sq)];
  };
  f32x16 dk[2], dv[2];
#pragma unroll
  for (int d = 0; d < 2; ++d) {
    zero(dk[d]);
    zero(dv[d]);
  }
  const int erow = 32 * half + col;                  // this lane's row of P and dS
  auto iter = [&](int it, auto stage) {
    constexpr int cur = decltype(stage)::value;
    __builtin_amdgcn_sched_barrier(0);
    WAIT_VMCNT(0);                                   // the tile and lse have landed
    lds_barrier();
    const int row = it * TR + erow;
    const float lse = row < R ? lse_next : __builtin_inff();   // a missing row: P = 0
    if (it + 1 < it1) gload(it + 1, cur ^ 1);
    const char* qs = smem + STAGES + cur * 2 * TILE;
    const char* gs = qs + TILE;
    f32x16 s, dp;
    zero(s);
    zero(dp);
#pragma unroll
    for (int ds = 0; ds < 8; ++ds) {
      s = mfma(tile_rows(smem + KT, 32 * kg, col, h, ds), tile_rows(qs, 32 * half, col, h, ds), s);
      dp = mfma(vf[ds], tile_rows(gs, 32 * half, col, h, ds), dp);
    }
    // element v: key 32 kg + 8 (v / 4) + 4 h + v % 4
#pragma unroll
    for (int v = 0; v < 16; ++v) s[v] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[v], c, -lse));
    if (len < 32 * kg + 32) {
#pragma unroll
      for (int v = 0; v < 16; ++v)
        if (32 * kg + 8 * (v >> 2) + 4 * h + (v & 3) >= len) s[v] = 0.0f;
    }
    float d = 0.0f;
#pragma unroll
    for (int v = 0; v < 16; ++v) d = __builtin_fmaf(s[v], dp[v], d);
    d += __shfl_xor(d, 32);
    auto put = [&](char* e, f32x16 x) {   // four consecutive keys a lane and write
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const bf16x4 o = {(__bf16)x[4 * q + 0], (__bf16)x[4 * q + 1], (__bf16)x[4 * q + 2], (__bf16)x[4 * q + 3]};
        lds_write(e + tile_off(erow, 64 * kg + 16 * q + 8 * h), o);
      }
    };
    put(smem + EP, s);
    if (h == 0) lds_write(smem + DSUM + (kg * TR + erow) * 4, d);
    lds_barrier();
    float D = 0.0f;
#pragma unroll
    for (int g = 0; g < 4; ++g) D += lds_read<float>(smem + DSUM + (g * TR + erow) * 4);
#pragma unroll
    for (int v = 0; v < 16; ++v) dp[v] = s[v] * (dp[v] - D);
    put(smem + ES, dp);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const bf16x8 pf = tr.read(smem + EP, u, kg);
#pragma unroll
      for (int e = 0; e < 2; ++e) dv[e] = mfma(tr.read(gs, u, 2 * half + e), pf, dv[e]);
    }
    lds_barrier();
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const bf16x8 df = tr.read(smem + ES, u, kg);
#pragma unroll
      for (int e = 0; e < 2; ++e) dk[e] = mfma(tr.read(qs, u, 2 * half + e), df, dk[e]);
    }
    f32x16 dq;
    zero(dq);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      // keys 16 u + 4 h.. and 16 u + 8 + 4 h.. of this lane's row, the order of the transposed reads
      const lds_i16x4_t lo = lds_read<lds_i16x4_t>(smem + ES + tile_off(erow, 32 * u + 8 * h));
      const lds_i16x4_t hi = lds_read<lds_i16x4_t>(smem + ES + tile_off(erow, 32 * u + 16 + 8 * h));
      dq = mfma(tr.read(smem + KT, u, kg),
                __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7)), dq);
    }
    if (len == 0) zero(dq);   // a row of dO that is not finite, times weights of 0
    const int rc = min(row, R - 1), sq = p.by_g.quot(rc);
    store_rows<1>(smem + ROWS + w * row_area<1, __bf16>(), (__bf16*)p.dQ,
                  ((int64_t)b * p.Sq + sq) * p.lddq + (kvh * p.G + p.by_g.rem(rc, sq)) * DH + 32 * kg, R - it * TR - 32 * half,
                  &dq, p.scale, lane);
  };
  if (it0 < it1) gload(it0, 0);
  for (int it = it0; it < it1; it += 2) {
    iter(it, std::integral_constant<int, 0>{});
    if (it + 1 < it1) iter(it + 1, std::integral_constant<int, 1>{});
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
    store_rows<2>(area, p.dKpart, at, rows, dk, p.scale, lane);
    store_rows<2>(area, p.dVpart, at, rows, dv, 1.0f, lane);
  } else {
    store_rows<2>(area, (__bf16*)p.dK, tk * p.lddk + kvh * DH + 64 * half, rows, dk, p.scale, lane);
    store_rows<2>(area, (__bf16*)p.dV, tk * p.lddv + kvh * DH + 64 * half, rows, dv, 1.0f, lane);
  }
}

// Four columns a thread; the parts' loads in flight together.
__global__ __launch_bounds__(256) void part_sum_kernel(PartSum p) {
  const int64_t stride = p.rows * p.cols, quads = stride / 4;
  const int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (q >= quads) return;
  const float* src = p.part[blockIdx.y] + 4 * q;
  f32x4 s = *(const f32x4*)src;
#pragma unroll 8
  for (int i = 1; i < p.parts; ++i) s += *(const f32x4*)(src + i * stride);
  const int64_t row = quads < ((int64_t)1 << 31) ? p.by_cols4.quot((int)q) : q / (p.cols / 4);
  *(bf16x4*)(p.out[blockIdx.y] + row * p.ld[blockIdx.y] + 4 * (q - row * (p.cols / 4))) =
      bf16x4{(__bf16)s[0], (__bf16)s[1], (__bf16)s[2], (__bf16)s[3]};
}

constexpr int64_t kCUs = 256;

}  // namespace

CrossBwdChoice cross_bwd_choice(int64_t B, int64_t Sq, int64_t Sk, int64_t Hq, int64_t Hk) {
  // A tile of 64 streamed rows takes a workgroup 2.8 us in the one pass, 1.45 us in
  // dq and 3 us in dkv; 1000 rows of a part cost 0.15 us.  One part / these: 2 x 4096
  // queries over 77 keys, 8 heads 187 / 30 us; 200 queries over 2048 keys, 4 heads
  // 77 / 36; 2048 queries over 200 keys, 4 heads 128 / 45; 500 over 500, 2 heads 53 /
  // 34.
  const int64_t R = Hq / Hk * Sq, rows = (R + 63) / 64, keys = (Sk + 63) / 64;
  auto most = [](int64_t grid, int64_t tiles) { return grid > 0 ? std::min(kCUs / grid, tiles) : 1; };
  const double q_us = 1.5e-4 * (double)(B * Sq * Hq), k_us = 2 * 1.5e-4 * (double)(B * Sk * Hk);
  // without keys the dq pass alone runs, and writes zeros
  if (Sk > 0 && Sk <= 128) return {true, 1, best_parts(most(B * Hk, rows), rows, 2.8, k_us)};
  return {false, best_parts(most(B * Hk * ((R + 127) / 128), keys), keys, 1.45, q_us),
          best_parts(most(B * Hk * ((Sk + 255) / 256), rows), rows, 3.0, k_us)};
}

hipError_t launch_cross_backward(const CrossBwdParams& p, CrossBwdPass pass, hipStream_t s) {
  const int64_t nbh = (int64_t)p.B * p.Hk;
  const bool even = 16 % p.G == 0;
  if (pass == CROSS_DQ) {
    const int64_t blocks = ((int64_t)p.G * p.Sq + 127) / 128;
    hipLaunchKernelGGL(cross_bwd_dq_kernel, dim3((unsigned)(blocks * nbh * p.q_parts)), dim3(NT), 0, s, p);
  } else if (pass == CROSS_ALL) {
    hipLaunchKernelGGL(even ? cross_bwd_one_pass_kernel<true> : cross_bwd_one_pass_kernel<false>,
                       dim3((unsigned)(nbh * p.k_parts)), dim3(2 * NT), 0, s, p);
  } else {
    const int64_t blocks = ((int64_t)p.Sk + 255) / 256;
    hipLaunchKernelGGL(even ? cross_bwd_dkv_kernel<true> : cross_bwd_dkv_kernel<false>,
                       dim3((unsigned)(blocks * nbh * p.k_parts)), dim3(2 * NT), 0, s, p);
  }
  return hipGetLastError();
}

hipError_t launch_part_sum(const PartSum& p, hipStream_t s) {
  const dim3 grid((unsigned)((p.rows * p.cols / 4 + 255) / 256), (unsigned)p.n);
  hipLaunchKernelGGL(part_sum_kernel, grid, dim3(256), 0, s, p);
  return hipGetLastError();
}

}  // namespace partir
