// Gradients of attention to another sequence, d_head = 128, bf16.
//
// With P = 2^(c S - lse) (c = scale log2 e, lse the forward's base-2
// log-sum-exp; P = 0 for keys at and behind len_b):
//     D  = rowsum(dO * O)             dV = P^T dO        dP = dO V^T
//     dS = P * (dP - D)               dQ = scale dS K    dK = scale dS^T Q
// Each pass holds one axis of the scores in registers and streams the other
// through LDS, so that a gradient has one writer and a fixed order (no
// atomics), the G query heads of a key head included:
//  * dq: workgroup = 128 of the G Sq query rows of a (sequence, key head), 4
//    waves x 32, keys in tiles of 64; S^T = K Q^T and dP^T = V dO^T put one row
//    on a lane, dQ^T += K^T dS^T.  It also writes D.
//  * dv and dk: workgroup = 128 keys of a (sequence, key head), 4 waves x 32;
//    the rows of its G heads in tiles of 64, head after head; S = Q K^T and dP =
//    dO V^T put one key on a lane, dV^T += dO^T P, dK^T += Q^T dS.
// Where the axis that is held is short (few queries in dq, few keys in dk and
// dv) the streamed one is shared out over parts, whose float32 results an
// ordered reduction adds.  P and dS are rounded to bf16 for their products
// (within 2^-8 of their value), sums are float32.
//
// Rows and keys past their end are zero rows of the tiles; P is set to 0 for
// keys behind len_b in dq, and the statistics of missing rows make P 0 in dk
// and dv.  Keys behind len_b get zero gradients.
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

// A lane's 64 of the 128 x 32 results of a wave: columns 32 d + 8 g + 4 h.. of
// its row, as bf16 or as float32.
__device__ __forceinline__ void store_row(uint16_t* out, const f32x16* a, float f, int h) {
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *(bf16x4*)(out + 32 * d + 8 * g + 4 * h) = bf16x4{(__bf16)(a[d][4 * g + 0] * f), (__bf16)(a[d][4 * g + 1] * f),
                                                        (__bf16)(a[d][4 * g + 2] * f), (__bf16)(a[d][4 * g + 3] * f)};
}
__device__ __forceinline__ void store_row(float* out, const f32x16* a, float f, int h) {
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *(f32x4*)(out + 32 * d + 8 * g + 4 * h) =
          f32x4{a[d][4 * g + 0] * f, a[d][4 * g + 1] * f, a[d][4 * g + 2] * f, a[d][4 * g + 3] * f};
}

__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(2, 2)))
void cross_bwd_dq_kernel(CrossBwdParams p) {
  __shared__ __attribute__((aligned(1024))) char smem[2 * 2 * TILE];
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = lane >> 5, col = lane & 31;

  const int R = p.G * p.Sq, nbh = p.B * p.Hk;
  const int bh = blockIdx.x % nbh, rest = blockIdx.x / nbh;
  const int part = rest % p.q_parts, qb = rest / p.q_parts;
  const int b = bh / p.Hk, kvh = bh - b * p.Hk;
  const CrossRange range = cross_range(key_count(p, b), p.q_parts, part);
  const int i = qb * 128 + 32 * w + col;
  const int ic = min(i, R - 1), sq = ic / p.G;
  const int64_t tq = (int64_t)b * p.Sq + sq;
  const int head = kvh * p.G + ic - sq * p.G;

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
  const float Dq = dsum + __shfl_xor(dsum, 32);
  const float lse = p.lse[tq * p.Hq + head];
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
  TileTr tr;
  tr.init(lane);
  f32x16 dq[4];
#pragma unroll
  for (int d = 0; d < 4; ++d) zero(dq[d]);
  const float c = p.scale_log2;
  auto iter = [&](int kb, auto stage) {
    constexpr int cur = decltype(stage)::value;
    if (kb + 1 < nkb) gload(kb + 1, cur ^ 1);
    const char* ks = smem + cur * 2 * TILE;
    const char* vs = ks + TILE;
    const int left = nkeys - kb * TR;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      f32x16 s, dp;
      zero(s);
      zero(dp);
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
        put2(dsf[v >> 3], v & 7, pr[v] * (dp[v] - Dq), pr[v + 1] * (dp[v + 1] - Dq));
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
  if (i >= R) return;
  if (p.q_parts > 1)
    store_row(p.dQpart + (((int64_t)part * p.B * p.Sq + tq) * p.Hq + head) * DH, dq, p.scale, h);
  else
    store_row(p.dQ + tq * p.lddq + head * DH, dq, p.scale, h);
}

// MODE 1: dV (S and P, dV^T += dO^T P); MODE 2: dK (S, P and dP, dK^T += Q^T
// dS).  One pass doing both would hold twice the accumulators, which leaves one
// wave a SIMD; forming S again costs less.
template <int MODE>
__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(2, 2)))
void cross_bwd_dkv_kernel(CrossBwdParams p) {
  constexpr bool DO_K = MODE == 2;
  __shared__ __attribute__((aligned(1024))) char smem[2 * 2 * TILE];
  __shared__ float stat[2][2][TR];   // [stage][-lse / c, -D][row]
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = lane >> 5, col = lane & 31;

  const int nbh = p.B * p.Hk;
  const int bh = blockIdx.x % nbh, rest = blockIdx.x / nbh;
  const int part = rest % p.k_parts, kblk = rest / p.k_parts;
  const int b = bh / p.Hk, kvh = bh - b * p.Hk;
  const int len = key_count(p, b);
  const int kj = kblk * 128 + 32 * w + col;          // this lane's key
  const int64_t tk = (int64_t)b * p.Sk + kj;

  f32x16 acc[4];
#pragma unroll
  for (int d = 0; d < 4; ++d) zero(acc[d]);
  // workgroup-uniform: keys behind len_b get zeros
  if (kblk * 128 < len) {
    bf16x8 kf[8], vf[8];
    {
      const int64_t t = (int64_t)b * p.Sk + min(kj, p.Sk - 1);
      const uint16_t* krow = p.K + t * p.ldk + kvh * DH + 8 * h;
      const uint16_t* vrow = p.V + t * p.ldv + kvh * DH + 8 * h;
#pragma unroll
      for (int ds = 0; ds < 8; ++ds) {
        kf[ds] = *(const bf16x8*)(krow + 16 * ds);
        if (DO_K) vf[ds] = *(const bf16x8*)(vrow + 16 * ds);
      }
    }
    // items: the 64-row tiles of head 0, of head 1, ...; a part takes a run of them
    const int nqb = (p.Sq + TR - 1) / TR;
    const int64_t items = (int64_t)p.G * nqb, per = (items + p.k_parts - 1) / p.k_parts;
    const int64_t it0 = min(items, part * per), it1 = min(items, it0 + per);
    const float inv_c = 1.0f / p.scale_log2;
    float st_l = 0.0f, st_d = 0.0f;
    auto gload = [&](int64_t it, int buf) {
      const int g = (int)(it / nqb), qb = (int)(it - (int64_t)g * nqb), head = kvh * p.G + g;
      const int rows = min(TR, p.Sq - qb * TR);
      const int64_t t0 = (int64_t)b * p.Sq + qb * TR;
      char* t = smem + buf * 2 * TILE;
      tile_load<TR, 4>(p.Q + t0 * p.ldq + head * DH, p.ldq, rows, t, w, lane);
      tile_load<TR, 4>(p.dO + t0 * p.ldg + head * DH, p.ldg, rows, t + TILE, w, lane);
      if (tid < TR) {
        const int64_t at = (t0 + tid) * p.Hq + head;
        st_l = tid < rows ? p.lse[at] : __builtin_inff();   // a missing row: P = 2^-inf
        if (DO_K) st_d = tid < rows ? p.Dstat[at] : 0.0f;
      }
    };
    auto sstore = [&](int buf) {
      if (tid < TR) {
        stat[buf][0][tid] = -st_l * inv_c;
        stat[buf][1][tid] = -st_d;
      }
    };
    TileTr tr;
    tr.init(lane);
    const float c = p.scale_log2;
    auto iter = [&](int64_t it, auto stage) {
      constexpr int cur = decltype(stage)::value;
      if (it + 1 < it1) gload(it + 1, cur ^ 1);
      const char* qs = smem + cur * 2 * TILE;
      const char* gs = qs + TILE;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        // the accumulators start at -lse / c and -D of their rows
        f32x16 s, dp;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f32x4 l4 = *(const f32x4*)&stat[cur][0][32 * t + 8 * q + 4 * h];
#pragma unroll
          for (int j = 0; j < 4; ++j) s[4 * q + j] = l4[j];
          if (DO_K) {
            const f32x4 d4 = *(const f32x4*)&stat[cur][1][32 * t + 8 * q + 4 * h];
#pragma unroll
            for (int j = 0; j < 4; ++j) dp[4 * q + j] = d4[j];
          }
        }
#pragma unroll
        for (int ds = 0; ds < 8; ++ds) {
          s = mfma(tile_rows(qs, 32 * t, col, h, ds), kf[ds], s);
          if (DO_K) dp = mfma(tile_rows(gs, 32 * t, col, h, ds), vf[ds], dp);
        }
        bf16x8 pf[2];
#pragma unroll
        for (int v = 0; v < 16; v += 2) {
          const float p0 = __builtin_amdgcn_exp2f(s[v] * c), p1 = __builtin_amdgcn_exp2f(s[v + 1] * c);
          if (DO_K)
            put2(pf[v >> 3], v & 7, p0 * dp[v], p1 * dp[v + 1]);
          else
            put2(pf[v >> 3], v & 7, p0, p1);
        }
#pragma unroll
        for (int uu = 0; uu < 2; ++uu)
#pragma unroll
          for (int d = 0; d < 4; ++d) acc[d] = mfma(tr.read(DO_K ? qs : gs, 2 * t + uu, d), pf[uu], acc[d]);
      }
      if (it + 1 < it1) sstore(cur ^ 1);
      WAIT_VMCNT(0);
      __syncthreads();
    };
    if (it0 < it1) {
      gload(it0, 0);
      sstore(0);
    }
    WAIT_VMCNT(0);
    __syncthreads();
    for (int64_t it = it0; it < it1; it += 2) {
      iter(it, std::integral_constant<int, 0>{});
      if (it + 1 < it1) iter(it + 1, std::integral_constant<int, 1>{});
    }
    if (kj >= len) {   // a lane's key is its own column: what its sums hold goes nowhere else
#pragma unroll
      for (int d = 0; d < 4; ++d) zero(acc[d]);
    }
  }
  if (kj >= p.Sk) return;
  const float f = DO_K ? p.scale : 1.0f;
  if (p.k_parts > 1)
    store_row((DO_K ? p.dKpart : p.dVpart) + (((int64_t)part * p.B * p.Sk + tk) * p.Hk + kvh) * DH, acc, f, h);
  else
    store_row((DO_K ? p.dK + tk * p.lddk : p.dV + tk * p.lddv) + kvh * DH, acc, f, h);
}

constexpr int64_t kCUs = 256;

}  // namespace

void cross_bwd_choice(int64_t B, int64_t Sq, int64_t Sk, int64_t Hq, int64_t Hk, int* q_parts, int* k_parts) {
  // Parts until there is a workgroup for every CU, none of them shorter than 4
  // tiles of the streamed axis.
  auto parts = [](int64_t grid, int64_t tiles) {
    int64_t n = grid > 0 ? kCUs / grid : 1;
    if (n > tiles / 4) n = tiles / 4;
    return (int)(n > 1 ? n : 1);
  };
  const int64_t G = Hq / Hk;
  *q_parts = parts(B * Hk * ((G * Sq + 127) / 128), (Sk + 63) / 64);
  *k_parts = parts(B * Hk * ((Sk + 127) / 128), G * ((Sq + 63) / 64));
}

hipError_t launch_cross_backward(const CrossBwdParams& p, CrossBwdPass pass, hipStream_t s) {
  const int64_t nbh = (int64_t)p.B * p.Hk;
  if (pass == CROSS_DQ) {
    const int64_t nqb = ((int64_t)p.G * p.Sq + 127) / 128;
    hipLaunchKernelGGL(cross_bwd_dq_kernel, dim3((unsigned)(nqb * nbh * p.q_parts)), dim3(NT), 0, s, p);
  } else {
    const dim3 grid((unsigned)((p.Sk + 127) / 128 * nbh * p.k_parts));
    if (pass == CROSS_DV)
      hipLaunchKernelGGL(cross_bwd_dkv_kernel<1>, grid, dim3(NT), 0, s, p);
    else
      hipLaunchKernelGGL(cross_bwd_dkv_kernel<2>, grid, dim3(NT), 0, s, p);
  }
  return hipGetLastError();
}

}  // namespace partir
