// Attention to another sequence, forward: O = softmax(scale Q K^T) V over the
// first len_b keys of each sequence, d_head = 128, bf16 in and out, any number
// of queries and keys, key heads shared by G query heads.
//
// A workgroup takes 32 QW rows of the G Sq query rows of one (sequence, key
// head); its QW x KG waves hold 32 rows each, and the KG key groups take every
// KG-th block of BKV keys through double-buffered LDS stages of their own.  A
// wave computes
//     S^T[BKV keys x 32 rows] = K_blk Q^T      (v_mfma_f32_32x32x16_bf16)
// so that a lane owns one row: maximum and sum of the running softmax are lane
// registers, and exp2(S^T - m), rounded to bf16 (within 2^-8 of its value, as
// the weights of partir_attention), is the B operand of
//     O^T[128 x 32 rows] += V_blk^T P^T
// with V^T from transposed LDS reads.  Sums and O are float32; groups and key
// parts join by (m, l, O) (+) (m', l', O'), in a fixed order.
//
// Keys at and behind len_b are never read: their tile rows are zeros (the
// descriptor ends before them), so what the padding holds, NaN included, does
// not reach a product, and their scores are -inf.  A sequence without keys
// gives 0 and a log-sum-exp of -inf.
#include <type_traits>

#include "attention_tiles.h"
#include "operators.h"

namespace partir {
namespace {

__device__ __forceinline__ int key_count(const CrossParams& p, int b) {
  return p.lens ? min(max(p.lens[b], 0), p.Sk) : p.Sk;
}

template <int QW, int KG, int BKV>
__global__ __launch_bounds__(64 * QW * KG) void cross_attention_kernel(CrossParams p) {
  constexpr int NSUB = BKV / 32;
  constexpr int T_BYTES = BKV * ROWB, STAGE = 2 * T_BYTES;      // K tile, then V tile
  constexpr int MERGE = (KG - 1) * QW * 64 * 66 * 4;            // O, m and l of the other key groups
  constexpr int LDS = KG * 2 * STAGE > MERGE ? KG * 2 * STAGE : MERGE;
  __shared__ __attribute__((aligned(1024))) char smem[LDS];

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int w = wave % QW, kg = wave / QW;
  const int h = lane >> 5, col = lane & 31;

  const int R = p.G * p.Sq, nqb = (R + 32 * QW - 1) / (32 * QW), nbh = p.B * p.Hk;
  int qb, bh, split;
  if (p.nsplit == 1 && (nbh & 7) == 0) {
    // Workgroup i runs on XCD i mod 8: an XCD takes one (sequence, key head)
    // after the other, whose K and V stay in its L2.
    const int j = blockIdx.x >> 3;
    const int n = j / nqb;
    bh = n * 8 + (blockIdx.x & 7);
    qb = j - n * nqb;
    split = 0;
  } else {
    bh = blockIdx.x % nbh;
    const int r = blockIdx.x / nbh;
    split = r % p.nsplit;
    qb = r / p.nsplit;
  }
  const int b = bh / p.Hk, kvh = bh - b * p.Hk;
  const CrossRange range = cross_range(key_count(p, b), p.nsplit, split);
  if (p.nsplit > 1 && split >= range.parts) return;   // the combine does not read it

  // this lane's row: queries (B operand of S^T) in registers
  const int i = qb * 32 * QW + 32 * w + col;
  const int ic = min(i, R - 1), sq = ic / p.G;
  const int64_t tq = (int64_t)b * p.Sq + sq;
  const int head = kvh * p.G + ic - sq * p.G;
  bf16x8 qf[8];
  {
    const uint16_t* qrow = p.Q + tq * p.ldq + head * DH + 8 * h;
#pragma unroll
    for (int ds = 0; ds < 8; ++ds) qf[ds] = *(const bf16x8*)(qrow + 16 * ds);
  }

  const uint16_t* kbase = p.K + (int64_t)b * p.Sk * p.ldk + kvh * DH;
  const uint16_t* vbase = p.V + (int64_t)b * p.Sk * p.ldv + kvh * DH;
  char* const stages = smem + kg * 2 * STAGE;
  // key block kb of the part; the addresses are 64-bit, so a part may hold any
  // number of bytes
  auto gload = [&](int kb, int buf) {
    const int64_t k0 = range.begin + (int64_t)kb * BKV;
    const int rows = (int)min((int64_t)BKV, range.end - k0);
    tile_load<BKV, QW>(kbase + k0 * p.ldk, p.ldk, rows, stages + buf * STAGE, w, lane);
    tile_load<BKV, QW>(vbase + k0 * p.ldv, p.ldv, rows, stages + buf * STAGE + T_BYTES, w, lane);
  };

  f32x16 oacc[4];
#pragma unroll
  for (int d = 0; d < 4; ++d) zero(oacc[d]);
  float m_run = -1e30f, l_run = 0.0f;
  TileTr tr;
  tr.init(lane);
  const int nkb = (range.end - range.begin + BKV - 1) / BKV;
  const float sl2 = p.scale_log2;

  if (kg < nkb) gload(kg, 0);
  WAIT_VMCNT(0);
  __syncthreads();
  // Two blocks a trip, so that a block's stage is a constant and folds into
  // the reads' offsets.
  auto block = [&](auto stage_c, int kb) {
    constexpr int cur = decltype(stage_c)::value;
    if (kb + KG < nkb) gload(kb + KG, cur ^ 1);
    if (KG == 1 || kb < nkb) {
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
      const int left = range.end - (range.begin + kb * BKV);   // keys from this block on
      if (left < BKV) {
#pragma unroll
        for (int t = 0; t < NSUB; ++t)
#pragma unroll
          for (int v = 0; v < 16; ++v)
            if (32 * t + 8 * (v >> 2) + 4 * h + (v & 3) >= left) sacc[t][v] = -__builtin_inff();
      }
      float lsum = 0.0f;
      bf16x8 pf[2 * NSUB];
      auto weights = [&]() {
        lsum = 0.0f;
#pragma unroll
        for (int t = 0; t < NSUB; ++t)
#pragma unroll
          for (int v = 0; v < 16; ++v) {
            const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[t][v], sl2, -m_run));
            lsum += e;
            pf[2 * t + (v >> 3)][v & 7] = (__bf16)e;
          }
      };
      // m moves only where the block's maximum is more than 8 (log2 units)
      // above it: weights stay below 2^8, exact range in float32 and bf16, and
      // O is rescaled in few blocks.  A lane whose weights sum to at most 2^8
      // has none above, so the maximum is taken only where some lane's sum is
      // larger (or inf / NaN, as on the first block, where m is -1e30).
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
#pragma unroll
      for (int u = 0; u < BKV / 16; ++u)
#pragma unroll
        for (int d = 0; d < 4; ++d) oacc[d] = mfma(tr.read(vs, u, d), pf[u], oacc[d]);
    }
    WAIT_VMCNT(0);   // this wave's loads of the next tiles have landed
    __syncthreads();
  };
  // every barrier is the workgroup's: the trip count does not depend on the group
  for (int kb = 0; kb < nkb; kb += 2 * KG) {
    block(std::integral_constant<int, 0>{}, kb + kg);
    if (kb + KG < nkb) block(std::integral_constant<int, 1>{}, kb + KG + kg);
  }

  float l_tot = l_run + __shfl_xor(l_run, 32);
  if constexpr (KG > 1) {
    // the groups' (m, l, O) into group 0's, in order; the stages are free (the
    // loop ended on a barrier with no load in flight)
    constexpr int PER = QW * 64;
    auto area = [&](int g) { return smem + (g - 1) * PER * 66 * 4; };
    if (kg > 0) {
      f32x4* mo = (f32x4*)area(kg) + (w * 64 + lane);
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          mo[(4 * d + g) * PER] = f32x4{oacc[d][4 * g + 0], oacc[d][4 * g + 1], oacc[d][4 * g + 2], oacc[d][4 * g + 3]};
      ((float2*)(area(kg) + PER * 64 * 4))[w * 64 + lane] = make_float2(m_run, l_tot);
    }
    __syncthreads();
    if (kg > 0) return;
#pragma unroll
    for (int g2 = 1; g2 < KG; ++g2) {
      const f32x4* mo = (const f32x4*)area(g2) + (w * 64 + lane);
      const float2 o = ((const float2*)(area(g2) + PER * 64 * 4))[w * 64 + lane];
      const float m_new = fmaxf(m_run, o.x);   // a group without keys holds (-1e30, 0, 0)
      const float a0 = __builtin_amdgcn_exp2f(m_run - m_new), a1 = __builtin_amdgcn_exp2f(o.x - m_new);
      l_tot = a0 * l_tot + a1 * o.y;
      m_run = m_new;
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const f32x4 v = mo[(4 * d + g) * PER];
#pragma unroll
          for (int e = 0; e < 4; ++e) oacc[d][4 * g + e] = a0 * oacc[d][4 * g + e] + a1 * v[e];
        }
    }
  }
  if (i >= R) return;
  const int64_t row = tq * p.Hq + head;
  if (p.nsplit > 1) {
    const int64_t at = (int64_t)split * p.B * p.Sq * p.Hq + row;
    float* orow = p.Opart + at * DH;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *(f32x4*)(orow + 32 * d + 8 * g + 4 * h) =
            f32x4{oacc[d][4 * g + 0], oacc[d][4 * g + 1], oacc[d][4 * g + 2], oacc[d][4 * g + 3]};
    if (h == 0) p.MLpart[at] = make_float2(m_run, l_tot);
    return;
  }
  if (p.lse && h == 0) p.lse[row] = nkb > 0 ? m_run + __builtin_amdgcn_logf(l_tot) : -__builtin_inff();
  const float inv = nkb > 0 ? 1.0f / l_tot : 0.0f;
  uint16_t* orow = p.O + tq * p.ldo + head * DH;
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *(bf16x4*)(orow + 32 * d + 8 * g + 4 * h) =
          bf16x4{(__bf16)(oacc[d][4 * g + 0] * inv), (__bf16)(oacc[d][4 * g + 1] * inv),
                 (__bf16)(oacc[d][4 * g + 2] * inv), (__bf16)(oacc[d][4 * g + 3] * inv)};
}

// O = sum_s w_s o_s / sum_s w_s l_s, w_s = 2^(m_s - M), M = max m_s.  A row of
// 128 takes 32 threads, 4 columns each, in each of 8 groups that share the
// parts (s = group, group + 8, ..); the groups are added in order.  The parts'
// rows are read once, all groups' loads in flight together: 32 parts of 32 rows
// 22 us with one group, 5 with eight.
__global__ __launch_bounds__(256) void cross_combine_kernel(CrossParams p) {
  __shared__ f32x4 acc_s[8][32];
  __shared__ float l_s[8];
  const int64_t row = blockIdx.x, rows = (int64_t)p.B * p.Sq * p.Hq;
  const int grp = threadIdx.x >> 5, c4 = threadIdx.x & 31;
  const int64_t tq = row / p.Hq;
  const int head = (int)(row - tq * p.Hq), b = (int)(tq / p.Sq);
  const int parts = cross_range(key_count(p, b), p.nsplit, 0).parts;
  float M = -3.0e38f;
  for (int s = c4; s < parts; s += 32) M = fmaxf(M, p.MLpart[s * rows + row].x);
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) M = fmaxf(M, __shfl_xor(M, o));
  float L = 0.0f;
  f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
  for (int s = grp; s < parts; s += 8) {
    const float2 ml = p.MLpart[s * rows + row];
    const float f = __builtin_amdgcn_exp2f(ml.x - M);
    L += f * ml.y;
    acc += f * *(const f32x4*)(p.Opart + (s * rows + row) * DH + 4 * c4);
  }
  acc_s[grp][c4] = acc;
  if (c4 == 0) l_s[grp] = L;
  __syncthreads();
  if (grp > 0) return;
#pragma unroll
  for (int g = 1; g < 8; ++g) {
    acc += acc_s[g][c4];
    L += l_s[g];
  }
  if (p.lse && c4 == 0) p.lse[row] = parts ? M + __builtin_amdgcn_logf(L) : -__builtin_inff();
  const float inv = parts ? 1.0f / L : 0.0f;
  *(bf16x4*)(p.O + tq * p.ldo + head * DH + 4 * c4) =
      bf16x4{(__bf16)(acc[0] * inv), (__bf16)(acc[1] * inv), (__bf16)(acc[2] * inv), (__bf16)(acc[3] * inv)};
}

constexpr int64_t kCUs = 256;   // compute units of an MI355X: plans do not need a GPU

}  // namespace

CrossChoice cross_choice(int64_t B, int64_t Sq, int64_t Sk, int64_t Hq, int64_t Hk) {
  const int64_t rows = Hq / Hk * Sq, blocks = (Sk + 63) / 64;
  CrossChoice c;
  c.qw = rows <= 32 ? 1 : 4;
  const int64_t grid = B * Hk * ((rows + 32 * c.qw - 1) / (32 * c.qw));
  c.nsplit = 1;
  if (grid < kCUs) {
    // the key axis in parts until there is a workgroup for every CU, none of
    // them shorter than 4 blocks of 64 keys
    int64_t n = kCUs / (grid > 0 ? grid : 1);
    if (n > blocks / 4) n = blocks / 4;
    if (n > 1) c.nsplit = (int)n;
  }
  if (c.qw == 1) {
    c.kg = 4;
    c.block = 32;
  } else if (grid * c.nsplit <= kCUs) {
    c.kg = 2;
    c.block = 64;
  } else {
    c.kg = 1;
    c.block = 32;
  }
  return c;
}

hipError_t launch_cross_attention(const CrossParams& p, const CrossChoice& c, hipStream_t s) {
  const int64_t rows = (int64_t)p.G * p.Sq, nqb = (rows + 32 * c.qw - 1) / (32 * c.qw);
  const dim3 grid((unsigned)(nqb * p.B * p.Hk * p.nsplit));
  if (c.qw == 1)
    hipLaunchKernelGGL((cross_attention_kernel<1, 4, 32>), grid, dim3(256), 0, s, p);
  else if (c.kg == 2)
    hipLaunchKernelGGL((cross_attention_kernel<4, 2, 64>), grid, dim3(512), 0, s, p);
  else
    hipLaunchKernelGGL((cross_attention_kernel<4, 1, 32>), grid, dim3(256), 0, s, p);
  return hipGetLastError();
}

hipError_t launch_cross_combine(const CrossParams& p, hipStream_t s) {
  const int64_t rows = (int64_t)p.B * p.Sq * p.Hq;
  hipLaunchKernelGGL(cross_combine_kernel, dim3((unsigned)rows), dim3(256), 0, s, p);
  return hipGetLastError();
}

}  // namespace partir
