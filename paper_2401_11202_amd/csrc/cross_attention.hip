// Attention to another sequence, forward: O = softmax(scale Q K^T) V over the
// first len_b keys of each sequence, d_head = 128, bf16 in and out, any number
// of queries and keys, key heads shared by G query heads.  The kernel and how it
// computes: cross_attention_kernel.h.
//
// Keys at and behind len_b are never read: their tile rows are zeros (the
// descriptor ends before them), so what the padding holds, NaN included, does
// not reach a product, and their scores are -inf.  A sequence without keys
// gives 0 and a log-sum-exp of -inf.
//
// What bounds it.  Many rows: the matrix units, and exp2 and the conversions of
// a score, which take about as long (16 cycles of the first, 4 a value elsewhere)
// and lie behind one another's time only in part, with three waves a SIMD: busy
// 57 and 45 % of the time, they still add up to all of it.  4 x 4096 queries over up to 2048 keys, 32 / 8 heads (0.44 TFLOP): 430 us, 1.02
// PFLOP/s.  With 64-key blocks and two stages (two waves a SIMD) 452, with two key
// groups 456.  Few rows: the reading of K and V; 131072 keys of 8 key heads (537
// MB): 93 us, 5.8 TB/s, and 5 for the join; 32 sequences of up to 1501 keys (109
// MB): 27 us.
#include <algorithm>

#include "cross_attention_kernel.h"

namespace partir {
namespace {

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
  const int parts = cross_range(clamp_len(p.lens, b, p.Sk), p.by_split, 0).parts;
  float M = kNoMax;
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
  // The key axis in parts where workgroups are few.  A workgroup takes 0.33 us for
  // 64 keys of a tile of 32 rows and 0.77 us of one of 128 (measured at 8 to 64
  // workgroups); 1000 rows of a part cost 0.2 us.  Unsplit / split so: 1 query, 32/8
  // heads, 4096 keys 27 / 15 us, 1024 keys 10.5 / 14.5; 512 queries, 4 heads, 2048
  // keys 32 / 18; 1024 queries, 8 heads, 1024 keys 21 / 25.  Above 64 parts joining
  // them costs more than it saves (one key head, 65536 keys: 16 us with 64, 19
  // with 256).
  const int64_t most = grid > 0 ? std::min<int64_t>(std::min(kCUs / grid, blocks), 64) : 1;
  c.nsplit = best_parts(most, blocks, c.qw == 1 ? 0.33 : 0.77, 2e-4 * (double)(B * Sq * Hq));
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
    hipLaunchKernelGGL((cross_attention_kernel<1, 4, 32, 2, 1, 0>), grid, dim3(256), 0, s, p);
  else if (c.kg == 2)
    hipLaunchKernelGGL((cross_attention_kernel<4, 2, 64, 2, 2, 0>), grid, dim3(512), 0, s, p);
  else
    hipLaunchKernelGGL((cross_attention_kernel<4, 1, 32, 3, 3, 0>), grid, dim3(256), 0, s, p);
  return hipGetLastError();
}

hipError_t launch_cross_combine(const CrossParams& p, hipStream_t s) {
  const int64_t rows = (int64_t)p.B * p.Sq * p.Hq;
  hipLaunchKernelGGL(cross_combine_kernel, dim3((unsigned)rows), dim3(256), 0, s, p);
  return hipGetLastError();
}

}  // namespace partir
