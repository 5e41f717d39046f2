// Masked attention, forward: O = softmax(z) V over the keys that a query sees,
//   z = cap tanh(scale q k / cap) - slope_h |p - j|   (cap and slopes as given)
// for query position p and key j; attention_mask.h says which keys those are.  The
// kernel is that of attention to another sequence (cross_attention_kernel.h) in its
// masked forms: a workgroup takes the keys from the first to the last block that a
// row of it may see, a wave passes blocks that none of its rows sees, and only
// blocks across a limit or a border of documents compare keys one by one.
#include <algorithm>

#include "cross_attention_kernel.h"

namespace partir {
namespace {

// The joined parts of a row, as cross_combine_kernel; every part of a row has its
// statistics, and one without a key that the row sees weighs nothing.
__global__ __launch_bounds__(256) void masked_combine_kernel(MaskedParams p) {
  __shared__ f32x4 acc_s[8][32];
  __shared__ float l_s[8];
  const int64_t row = blockIdx.x, rows = (int64_t)p.B * p.Sq * p.Hq;
  const int grp = threadIdx.x >> 5, c4 = threadIdx.x & 31;
  const int64_t tq = row / p.Hq;
  const int head = (int)(row - tq * p.Hq);
  float M = kNoMax;
  for (int s = c4; s < p.nsplit; s += 32) M = fmaxf(M, p.MLpart[s * rows + row].x);
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) M = fmaxf(M, __shfl_xor(M, o));
  float L = 0.0f;
  f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
  for (int s = grp; s < p.nsplit; s += 8) {
    const float2 ml = p.MLpart[s * rows + row];
    const float f = ml.y != 0.0f ? __builtin_amdgcn_exp2f(ml.x - M) : 0.0f;
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
  const bool seen = L != 0.0f;
  if (p.lse && c4 == 0) p.lse[row] = seen ? M + __builtin_amdgcn_logf(L) : -__builtin_inff();
  const float inv = seen ? 1.0f / L : 0.0f;
  *(bf16x4*)(p.O + tq * p.ldo + head * DH + 4 * c4) =
      bf16x4{(__bf16)(acc[0] * inv), (__bf16)(acc[1] * inv), (__bf16)(acc[2] * inv), (__bf16)(acc[3] * inv)};
}

// The least and largest document of every 64 valid positions of a sequence: a wave
// a block.  A block without valid positions meets none.
__global__ __launch_bounds__(256) void doc_table_kernel(DocTables t) {
  const int which = blockIdx.y, lane = threadIdx.x & 63;
  const int64_t n = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int blocks = t.blocks[which];
  if (n >= (int64_t)t.B * blocks) return;
  const int b = (int)(n / blocks), s = (int)(n - (int64_t)b * blocks) * 64 + lane;
  int lo = 2147483647, hi = -2147483647 - 1;
  if (s < clamp_len(t.lens[which], b, t.S[which])) lo = hi = t.docs[which][(int64_t)b * t.S[which] + s];
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    lo = min(lo, __shfl_xor(lo, o));
    hi = max(hi, __shfl_xor(hi, o));
  }
  if (lane == 0) t.table[which][n] = make_int2(lo, hi);
}

template <int F>
void launch_form(const MaskedParams& p, const CrossChoice& c, hipStream_t s) {
  const int64_t rows = (int64_t)p.G * p.Sq, nqb = (rows + 32 * c.qw - 1) / (32 * c.qw);
  const dim3 grid((unsigned)(nqb * p.B * p.Hk * p.nsplit));
  if (c.qw == 1)
    hipLaunchKernelGGL((cross_attention_kernel<1, 4, 32, 2, 1, F>), grid, dim3(256), 0, s, p);
  else if (c.kg == 2)
    hipLaunchKernelGGL((cross_attention_kernel<4, 2, 64, 2, 2, F>), grid, dim3(512), 0, s, p);
  else
    hipLaunchKernelGGL((cross_attention_kernel<4, 1, 32, 3, 3, F>), grid, dim3(256), 0, s, p);
}

}  // namespace

hipError_t launch_masked_attention(const MaskedParams& p, int form, const CrossChoice& c, hipStream_t s) {
  switch (form & (kCap | kBias)) {
    case 0: launch_form<kMasked>(p, c, s); break;
    case kCap: launch_form<kMasked | kCap>(p, c, s); break;
    case kBias: launch_form<kMasked | kBias>(p, c, s); break;
    default: launch_form<kMasked | kCap | kBias>(p, c, s);
  }
  return hipGetLastError();
}

hipError_t launch_masked_combine(const MaskedParams& p, hipStream_t s) {
  const int64_t rows = (int64_t)p.B * p.Sq * p.Hq;
  hipLaunchKernelGGL(masked_combine_kernel, dim3((unsigned)rows), dim3(256), 0, s, p);
  return hipGetLastError();
}

hipError_t launch_doc_tables(const DocTables& t, hipStream_t s) {
  const int64_t most = (int64_t)t.B * std::max(t.blocks[0], t.blocks[1]);
  hipLaunchKernelGGL(doc_table_kernel, dim3((unsigned)((most + 3) / 4), 2), dim3(256), 0, s, t);
  return hipGetLastError();
}

}  // namespace partir
