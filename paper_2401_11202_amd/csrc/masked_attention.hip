// Masked attention, forward: O = softmax(z) V over the keys that a query sees,
//   z = cap tanh(scale q k / cap) - slope_h |p - j|   (cap and slopes as given)
// for query position p and key j; attention_mask.h says which keys those are.  The
// kernel is that of attention to another sequence (cross_attention_kernel.h) in its
// masked forms: a workgroup takes the keys from the first to the last block that a
// row of it may see, a wave passes blocks that none of its rows sees, and only
// blocks across an end of some row's interval compare keys one by one.
//
// What bounds it.  A token a sequence: reading K and V; 65537 keys of 16 heads, bias
// (537 MB): 98 us, 5.5 TB/s, and 4.6 for the join of the parts; 16 sequences of up to
// 4099 keys, 8 key heads, capped (161 MB): 39 to 41, ragged lengths on equal parts.  Many
// rows: without a cap or documents the times are those of attention to another
// sequence (2 x 4096 tokens, 32 / 8 heads, no mask: 505 and 501 us; causal, 0.27 TFLOP:
// 276, and 447 with a bias, whose six instructions a score are vector work too).  A cap
// costs vector work, with the matrix units' behind it in part only:
// 2 x 4096 tokens, 32 / 8 heads, causal (0.27 TFLOP): 355 to 377 us, vector units busy 66
// % of the time, matrix units 37; 509 queries over 8192 keys: 95, in 54 and 32 %, and
// 5.7 for the join.  Documents of 400 tokens on average, 4 x 2048, 32 heads: 94 us for
// 380 MB of which 268 are needed: a block's rows of K and V are read again by each of the
// row blocks that a document spans.
#include <algorithm>

#include "cross_attention_kernel.h"

namespace partir {
namespace {

// The joined parts of a row: O = sum_s w_s o_s / sum_s w_s l_s, w_s = 2^(m_s - M), M =
// max m_s; every part of a row has its statistics, and one without a key that the row
// sees weighs nothing.  A row of 128 takes 32 threads, 4 columns each, in each of GRP
// groups that share the parts (s = group, group + GRP, ..) and are added in order; 8 /
// GRP rows a workgroup.  With two parts the eight groups of a row would idle but two:
// 16288 rows 15 us so, 6 with one group a row.
template <int GRP>
__global__ __launch_bounds__(256) void masked_combine_kernel(MaskedParams p) {
  constexpr int ROWS = 8 / GRP;
  __shared__ f32x4 acc_s[8][32];
  __shared__ float l_s[8];
  const int64_t rows = (int64_t)p.B * p.Sq * p.Hq;
  const int slot = threadIdx.x >> 5, grp = slot % GRP, c4 = threadIdx.x & 31;
  const int64_t row = min((int64_t)blockIdx.x * ROWS + slot / GRP, rows - 1);   // the last one more than once
  const int64_t tq = row / p.Hq;
  const int head = (int)(row - tq * p.Hq);
  float M = kNoMax;
  for (int s = c4; s < p.nsplit; s += 32) M = fmaxf(M, p.MLpart[s * rows + row].x);
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) M = fmaxf(M, __shfl_xor(M, o));
  float L = 0.0f;
  f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
  for (int s = grp; s < p.nsplit; s += GRP) {
    const float2 ml = p.MLpart[s * rows + row];
    const float f = ml.y != 0.0f ? __builtin_amdgcn_exp2f(ml.x - M) : 0.0f;
    L += f * ml.y;
    acc += f * *(const f32x4*)(p.Opart + (s * rows + row) * DH + 4 * c4);
  }
  if constexpr (GRP > 1) {
    acc_s[slot][c4] = acc;
    if (c4 == 0) l_s[slot] = L;
    __syncthreads();
    if (grp > 0) return;
#pragma unroll
    for (int g = 1; g < GRP; ++g) {
      acc += acc_s[slot + g][c4];
      L += l_s[slot + g];
    }
  }
  const bool seen = L != 0.0f;
  if (p.lse && c4 == 0) p.lse[row] = seen ? M + __builtin_amdgcn_logf(L) : -__builtin_inff();
  const float inv = seen ? 1.0f / L : 0.0f;
  *(bf16x4*)(p.O + tq * p.ldo + head * DH + 4 * c4) =
      bf16x4{(__bf16)(acc[0] * inv), (__bf16)(acc[1] * inv), (__bf16)(acc[2] * inv), (__bf16)(acc[3] * inv)};
}

// The keys of every query's document.  A workgroup takes 1024 queries of a sequence:
// it lists the runs of equal numbers of the sequence's valid keys, and where no
// number has two runs, and there are at most kRuns, a query's keys are the run of
// its number.  The run at the query's own position is looked at first, which is the
// one where queries and keys are the same tokens.  4 x 2048 tokens of some five
// documents each: 5.5 us, a launch and a chain of loads and barriers.  Many documents:
// the comparison of every two runs, in each workgroup again.  1 x 8192 tokens: 9 us
// with 32 documents, 14 with 128, 34 with 512, 320 with 2048, 1270 with 4096.
constexpr int kRuns = 4096, kDocThreads = 1024;
__global__ __launch_bounds__(kDocThreads) void doc_rows_kernel(DocRows t) {
  __shared__ __attribute__((aligned(16))) int id[kRuns];
  __shared__ int first[kRuns + 1];
  __shared__ int wave_sum[17];
  __shared__ int in_pieces;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int chunks = (t.Sq + kDocThreads - 1) / kDocThreads;
  for (int64_t job = blockIdx.x; job < (int64_t)chunks * t.B; job += gridDim.x) {
    const int b = (int)(job / chunks), chunk = (int)(job - (int64_t)b * chunks);
    const int klen = clamp_len(t.k_lens, b, t.Sk), qlen = clamp_len(t.q_lens, b, t.Sq);
    const int32_t* kd = t.k_docs + (int64_t)b * t.Sk;
    // starts of runs among this thread's keys, and how many lie before them
    const int per = (klen + kDocThreads - 1) / kDocThreads;
    const int j0 = min(tid * per, klen), j1 = min(j0 + per, klen);
    int count = 0;
    for (int j = j0; j < j1; ++j) count += j == 0 || kd[j] != kd[j - 1];
    int before = count;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int x = __shfl_up(before, o);
      if (lane >= o) before += x;
    }
    if (lane == 63) wave_sum[wave] = before;
    if (tid == 0) in_pieces = 0;
    __syncthreads();
    int runs = 0, base = 0;
    for (int w = 0; w < kDocThreads / 64; ++w) {
      if (w == wave) base = runs;
      runs += wave_sum[w];
    }
    before += base - count;
    const bool listed = runs <= kRuns;   // the same in every thread
    if (listed) {
      for (int j = j0; j < j1; ++j)
        if (j == 0 || kd[j] != kd[j - 1]) {
          id[before] = kd[j];
          first[before++] = j;
        }
      if (tid == 0) first[runs] = klen;
      __syncthreads();
      for (int r = tid; r < runs; r += kDocThreads) {
        const int mine = id[r];
        bool twice = false;
        for (int k = 0; k < runs; ++k) twice |= id[k] == mine && k != r;
        if (twice) in_pieces = 1;
      }
    } else if (tid == 0) {
      in_pieces = 1;
    }
    __syncthreads();
    const bool by_id = in_pieces != 0;
    if (chunk == 0 && tid == 0) t.by_id[b] = by_id;
    const int s = chunk * kDocThreads + tid;
    int2 e = make_int2(0, 0);
    if (s < qlen) {
      if (by_id) {
        e = make_int2(0, klen);
      } else if (runs > 0) {
        const int mine = t.q_docs[(int64_t)b * t.Sq + s];
        int a = 0, z = runs;             // the run that holds position s, if any does
        while (z - a > 1) {
          const int mid = (a + z) >> 1;
          (first[mid] <= s ? a : z) = mid;
        }
        if (id[a] != mine)
          for (a = 0; a < runs && id[a] != mine; ++a) {}
        if (a < runs) e = make_int2(first[a], first[a + 1]);
      }
    }
    if (s < t.Sq) t.rows[(int64_t)b * t.Sq + s] = e;
    int lo = e.y > e.x ? e.x : kNowhere, hi = e.y;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
      lo = min(lo, __shfl_xor(lo, o));
      hi = max(hi, __shfl_xor(hi, o));
    }
    if (lane == 0 && s < t.Sq) t.blocks[(int64_t)b * t.q_blocks + (s >> 6)] = make_int2(lo, hi);
    __syncthreads();                   // the next sequence takes the same memory
  }
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
  if (p.nsplit <= 4)
    hipLaunchKernelGGL(masked_combine_kernel<1>, dim3((unsigned)((rows + 7) / 8)), dim3(256), 0, s, p);
  else
    hipLaunchKernelGGL(masked_combine_kernel<8>, dim3((unsigned)rows), dim3(256), 0, s, p);
  return hipGetLastError();
}

hipError_t launch_doc_rows(const DocRows& t, hipStream_t s) {
  const int64_t chunks = ((int64_t)t.Sq + kDocThreads - 1) / kDocThreads;
  const int64_t grid = std::min<int64_t>(chunks * t.B, 1 << 20);   // a launch is fewer than 2^32 threads
  hipLaunchKernelGGL(doc_rows_kernel, dim3((unsigned)grid), dim3(kDocThreads), 0, s, t);
  return hipGetLastError();
}

}  // namespace partir
