// Launch interface between operators_api.cpp and the kernels of the operators
// around the loop nests: rotary positions and per-head norms, cross attention,
// the global norm of gradients.  Plain structs passed by value.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace partir {

// Division of 0 <= n < 2^31 by a divisor that the host knows: a high product,
// an addition and a shift (with L = ceil(log2 d) and m = floor(2^32 (2^L - d) /
// d) + 1, n / d = (hi32(m n) + n) >> L), where the compiler's division by a
// variable is some 30 dependent instructions before a kernel's first load.
struct Div {
  uint32_t m, l, d;
  static Div by(uint32_t d) {
    uint32_t l = 0;
    while (((uint64_t)1 << l) < d) ++l;
    return Div{(uint32_t)((((uint64_t)1 << 32) * (((uint64_t)1 << l) - d)) / d + 1), l, d};
  }
  __device__ __forceinline__ int quot(int n) const {
    return (int)((__umulhi(m, (uint32_t)n) + (uint32_t)n) >> l);
  }
  __device__ __forceinline__ int rem(int n, int q) const { return n - q * (int)d; }
};

// ---- rotary positions, alone or after a norm of each head (rotary.hip) ------
// Index 0 is the queries, 1 the keys; a tensor without heads is not read.
struct RotaryParams {
  const void* x[2];        // [T, H[i] dh], bf16 or f32, leading dim ldx[i]
  const void* dy[2];       // backward: cotangents of the outputs
  void* y[2];              // output (backward: gradient of x)
  const float* g[2];       // gains [dh] of the norm, or NULL: 1
  float* dgpart;           // backward: [parts][2][dh] partial gain gradients
  const double* freqs;     // [rd / 2] radians per position
  const void* pos;         // [T] positions, or NULL: row t stands at t mod S
  int64_t ldx[2], lddy[2], ldy[2];
  int64_t T, S;
  int H[2];
  Div by_s, by_half, by_h, by_hw[2];   // S, rd / 2, H[0] + H[1], each H (1 for 0)
  int dh, rd;
  int pos64;               // positions are int64 (else int32)
  int vec;                 // values of a load (8, 4, 2, 1): 2 vec divides rd and dh
  int tb;                  // tokens of a block
  int64_t blocks;          // blocks of tb tokens; workgroup w takes w, w + grid, ...
  int grid;
  float magnitude;         // factor of the rotated part
  float sign;              // 1, or -1 for the transposed rotation
  float eps;
};
// The token block, load width and grid of a call (host rule; the pointers are
// not looked at).  Sets vec, tb, blocks, grid and the divisors.
enum RotaryPass { ROTARY, ROTARY_NORM, ROTARY_NORM_BWD };
void rotary_choice(RotaryParams& p, bool bf16, RotaryPass pass);
hipError_t launch_rotary(const RotaryParams& p, bool bf16, bool interleaved, bool norm, hipStream_t s);
// Gradients of the norm and rotation together; gain gradients as partials.
hipError_t launch_qk_norm_backward(const RotaryParams& p, bool bf16, bool interleaved, hipStream_t s);
// dg[i][d] = sum over the parts, in order (a NULL dg[i] is skipped)
hipError_t launch_gain_reduce(const float* dgpart, int parts, int dh, float* dgq, float* dgk, hipStream_t s);

// ---- attention to another sequence (cross_attention.hip) --------------------
// d_head = 128, bf16.  Query head h reads key head h / G, G = Hq / Hk.  The
// G Sq query rows of a (sequence, key head) are numbered i = s G + g (position
// s, head kvh G + g) and tiled together, so that a single token's shared heads
// fill one tile.
struct CrossParams {
  const uint16_t* Q;
  const uint16_t* K;
  const uint16_t* V;
  uint16_t* O;
  float* lse;              // [B Sq][Hq] base-2 log-sum-exp of the scaled scores, or NULL
  const int32_t* lens;     // [B] valid keys of each sequence, or NULL: Sk
  int64_t ldq, ldk, ldv, ldo;
  int B, Sq, Sk, Hq, Hk, G;
  Div by_g, by_hk, by_nbh, by_nqb, by_split;   // G, Hk, B Hk, the row blocks of a (sequence, key head), nsplit
  float scale_log2;        // scale * log2(e)
  // key axis in nsplit parts (see cross_range): unnormalised outputs and
  // softmax statistics of the parts, joined by the combine launch
  int nsplit;
  float* Opart;            // [nsplit][B Sq Hq][128]
  float2* MLpart;          // [nsplit][B Sq Hq] (m, l)
};
// The kernel of a launch: waves over queries and key groups of a workgroup,
// keys of a block, parts of the key axis.
struct CrossChoice {
  int qw, kg, block, nsplit;
};
CrossChoice cross_choice(int64_t B, int64_t Sq, int64_t Sk, int64_t Hq, int64_t Hk);
hipError_t launch_cross_attention(const CrossParams& p, const CrossChoice& c, hipStream_t s);
hipError_t launch_cross_combine(const CrossParams& p, hipStream_t s);

// The count of parts, up to `most`, that takes the least time: n parts leave a
// workgroup steps / n steps of step_us, and from two on cost a launch that joins
// them (about 5 us) and part_us each, their float32 rows written and read.
inline int best_parts(int64_t most, int64_t steps, double step_us, double part_us) {
  int best = 1;
  double least = (double)steps * step_us;
  for (int64_t n = 2; n <= most;) {
    const double us = (double)((steps + n - 1) / n) * step_us + 5.0 + (double)n * part_us;
    if (us < least) {
      least = us;
      best = (int)n;
    }
    n = n < most && 2 * n > most ? most : 2 * n;   // powers of two, and the most
  }
  return best;
}

// Keys of part `split` of nsplit of a sequence with len keys: whole blocks of
// 64, shared out evenly; parts behind the last block are empty.
struct CrossRange {
  int begin, end, parts;   // [begin, end), and how many parts hold keys
};
__device__ __forceinline__ CrossRange cross_range(int len, const Div& by_split, int split) {
  const int nblk = (len + 63) / 64;
  if (by_split.d == 1) return CrossRange{0, len, nblk > 0};
  const int per = by_split.quot(nblk + (int)by_split.d - 1);
  CrossRange r;
  r.parts = per ? (nblk + per - 1) / per : 0;
  const long long b = (long long)split * per * 64, e = b + (long long)per * 64;
  r.begin = (int)(b < len ? b : len);
  r.end = (int)(e < len ? e : len);
  return r;
}

// Gradients (cross_attention_bwd.hip).  Up to 128 keys a sequence: one pass.
// Above: a dq pass, which takes the key axis in q_parts parts, and one for dk and
// dv.  A pass that yields dk and dv takes the query rows in k_parts; more than
// one part means fp32 partials for an ordered reduction.
struct CrossBwdParams {
  const uint16_t *Q, *K, *V, *O, *dO;
  const float* lse;
  float* Dstat;            // [B Sq][Hq] rowsums of dO * O, from the dq pass for the other
  uint16_t *dQ, *dK, *dV;
  float *dQpart, *dKpart, *dVpart;   // [parts][rows][heads * 128]
  const int32_t* lens;
  int64_t ldq, ldk, ldv, ldo, ldg, lddq, lddk, lddv;
  int B, Sq, Sk, Hq, Hk, G;
  int q_parts, k_parts;
  // G, Hk, B Hk, the 128-row blocks of a (sequence, key head), the counts of parts
  Div by_g, by_hk, by_nbh, by_nqb, by_q_parts, by_k_parts;
  float scale, scale_log2;
};
struct CrossBwdChoice {
  bool one_pass;
  int q_parts, k_parts;
};
CrossBwdChoice cross_bwd_choice(int64_t B, int64_t Sq, int64_t Sk, int64_t Hq, int64_t Hk);
enum CrossBwdPass { CROSS_ALL, CROSS_DQ, CROSS_DKV };
hipError_t launch_cross_backward(const CrossBwdParams& p, CrossBwdPass pass, hipStream_t s);
// Sums of parts of up to two matrices [rows, cols] with as many columns: out
// (bf16, leading dim ld) = sum over the parts, in order.
struct PartSum {
  const float* part[2];
  uint16_t* out[2];
  int64_t ld[2];
  int64_t rows;
  int cols, parts, n;      // n matrices
  Div by_cols4;            // cols / 4
};
hipError_t launch_part_sum(const PartSum& p, hipStream_t s);

// ---- global norm of many tensors (grad_norm.hip) ----------------------------
constexpr int kGradTensors = 144;             // tensors of one launch's table, which fills 4 KiB of arguments
constexpr int kGradChunkBytes = 32768;        // bytes of one step of a workgroup
constexpr int kGradMaxWorkgroups = 2048;
constexpr int kGradDirect = 2048;             // partial sums that a launch adds as they are
constexpr int kGradFolded = 256;              // more of them are added to these first
struct GradTable {
  const void* in[kGradTensors];
  void* out[kGradTensors];
  uint64_t size[kGradTensors];                // elements, kGradBf16 added for bf16 (else float32)
  uint32_t chunk0[kGradTensors + 1];          // first chunk of each tensor; [n] = all (at most 2^31)
  int n;
};
constexpr uint64_t kGradBf16 = (uint64_t)1 << 63;
static_assert(sizeof(GradTable) + 32 <= 4096, "with the other arguments of a launch");
// partial[w] = sum of squares of workgroup w's chunks
hipError_t launch_grad_sumsq(const GradTable& t, double* partial, int workgroups, hipStream_t s);
// folded[w] = the sum of run w of kGradFolded even runs of partial[0..n)
hipError_t launch_grad_fold(const double* partial, int n, double* folded, hipStream_t s);
// norm = sqrt(sum of partial[0..n))
hipError_t launch_grad_norm(const double* partial, int n, float* norm, hipStream_t s);
// out = in * (norm > max_norm ? max_norm / norm : 1) with the norm of the
// partials, which is also stored where `norm` is not NULL
hipError_t launch_grad_scale(const GradTable& t, const double* partial, int n, double max_norm, float* norm,
                             int workgroups, hipStream_t s);

}  // namespace partir
