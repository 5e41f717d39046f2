// Launch interface between operators_api.cpp and the kernels of the operators
// around the loop nests: rotary positions and per-head norms, cross attention,
// the global norm of gradients.  Plain structs passed by value.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace partir {

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
// not looked at).  Sets vec, tb, blocks and grid.
void rotary_choice(RotaryParams& p, bool bf16, bool backward);
constexpr int kRotaryMaxGrid = 2048, kRotaryMaxBwdGrid = 1024;
hipError_t launch_rotary(const RotaryParams& p, bool bf16, bool interleaved, bool norm, hipStream_t s);
// Gradients of the norm and rotation together; gain gradients as partials.
hipError_t launch_qk_norm_backward(const RotaryParams& p, bool bf16, bool interleaved, hipStream_t s);
// dg[i][d] = sum over the parts, in order (a NULL dg[i] is skipped)
hipError_t launch_gain_reduce(const float* dgpart, int parts, int dh, float* dgq, float* dgk, hipStream_t s);

// ---- global norm of many tensors (grad_norm.hip) ----------------------------
constexpr int kGradTensors = 112;             // tensors of one launch's table
constexpr int kGradChunkBytes = 32768;        // bytes of one step of a workgroup
constexpr int kGradMaxWorkgroups = 2048;
struct GradTable {
  const void* in[kGradTensors];
  void* out[kGradTensors];
  int64_t numel[kGradTensors];
  int64_t chunk0[kGradTensors + 1];           // first chunk of each tensor; [n] = all
  uint8_t bf16[kGradTensors];
  int n;
};
// partial[w] = sum of squares of workgroup w's chunks
hipError_t launch_grad_sumsq(const GradTable& t, double* partial, int workgroups, hipStream_t s);
// norm = sqrt(sum of partial[0..n))
hipError_t launch_grad_norm(const double* partial, int n, float* norm, hipStream_t s);
// out = in * (norm > max_norm ? max_norm / norm : 1) with the norm of the
// partials, which is also stored where `norm` is not NULL
hipError_t launch_grad_scale(const GradTable& t, const double* partial, int n, double max_norm, float* norm,
                             int workgroups, hipStream_t s);

}  // namespace partir
