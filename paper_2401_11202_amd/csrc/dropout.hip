// Dropout from a counter-based generator, alone or on top of a residual:
//   y = r + (kept ? x * 65536 / kept_of_65536 : 0)
// with the mask of philox.h, which is never stored; its transpose is itself, so
// the gradient of x is this kernel on the cotangent of y.
//
// A lane takes eight columns of a row at a time, one counter; a workgroup takes
// PER runs of 256 such groups of the matrix in row-major order.  What is dropped
// is 0 whatever x holds there.
//
// What bounds it: HBM, with the generator's products close behind (the vector units
// are busy for 66 % of the time).  8192 x 13824 in bf16 (453 MB): 81 us, 5.6 TB/s; 77 x
// 512 on a float32 residual: 4.2 us, a launch.
#include <type_traits>

#include "operators.h"
#include "runs.h"

namespace partir {
namespace {

constexpr int NT = 256;
constexpr int PER = 4;

template <typename TX, typename TY>
__global__ __launch_bounds__(NT) void dropout_kernel(DropoutParams p) {
  Philox rng;
  rng.init(p.drop.seed);
  // the workgroup's first group of eight columns; rows below it by a 32-bit division
  const int64_t g0 = (int64_t)blockIdx.x * (NT * PER);
  const int64_t row0 = g0 / p.cols8;
  const int in0 = (int)(g0 - row0 * p.cols8);
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const int i = in0 + u * NT + (int)threadIdx.x, dr = p.by_cols8.quot(i), c8 = p.by_cols8.rem(i, dr);
    const int64_t row = row0 + dr;
    if (row >= p.T) return;
    const TX* x = (const TX*)p.x + row * p.ldx + 8 * c8;
    const TY* r = p.r ? (const TY*)p.r + row * p.ldr + 8 * c8 : nullptr;
    TY* y = (TY*)p.y + row * p.ldy + 8 * c8;
    const uint32_t keep = rng.keep8(c8, p.drop.row0 + (uint32_t)row, p.drop.kept);
    const int left = p.D - 8 * c8;
    float v[8], b[8];
    if (left >= 8) {
      Run<TX, 8>::load(x, v);
      if (r) Run<TY, 8>::load(r, b);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v[e] = e < left ? (float)x[e] : 0.0f;
        b[e] = r && e < left ? (float)r[e] : 0.0f;
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[e] = keep >> e & 1 ? v[e] * p.drop.factor : 0.0f;
      if (r) v[e] += b[e];
    }
    if (left >= 8) {
      Run<TY, 8>::store(y, v);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < left) y[e] = (TY)v[e];
    }
  }
}

}  // namespace

hipError_t launch_dropout(const DropoutParams& p, bool x_bf16, bool y_bf16, hipStream_t s) {
  const int64_t groups = p.T * p.cols8;
  const dim3 grid((unsigned)((groups + NT * PER - 1) / (NT * PER)));
  auto go = [&](auto x, auto y) {
    hipLaunchKernelGGL((dropout_kernel<decltype(x), decltype(y)>), grid, dim3(NT), 0, s, p);
  };
  if (x_bf16)
    y_bf16 ? go(__bf16(), __bf16()) : go(__bf16(), float());
  else
    y_bf16 ? go(float(), __bf16()) : go(float(), float());
  return hipGetLastError();
}

}  // namespace partir
