// The global norm of many tensors, N = sqrt(sum of x^2 over all of them), and
// their clipping to it: x <- x min(1, max_norm / N).
//
// Two passes over the tensors with the partial sums between them, each one
// launch for up to kGradTensors tensors: the table of the tensors travels in
// the kernel arguments, so nothing is uploaded and nothing kept.  A workgroup
// takes a run of consecutive 32 KiB chunks, 16 bytes a lane and load, eight
// loads in flight; chunks never cross a tensor.  Squares are summed in float64:
// float32 overflows from 2e19 on and loses the small tensors of a sum of 1e9
// terms; conversions and adds of float64 are well within what the load rate
// leaves.  The partial sums are added in a fixed order by every workgroup of the
// second pass for itself, which saves a launch between; more than kGradDirect of
// them are added to kGradFolded by a launch first.
//
// A tensor off a 16-byte boundary has every chunk start and end off one: single
// values there, and one load at a time between them.  Where input and output lie
// differently to the boundary, scaling goes by single values.  128 tensors of
// 2^20 values, replayed, norm / clipping apart: float32 108 / 335 us aligned, 143 /
// 412 at 8 bytes from the boundary, 114 / 498 with the output alone there; bf16 59 /
// 182, 66 / 213, 58 / 370.
//
// What bounds it is HBM: one read for the norm, one read and one write for the
// scaling, which is left out where nothing would change (in place, N <=
// max_norm).  493e6 float32 values: 370 us for the norm (5.3 TB/s), 758 for the
// scaling (5.2 TB/s), what a copy reaches.
#include "operators.h"

namespace partir {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
constexpr int NT = 256;

// the sum over the workgroup, in every thread
__device__ __forceinline__ double block_sum(double v, double* red) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = red[0];
#pragma unroll
  for (int w = 1; w < NT / 64; ++w) v += red[w];
  __syncthreads();
  return v;
}

// Elements before the first 16-byte boundary of p (at most n).
template <typename T>
__device__ __forceinline__ int head_of(const T* p, int n) {
  const int off = (int)((uintptr_t)p & 15);
  const int h = off ? (16 - off) / (int)sizeof(T) : 0;
  return h < n ? h : n;
}

__device__ __forceinline__ void add_sq(double& s, float v) { s = __builtin_fma((double)v, (double)v, s); }

template <typename T, typename VEC>
__device__ __forceinline__ double chunk_sumsq(const T* x, int n) {
  constexpr int E = 16 / sizeof(T);
  const int tid = threadIdx.x;
  double s0 = 0.0, s1 = 0.0;
  const int head = head_of(x, n);
  if (tid < head) add_sq(s0, (float)x[tid]);
  const int nv = (n - head) / E;
  const VEC* xv = (const VEC*)(x + head);
  const int done = head + nv * E;
  if (tid < n - done) add_sq(s1, (float)x[done + tid]);
  constexpr int U = kGradChunkBytes / 16 / NT;
  if (nv == U * NT) {   // a whole chunk: every load before the first sum
    VEC v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = xv[u * NT + tid];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < E; e += 2) {
        add_sq(s0, (float)v[u][e]);
        add_sq(s1, (float)v[u][e + 1]);
      }
  } else {
    for (int i = tid; i < nv; i += NT) {
      const VEC v = xv[i];
#pragma unroll
      for (int e = 0; e < E; e += 2) {
        add_sq(s0, (float)v[e]);
        add_sq(s1, (float)v[e + 1]);
      }
    }
  }
  return s0 + s1;
}

// x f with f in float64: a factor below float32's normal range keeps its
// bits, and float32 values take a single rounding.
template <typename T>
__device__ __forceinline__ T scaled(T x, double f) {
  return (T)(float)((double)(float)x * f);
}

template <typename T, typename VEC>
__device__ __forceinline__ void chunk_scale(const T* x, T* y, int n, double f) {
  constexpr int E = 16 / sizeof(T);
  const int tid = threadIdx.x;
  if (((uintptr_t)x ^ (uintptr_t)y) & 15) {   // no common alignment: one value at a time
    for (int i = tid; i < n; i += NT) y[i] = scaled(x[i], f);
    return;
  }
  const int head = head_of(x, n);
  if (tid < head) y[tid] = scaled(x[tid], f);
  const int nv = (n - head) / E;
  const VEC* xv = (const VEC*)(x + head);
  VEC* yv = (VEC*)(y + head);
  const int done = head + nv * E;
  if (tid < n - done) y[done + tid] = scaled(x[done + tid], f);
  constexpr int U = kGradChunkBytes / 16 / NT;
  if (nv == U * NT) {
    VEC v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = xv[u * NT + tid];
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int e = 0; e < E; ++e) v[u][e] = scaled((T)v[u][e], f);
      yv[u * NT + tid] = v[u];
    }
  } else {
    for (int i = tid; i < nv; i += NT) {
      VEC v = xv[i];
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = scaled((T)v[e], f);
      yv[i] = v;
    }
  }
}

// Calls f(tensor, whether it is bf16, first element, elements) for this
// workgroup's chunks.
template <typename F>
__device__ __forceinline__ void for_chunks(const GradTable& t, F f) {
  const int64_t all = t.chunk0[t.n];
  const int64_t c0 = all * blockIdx.x / gridDim.x, c1 = all * (blockIdx.x + 1) / gridDim.x;
  if (c0 >= c1) return;
  int lo = 0, hi = t.n - 1;   // the last tensor that starts at or before chunk c0
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.chunk0[mid] <= c0) lo = mid; else hi = mid - 1;
  }
  int64_t c = c0;
  while (c < c1) {
    const bool bf16 = (t.size[lo] & kGradBf16) != 0;
    const int64_t n = (int64_t)(t.size[lo] & ~kGradBf16), last = t.chunk0[lo + 1], first = t.chunk0[lo];
    const int64_t step = kGradChunkBytes / (bf16 ? 2 : 4);
    for (; c < c1 && c < last; ++c) {
      const int64_t at = (c - first) * step;
      f(lo, bf16, at, (int)(n - at < step ? n - at : step));
    }
    ++lo;
  }
}

__global__ __launch_bounds__(NT) void grad_sumsq_kernel(GradTable t, double* partial) {
  __shared__ double red[NT / 64];
  double s = 0.0;
  for_chunks(t, [&](int i, bool bf16, int64_t at, int n) {
    s += bf16 ? chunk_sumsq<__bf16, bf16x8>((const __bf16*)t.in[i] + at, n)
              : chunk_sumsq<float, f32x4>((const float*)t.in[i] + at, n);
  });
  s = block_sum(s, red);
  if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

// the sum of partial[i0 .. i1), in every thread
__device__ __forceinline__ double sum_of(const double* partial, int i0, int i1, double* red) {
  double s = 0.0;
  for (int i = i0 + (int)threadIdx.x; i < i1; i += NT) s += partial[i];
  return block_sum(s, red);
}

__device__ __forceinline__ double norm_of(const double* partial, int n, double* red) {
  return sqrt(sum_of(partial, 0, n, red));
}

__global__ __launch_bounds__(NT) void grad_fold_kernel(const double* partial, int n, double* folded) {
  __shared__ double red[NT / 64];
  const int i0 = (int)((int64_t)n * blockIdx.x / gridDim.x), i1 = (int)((int64_t)n * (blockIdx.x + 1) / gridDim.x);
  const double s = sum_of(partial, i0, i1, red);
  if (threadIdx.x == 0) folded[blockIdx.x] = s;
}

__global__ __launch_bounds__(NT) void grad_norm_kernel(const double* partial, int n, float* norm) {
  __shared__ double red[NT / 64];
  const double v = norm_of(partial, n, red);
  if (threadIdx.x == 0) *norm = (float)v;
}

__global__ __launch_bounds__(NT) void grad_scale_kernel(GradTable t, const double* partial, int n, double max_norm,
                                                        float* norm) {
  __shared__ double red[NT / 64];
  const double v = norm_of(partial, n, red);
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)v;
  // Elements are at most 2^128 and at most 2^44 of them: the norm is infinite or
  // NaN only where one of them is, and then scales nothing.
  const bool clip = v > max_norm && v <= 1.0e300;
  const double f = clip ? max_norm / v : 1.0;
  for_chunks(t, [&](int i, bool bf16, int64_t at, int m) {
    if (!clip && t.in[i] == t.out[i]) return;
    if (bf16)
      chunk_scale<__bf16, bf16x8>((const __bf16*)t.in[i] + at, (__bf16*)t.out[i] + at, m, f);
    else
      chunk_scale<float, f32x4>((const float*)t.in[i] + at, (float*)t.out[i] + at, m, f);
  });
}

}  // namespace

hipError_t launch_grad_sumsq(const GradTable& t, double* partial, int workgroups, hipStream_t s) {
  hipLaunchKernelGGL(grad_sumsq_kernel, dim3((unsigned)workgroups), dim3(NT), 0, s, t, partial);
  return hipGetLastError();
}

hipError_t launch_grad_fold(const double* partial, int n, double* folded, hipStream_t s) {
  hipLaunchKernelGGL(grad_fold_kernel, dim3(kGradFolded), dim3(NT), 0, s, partial, n, folded);
  return hipGetLastError();
}

hipError_t launch_grad_norm(const double* partial, int n, float* norm, hipStream_t s) {
  hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(NT), 0, s, partial, n, norm);
  return hipGetLastError();
}

hipError_t launch_grad_scale(const GradTable& t, const double* partial, int n, double max_norm, float* norm,
                             int workgroups, hipStream_t s) {
  hipLaunchKernelGGL(grad_scale_kernel, dim3((unsigned)workgroups), dim3(NT), 0, s, t, partial, n, max_norm, norm);
  return hipGetLastError();
}

}  // namespace partir
