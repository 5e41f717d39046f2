// Device helpers: runs of values of a row, loaded and stored with one access
// each.
#pragma once
#include <hip/hip_runtime.h>

namespace partir {

// V values of a row: as they are stored, and in float32 registers
template <typename T, int V>
struct Run;
template <int V>
struct Run<float, V> {
  typedef float raw __attribute__((ext_vector_type(V)));
  static __device__ __forceinline__ void load(const float* p, float* v) {
    typedef float vec __attribute__((ext_vector_type(V)));
    const vec x = *(const vec*)p;
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = x[e];
  }
  static __device__ __forceinline__ void store(float* p, const float* v) {
    typedef float vec __attribute__((ext_vector_type(V)));
    vec x;
#pragma unroll
    for (int e = 0; e < V; ++e) x[e] = v[e];
    *(vec*)p = x;
  }
};
template <int V>
struct Run<__bf16, V> {
  typedef __bf16 raw __attribute__((ext_vector_type(V)));
  static __device__ __forceinline__ void load(const __bf16* p, float* v) {
    typedef __bf16 vec __attribute__((ext_vector_type(V)));
    const vec x = *(const vec*)p;
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = (float)x[e];
  }
  static __device__ __forceinline__ void store(__bf16* p, const float* v) {
    typedef __bf16 vec __attribute__((ext_vector_type(V)));
    vec x;
#pragma unroll
    for (int e = 0; e < V; ++e) x[e] = (__bf16)v[e];   // the one rounding, to the tensor's type
    *(vec*)p = x;
  }
};

}  // namespace partir
