// Rotary positions of queries and keys, alone or after an RMS norm of every
// head, and the gradients of both.
//
// A head x of dh values, with pairs (a_i, b_i), i < rd / 2, in its first rd
// values -- a_i = x[2 i], b_i = x[2 i + 1] (interleaved) or a_i = x[i], b_i =
// x[i + rd / 2] (halves) -- and the angle theta_i = position * freqs[i]:
//   n = x                                       or, with the norm,
//   n = g x r,  r = 1 / sqrt(mean(x^2) + eps)   over all dh values
//   (a, b) -> m (a cos - b sin, a sin + b cos), the values from rd on kept.
// Gradients: the rotation is linear, so its transpose (sin negated) takes dy to
// dn; then with u = g dn:
//   dx = r (u - x r^2 mean(x u)),   dg = sum over rows of dn x r.
// r is formed again from x, which the backward pass reads anyway.
//
// Angles.  position * freqs[i] runs to millions of radians, where a float32
// product has lost the angle.  It is formed in turns (theta / 2 pi) in float64
// and reduced to its fraction there; only the fraction, within half a turn, is
// rounded to float32.
//
// Layout.  A workgroup takes tb tokens: it first puts the tb x rd/2 cosines and
// sines into LDS, once for all heads, then a group of `lanes` lanes takes a
// (token, head) row at a time, a lane two runs of V values: the V first and the
// V second members of V pairs, or the 2 V values around them where pairs are
// neighbours, or 2 V values of the part that is not rotated.  Every row is read
// and written once, 16 bytes a lane and access where rd and dh allow.
//
// What bounds it is HBM: 2 (forward) or 3 (backward) x T H dh values.  bf16 heads
// of 128, 8192 tokens: the rotation of 80 heads 66 us (335 MB, 5.1 TB/s, the rate
// of a copy of that size), with the norm 64 heads 55 us (268 MB, 4.9 TB/s), the
// gradients 85 us (403 MB, 4.7 TB/s) and 5 us for the gains' partials.  A few
// tokens take 4 to 5 us, most of it the launch and two dependent loads.
#include "operators.h"

namespace partir {
namespace {

constexpr int NT = 256;
constexpr int MAX_PAIRS = 128;     // rd <= 256
constexpr int MAX_TB = 16;

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

// smallest power of two that is at least n
__device__ __host__ __forceinline__ int pow2_ceil(int n) {
  int r = 1;
  while (r < n) r <<= 1;
  return r;
}

// cos and sin (times the magnitude) of tokens [t0, t0 + nt) into cs[token][pair]
__device__ __forceinline__ void angles(const RotaryParams& p, int64_t t0, int nt, float2* cs) {
  const int half = p.rd >> 1;
  for (int e = threadIdx.x; e < nt * half; e += NT) {
    const int k = p.by_half.quot(e), i = p.by_half.rem(e, k);
    const int64_t t = t0 + k;
    double pos;
    if (p.pos)
      pos = p.pos64 ? (double)((const int64_t*)p.pos)[t] : (double)((const int32_t*)p.pos)[t];
    else
      pos = (double)p.by_s.rem((int)t, p.by_s.quot((int)t));
    const double turns = pos * (p.freqs[i] * 0.15915494309189533577);   // 1 / (2 pi)
    const float f = (float)(turns - rint(turns));
    float s, c;
    sincospif(2.0f * f, &s, &c);
    cs[e] = make_float2(c * p.magnitude, s * (p.magnitude * p.sign));
  }
}

// One lane's share of a row: C chunks of two runs of V values.  Chunk c of lane
// li is number li + 64 c (C > 1 only where one row takes the whole wave).
template <int V, int C, bool INTER>
struct Lane {
  int o0[C], o1[C], pair[C];   // offsets of the two runs; first pair (-1: not rotated)
  bool on[C];
  __device__ __forceinline__ void init(const RotaryParams& p, int li) {
    const int rl = p.rd / (2 * V), nl = p.dh / (2 * V);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int k = li + 64 * c;
      on[c] = k < nl;
      const bool rot = k < rl;
      pair[c] = rot ? k * V : -1;
      o0[c] = rot && !INTER ? k * V : 2 * k * V;
      o1[c] = rot && !INTER ? (p.rd >> 1) + k * V : o0[c] + V;
    }
  }
  // v[c][0..V) first run, v[c][V..2V) second
  template <typename T>
  __device__ __forceinline__ void load(const T* row, float (*v)[2 * V]) const {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (on[c]) {
        Run<T, V>::load(row + o0[c], v[c]);
        Run<T, V>::load(row + o1[c], v[c] + V);
      } else {
#pragma unroll
        for (int e = 0; e < 2 * V; ++e) v[c][e] = 0.0f;
      }
    }
  }
  // the row as it is stored (a lane without values takes the first ones), and
  // those values as load gives them
  template <typename T>
  __device__ __forceinline__ void fetch(const T* row, typename Run<T, V>::raw (*x)[2]) const {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      x[c][0] = *(const typename Run<T, V>::raw*)(row + (on[c] ? o0[c] : 0));
      x[c][1] = *(const typename Run<T, V>::raw*)(row + (on[c] ? o1[c] : 0));
    }
  }
  template <typename T>
  __device__ __forceinline__ void widen(const typename Run<T, V>::raw (*x)[2], float (*v)[2 * V]) const {
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int e = 0; e < 2 * V; ++e) v[c][e] = on[c] ? (float)x[c][e / V][e % V] : 0.0f;
  }
  template <typename T>
  __device__ __forceinline__ void store(T* row, const float (*v)[2 * V]) const {
#pragma unroll
    for (int c = 0; c < C; ++c)
      if (on[c]) {
        Run<T, V>::store(row + o0[c], v[c]);
        Run<T, V>::store(row + o1[c], v[c] + V);
      }
  }
  // turns the pairs of v by the token's angles
  __device__ __forceinline__ void rotate(const float2* cs, float (*v)[2 * V]) const {
#pragma unroll
    for (int c = 0; c < C; ++c)
      if (pair[c] >= 0) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float2 w = cs[pair[c] + e];
          float& a = INTER ? v[c][2 * e] : v[c][e];
          float& b = INTER ? v[c][2 * e + 1] : v[c][V + e];
          const float ra = a * w.x - b * w.y, rb = a * w.y + b * w.x;
          a = ra;
          b = rb;
        }
      }
  }
};

// sum over the `lanes` (a power of two) neighbouring lanes of a row
__device__ __forceinline__ float row_sum(float v, int lanes) {
  for (int o = lanes >> 1; o >= 1; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

template <typename T, int V, bool INTER, bool NORM>
__global__ __launch_bounds__(NT) void rotary_kernel(RotaryParams p) {
  constexpr int C = V == 1 ? 2 : 1;
  __shared__ float2 cs[MAX_TB * MAX_PAIRS];
  const int lanes = min(64, pow2_ceil(p.dh / (2 * V)));
  const int slots = NT / lanes, slot = threadIdx.x / lanes, li = threadIdx.x & (lanes - 1);
  const int half = p.rd >> 1, H = p.H[0] + p.H[1];
  Lane<V, C, INTER> lane;
  lane.init(p, li);
  float g[2][C][2 * V];
  if (NORM) {
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      if (p.g[w])
        lane.load(p.g[w], g[w]);
      else
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int e = 0; e < 2 * V; ++e) g[w][c][e] = 1.0f;
    }
  }
  const float inv_dh = 1.0f / (float)p.dh;
  for (int64_t blk = blockIdx.x; blk < p.blocks; blk += gridDim.x) {
    const int64_t t0 = blk * p.tb;
    const int nt = (int)min((int64_t)p.tb, p.T - t0);
    __syncthreads();   // the last block's angles are done with
    angles(p, t0, nt, cs);
    __syncthreads();
    // With the norm a row's loads go out while the one before is summed (8192 tokens
    // of 64 heads: 60 us without, 55 so); the rotation alone, and the gradients with
    // twice the registers, lose by it (8192 x 80 heads: 67 without, 71 so).
    typename Run<T, V>::raw next[C][2];
    auto fetch = [&](int r) {
      r = min(r, nt * H - 1);
      const int k = p.by_h.quot(r), hh = p.by_h.rem(r, k), w = hh >= p.H[0];
      lane.fetch((const T*)p.x[w] + (t0 + k) * p.ldx[w] + (w ? hh - p.H[0] : hh) * p.dh, next);
    };
    if (NORM) fetch(slot);
    for (int r = slot; r < nt * H; r += slots) {
      const int k = p.by_h.quot(r), hh = p.by_h.rem(r, k);
      const int w = hh >= p.H[0];
      const int head = w ? hh - p.H[0] : hh;
      const T* x = (const T*)p.x[w] + (t0 + k) * p.ldx[w] + head * p.dh;
      float v[C][2 * V];
      if (NORM) {
        lane.template widen<T>(next, v);
        fetch(r + slots);
      } else {
        lane.load(x, v);
      }
      if (NORM) {
        float ss = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int e = 0; e < 2 * V; ++e) ss += v[c][e] * v[c][e];
        const float rs = 1.0f / sqrtf(row_sum(ss, lanes) * inv_dh + p.eps);
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int e = 0; e < 2 * V; ++e) v[c][e] = v[c][e] * rs * (w ? g[1][c][e] : g[0][c][e]);
      }
      lane.rotate(cs + k * half, v);
      lane.store((T*)p.y[w] + (t0 + k) * p.ldy[w] + head * p.dh, v);
    }
  }
}

// Gradients of the norm and rotation.  The queries' rows first, then the keys',
// so that one set of accumulators holds a lane's share of the gain gradient;
// the workgroup's rows are added within lanes, then over the row groups of a
// wave, then over its waves, in a fixed order, into one partial per workgroup.
template <typename T, int V, bool INTER>
__global__ __launch_bounds__(NT) void qk_norm_backward_kernel(RotaryParams p) {
  constexpr int C = V == 1 ? 2 : 1;
  __shared__ float2 cs[MAX_TB * MAX_PAIRS];
  __shared__ float red[NT / 64][2 * MAX_PAIRS];
  const int lanes = min(64, pow2_ceil(p.dh / (2 * V)));
  const int slots = NT / lanes, slot = threadIdx.x / lanes, li = threadIdx.x & (lanes - 1);
  const int half = p.rd >> 1, wave = threadIdx.x >> 6;
  Lane<V, C, INTER> lane;
  lane.init(p, li);
  const float inv_dh = 1.0f / (float)p.dh;
  for (int w = 0; w < 2; ++w) {
    float g[C][2 * V], dg[C][2 * V];
    if (p.g[w])
      lane.load(p.g[w], g);
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int e = 0; e < 2 * V; ++e) {
        if (!p.g[w]) g[c][e] = 1.0f;
        dg[c][e] = 0.0f;
      }
    const int H = p.H[w];
    for (int64_t blk = blockIdx.x; blk < p.blocks && H > 0; blk += gridDim.x) {
      const int64_t t0 = blk * p.tb;
      const int nt = (int)min((int64_t)p.tb, p.T - t0);
      __syncthreads();
      angles(p, t0, nt, cs);
      __syncthreads();
      for (int r = slot; r < nt * H; r += slots) {
        const int k = p.by_hw[w].quot(r), head = p.by_hw[w].rem(r, k);
        float x[C][2 * V], u[C][2 * V];
        lane.load((const T*)p.x[w] + (t0 + k) * p.ldx[w] + head * p.dh, x);
        lane.load((const T*)p.dy[w] + (t0 + k) * p.lddy[w] + head * p.dh, u);
        lane.rotate(cs + k * half, u);   // dn
        float ss = 0.0f, xu = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int e = 0; e < 2 * V; ++e) {
            ss += x[c][e] * x[c][e];
            xu += x[c][e] * (u[c][e] * g[c][e]);
          }
        for (int o = lanes >> 1; o >= 1; o >>= 1) {
          ss += __shfl_xor(ss, o);
          xu += __shfl_xor(xu, o);
        }
        const float rs = 1.0f / sqrtf(ss * inv_dh + p.eps);
        const float k2 = rs * rs * (xu * inv_dh);
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int e = 0; e < 2 * V; ++e) {
            dg[c][e] += u[c][e] * (x[c][e] * rs);
            u[c][e] = rs * (u[c][e] * g[c][e] - x[c][e] * k2);
          }
        lane.store((T*)p.y[w] + (t0 + k) * p.ldy[w] + head * p.dh, u);
      }
    }
    // the row groups of a wave (lanes apart), then the waves
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int e = 0; e < 2 * V; ++e) {
        float v = dg[c][e];
        for (int o = lanes; o < 64; o <<= 1) v += __shfl_xor(v, o);
        if ((int)(threadIdx.x & 63) < lanes && lane.on[c]) red[wave][e < V ? lane.o0[c] + e : lane.o1[c] + e - V] = v;
      }
    __syncthreads();
    for (int d = threadIdx.x; d < p.dh; d += NT) {
      float v = red[0][d];
#pragma unroll
      for (int q = 1; q < NT / 64; ++q) v += red[q][d];
      p.dgpart[((int64_t)blockIdx.x * 2 + w) * p.dh + d] = v;
    }
    __syncthreads();
  }
}

// 8 columns and 32 groups of parts a workgroup: the parts of a group in order
// (i = group, group + 32, ..), then the groups in order.  With 1024 parts every
// thread adds 32 values whose loads are in flight together.
__global__ __launch_bounds__(256) void gain_reduce_kernel(const float* part, int parts, int dh, float* dgq, float* dgk) {
  __shared__ float red[32][9];
  const int w = blockIdx.y, col = threadIdx.x & 7, grp = threadIdx.x >> 3;
  const int d = blockIdx.x * 8 + col;   // dh is a multiple of 8
  float* out = w ? dgk : dgq;
  if (!out) return;
  float s = 0.0f;
#pragma unroll 8
  for (int i = grp; i < parts; i += 32) s += part[((int64_t)i * 2 + w) * dh + d];
  red[grp][col] = s;
  __syncthreads();
  if (grp == 0) {
#pragma unroll
    for (int i = 1; i < 32; ++i) s += red[i][col];
    out[d] = s;
  }
}

template <typename T, int V, bool INTER, bool NORM>
hipError_t fwd(const RotaryParams& p, hipStream_t s) {
  hipLaunchKernelGGL((rotary_kernel<T, V, INTER, NORM>), dim3((unsigned)p.grid), dim3(NT), 0, s, p);
  return hipGetLastError();
}
template <typename T, int V, bool NORM>
hipError_t fwd(const RotaryParams& p, bool inter, hipStream_t s) {
  return inter ? fwd<T, V, true, NORM>(p, s) : fwd<T, V, false, NORM>(p, s);
}
template <typename T, bool NORM>
hipError_t fwd(const RotaryParams& p, bool inter, hipStream_t s) {
  switch (p.vec) {
    case 8: return fwd<T, sizeof(T) == 2 ? 8 : 4, NORM>(p, inter, s);   // 8 with 16-bit values only
    case 4: return fwd<T, 4, NORM>(p, inter, s);
    case 2: return fwd<T, 2, NORM>(p, inter, s);
    default: return fwd<T, 1, NORM>(p, inter, s);
  }
}
template <typename T, int V>
hipError_t bwd(const RotaryParams& p, bool inter, hipStream_t s) {
  if (inter)
    hipLaunchKernelGGL((qk_norm_backward_kernel<T, V, true>), dim3((unsigned)p.grid), dim3(NT), 0, s, p);
  else
    hipLaunchKernelGGL((qk_norm_backward_kernel<T, V, false>), dim3((unsigned)p.grid), dim3(NT), 0, s, p);
  return hipGetLastError();
}
template <typename T>
hipError_t bwd(const RotaryParams& p, bool inter, hipStream_t s) {
  switch (p.vec) {
    case 8: return bwd<T, sizeof(T) == 2 ? 8 : 4>(p, inter, s);
    case 4: return bwd<T, 4>(p, inter, s);
    case 2: return bwd<T, 2>(p, inter, s);
    default: return bwd<T, 1>(p, inter, s);
  }
}

}  // namespace

void rotary_choice(RotaryParams& p, bool bf16, RotaryPass pass) {
  int v = bf16 ? 8 : 4;
  while (v > 1 && (p.rd % (2 * v) || p.dh % (2 * v))) v >>= 1;
  p.vec = v;
  const int lanes = pow2_ceil(p.dh / (2 * v)) < 64 ? pow2_ceil(p.dh / (2 * v)) : 64;
  const int64_t slots = NT / lanes;
  // Tokens of a block: enough rows for every row group where there are that
  // many, few enough that the blocks fill the chip.  The rotation alone likes many
  // short workgroups (8192 x 80 heads of 128: 75 us with 2048, 67 with 8192), with
  // the norm the gains that each of them reads first count (8192 x 64 heads: 60
  // with 2048, 69 with 8192), and the gradients leave a partial each.
  const int64_t max_grid = pass == ROTARY ? 8192 : pass == ROTARY_NORM ? 2048 : 1024;
  const int H = p.H[0] + p.H[1];
  int64_t want = p.T * H / max_grid;
  if (want < slots) want = slots;
  int64_t tb = H > 0 ? (want + H - 1) / H : 1;
  if (tb > MAX_TB) tb = MAX_TB;
  if (tb < 1) tb = 1;
  p.tb = (int)tb;
  p.blocks = (p.T + tb - 1) / tb;
  p.grid = (int)(p.blocks < max_grid ? p.blocks : max_grid);
  auto by = [](int64_t d) { return Div::by((uint32_t)(d > 1 ? d : 1)); };
  p.by_s = by(p.S < p.T ? p.S : p.T);   // S >= T: row t stands at t
  p.by_half = by(p.rd / 2);
  p.by_h = by(H);
  for (int w = 0; w < 2; ++w) p.by_hw[w] = by(p.H[w]);
}

hipError_t launch_rotary(const RotaryParams& p, bool bf16, bool interleaved, bool norm, hipStream_t s) {
  if (bf16) return norm ? fwd<__bf16, true>(p, interleaved, s) : fwd<__bf16, false>(p, interleaved, s);
  return norm ? fwd<float, true>(p, interleaved, s) : fwd<float, false>(p, interleaved, s);
}

hipError_t launch_qk_norm_backward(const RotaryParams& p, bool bf16, bool interleaved, hipStream_t s) {
  return bf16 ? bwd<__bf16>(p, interleaved, s) : bwd<float>(p, interleaved, s);
}

hipError_t launch_gain_reduce(const float* dgpart, int parts, int dh, float* dgq, float* dgk, hipStream_t s) {
  hipLaunchKernelGGL(gain_reduce_kernel, dim3((unsigned)(dh / 8), 2), dim3(256), 0, s, dgpart, parts, dh, dgq, dgk);
  return hipGetLastError();
}

}  // namespace partir
