// The join of a block's output y with the residual stream x, and its gradients:
//   u = g_post y r1, r1 = 1 / sqrt(mean(y^2) + eps)   (or u = y)
//   h = x + a u,  a = scale * gate * (kept ? factor : 0)
//   n = g_pre h r2,  r2 = 1 / sqrt(mean(h^2) + eps)   (the next block's norm)
// For cotangents dh and dn, with v = g_pre dn:
//   dx = dh + r2 (v - h r2^2 mean(h v))               the whole gradient of h
//   du = a dx,  dy = r1 (g_post du - y r1^2 mean(y g_post du))   (or dy = du)
//   dg_pre = sum dn h r2,  dg_post = sum du y r1,
//   dgate  = sum over the rows of a gate's row of scale * factor u dx.
// The gradients form h again from x and y, in float32, so that a bf16 stream
// costs them nothing in exactness.  mean(y g_post du) is taken from sums of the
// terms of dx, which need r1 only: two reductions over a row instead of three.
//
// A row is one wave's up to 512 columns, else a workgroup's of as many waves as
// it takes at 8 columns a lane (16 from 8192 columns on).  In the gradients a
// workgroup keeps its columns' sums over all of its rows in registers.
//
// What bounds it: HBM.  8192 x 5120, float32 stream, bf16 block, dropout: forward 97 to
// 102 us (503 MB, 5.0 TB/s), gradients 153 (761 MB, 5.0) and 5 for the sum of the parts.
// 4084 x 1000 in bf16 with post norm and gates: 12.4, 21 and 4 us, chains of a row's
// loads, its two sums and its stores (34 and 53 MB).  The forward loads its gains behind
// the sums: in front of them they take 12.4 -> 11.9 us there, but registers from the
// waves that hide the loads of the first (96 -> 102).
//
// Above 4096 columns the gradients' workgroups have 9 to 16 waves, so 128 registers a
// lane, and with a post norm or a gate that is not enough: 4 to 52 registers lie in
// scratch memory, and above 8192 columns, with 16 columns a lane, 45 to 348 in every form.
// These forms are bound by that.  Gradients in us, float32 stream, bf16 block, dropout,
// a gate's row for 2048 rows; the bytes at 5.06 TB/s:
//                  bytes   plain   post norm   gate   both
//   8192 x 4096      119     119         143    131    148
//   8192 x 5120      149     155         242    190    402
//   8192 x 8192      239     246         318    263    558
//   3000 x 12288     131     354         572    657   1212
//   3000 x 16384     175     409         726    870   1543
// The forward has no such limit: 95 to 114 us at 8192 x 5120, 92 to 108 at 3000 x 12288.
#include <algorithm>
#include <type_traits>

#include "operators.h"
#include "runs.h"

namespace partir {
namespace {

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// Sums over a row: over its wave, and over the workgroup's waves where a row takes
// all of them.  Two buffers in turn need one barrier a sum: who writes a buffer
// again has met everyone at the other's barrier, behind their reads of this one.
struct RowSum {
  float (*red)[16][8];   // [2][wave][value]
  int waves, wave, turn, base;   // base: the first wave of the row
  template <int N>
  __device__ __forceinline__ void operator()(float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
    if (waves == 1) return;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) red[turn][wave][i] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = 0.0f;
    for (int w = 0; w < waves; ++w)
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] += red[turn][base + w][i];
    turn ^= 1;
  }
};

// This lane's columns: chunk c is columns 8 (li + c * lanes) .. + 7.
template <int C>
struct Columns {
  int at[C];
  bool on[C];
  __device__ __forceinline__ Columns(const JoinParams& p, int li) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      at[c] = 8 * (li + c * 64 * p.waves);
      on[c] = at[c] < p.D;
    }
  }
};

template <int C>
__device__ __forceinline__ void load_gain(const float* g, const Columns<C>& k, float one, float (&v)[C][8]) {
#pragma unroll
  for (int c = 0; c < C; ++c) {
    if (g && k.on[c])
      Run<float, 8>::load(g + k.at[c], v[c]);
    else
#pragma unroll
      for (int e = 0; e < 8; ++e) v[c][e] = one;
  }
}

template <typename T, int C>
__device__ __forceinline__ void load_row(const void* p, int64_t off, const Columns<C>& k, float (&v)[C][8]) {
#pragma unroll
  for (int c = 0; c < C; ++c) {
    if (k.on[c])
      Run<T, 8>::load((const T*)p + off + k.at[c], v[c]);
    else
#pragma unroll
      for (int e = 0; e < 8; ++e) v[c][e] = 0.0f;
  }
}

template <typename T, int C>
__device__ __forceinline__ void store_row(void* p, int64_t off, const Columns<C>& k, const float (&v)[C][8]) {
#pragma unroll
  for (int c = 0; c < C; ++c)
    if (k.on[c]) Run<T, 8>::store((T*)p + off + k.at[c], v[c]);
}

template <typename TX, typename TY, int C>
__global__ __launch_bounds__(1024) void join_kernel(JoinParams p) {
  __shared__ float red[2][16][8];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t w = p.waves == 1 ? (int64_t)blockIdx.x * (blockDim.x >> 6) + wave : blockIdx.x;
  if (w >= p.workers) return;                        // whole waves, and only where a row is one wave's
  const Columns<C> k(p, p.waves == 1 ? lane : (int)threadIdx.x);
  RowSum sum{red, p.waves, wave, 0, 0};
  Philox rng;
  if (p.drop.seed) rng.init(p.drop.seed);
  const float inv_d = 1.0f / (float)p.D;
  for (int64_t t = w; t < p.T; t += p.workers) {
    float x[C][8], y[C][8], g[C][8];
    load_row<TX>(p.x, t * p.ldx, k, x);
    load_row<TY>(p.y, t * p.ldy, k, y);
    if (p.post) {
      float s[1] = {0.0f};
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) s[0] += y[c][e] * y[c][e];
      sum(s);
      const float r1 = rsqrtf(s[0] * inv_d + p.eps);
      load_gain(p.g_post, k, 1.0f, g);
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) y[c][e] = y[c][e] * r1 * g[c][e];
    }
    load_gain(p.gate ? p.gate + t / p.gate_rows * p.ldgate : nullptr, k, 1.0f, g);
    float s[1] = {0.0f};
#pragma unroll
    for (int c = 0; c < C; ++c) {
      uint32_t keep = 0xFF;
      if (p.drop.seed) keep = rng.keep8((uint32_t)k.at[c] >> 3, p.drop.row0 + (uint32_t)t, p.drop.kept);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[c][e] += keep >> e & 1 ? p.scale * g[c][e] * y[c][e] : 0.0f;
        s[0] += k.on[c] ? x[c][e] * x[c][e] : 0.0f;
      }
    }
    store_row<TX>(p.h, t * p.ldh, k, x);
    if (p.n) {
      sum(s);
      const float r2 = rsqrtf(s[0] * inv_d + p.eps);
      load_gain(p.g_pre, k, 1.0f, g);
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) x[c][e] = x[c][e] * r2 * g[c][e];
      store_row<TY>(p.n, t * p.ldn, k, x);
    }
  }
}

// A row as it is stored.
template <typename T, int C>
struct Raw {
  typename Run<T, 8>::raw v[C];
  __device__ __forceinline__ void load(const void* p, int64_t off, const Columns<C>& k) {
#pragma unroll
    for (int c = 0; c < C; ++c)
      if (k.on[c]) v[c] = *(const typename Run<T, 8>::raw*)((const T*)p + off + k.at[c]);
  }
  __device__ __forceinline__ void get(const Columns<C>& k, float (&x)[C][8]) const {
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) x[c][e] = k.on[c] ? (float)v[c][e] : 0.0f;
  }
};

// The rows of a workgroup are shared out over its teams of p.waves waves.  Where a
// gate's row has rows enough for a workgroup, or there is no gate, a workgroup has a
// chunk of one gate's row and its teams take every teams-th row; else a team has
// whole gate rows, and stores each one's gradient itself.  The teams' sums are added
// in LDS, so that a workgroup leaves one partial row of each gradient.  A row's
// loads go out before the sums of the row before are taken.
template <typename TX, typename TY, int C, int MOST, bool POST, bool GATE>
__global__ __launch_bounds__(MOST) void join_bwd_kernel(JoinParams p) {
  __shared__ float red[2][16][8];
  __shared__ __attribute__((aligned(16))) float acc[8][64][8];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int team = wave / p.waves, in_team = wave - team * p.waves;
  const Columns<C> k(p, 64 * in_team + lane);
  RowSum sum{red, p.waves, wave, 0, team * p.waves};
  Philox rng;
  if (p.drop.seed) rng.init(p.drop.seed);
  const float inv_d = 1.0f / (float)p.D;
  const bool next = p.dn != nullptr;
  // this team's rows: t0, t0 + step, .. below end; `turns` of them in every team of the workgroup
  int64_t t0, end, step, turns;
  if (p.chunks > 0) {
    const int64_t group = blockIdx.x / p.chunks, first = group * p.span + (blockIdx.x - group * p.chunks) * p.per;
    end = min(min(first + p.per, (group + 1) * p.span), p.T);
    t0 = first + team;
    step = p.teams;
    turns = (p.per + p.teams - 1) / p.teams;
  } else {
    t0 = ((int64_t)blockIdx.x * p.teams + team) * p.per;
    end = min(t0 + p.per, p.T);
    step = 1;
    turns = p.per;
  }
  float gpost[C][8], gpre[C][8], gate[C][8], apost[C][8], apre[C][8], agate[C][8];
  // 16 columns a lane leave no room for a second row's loads and for the gains
  constexpr bool AHEAD = C == 1;
  auto gains = [&]() {
    load_gain(p.g_post, k, 1.0f, gpost);
    load_gain(p.g_pre, k, 1.0f, gpre);
  };
  if (AHEAD) gains();
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      apost[c][e] = apre[c][e] = agate[c][e] = 0.0f;
      gate[c][e] = 1.0f;
    }
  Raw<TX, C> rx, rdh;
  Raw<TY, C> ry, rdn;
  auto fetch = [&](int64_t t) {
    ry.load(p.y, t * p.ldy, k);
    if (next) {
      rx.load(p.x, t * p.ldx, k);
      rdn.load(p.dn, t * p.lddn, k);
    }
    if (p.dh) rdh.load(p.dh, t * p.lddh, k);
  };
  if (AHEAD && t0 < end) fetch(t0);
  int64_t group = -1, group_end = t0;                // the gate's row that the sums are of, and where it ends
  for (int64_t n = 0; n < turns; ++n) {
    const int64_t t = t0 + n * step;
    const bool live = t < end;                       // the same in a team, not in a workgroup
    if (GATE && live && t >= group_end) {
      if (p.dgate_rows && group >= 0) {              // whole gate rows: each is stored where it belongs
        store_row<float>(p.dgate_rows, group * p.D, k, agate);
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int e = 0; e < 8; ++e) agate[c][e] = 0.0f;
      }
      group = t / p.gate_rows;
      group_end = (group + 1) * p.gate_rows;
      if (AHEAD) load_gain(p.gate + group * p.ldgate, k, 1.0f, gate);
    }
    if (!AHEAD) {
      if (live) fetch(t);
      gains();
      if (GATE && live) load_gain(p.gate + group * p.ldgate, k, 1.0f, gate);
    }
    float x[C][8], y[C][8], dh[C][8], v[C][8];
    ry.get(k, y);
    if (next) {
      rx.get(k, x);
      rdn.get(k, v);
    }
    if (p.dh) rdh.get(k, dh);
    if (AHEAD && t + step < end) fetch(t + step);
    float r1 = 1.0f, r2 = 0.0f;
    if constexpr (POST) {
      float s[1] = {0.0f};
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) s[0] += y[c][e] * y[c][e];
      sum(s);
      r1 = rsqrtf(s[0] * inv_d + p.eps);
    }
    uint32_t keep[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      keep[c] = k.on[c] ? 0xFF : 0;
      if (p.drop.seed && k.on[c]) keep[c] = rng.keep8((uint32_t)k.at[c] >> 3, p.drop.row0 + (uint32_t)t, p.drop.kept);
    }
    // sums of h^2, h v, and of z dh, z v, z h with z = a g_post y
    float s[POST ? 5 : 2];
#pragma unroll
    for (int i = 0; i < (POST ? 5 : 2); ++i) s[i] = 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (!p.dh) dh[c][e] = 0.0f;
        const float z = keep[c] >> e & 1 ? p.scale * gate[c][e] * (POST ? gpost[c][e] * y[c][e] : y[c][e]) : 0.0f;
        if (next) {
          x[c][e] += z * r1;                         // h
          const float gv = gpre[c][e] * v[c][e];
          s[0] += x[c][e] * x[c][e];
          s[1] += x[c][e] * gv;
          if constexpr (POST) {
            s[3] += z * gv;
            s[4] += z * x[c][e];
          }
        }
        if constexpr (POST) s[2] += z * dh[c][e];
      }
    if (next || POST) sum(s);
    float m = 0.0f, q = 0.0f;
    if (next) {
      r2 = rsqrtf(s[0] * inv_d + p.eps);
      m = r2 * r2 * (s[1] * inv_d);
    }
    if constexpr (POST) q = r1 * r1 * inv_d * (s[2] + r2 * (s[3] - m * s[4]));   // r1^2 mean(y g_post du)
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (next) {
          if (live) apre[c][e] += v[c][e] * x[c][e] * r2;
          dh[c][e] += r2 * (gpre[c][e] * v[c][e] - x[c][e] * m);
        }
        const bool on = keep[c] >> e & 1;
        const float kept = on ? p.scale * dh[c][e] : 0.0f;
        const float yr = y[c][e] * r1, du = gate[c][e] * kept;
        if (GATE && live) agate[c][e] += on ? kept * (POST ? gpost[c][e] * yr : yr) : 0.0f;
        if constexpr (POST) {
          if (live) apost[c][e] += du * yr;
          y[c][e] = r1 * (gpost[c][e] * du - y[c][e] * q);
        } else {
          y[c][e] = du;
        }
      }
    if (live) {
      store_row<TX>(p.dx, t * p.lddx, k, dh);
      store_row<TY>(p.dy, t * p.lddy, k, y);
    }
  }
  if (GATE && p.dgate_rows && group >= 0) store_row<float>(p.dgate_rows, group * p.D, k, agate);
  // the teams' sums, in order, into the workgroup's row of a matrix of parts
  auto leave = [&](float* part, float (&a)[C][8]) {
    if (!part) return;
    if (p.teams > 1) {                               // C = 1
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[wave & 7][lane][e] = a[0][e];
      __syncthreads();
      if (team == 0)
        for (int i = 1; i < p.teams; ++i)
#pragma unroll
          for (int e = 0; e < 8; ++e) a[0][e] += acc[i * p.waves + in_team][lane][e];
      __syncthreads();
    }
    if (team == 0) store_row<float>(part, (int64_t)blockIdx.x * p.D, k, a);
  };
  leave(p.part_post, apost);
  leave(p.part_pre, apre);
  if (p.chunks > 0) leave(p.part_gate, agate);
}

// out[o][d] = sum over parts [o * parts, (o + 1) * parts) of part[.][d], for the
// matrices of a launch; 64 columns and 16 runs of the parts a workgroup, in order.
__global__ __launch_bounds__(1024) void join_reduce_kernel(JoinSums q) {
  __shared__ float acc[16][64];
  int o = blockIdx.y, i = 0;
  while (o >= q.outs[i]) o -= q.outs[i++];
  const int d = blockIdx.x * 64 + (threadIdx.x & 63), run = threadIdx.x >> 6;
  const int64_t parts = q.parts[i], per = (parts + 15) / 16;
  float s = 0.0f;
  if (d < q.D) {
    const float* src = q.part[i] + (int64_t)o * parts * q.D + d;
    const int64_t end = min(parts, (run + 1) * per);
#pragma unroll 8
    for (int64_t k = run * per; k < end; ++k) s += src[k * q.D];
  }
  acc[run][threadIdx.x & 63] = s;
  __syncthreads();
  if (run == 0 && d < q.D) {
#pragma unroll
    for (int r = 1; r < 16; ++r) s += acc[r][threadIdx.x];
    q.out[i][(int64_t)o * q.D + d] = s;
  }
}

constexpr int64_t kCUs = 256;

template <typename F>
void by_types(bool x_bf16, bool y_bf16, bool wide, F go) {
  auto chunks = [&](auto x, auto y) {
    wide ? go(x, y, std::integral_constant<int, 2>()) : go(x, y, std::integral_constant<int, 1>());
  };
  if (x_bf16)
    y_bf16 ? chunks(__bf16(), __bf16()) : chunks(__bf16(), float());
  else
    y_bf16 ? chunks(float(), __bf16()) : chunks(float(), float());
}

}  // namespace

void join_choice(JoinParams& p, bool backward) {
  const int groups = (p.D + 7) / 8, chunk = groups > 1024 ? 2 : 1;
  p.waves = std::max(1, (groups + 64 * chunk - 1) / (64 * chunk));
  if (!backward) {
    p.workers = std::min<int64_t>(p.T, 1 << 20);   // a launch is fewer than 2^32 threads
    return;
  }
  // Workgroups of 8 to 16 waves, two a CU (one from 9 waves on); less than 4 rows a
  // team only where there are fewer, since each leaves a row of partial sums.
  p.teams = p.waves >= 5 ? 1 : 8 / p.waves;
  const int64_t most = kCUs * (p.waves * p.teams > 8 ? 1 : 2);
  const int64_t span = std::min(p.gate_rows, p.T);
  const int64_t wgs = std::max<int64_t>(1, std::min<int64_t>(most, (p.T + 4 * p.teams - 1) / (4 * p.teams)));
  const int64_t per = (p.T + wgs - 1) / wgs;
  if (span >= per) {                     // a workgroup: a chunk of one gate's row
    p.span = span;
    p.chunks = (span + per - 1) / per;
    p.per = (span + p.chunks - 1) / p.chunks;
    p.chunks = (span + p.per - 1) / p.per;
    p.workers = (p.T + span - 1) / span * p.chunks;
  } else {                               // a team: whole gate rows
    const int64_t rows = (per + p.teams - 1) / p.teams;
    p.per = p.span = (rows + span - 1) / span * span;
    p.chunks = 0;
    p.workers = (p.T + p.per * p.teams - 1) / (p.per * p.teams);
  }
}

hipError_t launch_join(const JoinParams& p, bool x_bf16, bool y_bf16, hipStream_t s) {
  const int64_t per = p.waves == 1 ? 4 : 1;
  const dim3 grid((unsigned)((p.workers + per - 1) / per)), block((unsigned)(64 * (p.waves == 1 ? 4 : p.waves)));
  by_types(x_bf16, y_bf16, p.D > 8192, [&](auto x, auto y, auto c) {
    hipLaunchKernelGGL((join_kernel<decltype(x), decltype(y), decltype(c)::value>), grid, block, 0, s, p);
  });
  return hipGetLastError();
}

hipError_t launch_join_backward(const JoinParams& p, bool x_bf16, bool y_bf16, hipStream_t s) {
  const dim3 grid((unsigned)p.workers), block((unsigned)(64 * p.waves * p.teams));
  by_types(x_bf16, y_bf16, p.D > 8192, [&](auto x, auto y, auto c) {
    auto go = [&](auto post, auto gate) {
      constexpr int C = decltype(c)::value;
      constexpr bool P = decltype(post)::value, G = decltype(gate)::value;
      // up to 8 waves may take twice the registers that 16 may, which are too few for
      // most forms (the figures at the top)
      if (C == 1 && p.waves * p.teams <= 8)
        hipLaunchKernelGGL((join_bwd_kernel<decltype(x), decltype(y), 1, 512, P, G>), grid, block, 0, s, p);
      else
        hipLaunchKernelGGL((join_bwd_kernel<decltype(x), decltype(y), C, 1024, P, G>), grid, block, 0, s, p);
    };
    typedef std::true_type yes;
    typedef std::false_type no;
    if (p.post)
      p.gate ? go(yes(), yes()) : go(yes(), no());
    else
      p.gate ? go(no(), yes()) : go(no(), no());
  });
  return hipGetLastError();
}

hipError_t launch_join_reduce(const JoinSums& q, hipStream_t s) {
  int64_t outs = 0;
  for (int i = 0; i < q.n; ++i) outs += q.outs[i];
  hipLaunchKernelGGL(join_reduce_kernel, dim3((unsigned)((q.D + 63) / 64), (unsigned)outs), dim3(1024), 0, s, q);
  return hipGetLastError();
}

}  // namespace partir
