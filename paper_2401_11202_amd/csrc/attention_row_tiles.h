// Device helpers of the attention gradient kernels: tiles of query rows of Q and dO,
// and the way of a wave's results out.
#pragma once
#include "attention_tiles.h"
#include "operators.h"

namespace partir {
namespace {

constexpr int NT = 256;
constexpr int TR = 64;                 // rows of a streamed tile
constexpr int TILE = TR * ROWB;

// The ROWS-row tiles of the first `rows` of the G Sq query rows of a (sequence, key head), Q and dO
// side by side: row i is position i / G of head i mod G.  Addresses ascend with
// the rows, so a descriptor that ends with the tile's last row makes those
// behind it zeros.  Where G divides 16, a lane's rows lie at one offset from a
// tile's first position and a fixed step apart; else each is divided by G (8 %
// of dkv's time).
template <bool EVEN, int WAVES = 4, int ROWS = TR>
struct RowTiles {
  const uint16_t *q, *g;
  int64_t ldq, ldg;
  Div by_g;
  int R, w, lane;
  uint32_t oq, og, chunk;
  __device__ __forceinline__ RowTiles(const CrossBwdParams& p, int b, int kvh, int rows, int w_, int lane_)
      : q(p.Q + (int64_t)b * p.Sq * p.ldq + kvh * p.G * DH), g(p.dO + (int64_t)b * p.Sq * p.ldg + kvh * p.G * DH), ldq(p.ldq),
        ldg(p.ldg), by_g(p.by_g), R(rows), w(w_), lane(lane_) {
    const int l4 = lane >> 4, r = 4 * w + l4, s = by_g.quot(r);
    chunk = ((lane & 15) ^ (l4 << 2) ^ (w & 3)) << 4;   // row 4 WAVES j + r sits at the same chunk for every j
    const uint32_t in = (uint32_t)by_g.rem(r, s) * ROWB + chunk;
    oq = (uint32_t)s * (uint32_t)(ldq * 2) + in;
    og = (uint32_t)s * (uint32_t)(ldg * 2) + in;
  }
  __device__ __forceinline__ void load(int it, char* tile) const {
    const int i0 = it * ROWS, s0 = by_g.quot(i0), last = min(i0 + ROWS, R) - 1, sl = by_g.quot(last);
    const uint32_t tail = (uint32_t)by_g.rem(last, sl) * ROWB + ROWB;
    const __amdgpu_buffer_rsrc_t rq = make_rsrc(q + s0 * ldq, (uint32_t)((sl - s0) * ldq * 2) + tail);
    const __amdgpu_buffer_rsrc_t rg = make_rsrc(g + s0 * ldg, (uint32_t)((sl - s0) * ldg * 2) + tail);
    auto put = [&](int j, uint32_t a, uint32_t b) {
      char* const t = tile + (WAVES * j + w) * 1024;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rq, (lds_void*)t, 16, a, 0, 0, 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rg, (lds_void*)(t + ROWS * ROWB), 16, b, 0, 0, 0);
    };
    if constexpr (EVEN) {
      const uint32_t n = by_g.quot(4 * WAVES), sq = n * (uint32_t)(ldq * 2), sg = n * (uint32_t)(ldg * 2);
#pragma unroll
      for (int j = 0; j < ROWS / (4 * WAVES); ++j) put(j, oq + j * sq, og + j * sg);
    } else {
#pragma unroll
      for (int j = 0; j < ROWS / (4 * WAVES); ++j) {
        const int i = i0 + 4 * (WAVES * j + w) + (lane >> 4), s = by_g.quot(i);
        const uint32_t in = (uint32_t)by_g.rem(i, s) * ROWB + chunk;
        put(j, (uint32_t)(s - s0) * (uint32_t)(ldq * 2) + in, (uint32_t)(s - s0) * (uint32_t)(ldg * 2) + in);
      }
    }
  }
};

// A wave's 32 rows of 128 results times f, through its share of the tiles'
// memory (free behind the loops' last barrier), as bf16 or as float32 parts.
__device__ __forceinline__ void store(char* smem, int w, uint16_t* out, int64_t off, int rows, const f32x16* a, float f, int lane) {
  store_rows<4>(smem + w * row_area<4, __bf16>(), (__bf16*)out, off, rows, a, f, lane);
}
__device__ __forceinline__ void store(char* smem, int w, float* out, int64_t off, int rows, const f32x16* a, float f, int lane) {
  char* const area = smem + w * row_area<2, float>();
  store_rows<2>(area, out, off, rows, a, f, lane);
  store_rows<2>(area, out, off + 64, rows, a + 2, f, lane);
}

}  // namespace
}  // namespace partir
