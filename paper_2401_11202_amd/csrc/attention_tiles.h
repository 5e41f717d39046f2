// Device helpers of the cross attention kernels: [rows x 128] bf16 tiles in
// LDS, read as MFMA operands.
#pragma once
#include "lds_dma.h"

namespace partir {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int DH = 128;        // values of a head
constexpr int ROWB = 256;      // bytes of a tile row

// A tile holds 256-byte rows of sixteen 16-byte chunks; chunk c of row r sits
// at position c ^ tile_swz(r).  Row 4 b + a of a 16-row group (a, b < 4) gets
// 4 a + b: a row read (16 lanes on 16 consecutive rows, one chunk) lands on 16
// distinct positions, and so does half a transposed read (4 consecutive rows x
// one aligned 64-byte group), since the row's low two bits move it to another
// group.
__device__ __forceinline__ int tile_swz(int row) { return ((row & 3) << 2) | ((row >> 2) & 3); }
__device__ __forceinline__ int tile_off(int row, int colb) {
  return row * ROWB + (((colb >> 4) ^ tile_swz(row)) << 4) + (colb & 15);
}

// Operand of a 32-row MFMA block read row-wise: rows r0 + (lane & 31), chunk
// 2 ds + h of the contracted 128 values.
__device__ __forceinline__ bf16x8 tile_rows(const char* tile, int r0, int col, int h, int ds) {
  return lds_read<bf16x8>(tile + tile_off(r0 + col, (2 * ds + h) * 16));
}

// Operand X^T [columns 32 dt.., rows 16 u..] of a tile X; the 16 rows come in
// the order in which a 32x32 MFMA result holds them: element v of lane half h
// is row 8 (v / 4) + 4 h + v % 4.
struct TileTr {
  int row, colb;
  __device__ __forceinline__ void init(int lane) {
    const int j = lane & 15, g = lane >> 4;
    row = 4 * (g >> 1) + (j >> 2);
    colb = 2 * (16 * (g & 1) + 4 * (j & 3));
  }
  __device__ __forceinline__ bf16x8 read(const char* tile, int u, int dt) const {
    const lds_i16x4_t lo = lds_read_tr16(tile + tile_off(16 * u + row, 64 * dt + colb));
    const lds_i16x4_t hi = lds_read_tr16(tile + tile_off(16 * u + row + 8, 64 * dt + colb));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
};

// Streams `rows` rows of a [rows, 128] block of a bf16 matrix into an LDS tile
// of ROWS rows, WAVES waves sharing the loads (wave w of them), 1 KiB or four
// rows each.  The descriptor ends with the last of the rows: those behind it
// are written as zeros, whatever the memory there holds.  Its size and offsets are
// 32-bit: `rows` is at most ROWS, and 128 rows are as many as reach there at any
// leading dim (2^24 values at most).
template <int ROWS, int WAVES>
__device__ __forceinline__ void tile_load(const uint16_t* base, int64_t ld, int rows, char* tile, int w, int lane) {
  static_assert((int64_t)ROWS * 2 * (1 << 24) <= (int64_t)1 << 32, "a descriptor's offsets are 32-bit");
  const __amdgpu_buffer_rsrc_t rs = make_rsrc(base, rows > 0 ? (uint32_t)((rows - 1) * ld * 2 + ROWB) : 0);
  const int l4 = lane >> 4, ch = lane & 15;
  const uint32_t ldb = (uint32_t)(ld * 2);
#pragma unroll
  for (int j = 0; j < ROWS / (4 * WAVES); ++j) {
    const int r4 = WAVES * j + w;                // group of four rows
    const uint32_t off = (uint32_t)(4 * r4 + l4) * ldb + ((ch ^ (l4 << 2) ^ (r4 & 3)) << 4);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void*)(tile + r4 * 1024), 16, off, 0, 0, 0);
  }
}

// An LDS write through a restrict pointer, for lds_read's reason: a plain one
// waits for every LDS DMA in flight first.
template <typename T>
__device__ __forceinline__ void lds_write(char* __restrict__ p, T v) { *(T*)p = v; }

// A workgroup barrier that waits for this wave's LDS reads and writes but not
// for its loads in flight, as __syncthreads would.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_sched_barrier(0);
  WAIT_LGKMCNT(0);
  asm volatile("s_barrier" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// two fp32 values rounded to bf16 into elements i, i + 1 of x
__device__ __forceinline__ void put2(bf16x8& x, int i, float a, float b) {
  const f32x2 f = {a, b};
  const bf16x2 r = __builtin_convertvector(f, bf16x2);
  x[i] = r[0];
  x[i + 1] = r[1];
}

__device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ void zero(f32x16& a) {
#pragma unroll
  for (int v = 0; v < 16; ++v) a[v] = 0.0f;
}

// Stores a wave's results, 32 rows of ND blocks of 32 columns held as a 32x32
// MFMA leaves them (lane: row lane & 31; element v of block d: column 32 d + 8
// (v / 4) + 4 h + v % 4), times f, as T (bf16: the one rounding).  A lane's own
// values are 8- or 16-byte pieces of a row, and stores of such pieces, 64 rows
// apart, held the attention kernels up for 4 us at their end; so the rows pass
// through `area` in LDS (the wave's own, row_area bytes, 16-byte aligned) and
// leave whole, 16 bytes a lane.  off: where this lane's row starts in out, in
// values (both lanes of a row alike); rows from `rows` on are not stored.
template <int ND, typename T>
__host__ __device__ constexpr int row_area() { return 32 * (ND * 32 * (int)sizeof(T) + 16); }
template <int ND, typename T>
__device__ __forceinline__ void store_rows(char* area, T* out, int64_t off, int rows, const f32x16* a, float f, int lane) {
  typedef T vec4 __attribute__((ext_vector_type(4)));
  constexpr int PITCH = ND * 32 * sizeof(T) + 16, CPR = ND * 32 * sizeof(T) / 16, RPI = 64 / CPR;
  const int h = lane >> 5, col = lane & 31;
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *(vec4*)(area + col * PITCH + (32 * d + 8 * g + 4 * h) * sizeof(T)) =
          vec4{(T)(a[d][4 * g + 0] * f), (T)(a[d][4 * g + 1] * f), (T)(a[d][4 * g + 2] * f), (T)(a[d][4 * g + 3] * f)};
  const int r0 = lane / CPR, c = lane % CPR;
  const int lo = (int)(uint32_t)off, hi = (int)(off >> 32);
#pragma unroll
  for (int j = 0; j < 32 / RPI; ++j) {
    const int r = j * RPI + r0;
    const f32x4 v = *(const f32x4*)(area + r * PITCH + c * 16);
    const int64_t o = ((int64_t)__shfl(hi, r) << 32) | (uint32_t)__shfl(lo, r);
    if (r < rows) *(f32x4*)((char*)(out + o) + c * 16) = v;
  }
}

}  // namespace partir
