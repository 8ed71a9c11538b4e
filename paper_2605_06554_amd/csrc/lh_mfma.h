// lh_mfma.h -- LDS tiles and MFMA operands of the bf16 attention kernels (gfx950; layouts: k_sdpa_mfma.hip).
#pragma once

#include <type_traits>

#include "lh_common.h"

namespace lh {

typedef s16x4 __attribute__((address_space(3))) lds_s16x4;

__device__ __forceinline__ f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kRescale = 8.0f;  // lazy rescaling threshold (log2 units)

template <int N>
using IC = std::integral_constant<int, N>;

// Swizzle of the 16-byte chunks of a row. D = 128 (16 chunks per row): swap the two 2-bit halves
// of r % 16. D = 64 (8 chunks per row, two rows per 256-byte bank line): a bijection of (r / 2) % 8
// whose top bit follows bit 1 of r. The 16 lanes that read one logical chunk of 16 consecutive
// rows hit 16 different chunk positions: row and transposed reads are conflict free.
template <int D>
__device__ __forceinline__ int swz(int r) {
  if constexpr (D == 128) return ((r & 3) << 2) | ((r >> 2) & 3);
  else return (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
}

// Byte offsets of one lane inside any swizzled tile (row blocks start at multiples of 16).
template <int D>
struct LaneOff {
  int row[D / 16];  // row operand (A or B) of k-step kk: row l % 32, columns 16 kk + 8h .. +7
  int trl[D / 32];  // transposed operand, column block d, rows 4h + (l % 16) / 4 (slots 0-3)
  int trh[D / 32];  // the same 8 rows further (slots 4-7)
};

// rows0: first tile row of this wave's share (a multiple of 32)
template <int D>
__device__ __forceinline__ LaneOff<D> lane_offsets(int lane, int rows0) {
  constexpr int RB = 2 * D;
  LaneOff<D> o;
  const int h = lane >> 5, r = lane & 31, base = rows0 * RB;
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk) o.row[kk] = base + r * RB + (((2 * kk + h) ^ swz<D>(r)) << 4);
  const int r0 = 4 * h + ((lane & 15) >> 2);
#pragma unroll
  for (int d = 0; d < D / 32; ++d) {
    const int chunk = 4 * d + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    o.trl[d] = base + r0 * RB + ((chunk ^ swz<D>(r0)) << 4) + 8 * (lane & 1);
    o.trh[d] = base + (r0 + 8) * RB + ((chunk ^ swz<D>(r0 + 8)) << 4) + 8 * (lane & 1);
  }
  return o;
}

// Row operand at byte offset `off` (lane offset plus a constant) of an LDS tile.
__device__ __forceinline__ bf16x8 row8(const bf16_t* tile, int off) {
  return *reinterpret_cast<const bf16x8*>(reinterpret_cast<const char*>(tile) + off);
}

// Transposed operand: within each 16-lane group, lane i receives Mat[r0 + j][c0 + i] (j = 0..3)
// from the lanes' addresses (lane s points at Mat[r0 + s / 4][c0 + 4 (s % 4)]); two reads give
// slots 0-3 (rows +0..3) and 4-7 (rows +8..11).
__device__ __forceinline__ bf16x8 tr8(const bf16_t* tile, int off_lo, int off_hi) {
  typedef __attribute__((__vector_size__(8 * sizeof(short)))) short s16x8;
  const char* p = reinterpret_cast<const char*>(tile);
  const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + off_lo));
  const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + off_hi));
  s16x8 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  return __builtin_bit_cast(bf16x8, v);
}

__device__ __forceinline__ bf16x8 cvt8(const float* f) {
  typedef __attribute__((__vector_size__(8 * sizeof(float)))) float f32x8;
  f32x8 v = {f[0], f[1], f[2], f[3], f[4], f[5], f[6], f[7]};
  return __builtin_convertvector(v, bf16x8);
}

__device__ __forceinline__ bf16x8 gld8(const bf16_t* p) { return *reinterpret_cast<const bf16x8*>(p); }

// Waits until at most N of this wave's vector-memory loads are outstanding and every LDS
// access of the wave has completed (s_waitcnt vmcnt(N) lgkmcnt(0)), then joins the block
// barrier. The empty asm statements keep the compiler from moving memory accesses across.
template <int N>
__device__ __forceinline__ void sync_tiles() {
  static_assert(N >= 0 && N < 64, "vmcnt holds 6 bits");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4));
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

}  // namespace lh
