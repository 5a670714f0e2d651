// Device helpers shared by the attention kernels (gfx950): swizzled 64 x 64
// bf16 tiles in LDS, the 32x32x16 MFMA operands read from them, and the
// reductions over the two lanes that hold one row.
#pragma once

#include "pf_dma.h"

namespace pf {
namespace {

constexpr int D = 64;                    // head dim
constexpr int BQ = 64;                   // block size
constexpr int TILE = BQ * D * 2;         // bytes of a 64 x 64 bf16 tile
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// 2^x on the hardware exponential unit (v_exp_f32): results below 2^-126
// flush toward zero, which a softmax probability can afford; saves the
// range-reduction sequence the library exp2f adds for denormal outputs.
__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// x combined with the value of lane l ^ 32 by max or +: the swap exchanges
// the halves inside the VALU, where a lane shuffle would make a round trip
// through the LDS.
__device__ __forceinline__ float max_xor32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float add_xor32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)lo) |
         ((uint32_t)__builtin_bit_cast(uint16_t, (__bf16)hi) << 16);
}

// LDS tile: 64 rows of 128 bytes, the 16-byte chunk c of row r at position
// c ^ chunk_swz(r).  Row pairs (256 bytes, all 64 banks) get the eight
// values of the bit-reversed pair index: 16 rows at one chunk (fragment
// read) and 4 rows x 4 chunks (transpose read) both fall in distinct banks.
__device__ __forceinline__ int chunk_swz(int r) {
  return ((r & 2) << 1) | ((r & 4) >> 1) | ((r & 8) >> 3);
}

// Operand of a 32x32x16 MFMA from a tile: row r0 + l % 32, k = ks * 16 +
// (l / 32) * 8 + 0..7.
__device__ __forceinline__ bf16x8 frag_r(const uint8_t *tile, int r0, int ks, int lane) {
  const int r = r0 + (lane & 31), c = ks * 2 + (lane >> 5);
  return *(const bf16x8 *)(tile + r * 128 + ((c ^ chunk_swz(r)) << 4));
}
// Operand A[m][k] = tile[k][m], m = m0 + l % 32, k in the accumulator's row
// order: kb + 4 (l / 32) + 0..3, then kb + 8 + 4 (l / 32) + 0..3.
__device__ __forceinline__ bf16x8 frag_t(const uint8_t *tile, int kb, int m0, int lane) {
  const int g = lane >> 4, i = lane & 15;
  const int c = (m0 >> 3) + (g & 1) * 2 + ((i & 3) >> 1), half = (i & 1) << 3;
  const int k = kb + (g >> 1) * 4 + (i >> 2);
  const int lo_off = k * 128 + ((c ^ chunk_swz(k)) << 4) + half;
  const int hi_off = (k + 8) * 128 + ((c ^ chunk_swz(k + 8)) << 4) + half;
  const s16x4 lo = tr16(tile + lo_off), hi = tr16(tile + hi_off);
  const s16x8 v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  return __builtin_bit_cast(bf16x8, v);
}
// Registers 8 j .. 8 j + 7 of an accumulator as a bf16 K-operand.
__device__ __forceinline__ bf16x8 pack_k(const f32x16 &s, int j) {
  bf16x8 v;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = (__bf16)s[8 * j + e];
  return v;
}

#define MFMA32(a, b, c) __builtin_amdgcn_mfma_f32_32x32x16_bf16((a), (b), (c), 0, 0, 0)

}  // namespace
}  // namespace pf
