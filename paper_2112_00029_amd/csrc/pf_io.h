// Elements of one type <-> floats, V at a time (16 bytes, or single elements),
// and sums over a wave and a workgroup in a fixed order.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "pf_dma.h"

namespace pf {
namespace {

// V elements as they lie in memory: one 16-byte access, or one element.
template <typename T, int V>
struct Raw;
template <typename T>
struct Raw<T, 1> {
  T x;
};
template <>
struct Raw<bf16_t, 8> {
  u32x4 x;
};
template <>
struct Raw<float, 4> {
  f32x4 x;
};

// At any element's address: the hardware's 16-byte accesses need no more.
template <typename T, int V>
__device__ __forceinline__ Raw<T, V> ld_raw(const T *p) {
  typedef decltype(Raw<T, V>::x) at __attribute__((aligned(sizeof(T))));
  Raw<T, V> r;
  r.x = *(const at *)p;
  return r;
}
template <typename T, int V, bool NT = false>
__device__ __forceinline__ void st_raw(T *p, const Raw<T, V> &r) {
  typedef decltype(Raw<T, V>::x) at __attribute__((aligned(sizeof(T))));
  if constexpr (NT && V > 1) __builtin_nontemporal_store(r.x, (at *)p);
  else *(at *)p = r.x;
}

__device__ __forceinline__ float up(bf16_t x) { return __uint_as_float((uint32_t)x << 16); }
__device__ __forceinline__ float up(float x) { return x; }
__device__ __forceinline__ void down(bf16_t &o, float v) { o = __builtin_bit_cast(uint16_t, (__bf16)v); }
__device__ __forceinline__ void down(float &o, float v) { o = v; }

template <typename T, int V>
__device__ __forceinline__ void unpack(const Raw<T, V> &r, float (&v)[V]) {
  if constexpr (V == 1) {
    v[0] = up(r.x);
  } else if constexpr (V == 8) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[2 * e] = __uint_as_float(r.x[e] << 16);
      v[2 * e + 1] = __uint_as_float(r.x[e] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = r.x[e];
  }
}
// Rounds to nearest even.
template <typename T, int V>
__device__ __forceinline__ Raw<T, V> pack(const float (&v)[V]) {
  Raw<T, V> r;
  if constexpr (V == 1) {
    down(r.x, v[0]);
  } else if constexpr (V == 8) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      r.x[e] = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v[2 * e]) |
               ((uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v[2 * e + 1]) << 16);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) r.x[e] = v[e];
  }
  return r;
}
template <typename T, int V>
__device__ __forceinline__ Raw<T, V> zero_raw() {
  float z[V] = {};
  return pack<T, V>(z);
}

// Sum over the 64 lanes, the same in all of them: each step adds the value of
// another lane of the same row of 16, then of the rows before.
template <int CTRL, int ROWS>
__device__ __forceinline__ float dpp_add(float x) {
  const int y = __builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, ROWS, 0xf, false);
  return x + __int_as_float(y);
}
__device__ __forceinline__ float wave_sum(float x) {
  x = dpp_add<0x111, 0xf>(x);  // row_shr:1
  x = dpp_add<0x112, 0xf>(x);  // row_shr:2
  x = dpp_add<0x114, 0xf>(x);  // row_shr:4
  x = dpp_add<0x118, 0xf>(x);  // row_shr:8 (lane 15 of a row: its sum)
  x = dpp_add<0x142, 0xa>(x);  // row_bcast:15 into rows 1 and 3
  x = dpp_add<0x143, 0xc>(x);  // row_bcast:31 into rows 2 and 3
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}

// The same of doubles, whose halves move together.
template <int CTRL, int ROWS>
__device__ __forceinline__ double dpp_add(double x) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, CTRL, ROWS, 0xf, false);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), CTRL, ROWS, 0xf, false);
  return x + __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double wave_sum(double x) {
  x = dpp_add<0x111, 0xf>(x);
  x = dpp_add<0x112, 0xf>(x);
  x = dpp_add<0x114, 0xf>(x);
  x = dpp_add<0x118, 0xf>(x);
  x = dpp_add<0x142, 0xa>(x);
  x = dpp_add<0x143, 0xc>(x);
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)b, 63);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), 63);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// Sums of NV values over groups of TPR threads (a multiple of 64), the same in
// every thread of a group.  `box`: NV * (threads / 64) of them in LDS; a box is
// free again after the next barrier that follows.
template <int TPR, int NV, typename S>
__device__ __forceinline__ void group_sum(S (&v)[NV], S *box) {
#pragma unroll
  for (int i = 0; i < NV; ++i) v[i] = wave_sum(v[i]);
  if constexpr (TPR > 64) {
    constexpr int W = TPR / 64;
    const int w = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int i = 0; i < NV; ++i) box[w * NV + i] = v[i];
    }
    __syncthreads();
    const S *g = box + w / W * W * NV;
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] = 0;
#pragma unroll
    for (int k = 0; k < W; ++k)
#pragma unroll
      for (int i = 0; i < NV; ++i) v[i] += g[k * NV + i];
  }
}

}  // namespace
}  // namespace pf
