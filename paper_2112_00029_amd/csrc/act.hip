// Backward of the layer's epilogue: dY_pre = dY o act'(Y_pre) and the bias
// gradient, its column sums, in one pass over T x N.
//
// Every element is read twice and written once (read once for PF_ACT_NONE) with
// ten to thirty VALU instructions on it.  A thread owns one 16-byte column chunk and
// walks down the rows of its workgroup's part, eight fp32 sums (four for fp32 data) in
// registers; a workgroup is `cw` chunks wide and 256 / cw rows tall, its rows' sums are
// added through LDS in row order, and the parts of the token range leave one fp32 row
// of N sums each, which a second launch adds in part order.  Deterministic: no
// atomics.  16384 x 16384 GELU: 309 us, 5.2 TB/s (a large copy: 4.86), bound by
// memory; 2100 x 4096: 10.7 + 3.9 us, one round of workgroups and a second launch.
// Measured and not kept: two rows per step (319 -> 363 us).
//
// dY_pre goes past the caches when it is larger than they are (256 MiB): 16384 x 16384
// 319 -> 309 us, with the backward-data that reads it next 942 -> 936; smaller ones
// stay for that call (8192 x 4096 both calls 97 us, streamed 101; 2100 x 4096 51, 53).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "pf_act.h"
#include "pf_dma.h"
#include "pf_launch.h"

namespace pf {
namespace {

// 16 bytes <-> floats.
__device__ __forceinline__ void get16(const float *p, float (&v)[4]) {
  const f32x4 x = *(const f32x4 *)p;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = x[e];
}
__device__ __forceinline__ void get16(const bf16_t *p, float (&v)[8]) {
  const u32x4 x = *(const u32x4 *)p;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    v[2 * e] = __uint_as_float(x[e] << 16);
    v[2 * e + 1] = __uint_as_float(x[e] & 0xffff0000u);
  }
}
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)lo) |
         ((uint32_t)__builtin_bit_cast(uint16_t, (__bf16)hi) << 16);
}
__device__ __forceinline__ f32x4 words(const float (&v)[4]) { return f32x4{v[0], v[1], v[2], v[3]}; }
__device__ __forceinline__ u32x4 words(const float (&v)[8]) {
  return u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]),
               pack_bf16x2(v[6], v[7])};
}
__device__ __forceinline__ void put1(float *p, float v) { *p = v; }
__device__ __forceinline__ void put1(bf16_t *p, float v) {
  *p = __builtin_bit_cast(uint16_t, (__bf16)v);
}

// STREAM: a variant, not a branch, whose two stores the compiler would join.
template <typename T, bool STREAM>
__global__ __launch_bounds__(256) void act_bwd_kernel(ActBwdArgs a) {
  constexpr int V = 16 / sizeof(T);
  __shared__ float red[256 * V];
  const int cw = a.cw, rows = 256 / cw;
  const int ci = threadIdx.x % cw, ri = threadIdx.x / cw;
  const int grp = blockIdx.x % a.groups, part = blockIdx.x / a.groups;
  const int64_t chunk = (int64_t)grp * cw + ci;
  const bool live = chunk * V < a.N;
  const int64_t t0 = (int64_t)part * a.rows_per_part, t1 = min(a.T, t0 + a.rows_per_part);
  const T *dY = (const T *)a.dY + chunk * V, *Z = (const T *)a.Z + chunk * V;
  T *dZ = (T *)a.dZ + chunk * V;
  float sum[V];
#pragma unroll
  for (int e = 0; e < V; ++e) sum[e] = 0.f;
  if (live) {
    for (int64_t t = t0 + ri; t < t1; t += rows) {
      float d[V];
      get16(dY + t * a.N, d);
      if (a.act != kActNone) {
        float z[V];
        get16(Z + t * a.N, z);
        act_grad_apply<T>(a.act, d, z);
        const auto x = words(d);
        auto *p = (decltype(words(d)) *)(dZ + t * a.N);
        if constexpr (STREAM) __builtin_nontemporal_store(x, p);
        else *p = x;
      }
#pragma unroll
      for (int e = 0; e < V; ++e) sum[e] += d[e];
    }
  }
  if (!a.partials && !a.dbias) return;
#pragma unroll
  for (int e = 0; e < V; ++e) red[(ri * cw + ci) * V + e] = sum[e];
  __syncthreads();
  // Columns of the workgroup, summed over its rows in row order.
  for (int c = threadIdx.x; c < cw * V; c += 256) {
    const int64_t col = (int64_t)grp * cw * V + c;
    if (col >= a.N) continue;
    float s = 0.f;
    for (int r = 0; r < rows; ++r) s += red[r * cw * V + c];
    if (a.partials) a.partials[part * a.N + col] = s;
    else put1((T *)a.dbias + col, s);
  }
}

// dbias[c] = sum over the parts, in a fixed order: a workgroup takes 16 columns,
// 16 threads a column every 16th part each.
template <typename T>
__global__ __launch_bounds__(256) void act_dbias_kernel(const float *P, int nparts, int64_t N, T *dbias) {
  __shared__ float red[256];
  const int64_t col = (int64_t)blockIdx.x * 16 + (threadIdx.x & 15);
  const int q = threadIdx.x >> 4;
  float s = 0.f;
#pragma unroll 4
  for (int p = q; p < nparts; p += 16) s += P[(int64_t)p * N + col];
  red[threadIdx.x] = s;
  __syncthreads();
  if (q) return;
  for (int p = 1; p < 16; ++p) s += red[p * 16 + threadIdx.x];
  put1(dbias + col, s);
}

}  // namespace

hipError_t launch_act_bwd(int dtype, const ActBwdArgs &a, hipStream_t s) {
  const int64_t grid = (int64_t)a.groups * a.nparts;
  if (grid <= 0 || grid > 0x7fffffff || a.cw < 1 || a.cw > 64 || 256 % a.cw) return hipErrorInvalidValue;
  auto go = [&](auto kernel) { launch_kernel(kernel, dim3((unsigned)grid), dim3(256), s, a); };
  if (dtype == 0) a.stream ? go(act_bwd_kernel<bf16_t, true>) : go(act_bwd_kernel<bf16_t, false>);
  else a.stream ? go(act_bwd_kernel<float, true>) : go(act_bwd_kernel<float, false>);
  return hipGetLastError();
}

hipError_t launch_act_dbias(int dtype, const ActBwdArgs &a, hipStream_t s) {
  const int64_t grid = a.N / 16;  // N is a multiple of 32
  if (grid > 0x7fffffff) return hipErrorInvalidValue;
  if (dtype == 0)
    launch_kernel(act_dbias_kernel<bf16_t>, dim3((unsigned)grid), dim3(256), s,
                  (const float *)a.partials, a.nparts, a.N, (bf16_t *)a.dbias);
  else
    launch_kernel(act_dbias_kernel<float>, dim3((unsigned)grid), dim3(256), s,
                  (const float *)a.partials, a.nparts, a.N, (float *)a.dbias);
  return hipGetLastError();
}

}  // namespace pf
