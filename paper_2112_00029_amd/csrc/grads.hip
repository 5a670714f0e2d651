// Norm over all gradients of a model and their scaling to at most a given norm.
//
// The gradients are cut into chunks of kGradChunk elements (a table the plan
// holds); a workgroup takes every gridDim-th chunk.  Each pass is bound by memory:
// one read for the norm, one read and one write for the scaling.  Squares are
// summed in 64 bits, so no finite gradient overflows or vanishes: a conversion and
// a multiply-add per element, a quarter of the time the loads take.  Every
// workgroup leaves one sum; the scaling's workgroups each add those up (in one
// fixed order, so all find the same scale) instead of a launch of its own doing
// it.  The scaling walks the chunks backwards: what the norm read last may still
// lie in a cache.  Elements need no more than their own alignment (the hardware's
// 16-byte accesses take any address); a chunk's last elements are single.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "pf_io.h"
#include "pf_launch.h"

namespace pf {
namespace {

constexpr int GV = 8;  // elements per thread and step

template <typename T>
struct Grad8;
template <>
struct Grad8<bf16_t> {
  typedef unsigned int raw __attribute__((ext_vector_type(4), aligned(2)));
  raw x;
  __device__ __forceinline__ void load(const bf16_t *p) { x = *(const raw *)p; }
  __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[2 * e] = __uint_as_float(x[e] << 16);
      v[2 * e + 1] = __uint_as_float(x[e] & 0xffff0000u);
    }
  }
};
template <>
struct Grad8<float> {
  typedef float raw __attribute__((ext_vector_type(4), aligned(4)));
  raw x, y;
  __device__ __forceinline__ void load(const float *p) {
    x = *(const raw *)p;
    y = *(const raw *)(p + 4);
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = x[e];
      v[4 + e] = y[e];
    }
  }
};
__device__ __forceinline__ void put8(float *p, const float (&v)[8]) {
  typedef float raw __attribute__((ext_vector_type(4), aligned(4)));
  *(raw *)p = raw{v[0], v[1], v[2], v[3]};
  *(raw *)(p + 4) = raw{v[4], v[5], v[6], v[7]};
}
__device__ __forceinline__ void put8(bf16_t *p, const float (&v)[8]) {
  typedef unsigned int raw __attribute__((ext_vector_type(4), aligned(2)));
  const Raw<bf16_t, 8> r = pack<bf16_t, 8>(v);
  *(raw *)p = raw{r.x[0], r.x[1], r.x[2], r.x[3]};
}

__device__ __forceinline__ double block_sum(double x, double *box) {
#pragma unroll
  for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
  if ((threadIdx.x & 63) == 0) box[threadIdx.x >> 6] = x;
  __syncthreads();
  return (box[0] + box[1]) + (box[2] + box[3]);
}

// A whole chunk's elements, eight per thread and step; f(values, index) and, for
// the last n % 8, g(value, index).
template <typename T, typename F, typename G>
__device__ __forceinline__ void each(const T *p, int n, F f, G g) {
  constexpr int S = kGradChunk / (256 * GV);
  const int n8 = n / GV * GV;
  Grad8<T> x[S];
#pragma unroll
  for (int k = 0; k < S; ++k) {
    const int i = (k * 256 + (int)threadIdx.x) * GV;
    if (i < n8) x[k].load(p + i);
  }
#pragma unroll
  for (int k = 0; k < S; ++k) {
    const int i = (k * 256 + (int)threadIdx.x) * GV;
    if (i < n8) {
      float v[8];
      x[k].get(v);
      f(v, i);
    }
  }
  const int r = n8 + (int)threadIdx.x;
  if (r < n) g(up(p[r]), r);
}

__global__ __launch_bounds__(256) void grad_sumsq_kernel(GradArgs a) {
  __shared__ double box[4];
  double s0 = 0.0, s1 = 0.0;
  for (int c = blockIdx.x; c < a.nchunk; c += gridDim.x) {
    const GradChunk *k = a.chunks + c;
    const void *src = (const void *)ld_meta(&k->src);
    const int n = ld_meta(&k->n), types = ld_meta(&k->types);
    auto f = [&](const float (&v)[8], int) __attribute__((always_inline)) {
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        s0 = __builtin_fma((double)v[e], (double)v[e], s0);
        s1 = __builtin_fma((double)v[e + 1], (double)v[e + 1], s1);
      }
    };
    auto g = [&](float v, int) __attribute__((always_inline)) { s0 = __builtin_fma((double)v, (double)v, s0); };
    if (types & kGradSrcF32) each((const float *)src, n, f, g);
    else each((const bf16_t *)src, n, f, g);
  }
  const double s = block_sum(s0 + s1, box);
  if (threadIdx.x == 0) a.partials[blockIdx.x] = s;
}

// Total of the partials, the same in every thread of every workgroup.
__device__ __forceinline__ double total(const GradArgs &a, double *box) {
  double s = 0.0;
  for (int i = threadIdx.x; i < a.nparts; i += 256) s += a.partials[i];
  return block_sum(s, box);
}

__global__ __launch_bounds__(256) void grad_total_kernel(GradArgs a) {
  __shared__ double box[4];
  const double s = total(a, box);
  if (threadIdx.x) return;
  if (a.sumsq) *a.sumsq = s;
  if (a.norm) *a.norm = (float)sqrt(s);
}

__global__ __launch_bounds__(256) void grad_scale_kernel(GradArgs a) {
  __shared__ double box[4];
  const double s = total(a, box), norm = sqrt(s);
  if (a.norm && blockIdx.x == 0 && threadIdx.x == 0) *a.norm = (float)norm;
  // One if the norm is within the limit, or no number: then the caller sees it and
  // drops the step.
  const bool cut = norm > (double)a.max_norm && norm < __builtin_huge_val();
  const float scale = cut ? (float)((double)a.max_norm / norm) : 1.0f;
  for (int c = a.nchunk - 1 - (int)blockIdx.x; c >= 0; c -= gridDim.x) {
    const GradChunk *k = a.chunks + c;
    const void *src = (const void *)ld_meta(&k->src);
    void *dst = (void *)ld_meta(&k->dst);
    const int n = ld_meta(&k->n), types = ld_meta(&k->types);
    if (!cut && src == dst) continue;
    auto go = [&](auto *p, auto *q) __attribute__((always_inline)) {
      each(
          p, n,
          [&](const float (&v)[8], int i) __attribute__((always_inline)) {
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = v[e] * scale;
            put8(q + i, y);
          },
          [&](float v, int i) __attribute__((always_inline)) { down(q[i], v * scale); });
    };
    switch (types) {
      case 0: go((const bf16_t *)src, (bf16_t *)dst); break;
      case kGradSrcF32: go((const float *)src, (bf16_t *)dst); break;
      case kGradDstF32: go((const bf16_t *)src, (float *)dst); break;
      default: go((const float *)src, (float *)dst); break;
    }
  }
}

}  // namespace

hipError_t launch_grad_sumsq(const GradArgs &a, hipStream_t s) {
  launch_kernel(grad_sumsq_kernel, dim3((unsigned)a.nparts), dim3(256), s, a);
  return hipGetLastError();
}
hipError_t launch_grad_total(const GradArgs &a, hipStream_t s) {
  launch_kernel(grad_total_kernel, dim3(1), dim3(256), s, a);
  return hipGetLastError();
}
hipError_t launch_grad_scale(const GradArgs &a, int grid, hipStream_t s) {
  launch_kernel(grad_scale_kernel, dim3((unsigned)grid), dim3(256), s, a);
  return hipGetLastError();
}

}  // namespace pf
