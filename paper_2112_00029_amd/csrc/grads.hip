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
// lie in a cache, and stores go past the caches, which then hold more of it (289
// tensors of 298M elements, bf16 into fp32: 497 us with plain stores, 461 past the
// caches, 420 on four workgroups per CU instead of eight, 406 on three: 5.9 TB/s of
// two reads and a write; 44M elements 78, 58, 55, 56).  Elements need no more than
// their own alignment (the hardware's 16-byte accesses take any address); a chunk's
// last elements are single.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "pf_io.h"
#include "pf_launch.h"

namespace pf {
namespace {

// V elements as one access at any element's address: 16 bytes, or four bf16 that
// become (or were) 16 bytes of fp32, so that a wave's accesses are contiguous on both
// sides.
template <typename T, int V>
struct Grad;
template <>
struct Grad<bf16_t, 8> {
  typedef unsigned int raw __attribute__((ext_vector_type(4), aligned(2)));
};
template <>
struct Grad<bf16_t, 4> {
  typedef unsigned int raw __attribute__((ext_vector_type(2), aligned(2)));
};
template <>
struct Grad<float, 4> {
  typedef float raw __attribute__((ext_vector_type(4), aligned(4)));
};
template <int V, typename R>
__device__ __forceinline__ void get(const bf16_t *, const R &x, float (&v)[V]) {
#pragma unroll
  for (int e = 0; e < V / 2; ++e) {
    v[2 * e] = __uint_as_float(x[e] << 16);
    v[2 * e + 1] = __uint_as_float(x[e] & 0xffff0000u);
  }
}
template <int V, typename R>
__device__ __forceinline__ void get(const float *, const R &x, float (&v)[V]) {
#pragma unroll
  for (int e = 0; e < V; ++e) v[e] = x[e];
}
// NT: past the caches.
template <bool NT, int V>
__device__ __forceinline__ void put(float *p, const float (&v)[V]) {
  static_assert(V == 4, "16 bytes");
  typedef typename Grad<float, V>::raw raw;
  if constexpr (NT) __builtin_nontemporal_store(raw{v[0], v[1], v[2], v[3]}, (raw *)p);
  else *(raw *)p = raw{v[0], v[1], v[2], v[3]};
}
template <bool NT, int V>
__device__ __forceinline__ void put(bf16_t *p, const float (&v)[V]) {
  typename Grad<bf16_t, V>::raw r;
#pragma unroll
  for (int e = 0; e < V / 2; ++e)
    r[e] = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v[2 * e]) |
           ((uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v[2 * e + 1]) << 16);
  if constexpr (NT) __builtin_nontemporal_store(r, (typename Grad<bf16_t, V>::raw *)p);
  else *(typename Grad<bf16_t, V>::raw *)p = r;
}

// A chunk's addresses come out of memory: said to be global, they take global (not
// flat) accesses.
template <typename T>
__device__ __forceinline__ T *global_ptr(uint64_t x) {
  return (T *)(__attribute__((address_space(1))) T *)x;
}

__device__ __forceinline__ double block_sum(double x, double *box) {
#pragma unroll
  for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
  if ((threadIdx.x & 63) == 0) box[threadIdx.x >> 6] = x;
  __syncthreads();
  return (box[0] + box[1]) + (box[2] + box[3]);
}

// A whole chunk's elements, V per thread and step: all are loaded, then
// between() runs, then f(values, index) and, for the last n % V, g(value, index).
template <int V, typename T, typename B, typename F, typename G>
__device__ __forceinline__ void each(const T *p, int n, B between, F f, G g) {
  constexpr int S = kGradChunk / (256 * V);
  const int nv = n / V * V;
  typename Grad<T, V>::raw x[S];
#pragma unroll
  for (int k = 0; k < S; ++k) {
    const int i = (k * 256 + (int)threadIdx.x) * V;
    if (i < nv) x[k] = *(const typename Grad<T, V>::raw *)(p + i);
  }
  between();
#pragma unroll
  for (int k = 0; k < S; ++k) {
    const int i = (k * 256 + (int)threadIdx.x) * V;
    if (i < nv) {
      float v[V];
      get<V>(p, x[k], v);
      f(v, i);
    }
  }
  const int r = nv + (int)threadIdx.x;
  if (r < n) g(up(p[r]), r);
}

__global__ __launch_bounds__(256) void grad_sumsq_kernel(GradArgs a) {
  __shared__ double box[4];
  double s0 = 0.0, s1 = 0.0;
  for (int c = blockIdx.x; c < a.nchunk; c += gridDim.x) {
    const GradChunk *k = a.chunks + c;
    const uint64_t src = ld_meta(&k->src);
    const int n = ld_meta(&k->n), types = ld_meta(&k->types);
    auto f = [&](const auto &v, int) __attribute__((always_inline)) {
#pragma unroll
      for (int e = 0; e < (int)(sizeof(v) / sizeof(float)); e += 2) {
        s0 = __builtin_fma((double)v[e], (double)v[e], s0);
        s1 = __builtin_fma((double)v[e + 1], (double)v[e + 1], s1);
      }
    };
    auto g = [&](float v, int) __attribute__((always_inline)) { s0 = __builtin_fma((double)v, (double)v, s0); };
    auto no = [] {};
    if (types & kGradSrcF32) each<4>(global_ptr<const float>(src), n, no, f, g);
    else each<8>(global_ptr<const bf16_t>(src), n, no, f, g);
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

template <bool NT>
__global__ __launch_bounds__(256) void grad_scale_kernel(GradArgs a) {
  __shared__ double box[4];
  bool cut = false, known = false;
  float scale = 1.0f, pre = 1.0f;
  // The first chunk's loads are on their way before the total is formed (13 tensors of
  // 1.4M elements, whole call: 7.7 -> 7.4 us).
  auto settle = [&]() __attribute__((always_inline)) {
    if (known) return;
    known = true;
    const double norm = sqrt(total(a, box));
    if (a.norm && blockIdx.x == 0 && threadIdx.x == 0) *a.norm = (float)norm;
    // One if the norm is within the limit, or no number: then the caller sees it and
    // drops the step.
    cut = norm > (double)a.max_norm && norm < __builtin_huge_val();
    double s = cut ? (double)a.max_norm / norm : 1.0;
    // A factor near fp32's smallest takes two, the first a power of two: gradients that
    // it would cost digits vanish by the second.
    if (s < 0x1p-100) {
      pre = 0x1p-64f;
      s *= 0x1p64;
    }
    scale = (float)s;
  };
  for (int c = a.nchunk - 1 - (int)blockIdx.x; c >= 0; c -= gridDim.x) {
    const GradChunk *k = a.chunks + c;
    const uint64_t src = ld_meta(&k->src), dst = ld_meta(&k->dst);
    const int n = ld_meta(&k->n), types = ld_meta(&k->types);
    if (known && !cut && src == dst) continue;
    auto go = [&](auto *p, auto *q) __attribute__((always_inline)) {
      constexpr int V = sizeof(*p) + sizeof(*q) == 4 ? 8 : 4;
      each<V>(
          p, n, settle,
          [&](const float (&v)[V], int i) __attribute__((always_inline)) {
            if (!cut && src == dst) return;
            float y[V];
#pragma unroll
            for (int e = 0; e < V; ++e) y[e] = v[e] * pre * scale;
            put<NT, V>(q + i, y);
          },
          [&](float v, int i) __attribute__((always_inline)) {
            if (cut || src != dst) down(q[i], v * pre * scale);
          });
    };
    switch (types) {
      case 0: go(global_ptr<const bf16_t>(src), global_ptr<bf16_t>(dst)); break;
      case kGradSrcF32: go(global_ptr<const float>(src), global_ptr<bf16_t>(dst)); break;
      case kGradDstF32: go(global_ptr<const bf16_t>(src), global_ptr<float>(dst)); break;
      default: go(global_ptr<const float>(src), global_ptr<float>(dst)); break;
    }
  }
  settle();  // (a list without elements: the norm is still due)
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
  if (a.stream) launch_kernel(grad_scale_kernel<true>, dim3((unsigned)grid), dim3(256), s, a);
  else launch_kernel(grad_scale_kernel<false>, dim3((unsigned)grid), dim3(256), s, a);
  return hipGetLastError();
}

}  // namespace pf
