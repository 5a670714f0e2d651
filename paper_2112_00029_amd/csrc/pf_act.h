// Activations of the layer's epilogue and their derivatives, chosen by a
// launch argument (uniform over a launch).
//
//   gelu       x Phi(x)                      Phi(x) + x phi(x)
//   gelu_tanh  x s(y), y = 2 k (x + c x^3),  s + x s (1 - s) y',
//              k = sqrt(2 / pi), c = 0.044715   y' = 2 k (1 + 3 c x^2)
//   silu       x s(x)                        s + x s (1 - s)
//   relu       x for x > 0, else 0           1 for x > 0, else 0
// s(y) = 1 / (1 + exp(-y)); 0.5 (1 + tanh(y / 2)) is the same number.  Where 1 - s
// is needed too, both come from e = exp(-|y|), r = 1 / (1 + e): r and e r, whichever
// side, so that neither cancels or overflows.
// bf16 results take the hardware exponential and reciprocal (1 ulp each: far below
// their own rounding); fp32 results take the library's functions, and for GELU the
// forms of pf_gelu.h, which keep their digits in the negative tail: x (1 + erf(x / sqrt
// 2)) / 2 is 4 % off at -5 and zero from -5.6.
#pragma once

#include <hip/hip_runtime.h>

#include "pf_gelu.h"
#include "pf_internal.h"

namespace pf {
namespace {

// s = s(y), c = 1 - s(y).
template <typename T>
__device__ __forceinline__ void act_sigmoid(float y, float &s, float &c) {
  float e, r;
  if constexpr (sizeof(T) == 2) {
    e = __builtin_amdgcn_exp2f(fabsf(y) * -1.4426950408889634f);
    r = __builtin_amdgcn_rcpf(1.0f + e);
  } else {
    e = expf(-fabsf(y));
    r = 1.0f / (1.0f + e);
  }
  const float er = e * r;
  s = y < 0.f ? er : r;
  c = y < 0.f ? r : er;
}

constexpr float kTanh2k = 1.5957691216057308f;  // 2 sqrt(2 / pi)
constexpr float kTanhC = 0.044715f;

// s(y) alone, of y = -log2(e) y2 for bf16 results.
__device__ __forceinline__ float sigmoid2(float y2) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(y2));
}

// Phi(-a), a >= 0, for bf16 results: the exponential of a polynomial.  log2 Phi(-a)
// is smooth: one of degree 7 (fitted here over a <= 7 to the largest error, its
// leading coefficient negative, so that the tail goes on falling beyond) leaves it
// within 1.2e-5 of itself up to a = 7, a three-hundredth of half a bf16 step; past 7
// it is below 1.3e-12 and the fit falls faster than it does.
__device__ __forceinline__ float normal_tail_bf16(float a) {
  float q = -1.58825458e-06f;
  q = __builtin_fmaf(q, a, 5.61542814e-05f);
  q = __builtin_fmaf(q, a, -0.00088322388f);
  q = __builtin_fmaf(q, a, 0.00830325577f);
  q = __builtin_fmaf(q, a, -0.0535013936f);
  q = __builtin_fmaf(q, a, -0.458964258f);
  q = __builtin_fmaf(q, a, -1.15103567f);
  q = __builtin_fmaf(q, a, -1.00001395f);
  return __builtin_amdgcn_exp2f(q);
}
// GELU for bf16 results: max(x, 0) - |x| Phi(-|x|).  The epilogue has nothing to
// overlap with, so its instructions are time: 16384 x 4096 -> 16384 with
// pre-activations 801 us with pf_gelu.h's form (6e-8 of the CDF, 30 issue slots), 771
// with a reciprocal and a polynomial of degree 4 (21), 697 - 719 so (15; boxes
// differ).
__device__ __forceinline__ float gelu_bf16(float x) {
  // Keeps a * tail finite (one instruction; fminf quiets NaNs first).
  const float a = fabsf(__builtin_amdgcn_fmed3f(x, -1e4f, 1e4f));
  return __builtin_fmaf(-a, normal_tail_bf16(a), x < 0.f ? 0.f : x);
}
// Its derivative, Phi(x) + x phi(x), within 7e-6: the way back of 16384 x 16384 takes
// 319 us so (memory), 334 with pf_gelu.h's form (82 % of the issue slots).
__device__ __forceinline__ float gelu_grad_bf16(float x) {
  const float tail = normal_tail_bf16(fabsf(x));
  const float e = __builtin_amdgcn_exp2f(x * x * -0.72134752f);
  return __builtin_fmaf(x * 0.39894228040143268f, e, x < 0.f ? tail : 1.0f - tail);
}

template <typename T>
__device__ __forceinline__ float act_gelu(float x) {
  if constexpr (sizeof(T) == 2) return gelu_bf16(x);
  else return gelu_fast(x);
}
template <typename T>
__device__ __forceinline__ float act_gelu_grad(float x) {
  if constexpr (sizeof(T) == 2) return gelu_grad_bf16(x);
  else return gelu_grad_fast(x);
}
template <typename T>
__device__ __forceinline__ float act_gelu_tanh(float x) {
  if constexpr (sizeof(T) == 2) {
    constexpr float A = -1.4426950408889634f * kTanh2k;
    return x * sigmoid2(x * __builtin_fmaf(A * kTanhC, x * x, A));
  } else {
    return x * (1.0f / (1.0f + expf(-kTanh2k * __builtin_fmaf(kTanhC * x, x * x, x))));
  }
}
template <typename T>
__device__ __forceinline__ float act_gelu_tanh_grad(float x) {
  // Beyond |x| = 16, s (1 - s) is below 1e-125: the clamp only keeps the
  // square finite.
  const float z = fminf(fmaxf(x, -16.f), 16.f), z2 = z * z;
  float s, c;
  act_sigmoid<T>(kTanh2k * __builtin_fmaf(kTanhC * z, z2, z), s, c);
  const float g = __builtin_fmaf(z * s * c, kTanh2k * __builtin_fmaf(3 * kTanhC, z2, 1.0f), s);
  return x != x ? x : g;
}
template <typename T>
__device__ __forceinline__ float act_silu(float x) {
  if constexpr (sizeof(T) == 2) return x * sigmoid2(x * -1.4426950408889634f);
  else return x * (1.0f / (1.0f + expf(-x)));
}
template <typename T>
__device__ __forceinline__ float act_silu_grad(float x) {
  float s, c;
  act_sigmoid<T>(x, s, c);
  return __builtin_fmaf(x * c, s, s);
}

// v[i] = act(v[i]); T: the type the results are stored in.
template <typename T, int N>
__device__ __forceinline__ void act_apply(int act, float (&v)[N]) {
  switch (act) {
    case kActGelu:
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = act_gelu<T>(v[e]);
      break;
    case kActGeluTanh:
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = act_gelu_tanh<T>(v[e]);
      break;
    case kActSilu:
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = act_silu<T>(v[e]);
      break;
    case kActRelu:
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = v[e] < 0.f ? 0.f : v[e];
      break;
    default: break;
  }
}

// f[i] = act(x[i]), d[i] = act'(x[i]); the two share their exponentials.
template <typename T>
__device__ __forceinline__ void act_sigmoid_both(float x, float y, float dy, float &f, float &d) {
  float s, c;
  act_sigmoid<T>(y, s, c);
  f = x * s;
  d = __builtin_fmaf(x * s * c, dy, s);
}
template <typename T, int N>
__device__ __forceinline__ void act_both(int act, const float (&x)[N], float (&f)[N], float (&d)[N]) {
  switch (act) {
    case kActGelu:
#pragma unroll
      for (int e = 0; e < N; ++e) {
        if constexpr (sizeof(T) == 2) {
          const float v = x[e], a = fabsf(__builtin_amdgcn_fmed3f(v, -1e4f, 1e4f));
          const float tail = normal_tail_bf16(a);
          f[e] = __builtin_fmaf(-a, tail, v < 0.f ? 0.f : v);
          d[e] = __builtin_fmaf(v * 0.39894228040143268f, __builtin_amdgcn_exp2f(v * v * -0.72134752f),
                                v < 0.f ? tail : 1.0f - tail);
        } else {
          f[e] = act_gelu<T>(x[e]);
          d[e] = act_gelu_grad<T>(x[e]);
        }
      }
      break;
    case kActGeluTanh:
#pragma unroll
      for (int e = 0; e < N; ++e) {
        if constexpr (sizeof(T) == 2) {
          // (The clamp as in act_gelu_tanh_grad; s has its limits there.  The median
          // of a NaN is a bound: NaN is put back.)
          const float v = x[e], z = __builtin_amdgcn_fmed3f(v, -16.f, 16.f), z2 = z * z;
          float s, c;
          act_sigmoid<T>(kTanh2k * __builtin_fmaf(kTanhC * z, z2, z), s, c);
          f[e] = v * s;
          d[e] = __builtin_fmaf(z * s * c, kTanh2k * __builtin_fmaf(3 * kTanhC, z2, 1.0f), s);
          if (v != v) d[e] = v;
        } else {
          f[e] = act_gelu_tanh<T>(x[e]);
          d[e] = act_gelu_tanh_grad<T>(x[e]);
        }
      }
      break;
    case kActSilu:
#pragma unroll
      for (int e = 0; e < N; ++e) act_sigmoid_both<T>(x[e], x[e], 1.0f, f[e], d[e]);
      break;
    case kActRelu:
#pragma unroll
      for (int e = 0; e < N; ++e) {
        f[e] = x[e] < 0.f ? 0.f : x[e];
        d[e] = x[e] > 0.f ? 1.f : 0.f;
      }
      break;
    default:
#pragma unroll
      for (int e = 0; e < N; ++e) {
        f[e] = x[e];
        d[e] = 1.f;
      }
      break;
  }
}

// v[i] *= act'(x[i]).
template <typename T, int N>
__device__ __forceinline__ void act_grad_apply(int act, float (&v)[N], const float (&x)[N]) {
  switch (act) {
    case kActGelu:
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] *= act_gelu_grad<T>(x[e]);
      break;
    case kActGeluTanh:
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] *= act_gelu_tanh_grad<T>(x[e]);
      break;
    case kActSilu:
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] *= act_silu_grad<T>(x[e]);
      break;
    case kActRelu:
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = x[e] > 0.f ? v[e] : 0.f;
      break;
    default: break;
  }
}

}  // namespace
}  // namespace pf
