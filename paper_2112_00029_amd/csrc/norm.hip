// Layer normalisation of token rows, forward and backward.
//
//   n = (x - mean) rstd,  rstd = 1 / sqrt(mean((x - mean)^2) + eps)
//   y = n o w + b
//   dx = rstd (g - mean(g) - n mean(g o n)) + dR,  g = dy o w
//   dw = column sums of dy o n,  db = column sums of dy
//
// Every element is read once and written once (the backward reads two or three
// tensors): memory is the bound.  A row lives in the registers of TPR threads, 16
// elements each (32 for the backward's longest rows) or fewer, so that mean, variance
// and output need no second read; the sums cross the wave by DPP and the waves of a
// row through LDS, one barrier a sum.  Rows of at most 1024 elements take one wave and
// no barrier.  A workgroup
// walks over rows (its weights stay in registers, and in the backward its fp32
// sums of dw and db); the next row's loads are issued before the present row is
// worked on.  The backward's workgroups leave their sums as one row of fp32
// partials each, added in order by a second launch: no atomics, so the same call
// gives the same bits.  16384 x 4096 in bf16: forward 48.9 us, 5.5 TB/s, backward with an
// added gradient 109 us, 4.9 TB/s (a large copy: 4.9); 2509 x 768 backward 8 us and 4
// for the partials, launches more than memory.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "pf_io.h"
#include "pf_launch.h"

namespace pf {
namespace {

// A row's chunk from column col on lies at `from`.  Where V does not divide N (TAIL),
// the last chunk is the row's last V elements, of which those before `first` belong to
// the chunk before: they are taken as zeros and not stored.  (Odd widths and strides by
// single elements instead: backward of 184 rows of 9056, 9065 apart, 39 us for what
// takes 18.  With the zeros put in as the chunk is loaded, the next row's loads were
// waited for at once: 10543 x 323 21.5 us, 15.4 so; 320 columns take 13.6.)
template <int V, bool TAIL>
__device__ __forceinline__ int from(int col, int N) {
  return TAIL ? min(col, N - V) : col;
}
template <int V, bool TAIL>
__device__ __forceinline__ int first(int col, int N) {  // V: past the row
  if constexpr (TAIL) return min(max(col - (N - V), 0), V);
  else return col < N ? 0 : V;
}
// A row's raw chunks of this thread: chunk c covers columns (c TPR + i) V ...
template <typename T, int V, int C, int TPR, bool TAIL>
__device__ __forceinline__ void load_row(const T *p, int N, int i, Raw<T, V> (&r)[C]) {
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int col = (c * TPR + i) * V;
    r[c] = col < N ? ld_raw<T, V>(p + from<V, TAIL>(col, N)) : zero_raw<T, V>();
  }
}
// A chunk's values, zero before the k-th.
template <typename T, int V, bool TAIL>
__device__ __forceinline__ void values(const Raw<T, V> &r, int k, float (&v)[V]) {
  unpack<T, V>(r, v);
  if constexpr (TAIL) {
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = e < k ? 0.f : v[e];
  }
}
// A chunk to its place.
template <typename T, int V, bool TAIL>
__device__ __forceinline__ void store_chunk(T *p, int N, int col, const float (&v)[V]) {
  const int k = first<V, TAIL>(col, N);
  if (k == 0) {
    st_raw<T, V>(p + col, pack<T, V>(v));
  } else if (TAIL && k < V) {
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (e >= k) down(p[N - V + e], v[e]);
  }
}

template <typename T, int V, int C, int TPR, bool TAIL>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void norm_fwd_kernel(NormArgs a) {
  constexpr auto load = load_row<T, V, C, TPR, TAIL>;
  constexpr int BT = TPR < 256 ? 256 : TPR, RPB = BT / TPR;  // threads, rows at a time
  __shared__ double dbox[BT / 64];
  __shared__ float box[BT / 64];
  const int i = threadIdx.x % TPR, slot = threadIdx.x / TPR;
  const int N = (int)a.N;
  const T *X = (const T *)a.X;
  T *Y = (T *)a.Y;
  const double inv = 1.0 / (double)N;
  Raw<T, V> w[C], b[C];
  if (a.weight) load((const T *)a.weight, N, i, w);
  if (a.bias) load((const T *)a.bias, N, i, b);
  const int64_t step = (int64_t)gridDim.x * RPB;
  Raw<T, V> x[C], nx[C];
  int64_t t = (int64_t)blockIdx.x * RPB + slot;
  if (t < a.T) load(X + t * a.ldx, N, i, x);
  for (int64_t t0 = (int64_t)blockIdx.x * RPB; t0 < a.T; t0 += step, t += step) {
    const bool live = t < a.T;
    if (t + step < a.T) load(X + (t + step) * a.ldx, N, i, nx);
    // The mean from a sum in 64 bits, as m0 + m1: rows far from zero keep the digits of
    // their differences, and a mean near zero its own (16384 x 4096: off by 2.6e-8 of the
    // means' size, a rounding; the 64-bit sums cost no time there, 48.2 and 48.5 us).
    double sum[1] = {0.0};
    float d[C][V], sq[1] = {0.f};
#pragma unroll
    for (int c = 0; c < C; ++c) {
      values<T, V, TAIL>(x[c], first<V, TAIL>((c * TPR + i) * V, N), d[c]);
#pragma unroll
      for (int e = 0; e < V; ++e) sum[0] += (double)d[c][e];
    }
    group_sum<TPR, 1>(sum, dbox);
    const double mean = sum[0] * inv;
    const float m0 = (float)mean, m1 = (float)(mean - (double)m0);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int k = first<V, TAIL>((c * TPR + i) * V, N);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        d[c][e] = (TAIL ? e >= k : k == 0) ? (d[c][e] - m0) - m1 : 0.f;
        sq[0] = __builtin_fmaf(d[c][e], d[c][e], sq[0]);
      }
    }
    group_sum<TPR, 1>(sq, box);
    const float rstd = 1.0f / sqrtf(sq[0] * (float)inv + a.eps);
    if (live) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int col = (c * TPR + i) * V;
        float y[V], f[V];
#pragma unroll
        for (int e = 0; e < V; ++e) y[e] = d[c][e] * rstd;
        if (a.weight) {
          unpack<T, V>(w[c], f);
#pragma unroll
          for (int e = 0; e < V; ++e) y[e] *= f[e];
        }
        if (a.bias) {
          unpack<T, V>(b[c], f);
#pragma unroll
          for (int e = 0; e < V; ++e) y[e] += f[e];
        }
        store_chunk<T, V, TAIL>(Y + t * a.ldy, N, col, y);
      }
      if (i == 0) {
        if (a.mean) a.mean[t] = m0;
        if (a.rstd) a.rstd[t] = rstd;
      }
    }
#pragma unroll
    for (int c = 0; c < C; ++c) x[c] = nx[c];
  }
}

template <typename T, int V, int C, int TPR, bool TAIL>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void norm_bwd_kernel(NormArgs a) {
  constexpr auto load = load_row<T, V, C, TPR, TAIL>;
  constexpr int BT = TPR < 256 ? 256 : TPR, RPB = BT / TPR;
  __shared__ float box[2][2 * (BT / 64)];
  __shared__ float red[RPB > 1 ? (RPB - 1) * TPR * V * C : 1];
  const int i = threadIdx.x % TPR, slot = threadIdx.x / TPR;
  const int N = (int)a.N;
  const T *X = (const T *)a.X, *dY = (const T *)a.dY, *dR = (const T *)a.dR;
  T *dX = (T *)a.dX;
  const float inv = 1.0f / (float)N;
  Raw<T, V> w[C];
  if (a.weight) load((const T *)a.weight, N, i, w);
  float dw[C][V] = {}, db[C][V] = {};
  const int64_t step = (int64_t)gridDim.x * RPB;
  // (32 elements a thread leave no registers for a second row.)
  constexpr bool AHEAD = V * C <= 16;
  Raw<T, V> x[C], g[C], nx[C], ng[C];
  float mean = 0.f, rstd = 0.f, nmean = 0.f, nrstd = 0.f;
  int64_t t = (int64_t)blockIdx.x * RPB + slot;
  auto fetch = [&](int64_t r, Raw<T, V> (&xx)[C], Raw<T, V> (&gg)[C], float &m, float &s)
                   __attribute__((always_inline)) {
    load(X + r * a.ldx, N, i, xx);
    load(dY + r * a.lddy, N, i, gg);
    m = a.mean_in[r];
    s = a.rstd_in[r];
  };
  if (AHEAD && t < a.T) fetch(t, x, g, mean, rstd);
  int buf = 0;
  for (int64_t t0 = (int64_t)blockIdx.x * RPB; t0 < a.T; t0 += step, t += step) {
    const bool live = t < a.T;
    if (!AHEAD && live) fetch(t, x, g, mean, rstd);
    if (AHEAD && t + step < a.T) fetch(t + step, nx, ng, nmean, nrstd);
    Raw<T, V> r[C];
    if (dR && live) load(dR + t * a.lddr, N, i, r);
    float s[2] = {0.f, 0.f};
    // n of a chunk (zero past the row) and dy; formed again after the sums, which
    // costs less than the registers that would keep them.
    auto norm_of = [&](int c, float (&n)[V], float (&q)[V]) __attribute__((always_inline)) {
      const int k = first<V, TAIL>((c * TPR + i) * V, N);
      unpack<T, V>(x[c], n);
      values<T, V, TAIL>(g[c], k, q);
#pragma unroll
      for (int e = 0; e < V; ++e) n[e] = (TAIL ? e >= k : k == 0) ? (n[e] - mean) * rstd : 0.f;
    };
    if (live) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        float n[V], q[V], f[V];
        norm_of(c, n, q);
        if (a.weight) unpack<T, V>(w[c], f);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          dw[c][e] = __builtin_fmaf(q[e], n[e], dw[c][e]);
          db[c][e] += q[e];
          if (a.weight) q[e] *= f[e];
          s[0] += q[e];
          s[1] = __builtin_fmaf(q[e], n[e], s[1]);
        }
      }
    }
    // Boxes in turn: a group writes one while others still read the last.
    group_sum<TPR, 2>(s, box[buf]);
    buf ^= 1;
    if (live) {
      const float c1 = s[0] * inv, c2 = s[1] * inv;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int col = (c * TPR + i) * V;
        float n[V], y[V], f[V];
        norm_of(c, n, y);
        if (a.weight) unpack<T, V>(w[c], f);
#pragma unroll
        for (int e = 0; e < V; ++e)
          y[e] = rstd * ((a.weight ? y[e] * f[e] : y[e]) - __builtin_fmaf(n[e], c2, c1));
        if (dR) {
          unpack<T, V>(r[c], f);
#pragma unroll
          for (int e = 0; e < V; ++e) y[e] += f[e];
        }
        store_chunk<T, V, TAIL>(dX + t * a.lddx, N, col, y);
      }
    }
    if constexpr (AHEAD) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        x[c] = nx[c];
        g[c] = ng[c];
      }
      mean = nmean;
      rstd = nrstd;
    }
  }
  // The workgroup's sums: its row slots in order, dw then db; to the partials, or the
  // one workgroup of few rows to the results themselves.
  auto leave = [&](float (&v)[C][V], float *part, T *out, bool second) __attribute__((always_inline)) {
    if constexpr (RPB > 1) {
      if (second) __syncthreads();
      if (slot) {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int e = 0; e < V; ++e) red[(((slot - 1) * C + c) * V + e) * TPR + i] = v[c][e];
      }
      __syncthreads();
      if (slot) return;
#pragma unroll
      for (int k = 0; k < RPB - 1; ++k)
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int e = 0; e < V; ++e) v[c][e] += red[((k * C + c) * V + e) * TPR + i];
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = (c * TPR + i) * V;
      if (col >= N) continue;
      if (part) {
        const int k = first<V, TAIL>(col, N);
#pragma unroll
        for (int e = 0; e < V; ++e)
          if (!TAIL || e >= k) part[from<V, TAIL>(col, N) + e] = v[c][e];
      } else if (out) {
        store_chunk<T, V, TAIL>(out, N, col, v[c]);
      }
    }
  };
  if (!a.partials && (gridDim.x > 1 || (!a.dweight && !a.dbias))) return;
  float *P = a.partials ? a.partials + (int64_t)blockIdx.x * 2 * N : nullptr;
  leave(dw, P, (T *)a.dweight, false);
  leave(db, P ? P + N : P, (T *)a.dbias, true);
}

// Column sums of the partials [parts][2 N] into dw and db: 16 columns a workgroup,
// 64 threads a column every 64th part each, added in order.
template <typename T>
__global__ __launch_bounds__(1024) void norm_sum_kernel(NormArgs a) {
  __shared__ float red[16 * 16];
  const int64_t col = (int64_t)blockIdx.x * 16 + (threadIdx.x & 15), n2 = 2 * a.N;
  const int q = threadIdx.x >> 4, w = threadIdx.x >> 6;
  float s = 0.f;
  if (col < n2) {
#pragma unroll 4
    for (int p = q; p < a.parts; p += 64) s += a.partials[(int64_t)p * n2 + col];
  }
  s += __shfl_xor(s, 16);
  s += __shfl_xor(s, 32);
  if ((threadIdx.x & 63) < 16) red[w * 16 + (threadIdx.x & 15)] = s;
  __syncthreads();
  if (q || col >= n2) return;
  s = 0.f;
#pragma unroll
  for (int k = 0; k < 16; ++k) s += red[k * 16 + threadIdx.x];
  T *out = (T *)(col < a.N ? a.dweight : a.dbias);
  if (out) down(out[col < a.N ? col : col - a.N], s);
}

// f(V, C, TPR, TAIL) of a plan (capi_train.cpp): one of norm_plan_exists.
template <typename T, bool BACK, typename F>
bool norm_pick(const NormArgs &a, F f) {
  constexpr int VW = 16 / sizeof(T);
  if (a.N < VW) {  // (single elements)
    if (a.tpr != 64) return false;
    f(std::integral_constant<int, 1>{}, std::integral_constant<int, 1>{}, std::integral_constant<int, 64>{},
      std::false_type{});
    return true;
  }
  if ((int64_t)a.tpr * a.chunks * VW < a.N) return false;
  auto tpr = [&](auto c, auto t) -> bool {
    if constexpr (norm_plan_exists(VW, BACK, decltype(t)::value, decltype(c)::value)) {
      if (a.tpr != t || a.chunks != c) return false;
      constexpr std::integral_constant<int, VW> v{};
      if (a.N % VW) f(v, c, t, std::true_type{});
      else f(v, c, t, std::false_type{});
      return true;
    }
    return false;
  };
  auto chunks = [&](auto c) -> bool {
    return tpr(c, std::integral_constant<int, 64>{}) || tpr(c, std::integral_constant<int, 128>{}) ||
           tpr(c, std::integral_constant<int, 256>{}) || tpr(c, std::integral_constant<int, 512>{}) ||
           tpr(c, std::integral_constant<int, 1024>{});
  };
  return chunks(std::integral_constant<int, 1>{}) || chunks(std::integral_constant<int, 2>{}) ||
         chunks(std::integral_constant<int, 4>{}) || chunks(std::integral_constant<int, 8>{});
}

template <typename T>
hipError_t norm_fwd(const NormArgs &a, hipStream_t s) {
  const bool ok = norm_pick<T, false>(a, [&](auto v, auto c, auto t, auto tail) {
    constexpr int V = decltype(v)::value, C = decltype(c)::value, TPR = decltype(t)::value;
    launch_kernel(norm_fwd_kernel<T, V, C, TPR, decltype(tail)::value>, dim3((unsigned)a.parts), dim3(std::max(256, TPR)), s, a);
  });
  return ok ? hipGetLastError() : hipErrorInvalidValue;
}
template <typename T>
hipError_t norm_bwd(const NormArgs &a, hipStream_t s) {
  const bool ok = norm_pick<T, true>(a, [&](auto v, auto c, auto t, auto tail) {
    constexpr int V = decltype(v)::value, C = decltype(c)::value, TPR = decltype(t)::value;
    launch_kernel(norm_bwd_kernel<T, V, C, TPR, decltype(tail)::value>, dim3((unsigned)a.parts), dim3(std::max(256, TPR)), s, a);
  });
  return ok ? hipGetLastError() : hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_norm_fwd(int dtype, const NormArgs &a, hipStream_t s) {
  return dtype == 0 ? norm_fwd<bf16_t>(a, s) : norm_fwd<float>(a, s);
}
hipError_t launch_norm_bwd(int dtype, const NormArgs &a, hipStream_t s) {
  return dtype == 0 ? norm_bwd<bf16_t>(a, s) : norm_bwd<float>(a, s);
}
hipError_t launch_norm_sum(int dtype, const NormArgs &a, hipStream_t s) {
  const unsigned grid = (unsigned)((2 * a.N + 15) / 16);
  if (dtype == 0) launch_kernel(norm_sum_kernel<bf16_t>, dim3(grid), dim3(1024), s, a);
  else launch_kernel(norm_sum_kernel<float>, dim3(grid), dim3(1024), s, a);
  return hipGetLastError();
}

}  // namespace pf
