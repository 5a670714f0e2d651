// Way back through the gated product H = act(Zg) o Zu, Z = [Zg Zu] in blocks of b
// columns that alternate gate, other:
//
//   dZg = dH o Zu o act'(Zg),  dZu = dH o act(Zg),  dbias = column sums of dZ
//
// in one pass: three 16-byte loads and two stores per thread and row, act and act'
// from one set of exponentials.  Memory is the bound: 16384 x 16384 in bf16 takes 466
// us, 5.8 TB/s (a large copy: 4.9).  A thread owns one chunk of H's columns and walks
// down the rows of its workgroup's part, the next row's loads in flight, its 2 V
// column sums in registers; rows of the workgroup are added through LDS in row order,
// parts by a second launch in part order.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "pf_act.h"
#include "pf_io.h"
#include "pf_launch.h"

namespace pf {
namespace {

// STREAM: dZ is stored past the caches (a variant, as a branch's two stores would
// be joined).
template <typename T, bool STREAM>
__global__ __launch_bounds__(256) void gated_bwd_kernel(GatedBwdArgs a) {
  constexpr int V = 16 / sizeof(T);
  __shared__ float red[256 * 2 * V];
  const int cw = a.cw, rows = 256 / cw;
  const int ci = threadIdx.x % cw, ri = threadIdx.x / cw;
  const int grp = blockIdx.x % a.groups, part = blockIdx.x / a.groups;
  const int64_t n = ((int64_t)grp * cw + ci) * V;
  const bool live = n < a.N;
  const int64_t zc = (n / a.b) * 2 * a.b + n % a.b;  // its gate's column of Z
  const int64_t t0 = (int64_t)part * a.rows_per_part, t1 = min(a.T, t0 + a.rows_per_part);
  const T *dH = (const T *)a.dH + n, *Z = (const T *)a.Z + zc;
  T *dZ = (T *)a.dZ + zc;
  float sg[V] = {}, su[V] = {};
  if (live && t0 + ri < t1) {
    Raw<T, V> rd, rg, ru, nd, ng, nu;
    auto fetch = [&](int64_t t, Raw<T, V> &d, Raw<T, V> &g, Raw<T, V> &u) __attribute__((always_inline)) {
      d = ld_raw<T, V>(dH + t * a.N);
      g = ld_raw<T, V>(Z + t * 2 * a.N);
      u = ld_raw<T, V>(Z + t * 2 * a.N + a.b);
    };
    fetch(t0 + ri, nd, ng, nu);
    for (int64_t t = t0 + ri; t < t1; t += rows) {
      T *o = dZ + t * 2 * a.N;
      rd = nd;
      rg = ng;
      ru = nu;
      // (Past the end: this row again, whose dZ, which may be Z, is stored below.)
      fetch(t + rows < t1 ? t + rows : t, nd, ng, nu);
      float d[V], g[V], u[V], f[V], s[V];
      unpack<T, V>(rd, d);
      unpack<T, V>(rg, g);
      unpack<T, V>(ru, u);
      act_both<T>(a.act, g, f, s);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        g[e] = d[e] * u[e] * s[e];
        u[e] = d[e] * f[e];
        sg[e] += g[e];
        su[e] += u[e];
      }
      st_raw<T, V, STREAM>(o, pack<T, V>(g));
      st_raw<T, V, STREAM>(o + a.b, pack<T, V>(u));
    }
  }
  if (!a.partials && !a.dbias) return;
#pragma unroll
  for (int e = 0; e < V; ++e) {
    red[(ri * cw + ci) * 2 * V + e] = sg[e];
    red[(ri * cw + ci) * 2 * V + V + e] = su[e];
  }
  __syncthreads();
  for (int c = threadIdx.x; c < cw * 2 * V; c += 256) {
    const int64_t m = (int64_t)grp * cw * V + c / (2 * V) * V + c % V;  // column of H
    if (m >= a.N) continue;
    float s = 0.f;
    for (int r = 0; r < rows; ++r) s += red[r * cw * 2 * V + c];
    const int64_t col = (m / a.b) * 2 * a.b + m % a.b + (c % (2 * V) >= V ? a.b : 0);
    if (a.partials) a.partials[part * 2 * a.N + col] = s;
    else down(((T *)a.dbias)[col], s);
  }
}

}  // namespace

hipError_t launch_gated_bwd(int dtype, const GatedBwdArgs &a, hipStream_t s) {
  const int64_t grid = (int64_t)a.groups * a.nparts;
  if (grid <= 0 || grid > 0x7fffffff || a.cw < 1 || a.cw > 32 || 256 % a.cw) return hipErrorInvalidValue;
  auto go = [&](auto kernel) { launch_kernel(kernel, dim3((unsigned)grid), dim3(256), s, a); };
  if (dtype == 0) a.stream ? go(gated_bwd_kernel<bf16_t, true>) : go(gated_bwd_kernel<bf16_t, false>);
  else a.stream ? go(gated_bwd_kernel<float, true>) : go(gated_bwd_kernel<float, false>);
  return hipGetLastError();
}

}  // namespace pf
