// C ABI of the operators of a training step round the matrices: the way back
// through the gated product, layer normalisation, and the norm and clipping of all
// gradients.  Argument validation (all before any enqueue) and dispatch; see
// include/pixelfly.h for the contract.
#include "capi.h"

#include <cmath>
#include <new>

using namespace pf::capi;

namespace {

bool type_ok(int dt) { return dt == PF_BF16 || dt == PF_FP32; }

// ---------------------------------------------------------------------------
// Way back through the gated product
// ---------------------------------------------------------------------------
struct GatedPlan {
  int cw, groups, nparts;
  int64_t rows;
};
GatedPlan gated_plan(pf_dtype dt, int64_t T, int64_t N) {
  const int64_t chunks = N / (dt == PF_BF16 ? 8 : 4);
  GatedPlan p{};
  // Widest workgroup row, of 512 bytes at most, that leaves at most an eighth of its
  // chunks idle (16384 x 16384: rows of 4096 bytes 559 us, 1024 593, 512 466, 256 523;
  // 2100 x 4096 35.1, 22.2, 20.9, 20.6).
  p.cw = 32;
  while (p.cw > 4 && (chunks + p.cw - 1) / p.cw * p.cw * 7 > chunks * 8) p.cw /= 2;
  p.groups = (int)((chunks + p.cw - 1) / p.cw);
  const int tall = 256 / p.cw;
  // Eight workgroups per CU, each with at least two rows per thread.
  const int64_t want = std::max<int64_t>(1, 2048 / p.groups);
  const int64_t most = std::max<int64_t>(1, T / (2 * tall));
  p.rows = (T + std::min(want, most) - 1) / std::min(want, most);
  p.rows = (p.rows + tall - 1) / tall * tall;
  p.nparts = (int)((T + p.rows - 1) / p.rows);
  return p;
}
bool gated_dims_ok(pf_dtype dt, int64_t T, int64_t N) {
  return type_ok(dt) && T >= 1 && T <= ((int64_t)1 << 30) && N >= 32 && N % 32 == 0 &&
         N <= ((int64_t)1 << 24);
}
size_t gated_ws(const GatedPlan &p, int64_t N) {
  return p.nparts > 1 ? (size_t)p.nparts * 2 * N * sizeof(float) : 0;
}

}  // namespace

extern "C" {

size_t pf_linear_gated_workspace_bytes(pf_dtype dtype, int64_t T, int64_t N) {
  return gated_dims_ok(dtype, T, N) ? gated_ws(gated_plan(dtype, T, N), N) : 0;
}

pf_status pf_linear_gated_bwd(pf_dtype dtype, int64_t T, int64_t N, int32_t b, pf_activation act,
                              const void *dH, const void *Z, void *dZ, void *dbias, void *workspace,
                              size_t ws_bytes, void *stream) {
  if (!type_ok(dtype)) return fail(PF_ERR_INVALID_ARG, "bad dtype");
  if (!gated_dims_ok(dtype, T, N))
    return fail(PF_ERR_INVALID_ARG, "T must be in 1 .. 2^30, N a multiple of 32 up to 2^24");
  if (!kernel_block(b)) return fail(PF_ERR_UNSUPPORTED, "kernels support b in {32, 64, 128}");
  if (N % b) return fail(PF_ERR_INVALID_ARG, "b must divide N");
  if ((int)act < pf::kActNone || (int)act > pf::kActRelu) return fail(PF_ERR_INVALID_ARG, "bad activation");
  pf_status st;
  if ((st = need_ptr(dH, "dH")) != PF_OK || (st = need_ptr(Z, "Z")) != PF_OK ||
      (st = need_ptr(dZ, "dZ")) != PF_OK)
    return st;
  if (dbias && (st = need_ptr(dbias, "dbias")) != PF_OK) return st;
  const GatedPlan p = gated_plan(dtype, T, N);
  const size_t need = dbias ? gated_ws(p, N) : 0;
  if ((st = need_ws(need, workspace, ws_bytes)) != PF_OK) return st;
  hipStream_t s = (hipStream_t)stream;
  pf::GatedBwdArgs a{};
  a.dH = dH; a.Z = Z; a.dZ = dZ; a.dbias = dbias;
  a.partials = need ? (float *)workspace : nullptr;
  a.T = T; a.N = N; a.rows_per_part = p.rows;
  a.b = b; a.act = (int)act; a.cw = p.cw; a.groups = p.groups; a.nparts = p.nparts;
  // dZ larger than the caches.
  a.stream = 2 * T * N * (dtype == PF_BF16 ? 2 : 4) >= (int64_t)256 << 20;
  {
    Timed t(PF_KERNEL_GELU_BWD, s);
    if ((st = hip_status(pf::launch_gated_bwd((int)dtype, a, s), "gated backward kernel")) != PF_OK) return st;
  }
  if (!need) return PF_OK;
  pf::ActBwdArgs r{};
  r.dbias = dbias; r.partials = a.partials; r.N = 2 * N; r.nparts = p.nparts;
  Timed t(PF_KERNEL_REDUCE, s);
  return hip_status(pf::launch_act_dbias((int)dtype, r, s), "bias gradient sum");
}

}  // extern "C"

// ---------------------------------------------------------------------------
// Layer normalisation
// ---------------------------------------------------------------------------
namespace {

// Threads per row and chunks of 16 bytes per thread for rows of N elements, and the
// workgroups that share T rows.
struct NormPlan {
  int tpr, chunks, parts;
};
NormPlan norm_plan(pf_dtype dt, int64_t T, int64_t N, bool backward) {
  const int vw = dt == PF_BF16 ? 8 : 4;
  NormPlan p{};
  // 16 elements a thread; 32 for the longest rows of the backward, which keeps two sums
  // of each: 1024 threads have too few registers and 512 workgroups of them too many
  // partials (5000 x 16384 in bf16: 1024 threads, 128 / 256 / 512 workgroups, 224 / 163 /
  // 186 us, 512 threads, 256 workgroups, 148; fp32 1000 x 12000 127 / 109 / 128, 60).
  p.tpr = 64;
  while ((int64_t)p.tpr * 16 < N && !(backward && p.tpr == 512)) p.tpr *= 2;
  p.chunks = ((int64_t)p.tpr * 16 < N ? 32 : 16) / vw;
  // Fewer chunks where they cover the row.
  while (p.chunks > 1 && (int64_t)p.tpr * vw * (p.chunks / 2) >= N) p.chunks /= 2;
  const int64_t rpb = p.tpr < 256 ? 256 / p.tpr : 1;
  const int64_t rows = (T + rpb - 1) / rpb;
  // Forward: rows in plenty per CU, so that short ones still fill memory (16384 x
  // 4096: 8 workgroups per CU 52.5 us, 32 48.9).  Backward: two per CU, whose sums of dw
  // and db are then few (16384 x 4096, 1 / 2 / 3 / 4 per CU: 111, 109, 114, 125 us; 16384
  // x 1024 37, 32, 34, 37); four for many short rows (two / four: 65536 x 256 49.5 / 36.6
  // us, 20000 x 323 19.8 / 18.4, 16384 x 512 16.6 / 17.3, 65536 x 768 86.9 / 95.4).  All
  // of them take the same number of rows, or one less.
  const int64_t back = N <= 512 && rows > 4096 ? 4 : 2;
  const int64_t fill = 256 * (backward ? back : 32) * 256 / std::max(256, p.tpr);
  const int64_t it = (rows + fill - 1) / fill;
  p.parts = (int)((rows + it - 1) / it);
  return p;
}

pf_status check_norm(pf_dtype dt, int64_t T, int64_t N) {
  if (!type_ok(dt)) return fail(PF_ERR_INVALID_ARG, "bad dtype");
  if (T < 1 || T > ((int64_t)1 << 30) || N < 1) return fail(PF_ERR_INVALID_ARG, "T must be in 1 .. 2^30, N >= 1");
  if (N > pf::kNormMaxN)
    return fail(PF_ERR_UNSUPPORTED, "rows of more than " + std::to_string(pf::kNormMaxN) + " elements");
  return PF_OK;
}
// Rows of N elements, ld apart.
pf_status check_rows(const void *p, const char *name, int64_t N, int64_t ld) {
  pf_status st = need_ptr(p, name);
  if (st != PF_OK) return st;
  if (ld < N || ld > ((int64_t)1 << 32))
    return fail(PF_ERR_INVALID_ARG, std::string(name) + ": row stride below N or above 2^32");
  return PF_OK;
}
pf_status check_vector(const void *p, const char *name) { return p ? need_ptr(p, name) : PF_OK; }

}  // namespace

extern "C" {

pf_status pf_layernorm_fwd(pf_dtype dtype, int64_t T, int64_t N, float eps, const void *X, int64_t ldx,
                           const void *weight, const void *bias, void *Y, int64_t ldy, float *mean,
                           float *rstd, void *stream) {
  pf_status st = check_norm(dtype, T, N);
  if (st != PF_OK) return st;
  if (!(eps >= 0.f) || !std::isfinite(eps)) return fail(PF_ERR_INVALID_ARG, "eps must be finite and >= 0");
  if ((st = check_rows(X, "X", N, ldx)) != PF_OK || (st = check_rows(Y, "Y", N, ldy)) != PF_OK ||
      (st = check_vector(weight, "weight")) != PF_OK || (st = check_vector(bias, "bias")) != PF_OK ||
      (st = check_vector(mean, "mean")) != PF_OK || (st = check_vector(rstd, "rstd")) != PF_OK)
    return st;
  const NormPlan p = norm_plan(dtype, T, N, false);
  pf::NormArgs a{};
  a.X = X; a.weight = weight; a.bias = bias; a.Y = Y;
  a.mean = mean; a.rstd = rstd;
  a.T = T; a.N = N; a.ldx = ldx; a.ldy = ldy;
  a.eps = eps;
  a.tpr = p.tpr; a.chunks = p.chunks; a.parts = p.parts;
  hipStream_t s = (hipStream_t)stream;
  Timed t(PF_KERNEL_REDUCE, s);
  return hip_status(pf::launch_norm_fwd((int)dtype, a, s), "layer normalisation kernel");
}

size_t pf_layernorm_workspace_bytes(pf_dtype dtype, int64_t T, int64_t N) {
  if (!type_ok(dtype) || T < 1 || T > ((int64_t)1 << 30) || N < 1 || N > pf::kNormMaxN) return 0;
  const int parts = norm_plan(dtype, T, N, true).parts;
  return parts > 1 ? (size_t)parts * 2 * N * sizeof(float) : 0;
}

pf_status pf_layernorm_bwd(pf_dtype dtype, int64_t T, int64_t N, const void *dY, int64_t lddy, const void *X,
                           int64_t ldx, const void *weight, const float *mean, const float *rstd,
                           const void *dR, int64_t lddr, void *dX, int64_t lddx, void *dweight, void *dbias,
                           void *workspace, size_t ws_bytes, void *stream) {
  pf_status st = check_norm(dtype, T, N);
  if (st != PF_OK) return st;
  if ((st = check_rows(dY, "dY", N, lddy)) != PF_OK || (st = check_rows(X, "X", N, ldx)) != PF_OK ||
      (st = check_vector(weight, "weight")) != PF_OK || (st = need_ptr(mean, "mean")) != PF_OK ||
      (st = need_ptr(rstd, "rstd")) != PF_OK || (dR && (st = check_rows(dR, "dR", N, lddr)) != PF_OK) ||
      (st = check_rows(dX, "dX", N, lddx)) != PF_OK || (st = check_vector(dweight, "dweight")) != PF_OK ||
      (st = check_vector(dbias, "dbias")) != PF_OK)
    return st;
  const NormPlan p = norm_plan(dtype, T, N, true);
  const bool sums = dweight || dbias, many = p.parts > 1;
  if ((st = need_ws(sums && many ? (size_t)p.parts * 2 * N * sizeof(float) : 0, workspace, ws_bytes)) != PF_OK) return st;
  pf::NormArgs a{};
  a.X = X; a.weight = weight; a.dY = dY; a.dR = dR; a.dX = dX;
  a.dweight = dweight; a.dbias = dbias;
  a.mean_in = mean; a.rstd_in = rstd;
  a.partials = sums && many ? (float *)workspace : nullptr;
  a.T = T; a.N = N; a.ldx = ldx; a.lddy = lddy; a.lddr = lddr; a.lddx = lddx;
  a.tpr = p.tpr; a.chunks = p.chunks; a.parts = p.parts;
  hipStream_t s = (hipStream_t)stream;
  {
    Timed t(PF_KERNEL_REDUCE, s);
    if ((st = hip_status(pf::launch_norm_bwd((int)dtype, a, s), "layer normalisation backward kernel")) != PF_OK)
      return st;
  }
  if (!sums || !many) return PF_OK;
  Timed t(PF_KERNEL_REDUCE, s);
  return hip_status(pf::launch_norm_sum((int)dtype, a, s), "layer normalisation weight gradients");
}

}  // extern "C"

// ---------------------------------------------------------------------------
// Norm and clipping of all gradients
// ---------------------------------------------------------------------------
struct pf_grads {
  std::vector<pf::GradChunk> chunks;
  int64_t written = 0;  // bytes of the scaled gradients
  int device = -1;
  void *dev_mem = nullptr;
};

namespace {

// Workgroups of the passes: up to three per CU.
constexpr int kGradGrid = 768;
// Scaled gradients from here on are stored past the caches; fewer stay in them for
// the optimizer.
constexpr int64_t kGradStream = (int64_t)64 << 20;
constexpr int64_t kGradMaxChunks = (int64_t)1 << 24;
int grad_grid(const pf_grads *g) { return (int)std::min<size_t>(kGradGrid, std::max<size_t>(1, g->chunks.size())); }

// Chunks of the tensors; "" or an error.
std::string grad_chunks(int32_t n, const pf_grad_tensor *t, std::vector<pf::GradChunk> &out, int64_t &written) {
  struct Span {
    uint64_t lo, hi;
    int tensor;
    bool written;
  };
  std::vector<Span> spans;
  for (int32_t i = 0; i < n; ++i) {
    const std::string name = "tensor " + std::to_string(i);
    if (!type_ok(t[i].src_dtype) || !type_ok(t[i].dst_dtype)) return name + ": bad dtype";
    if (t[i].n < 0) return name + ": n is negative";
    if (t[i].n == 0) continue;
    // (2^37 elements in whole chunks; no card holds more.)
    if (t[i].n > kGradMaxChunks * pf::kGradChunk ||
        (int64_t)out.size() + (t[i].n + pf::kGradChunk - 1) / pf::kGradChunk > kGradMaxChunks)
      return name + ": too many elements";
    const int ss = t[i].src_dtype == PF_BF16 ? 2 : 4, ds = t[i].dst_dtype == PF_BF16 ? 2 : 4;
    const uint64_t src = (uint64_t)(uintptr_t)t[i].src, dst = (uint64_t)(uintptr_t)t[i].dst;
    if (!src || !dst) return name + ": src or dst is NULL";
    if (src % ss || dst % ds) return name + ": src or dst is not aligned to its elements";
    if (src == dst && ss != ds) return name + ": in place, but the types differ";
    if (src != dst) spans.push_back({src, src + (uint64_t)t[i].n * ss, i, false});
    spans.push_back({dst, dst + (uint64_t)t[i].n * ds, i, true});
    written += t[i].n * ds;
    const int types = (ss == 4 ? pf::kGradSrcF32 : 0) | (ds == 4 ? pf::kGradDstF32 : 0);
    for (int64_t e = 0; e < t[i].n; e += pf::kGradChunk)
      out.push_back({src + e * ss, dst + e * ds, (int32_t)std::min<int64_t>(pf::kGradChunk, t[i].n - e), types});
  }
  // What is written meets nothing else: in order of address, no span begins before
  // the furthest written end so far, and no written one before any end so far.
  std::sort(spans.begin(), spans.end(), [](const Span &x, const Span &y) { return x.lo < y.lo; });
  uint64_t end = 0, wend = 0;
  for (const Span &s : spans) {
    if (s.lo < wend || (s.written && s.lo < end))
      return "tensor " + std::to_string(s.tensor) + ": what is written overlaps another tensor";
    end = std::max(end, s.hi);
    if (s.written) wend = std::max(wend, s.hi);
  }
  return "";
}

pf_status grad_state(const pf_grads *g) {
  if (g->device < 0 || !g->dev_mem) return fail(PF_ERR_STATE, "gradient list not uploaded (call pf_grads_upload)");
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess || dev != g->device)
    return fail(PF_ERR_STATE, "gradient list was uploaded to another device");
  return PF_OK;
}

pf::GradArgs grad_args(const pf_grads *g) {
  pf::GradArgs a{};
  a.chunks = (const pf::GradChunk *)g->dev_mem;
  a.nchunk = (int)g->chunks.size();
  a.nparts = grad_grid(g);
  a.stream = g->written >= kGradStream;
  return a;
}

pf_status check_limit(float max_norm) {
  if (!(max_norm >= 0.f) || !std::isfinite(max_norm))
    return fail(PF_ERR_INVALID_ARG, "max_norm must be finite and >= 0");
  return PF_OK;
}
pf_status check_word(const void *p, size_t align, const char *name) {
  if ((uintptr_t)p % align) return fail(PF_ERR_INVALID_ARG, std::string(name) + " is misaligned");
  return PF_OK;
}

}  // namespace

extern "C" {

pf_status pf_grads_create(int32_t n, const pf_grad_tensor *tensors, pf_grads **out) {
  if (!out) return fail(PF_ERR_INVALID_ARG, "out is NULL");
  *out = nullptr;
  if (n < 0 || (n > 0 && !tensors)) return fail(PF_ERR_INVALID_ARG, "n below 0, or tensors is NULL");
  pf_grads *g = new (std::nothrow) pf_grads();
  if (!g) return fail(PF_ERR_NOMEM, "host allocation failed");
  std::string e;
  try {
    e = grad_chunks(n, tensors, g->chunks, g->written);
  } catch (const std::exception &) {
    delete g;
    return fail(PF_ERR_NOMEM, "host allocation failed");
  }
  if (!e.empty()) {
    delete g;
    return fail(PF_ERR_INVALID_ARG, e);
  }
  *out = g;
  return PF_OK;
}

pf_status pf_grads_upload(pf_grads *g, void *stream) {
  if (!g) return fail(PF_ERR_INVALID_ARG, "gradient list is NULL");
  if (g->dev_mem) return PF_OK;
  int dev = -1;
  pf_status st = hip_status(hipGetDevice(&dev), "hipGetDevice");
  if (st != PF_OK) return st;
  const size_t bytes = g->chunks.size() * sizeof(pf::GradChunk);
  void *mem = nullptr;
  if (hipMalloc(&mem, std::max<size_t>(bytes, 256)) != hipSuccess)
    return fail(PF_ERR_NOMEM, "hipMalloc for the gradient list failed");
  hipStream_t s = (hipStream_t)stream;
  hipError_t e = bytes ? hipMemcpyAsync(mem, g->chunks.data(), bytes, hipMemcpyHostToDevice, s) : hipSuccess;
  if (e == hipSuccess) e = hipStreamSynchronize(s);
  if (e != hipSuccess) {
    (void)hipFree(mem);
    return hip_status(e, "gradient list upload");
  }
  g->dev_mem = mem;
  g->device = dev;
  return PF_OK;
}

void pf_grads_destroy(pf_grads *g) {
  if (!g) return;
  if (g->dev_mem) {
    int cur = -1;
    (void)hipGetDevice(&cur);
    if (cur != g->device) (void)hipSetDevice(g->device);
    (void)hipFree(g->dev_mem);
    if (cur >= 0 && cur != g->device) (void)hipSetDevice(cur);
  }
  delete g;
}

size_t pf_grads_workspace_bytes(const pf_grads *g) { return g ? grad_grid(g) * sizeof(double) : 0; }

pf_status pf_grads_norm(const pf_grads *g, double *sumsq, float *norm, void *workspace, size_t ws_bytes,
                        void *stream) {
  if (!g) return fail(PF_ERR_INVALID_ARG, "gradient list is NULL");
  if (!sumsq && !norm) return fail(PF_ERR_INVALID_ARG, "sumsq and norm are NULL");
  pf_status st;
  if ((st = check_word(sumsq, 8, "sumsq")) != PF_OK || (st = check_word(norm, 4, "norm")) != PF_OK ||
      (st = need_ws(pf_grads_workspace_bytes(g), workspace, ws_bytes)) != PF_OK || (st = grad_state(g)) != PF_OK)
    return st;
  pf::GradArgs a = grad_args(g);
  a.partials = (double *)workspace;
  a.sumsq = sumsq;
  a.norm = norm;
  hipStream_t s = (hipStream_t)stream;
  {
    Timed t(PF_KERNEL_REDUCE, s);
    if ((st = hip_status(pf::launch_grad_sumsq(a, s), "gradient norm kernel")) != PF_OK) return st;
  }
  Timed t(PF_KERNEL_REDUCE, s);
  return hip_status(pf::launch_grad_total(a, s), "gradient norm sum");
}

pf_status pf_grads_scale(const pf_grads *g, float max_norm, const double *sumsq, void *stream) {
  if (!g) return fail(PF_ERR_INVALID_ARG, "gradient list is NULL");
  pf_status st;
  if ((st = check_limit(max_norm)) != PF_OK) return st;
  if (!sumsq) return fail(PF_ERR_INVALID_ARG, "sumsq is NULL");
  if ((st = check_word(sumsq, 8, "sumsq")) != PF_OK || (st = grad_state(g)) != PF_OK) return st;
  pf::GradArgs a = grad_args(g);
  const int grid = a.nparts;
  a.partials = const_cast<double *>(sumsq);
  a.nparts = 1;
  a.max_norm = max_norm;
  hipStream_t s = (hipStream_t)stream;
  Timed t(PF_KERNEL_REDUCE, s);
  return hip_status(pf::launch_grad_scale(a, grid, s), "gradient scaling kernel");
}

pf_status pf_grads_clip(const pf_grads *g, float max_norm, float *norm, void *workspace, size_t ws_bytes,
                        void *stream) {
  if (!g) return fail(PF_ERR_INVALID_ARG, "gradient list is NULL");
  pf_status st;
  if ((st = check_limit(max_norm)) != PF_OK || (st = check_word(norm, 4, "norm")) != PF_OK ||
      (st = need_ws(pf_grads_workspace_bytes(g), workspace, ws_bytes)) != PF_OK || (st = grad_state(g)) != PF_OK)
    return st;
  pf::GradArgs a = grad_args(g);
  a.partials = (double *)workspace;
  a.norm = norm;
  a.max_norm = max_norm;
  hipStream_t s = (hipStream_t)stream;
  {
    Timed t(PF_KERNEL_REDUCE, s);
    if ((st = hip_status(pf::launch_grad_sumsq(a, s), "gradient norm kernel")) != PF_OK) return st;
  }
  Timed t(PF_KERNEL_REDUCE, s);
  return hip_status(pf::launch_grad_scale(a, a.nparts, s), "gradient scaling kernel");
}

}  // extern "C"
