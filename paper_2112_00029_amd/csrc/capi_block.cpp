// C ABI of the operators round the matrices of a Transformer block: the way
// back through the layer's activation epilogue.  Argument validation (all
// before any enqueue) and dispatch; see include/pixelfly.h for the contract.
#include "capi.h"

using namespace pf::capi;

namespace {

// Launch plan of pf_linear_act_bwd: chunks per workgroup row, workgroups across
// the columns, parts of the token range.
struct ActPlan {
  int cw, groups, nparts;
  int64_t rows;
};
ActPlan act_plan(pf_dtype dt, int64_t T, int64_t N) {
  const int v = dt == PF_BF16 ? 8 : 4;
  const int64_t chunks = N / v;
  ActPlan p{};
  // Widest workgroup row that leaves at most an eighth of its chunks idle.
  p.cw = 64;
  while (p.cw > 4 && (chunks + p.cw - 1) / p.cw * p.cw * 7 > chunks * 8) p.cw /= 2;
  p.groups = (int)((chunks + p.cw - 1) / p.cw);
  const int tall = 256 / p.cw;
  // Eight workgroups per CU, each with at least four rows per thread.
  const int64_t want = std::max<int64_t>(1, 2048 / p.groups);
  const int64_t most = std::max<int64_t>(1, T / (4 * tall));
  p.rows = (T + std::min(want, most) - 1) / std::min(want, most);
  p.rows = (p.rows + tall - 1) / tall * tall;
  p.nparts = (int)((T + p.rows - 1) / p.rows);
  return p;
}

bool act_dims_ok(pf_dtype dt, int64_t T, int64_t N) {
  return (dt == PF_BF16 || dt == PF_FP32) && T >= 1 && T <= ((int64_t)1 << 30) && N >= 32 &&
         N % 32 == 0 && N <= ((int64_t)1 << 24);
}

size_t act_ws(const ActPlan &p, int64_t N) {
  return p.nparts > 1 ? (size_t)p.nparts * N * sizeof(float) : 0;
}

}  // namespace

extern "C" {

size_t pf_linear_act_workspace_bytes(pf_dtype dtype, int64_t T, int64_t N) {
  if (!act_dims_ok(dtype, T, N)) return 0;
  return act_ws(act_plan(dtype, T, N), N);
}

pf_status pf_linear_act_bwd(pf_dtype dtype, int64_t T, int64_t N, pf_activation act, const void *dY,
                            const void *Y_pre, void *dY_pre, void *dbias, void *workspace,
                            size_t ws_bytes, void *stream) {
  if (dtype != PF_BF16 && dtype != PF_FP32) return fail(PF_ERR_INVALID_ARG, "bad dtype");
  if (!act_dims_ok(dtype, T, N))
    return fail(PF_ERR_INVALID_ARG, "T must be in 1 .. 2^30, N a multiple of 32 up to 2^24");
  if ((int)act < pf::kActNone || (int)act > pf::kActRelu) return fail(PF_ERR_INVALID_ARG, "bad activation");
  pf_status st;
  if ((st = need_ptr(dY, "dY")) != PF_OK) return st;
  if (act == PF_ACT_NONE) {
    if (Y_pre || dY_pre) return fail(PF_ERR_INVALID_ARG, "Y_pre or dY_pre given without an activation");
    if ((st = need_ptr(dbias, "dbias")) != PF_OK) return st;
  } else {
    if ((st = need_ptr(Y_pre, "Y_pre")) != PF_OK || (st = need_ptr(dY_pre, "dY_pre")) != PF_OK) return st;
    if (dbias && (st = need_ptr(dbias, "dbias")) != PF_OK) return st;
  }
  const ActPlan p = act_plan(dtype, T, N);
  const size_t need = dbias ? act_ws(p, N) : 0;
  if ((st = need_ws(need, workspace, ws_bytes)) != PF_OK) return st;
  hipStream_t s = (hipStream_t)stream;
  pf::ActBwdArgs a{};
  a.dY = dY; a.Z = Y_pre; a.dZ = dY_pre; a.dbias = dbias;
  a.partials = need ? (float *)workspace : nullptr;
  a.T = T; a.N = N; a.rows_per_part = p.rows;
  a.act = (int)act; a.cw = p.cw; a.groups = p.groups; a.nparts = p.nparts;
  {
    Timed t(PF_KERNEL_GELU_BWD, s);
    if ((st = hip_status(pf::launch_act_bwd((int)dtype, a, s), "activation backward kernel")) != PF_OK)
      return st;
  }
  if (!need) return PF_OK;
  Timed t(PF_KERNEL_REDUCE, s);
  return hip_status(pf::launch_act_dbias((int)dtype, a, s), "bias gradient sum");
}

}  // extern "C"
