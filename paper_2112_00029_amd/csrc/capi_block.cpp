// C ABI of the operators round the matrices of a Transformer block: the way
// back through the layer's activation epilogue, and attention with a relative
// position bias.  Argument validation (all before any enqueue) and dispatch;
// see include/pixelfly.h for the contract.
#include "capi.h"

#include <new>

#include "relpos.h"

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
  a.stream = T * N * (dtype == PF_BF16 ? 2 : 4) >= (int64_t)256 << 20;
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

// ---------------------------------------------------------------------------
// Relative position bias
// ---------------------------------------------------------------------------
namespace {

// Checks shared by the two ways of making a plan.
pf_status relpos_dims(int64_t seq, int32_t n_buckets, const void *out) {
  if (!out) return fail(PF_ERR_INVALID_ARG, "out is NULL");
  if (seq < 64 || seq % 64 || seq / 64 > 16384)
    return fail(PF_ERR_INVALID_ARG, "seq must be a multiple of 64, 64 .. 2^20");
  if (n_buckets < 1 || n_buckets > pf::kRelposMaxBuckets)
    return fail(PF_ERR_INVALID_ARG, "n_buckets must be in 1 .. " + std::to_string(pf::kRelposMaxBuckets));
  return PF_OK;
}

pf_status relpos_state(const pf_relpos *R) {
  if (R->device < 0 || !R->dev_mem)
    return fail(PF_ERR_STATE, "position bias plan not uploaded (call pf_relpos_upload)");
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess || dev != R->device)
    return fail(PF_ERR_STATE, "position bias plan was uploaded to another device");
  return PF_OK;
}

// Kernels address one head's rows of a sequence with 32-bit byte offsets, up
// to 64 rows before the first and past the last included.
constexpr int64_t kMaxToken = (int64_t)1 << 24;
pf_status check_rows(const pf_attn_tensor *t, const char *name, int64_t rows, bool out, int32_t B, int32_t heads) {
  const std::string n = name;
  if (!t) return fail(PF_ERR_INVALID_ARG, n + " is NULL");
  pf_status st = need_ptr(t->data, name);
  if (st != PF_OK) return st;
  if (t->seq % 8 || t->head % 8 || t->token % 8)
    return fail(PF_ERR_INVALID_ARG, n + ": strides must be multiples of 8 elements");
  if (t->token < 64 || t->seq < 0 || t->head < 0)
    return fail(PF_ERR_INVALID_ARG, n + ": token stride below 64, or a negative stride");
  if (t->token > kMaxToken || (rows + 64) * t->token * 2 > 0x7fffffff)
    return fail(PF_ERR_UNSUPPORTED, n + ": a head's rows of one sequence span 2^31 bytes or more");
  if (out) {
    // Rows of different tokens, heads or sequences must not meet: by ascending
    // stride, each dimension steps past all that the smaller ones cover.
    struct Dim {
      int64_t stride, n;
    } dim[3] = {{t->token, rows}, {t->head, heads}, {t->seq, B}};
    std::sort(dim, dim + 3, [](const Dim &x, const Dim &y) { return x.stride < y.stride; });
    __int128 span = 64;
    for (const Dim &x : dim) {
      if (x.n == 1) continue;
      if (x.stride < span)
        return fail(PF_ERR_INVALID_ARG, n + " is written: its tokens, heads and sequences must not overlap");
      span += (__int128)x.stride * (x.n - 1);
    }
  }
  return PF_OK;
}

struct RelposDims {
  int32_t B, H, H_kv, Sq, Skv, d;
  float scale;
};
pf_status check_relpos(const pf_layout *L, const pf_relpos *R, const RelposDims &m, const float *bias,
                       const int32_t *q_start, const int32_t *kv_len) {
  pf_status st = check_layout_arg(L);
  if (st != PF_OK) return st;
  if (!R) return fail(PF_ERR_INVALID_ARG, "position bias plan is NULL");
  if (L->n_out != L->n_in || L->n_out != R->seq)
    return fail(PF_ERR_INVALID_ARG, "layout must be square with the plan's sequence length as its side");
  if (L->b != 64 || m.d != 64) return fail(PF_ERR_UNSUPPORTED, "attention supports b = 64, d = 64");
  if (m.B < 1 || m.H < 1 || m.H_kv < 1 || m.H % m.H_kv)
    return fail(PF_ERR_INVALID_ARG, "B, H and H_kv must be >= 1 and H_kv divide H");
  if (m.H > 65535) return fail(PF_ERR_UNSUPPORTED, "more than 65535 heads");
  if (m.Sq < 1 || m.Sq > R->seq || m.Skv < 1 || m.Skv > R->seq)
    return fail(PF_ERR_INVALID_ARG, "Sq and Skv must be in 1 .. the layout's side");
  if ((int64_t)m.B * m.H > 0x7fffffff / (R->nb + 1)) return fail(PF_ERR_INVALID_ARG, "too many blocks");
  // The bias enters the products in units of the unscaled score.
  if (!(m.scale >= 0x1p-40f && m.scale <= 0x1p40f))
    return fail(PF_ERR_INVALID_ARG, "scale must be in 2^-40 .. 2^40");
  if ((st = need_ptr(bias, "bias")) != PF_OK) return st;
  if (((uintptr_t)q_start | (uintptr_t)kv_len) & 3)
    return fail(PF_ERR_INVALID_ARG, "q_start or kv_len is not 4-byte aligned");
  return PF_OK;
}

pf::RowView view(const pf_attn_tensor *t) { return {t->data, t->seq, t->head, t->token}; }
pf::RowViewOut view_out(const pf_attn_tensor *t) { return {t->data, t->seq, t->head, t->token}; }

pf::RelposArgs relpos_args(const pf_layout *L, const pf_relpos *R, const RelposDims &m, const float *bias,
                           const int32_t *q_start, const int32_t *kv_len) {
  pf::RelposArgs a{};
  a.bias = bias;
  a.bias_ld = 4 * R->seq;
  a.q_start = q_start; a.kv_len = kv_len;
  a.info = R->d_info; a.order = R->d_order;
  a.row_ptr = L->d_row_ptr; a.col_idx = L->d_col_idx;
  a.col_ptr = L->d_col_ptr; a.row_idx = L->d_row_idx;
  a.B = m.B; a.H = m.H; a.Hkv = m.H_kv; a.G = m.H / m.H_kv;
  a.Sq = m.Sq; a.Skv = m.Skv; a.seq = (int)R->seq; a.nb = R->nb;
  a.nbucket = R->n_buckets;
  a.omin = R->omin; a.omax = R->omax;
  a.scale = m.scale;
  return a;
}

size_t up256(size_t x) { return (x + 255) / 256 * 256; }

// How a launch over blocks shares them among workgroups: the first nlong of a
// head's ntile in plong parts, the others in pshort (see pf::RelposArgs).
struct Parts {
  int nbh = 0, ntile = 0, nlong = 0, plong = 1, pshort = 1;
  int64_t slots() const {
    return (int64_t)nbh * ((plong > 1 ? (int64_t)nlong * plong : 0) +
                           (pshort > 1 ? (int64_t)(ntile - nlong) * pshort : 0));
  }
  // Every launch's workgroups and slots fit 31 bits (a join takes up to eight
  // workgroups a block).
  bool fits() const { return workgroups() <= 0x7fffffff / 8; }
  int64_t workgroups() const {
    return (int64_t)nbh * ((int64_t)nlong * plong + (int64_t)(ntile - nlong) * pshort);
  }
  void set(pf::RelposArgs &a) const {
    a.nbh = nbh; a.ntile = ntile; a.nlong = nlong; a.plong = plong; a.pshort = pshort;
  }
};

// Blocks (items) per part of the long lists: 8 x 12 x 4096 with a stripe, lists of
// 64 in parts of 16 / 12 / 8, backward 377 / 347 / 328 us, forward 133 / 129 / 121.
// Up to eight workgroups per CU: more long lists than that balance by themselves, and
// the slots stay below 64 MiB.
constexpr int kLongItems = 8;
constexpr int64_t kLongWG = 2048;
// The other lists are split where their blocks make fewer workgroups than `fill`, in
// parts of at least `least` items.  Rows (forward and dQ): 512 and 4; 12 heads x
// 2048, every block kept, 384 workgroups: two parts 35.4 us, three 38.1.  dK and
// dV, whose slots are twice as large: 1024 and 16; 4 x 4 x 2048 causal, four query
// heads each (512 workgroups, up to 128 items): one part 325 us, two 234; 4 x 4 x 1511
// (368, 24 items on average): two 68, three 77.
constexpr int kShortItems = 16;  // lists up to here stay whole
struct Split {
  int64_t fill, least;
};
constexpr Split kRowSplit{512, 4}, kColSplit{1024, 16};

// long_items: list length of the nlong leading blocks, items: of the others.
Parts choose_parts(int nbh, int ntile, int nlong, int64_t long_items, int64_t items, const Split &s) {
  Parts p;
  p.nbh = nbh;
  p.ntile = ntile;
  if (nlong > 0 && long_items > kShortItems) {
    p.nlong = std::min(nlong, ntile);
    p.plong = (int)std::max<int64_t>(1, std::min((long_items + kLongItems - 1) / kLongItems,
                                                 kLongWG / ((int64_t)nbh * p.nlong)));
  }
  const int64_t wg = (int64_t)nbh * (ntile - p.nlong);
  if (wg > 0 && wg < s.fill && items > kShortItems)
    p.pshort = (int)std::min((s.fill + wg - 1) / wg, (items + s.least - 1) / s.least);
  return p;
}

// Longest lists of a layout's block rows (or columns) as far as the plan's
// distances reach: of the leading stripes, and of the rest.
struct Lists {
  int nlong;
  int64_t long_items, items;
};
Lists row_lists(const pf_layout *L, const pf_relpos *R, bool columns) {
  const int64_t nb = L->nb_out, g = std::min<int64_t>(L->global_blocks, nb);
  // Key block - query block lies in omin .. omax; seen from a column the other
  // way round.
  const int64_t lo = columns ? -R->omax : R->omin, hi = columns ? -R->omin : R->omax;
  auto reach = [&](int64_t last) {  // blocks within lo .. hi of block `last`
    return std::max<int64_t>(0, std::min(nb - 1, last + hi) - std::max<int64_t>(0, last + lo) + 1);
  };
  Lists r{(int)g, g > 0 ? reach(g - 1) : 0, 0};
  const int64_t most = columns ? L->kmax_bwd : L->kmax_fwd;
  // With stripes the longest list is theirs: the others' average.
  r.items = g > 0 && g < nb ? (L->nnzb - g * nb + (nb - g) - 1) / (nb - g) : most;
  r.items = std::min(r.items, std::max<int64_t>(0, hi - lo + 1));
  return r;
}

Parts fwd_parts(const pf_layout *L, const pf_relpos *R, int32_t B, int32_t H, int32_t Sq, bool chunk) {
  const Lists l = row_lists(L, R, false);
  // A chunk starts anywhere in a block, and anywhere in its sequence: which of
  // its tiles are a stripe's is not known here.  A chunk inside a stripe pays for it (12
  // heads, the first 64 rows of 4096 with a stripe of one block: 58 us as a chunk, 15 as
  // the first rows of the sequence).
  return choose_parts(B * H, (Sq + (chunk ? 63 : 0) + 63) / 64, chunk ? 0 : l.nlong, l.long_items, l.items,
                      kRowSplit);
}
Parts dkv_parts(const pf_layout *L, const pf_relpos *R, int32_t B, int32_t H, int32_t Hkv, int32_t S) {
  const Lists l = row_lists(L, R, true);
  const int G = H / Hkv;
  return choose_parts(B * Hkv, (S + 63) / 64, l.nlong, l.long_items * G, l.items * G, kColSplit);
}
// Waves per (sequence, key/value head) of the decode kernel: lists of eight blocks
// or more are split up to 1024 waves in all, at least two blocks each (16 x 4 heads of
// 4096 keys: one wave 68 us, 1024 in all 16.6, 2048 19.2; 12 heads of 1000 keys: one
// 20.7, eight 12.3; seven blocks in two parts 12.3 against 11.7 in one).
Parts decode_parts(const pf_layout *L, const pf_relpos *R, int32_t B, int32_t Hkv) {
  const Lists l = row_lists(L, R, false);
  Parts p;
  p.nbh = B * Hkv;
  p.ntile = 1;
  if (l.items >= 8)
    p.pshort = (int)std::max<int64_t>(1, std::min<int64_t>((1024 + p.nbh - 1) / p.nbh, (l.items + 1) / 2));
  return p;
}
bool use_decode(int32_t Sq, int32_t H, int32_t Hkv) { return Sq == 1 && H / Hkv <= pf::kRelposDecodeRows; }

size_t fwd_slots(const pf_layout *L, const pf_relpos *R, int32_t B, int32_t H, int32_t Hkv, int32_t Sq, bool chunk) {
  if (use_decode(Sq, H, Hkv))
    return decode_parts(L, R, B, Hkv).slots() * pf::kRelposDecodeSlot * sizeof(float);
  return fwd_parts(L, R, B, H, Sq, chunk).slots() * pf::kRelposFwdSlot * sizeof(float);
}
// Backward workspace: delta, the bucket sums, slots (first dQ's, then dK and
// dV's).
struct BwdPlan {
  Parts dq, dkv;
  size_t partials, slots, total;
};
BwdPlan bwd_plan(const pf_layout *L, const pf_relpos *R, int32_t B, int32_t H, int32_t Hkv, int32_t S) {
  BwdPlan p;
  p.dq = fwd_parts(L, R, B, H, S, false);
  p.dkv = dkv_parts(L, R, B, H, Hkv, S);
  p.partials = up256((size_t)B * H * S * sizeof(float));
  p.slots = p.partials + up256((size_t)p.dq.workgroups() * R->n_buckets * sizeof(float));
  p.total = p.slots + std::max((size_t)p.dq.slots() * pf::kRelposAccFloats,
                               (size_t)p.dkv.slots() * 2 * pf::kRelposAccFloats) * sizeof(float);
  return p;
}

}  // namespace

extern "C" {

pf_status pf_relpos_create(int64_t seq, int32_t n_buckets, const int32_t *bucket, pf_relpos **out) {
  pf_status st = relpos_dims(seq, n_buckets, out);
  if (st != PF_OK) return st;
  if (!bucket) return fail(PF_ERR_INVALID_ARG, "bucket is NULL");
  pf_relpos *R = nullptr;
  try {
    R = new pf_relpos;
    const std::string err = pf::build_relpos(*R, seq, n_buckets, bucket);
    if (!err.empty()) {
      delete R;
      return fail(PF_ERR_INVALID_ARG, err);
    }
  } catch (const std::bad_alloc &) {
    delete R;
    return PF_ERR_NOMEM;
  }
  *out = R;
  return PF_OK;
}

pf_status pf_relpos_create_log(int64_t seq, int32_t n_buckets, int64_t max_distance, int32_t bidirectional,
                               pf_relpos **out) {
  pf_status st = relpos_dims(seq, n_buckets, out);
  if (st != PF_OK) return st;
  try {
    std::vector<int32_t> bucket;
    const std::string err = pf::log_buckets(seq, n_buckets, max_distance, bidirectional != 0, bucket);
    if (!err.empty()) return fail(PF_ERR_INVALID_ARG, err);
    return pf_relpos_create(seq, n_buckets, bucket.data(), out);
  } catch (const std::bad_alloc &) {
    return PF_ERR_NOMEM;
  }
}

pf_status pf_relpos_buckets_get(const pf_relpos *R, const int32_t **bucket, int64_t *seq, int32_t *n_buckets) {
  if (!R) return fail(PF_ERR_INVALID_ARG, "position bias plan is NULL");
  if (bucket) *bucket = R->bucket.data() + 1;
  if (seq) *seq = R->seq;
  if (n_buckets) *n_buckets = R->n_buckets;
  return PF_OK;
}

pf_status pf_relpos_upload(pf_relpos *R, void *stream) {
  if (!R) return fail(PF_ERR_INVALID_ARG, "position bias plan is NULL");
  if (R->dev_mem) return PF_OK;
  int dev = -1;
  pf_status st = hip_status(hipGetDevice(&dev), "hipGetDevice");
  if (st != PF_OK) return st;
  const size_t nb = R->bucket.size() * 4, ni = R->info.size() * 4, no = R->order.size() * 4;
  char *mem = nullptr;
  if (hipMalloc((void **)&mem, up256(nb) + up256(ni) + up256(std::max<size_t>(no, 4))) != hipSuccess)
    return fail(PF_ERR_NOMEM, "hipMalloc for the position bias plan failed");
  hipStream_t s = (hipStream_t)stream;
  hipError_t e = hipMemcpyAsync(mem, R->bucket.data(), nb, hipMemcpyHostToDevice, s);
  if (e == hipSuccess) e = hipMemcpyAsync(mem + up256(nb), R->info.data(), ni, hipMemcpyHostToDevice, s);
  if (e == hipSuccess && no)
    e = hipMemcpyAsync(mem + up256(nb) + up256(ni), R->order.data(), no, hipMemcpyHostToDevice, s);
  if (e == hipSuccess) e = hipStreamSynchronize(s);
  if (e != hipSuccess) {
    (void)hipFree(mem);
    return hip_status(e, "position bias plan upload");
  }
  R->d_bucket = (const int32_t *)mem;
  R->d_info = (const int32_t *)(mem + up256(nb));
  R->d_order = (const uint32_t *)(mem + up256(nb) + up256(ni));
  R->dev_mem = mem;
  R->device = dev;
  return PF_OK;
}

void pf_relpos_destroy(pf_relpos *R) {
  if (!R) return;
  if (R->dev_mem) {
    int cur = -1;
    (void)hipGetDevice(&cur);
    if (cur != R->device) (void)hipSetDevice(R->device);
    (void)hipFree(R->dev_mem);
    if (cur >= 0 && cur != R->device) (void)hipSetDevice(cur);
  }
  delete R;
}

size_t pf_relpos_bias_floats(const pf_relpos *R) { return R ? (size_t)R->seq * 4 : 0; }

pf_status pf_relpos_bias(const pf_relpos *R, int32_t H, const float *table, float *bias, void *stream) {
  if (!R) return fail(PF_ERR_INVALID_ARG, "position bias plan is NULL");
  if (H < 1 || H > 65535) return fail(PF_ERR_INVALID_ARG, "H must be in 1 .. 65535");
  pf_status st;
  if ((st = need_ptr(table, "table")) != PF_OK || (st = need_ptr(bias, "bias")) != PF_OK) return st;
  if ((st = relpos_state(R)) != PF_OK) return st;
  hipStream_t s = (hipStream_t)stream;
  Timed t(PF_KERNEL_REDUCE, s);
  return hip_status(pf::launch_relpos_bias({R->d_bucket, table, bias, (int)R->seq, R->n_buckets}, H, s),
                    "position bias kernel");
}

size_t pf_attn_relpos_workspace_bytes(const pf_layout *L, const pf_relpos *R, int32_t B, int32_t H, int32_t Sq) {
  if (!L || !R || B < 1 || H < 1 || H > 65535 || Sq < 1 || Sq > R->seq || L->n_out != R->seq || L->n_in != R->seq ||
      (int64_t)B * H > 0x7fffffff / (R->nb + 1))
    return 0;
  // For every number of key/value heads, and either form of the forward.
  size_t need = 0;
  for (int32_t k = 1; k <= H; ++k)
    if (H % k == 0)
      need = std::max({need, fwd_slots(L, R, B, H, k, Sq, false), fwd_slots(L, R, B, H, k, Sq, true),
                       bwd_plan(L, R, B, H, k, Sq).total});
  return up256(need);
}

pf_status pf_attn_relpos_fwd(const pf_layout *L, const pf_relpos *R, int32_t B, int32_t H, int32_t H_kv,
                             int32_t Sq, int32_t Skv, int32_t d, float scale, const pf_attn_tensor *Q,
                             const pf_attn_tensor *K, const pf_attn_tensor *V, const float *bias,
                             const pf_attn_tensor *O, float *lse, const int32_t *q_start,
                             const int32_t *kv_len, void *workspace, size_t ws_bytes, void *stream) {
  const RelposDims m{B, H, H_kv, Sq, Skv, d, scale};
  pf_status st = check_relpos(L, R, m, bias, q_start, kv_len);
  if (st != PF_OK) return st;
  if ((st = check_rows(Q, "Q", Sq, false, B, H)) != PF_OK || (st = check_rows(K, "K", Skv, false, B, H_kv)) != PF_OK ||
      (st = check_rows(V, "V", Skv, false, B, H_kv)) != PF_OK || (st = check_rows(O, "O", Sq, true, B, H)) != PF_OK ||
      (st = need_ptr(lse, "lse")) != PF_OK)
    return st;
  const bool dec = use_decode(Sq, H, H_kv);
  const Parts parts = dec ? decode_parts(L, R, B, H_kv) : fwd_parts(L, R, B, H, Sq, q_start != nullptr);
  if (!parts.fits()) return fail(PF_ERR_UNSUPPORTED, "too many blocks for one launch");
  const size_t need = fwd_slots(L, R, B, H, H_kv, Sq, q_start != nullptr);
  if ((st = need_ws(need, workspace, ws_bytes)) != PF_OK) return st;
  if ((st = check_state(L)) != PF_OK || (st = relpos_state(R)) != PF_OK) return st;
  pf::RelposArgs a = relpos_args(L, R, m, bias, q_start, kv_len);
  a.Q = view(Q); a.K = view(K); a.V = view(V); a.Oout = view_out(O);
  a.lse = lse;
  a.slots = (float *)workspace;
  hipStream_t s = (hipStream_t)stream;
  parts.set(a);
  {
    Timed t(PF_KERNEL_ATTN_FWD, s);
    st = hip_status(dec ? pf::launch_relpos_decode(a, s) : pf::launch_relpos_fwd(a, s),
                    "attention forward kernel");
  }
  if (st != PF_OK || !need) return st;
  Timed t(PF_KERNEL_REDUCE, s);
  return hip_status(dec ? pf::launch_relpos_decode_join(a, s) : pf::launch_relpos_fwd_join(a, s),
                    "attention forward join");
}

pf_status pf_attn_relpos_bwd(const pf_layout *L, const pf_relpos *R, int32_t B, int32_t H, int32_t H_kv,
                             int32_t S, int32_t d, float scale, const pf_attn_tensor *Q,
                             const pf_attn_tensor *K, const pf_attn_tensor *V, const float *bias,
                             const pf_attn_tensor *O, const float *lse, const pf_attn_tensor *dO,
                             const pf_attn_tensor *dQ, const pf_attn_tensor *dK, const pf_attn_tensor *dV,
                             float *dtable, const int32_t *kv_len, void *workspace, size_t ws_bytes,
                             void *stream) {
  const RelposDims m{B, H, H_kv, S, S, d, scale};
  pf_status st = check_relpos(L, R, m, bias, nullptr, kv_len);
  if (st != PF_OK) return st;
  if ((st = check_rows(Q, "Q", S, false, B, H)) != PF_OK || (st = check_rows(K, "K", S, false, B, H_kv)) != PF_OK ||
      (st = check_rows(V, "V", S, false, B, H_kv)) != PF_OK || (st = check_rows(O, "O", S, false, B, H)) != PF_OK ||
      (st = check_rows(dO, "dO", S, false, B, H)) != PF_OK || (st = check_rows(dQ, "dQ", S, true, B, H)) != PF_OK ||
      (st = check_rows(dK, "dK", S, true, B, H_kv)) != PF_OK ||
      (st = check_rows(dV, "dV", S, true, B, H_kv)) != PF_OK || (st = need_ptr(lse, "lse")) != PF_OK ||
      (st = need_ptr(dtable, "dtable")) != PF_OK)
    return st;
  const BwdPlan p = bwd_plan(L, R, B, H, H_kv, S);
  if (!p.dq.fits() || !p.dkv.fits()) return fail(PF_ERR_UNSUPPORTED, "too many blocks for one launch");
  if ((st = need_ws(p.total, workspace, ws_bytes)) != PF_OK) return st;
  if ((st = check_state(L)) != PF_OK || (st = relpos_state(R)) != PF_OK) return st;
  pf::RelposArgs a = relpos_args(L, R, m, bias, nullptr, kv_len);
  a.Q = view(Q); a.K = view(K); a.V = view(V); a.O = view(O); a.dO = view(dO);
  a.dQ = view_out(dQ); a.dK = view_out(dK); a.dV = view_out(dV);
  a.lse_in = lse;
  a.delta = (float *)workspace;
  a.partials = (float *)((char *)workspace + p.partials);
  a.slots = (float *)((char *)workspace + p.slots);
  hipStream_t s = (hipStream_t)stream;
  auto run = [&](pf_kernel_class k, const char *what, auto &&launch) {
    if (st != PF_OK) return;
    Timed t(k, s);
    st = hip_status(launch(), what);
  };
  p.dq.set(a);
  run(PF_KERNEL_ATTN_BWD_DQ, "attention dQ kernel", [&] { return pf::launch_relpos_bwd_dq(a, s); });
  if (p.dq.slots())
    run(PF_KERNEL_REDUCE, "dQ join", [&] { return pf::launch_relpos_bwd_join(false, a, s); });
  // The dQ launch's partials: whole rounds of the 8 XCDs.
  a.dtable = dtable;
  a.tab_wg = (H * ((R->n_buckets + pf::kRelposTabCols - 1) / pf::kRelposTabCols) + 7) / 8 * 8;
  a.tab_nl = p.dq.nlong * p.dq.plong;
  a.tab_ns = (p.dq.ntile - p.dq.nlong) * p.dq.pshort;
  p.dkv.set(a);
  run(PF_KERNEL_ATTN_BWD_DKV, "attention dK/dV kernel", [&] { return pf::launch_relpos_bwd_dkv(a, s); });
  if (p.dkv.slots())
    run(PF_KERNEL_REDUCE, "dK/dV join", [&] { return pf::launch_relpos_bwd_join(true, a, s); });
  return st;
}

}  // extern "C"
