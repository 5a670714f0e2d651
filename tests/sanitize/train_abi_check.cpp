// Host-only driver of the operators of a training step for the sanitizer build:
// gated layouts of many shapes against the mask they double, the launch plans of
// the gated product's way back and of layer normalisation (every row and column
// once, partials inside the workspace), gradient lists of random tensors against a
// count of the bytes they cover, and every entry point with bad arguments.  No device
// is used.  Exits 0 when every expectation holds.
#include <cstdint>
#include <cstdio>
#include <map>
#include <random>
#include <vector>

#include "layout.h"
#include "pixelfly.h"
#include "train_stubs.h"

static int g_fail = 0;
#define EXPECT(cond)                                                            \
  do {                                                                          \
    if (!(cond) && ++g_fail < 40)                                               \
      std::fprintf(stderr, "%s:%d: expectation failed: %s (%s)\n", __FILE__,    \
                   __LINE__, #cond, pf_last_error());                           \
  } while (0)

static void *const AT = (void *)0x100000;

// The pairs of a tile list: slots 2 p and 2 p + 1 hold blocks 2 i and 2 i + 1, each
// pair once.
static void check_pairs(const std::vector<pf::NTTile> &tiles, int G, int nb_out) {
  if (G % 2) return;  // (not a list of the gated forward)
  std::vector<int> seen(nb_out / 2, 0);
  for (const auto &t : tiles) {
    EXPECT(t.g % 2 == 0 && t.g >= 2 && t.g <= G);
    for (int p = 0; p + 1 < t.g; p += 2) {
      EXPECT(t.out_blk[p] % 2 == 0 && t.out_blk[p + 1] == t.out_blk[p] + 1 && t.out_blk[p + 1] < nb_out);
      if (t.out_blk[p] / 2 < nb_out / 2) ++seen[t.out_blk[p] / 2];
    }
  }
  for (int n : seen) EXPECT(n == 1);
}

static void layouts(std::mt19937 &rng) {
  for (int b : {32, 64, 128, 16})
    for (int i = 0; i < 60; ++i) {
      const int64_t no = 1 + rng() % 70, ni = 1 + rng() % 40;
      const int ms = 1 << rng() % 7;
      pf_layout *L = nullptr, *one = nullptr;
      EXPECT(pf_layout_create_gated(no * b, ni * b, b, ms, &L) == PF_OK);
      EXPECT(pf_layout_create(no * b, ni * b, b, ms, &one) == PF_OK);
      if (L && one) {
        EXPECT(L->gated && !one->gated && L->nnzb == 2 * one->nnzb && L->nb_out == 2 * one->nb_out);
        EXPECT(L->n_out == 2 * no * b && pf_layout_check(L) == PF_OK);
        for (int r = 0; r < L->nb_out; ++r) {
          EXPECT(L->row_ptr[r + 1] - L->row_ptr[r] == one->row_ptr[r / 2 + 1] - one->row_ptr[r / 2]);
          for (int k = L->row_ptr[r]; k < L->row_ptr[r + 1]; ++k)
            EXPECT(L->col_idx[k] == one->col_idx[one->row_ptr[r / 2] + k - L->row_ptr[r]]);
        }
        // The lists the gated forward takes: wide ones for blocks of 128, both others.
        if (b >= 32) {
          EXPECT(L->G_fwd_w % 2 == 0);
          if (b < 128) EXPECT(L->G_fwd % 2 == 0);
          check_pairs(L->fwd_tiles_w, L->G_fwd_w, L->nb_out);
          check_pairs(L->fwd_tiles, L->G_fwd, L->nb_out);
        }
      }
      pf_layout_destroy(L);
      pf_layout_destroy(one);
      std::vector<uint8_t> m(no * ni);
      for (auto &x : m) x = rng() % 3 == 0;
      for (int64_t r = 0; r < no; ++r) m[r * ni + rng() % ni] = 1;
      EXPECT(pf_layout_create_gated_from_mask((int)no, (int)ni, b, m.data(), &L) == PF_OK);
      if (L) {
        EXPECT(L->gated && pf_layout_check(L) == PF_OK);
        if (b >= 32) check_pairs(L->fwd_tiles_w, L->G_fwd_w, L->nb_out);
      }
      pf_layout_destroy(L);
    }
  pf_layout *L = (pf_layout *)AT;
  EXPECT(pf_layout_create_gated(64, 64, 32, 3, &L) == PF_ERR_INVALID_ARG && !L);
  EXPECT(pf_layout_create_gated(64, 64, 32, 2, nullptr) == PF_ERR_INVALID_ARG);
  EXPECT(pf_layout_create_gated_from_mask(2, 2, 32, nullptr, &L) == PF_ERR_INVALID_ARG && !L);
  EXPECT(pf_layout_create_gated((int64_t)1 << 45, 64, 32, 2, &L) == PF_ERR_INVALID_ARG && !L);
}

static void gated_bwd(std::mt19937 &rng) {
  for (int i = 0; i < 3000; ++i) {
    const pf_dtype dt = rng() % 2 ? PF_BF16 : PF_FP32;
    const int b = 32 << rng() % 3;
    const int64_t N = b * (1 + (int64_t)(rng() % 4 ? rng() % 40 : rng() % 4000));
    const int64_t T = rng() % 50 == 0 ? (int64_t)1 << 30 : 1 + rng() % (rng() % 3 ? 300 : 40000);
    const bool sums = rng() % 4 != 0;
    const size_t ws = pf_linear_gated_workspace_bytes(dt, T, N);
    pf::g_launches = pf::g_sums = 0;
    const pf_status st = pf_linear_gated_bwd(dt, T, N, b, PF_ACT_GELU, AT, AT, AT, sums ? AT : nullptr,
                                             ws ? AT : nullptr, ws, nullptr);
    EXPECT(st == PF_OK && pf::g_launches == 1);
    const pf::GatedBwdArgs &a = pf::g_gated;
    const int64_t v = dt == PF_BF16 ? 8 : 4;
    EXPECT(a.cw >= 1 && a.cw <= 64 && 256 % a.cw == 0);
    // Columns: the last group begins inside the row and ends at or past its end.
    EXPECT((int64_t)a.groups * a.cw * v >= N && ((int64_t)a.groups - 1) * a.cw * v < N);
    EXPECT(a.nparts >= 1 && a.nparts * a.rows_per_part >= T && (a.nparts - 1) * a.rows_per_part < T);
    EXPECT((int64_t)a.groups * a.nparts <= 0x7fffffff);
    EXPECT((pf::g_sums == 1) == (sums && a.nparts > 1));
    if (sums && a.nparts > 1) {
      EXPECT((size_t)a.nparts * 2 * N * sizeof(float) <= ws && a.partials == (float *)AT);
      EXPECT(pf::g_dbias.nparts == a.nparts && pf::g_dbias.N == 2 * N && pf::g_dbias.N % 16 == 0);
    } else {
      EXPECT(!a.partials);
    }
  }
}

static void norms(std::mt19937 &rng) {
  for (int i = 0; i < 6000; ++i) {
    const pf_dtype dt = rng() % 2 ? PF_BF16 : PF_FP32;
    const int64_t N = rng() % 3 ? 1 + rng() % 16384 : 8 * (1 + rng() % 2048);
    const int64_t T = rng() % 50 == 0 ? (int64_t)1 << 30 : 1 + rng() % (rng() % 3 ? 300 : 40000);
    const int64_t pad = rng() % 2 ? 0 : rng() % 40;
    const size_t ws = pf_layernorm_workspace_bytes(dt, T, N);
    const bool back = rng() % 2, sums = rng() % 4 != 0;
    pf::g_launches = pf::g_sums = 0;
    const pf_status st =
        back ? pf_layernorm_bwd(dt, T, N, AT, N + pad, AT, N + pad, AT, (float *)AT, (float *)AT, AT, N + pad, AT,
                                N + pad, sums ? AT : nullptr, nullptr, ws ? AT : nullptr, ws, nullptr)
             : pf_layernorm_fwd(dt, T, N, 1e-5f, AT, N + pad, AT, AT, AT, N + pad, nullptr, nullptr, nullptr);
    EXPECT(st == PF_OK && pf::g_launches == 1);
    const pf::NormArgs &a = pf::g_norm;
    const int vw = dt == PF_BF16 ? 8 : 4;
    EXPECT(a.tpr == 64 || a.tpr == 128 || a.tpr == 256 || a.tpr == 512 || a.tpr == 1024);
    EXPECT((int64_t)a.tpr * vw * a.chunks >= N && (N >= vw || a.tpr == 64));
    EXPECT(a.chunks == 1 || a.chunks == 2 || (vw == 4 && a.chunks == 4) ||
           (back && a.tpr == 512 && a.chunks == 32 / vw));
    EXPECT(!back || a.tpr <= 512);
    EXPECT(a.parts >= 1 && a.parts <= T);
    if (back) {
      EXPECT((pf::g_sums == 1) == (sums && a.parts > 1));
      if (sums && a.parts > 1) EXPECT((size_t)a.parts * 2 * N * sizeof(float) <= ws && a.partials == (float *)AT);
      else EXPECT(!a.partials);
    }
  }
}

// Random lists: refused exactly when a written byte is another span's.
static void lists(std::mt19937 &rng) {
  for (int i = 0; i < 4000; ++i) {
    const int n = rng() % 6;
    std::vector<pf_grad_tensor> t(n);
    std::map<uint64_t, int> reads, writes;
    bool bad = false;
    for (auto &x : t) {
      x.src_dtype = rng() % 2;
      x.dst_dtype = rng() % 2;
      x.n = rng() % 5 ? rng() % 20 : 0;
      const uint64_t src = 0x10000 + 4 * (rng() % 100);
      uint64_t dst = rng() % 2 ? src : 0x10000 + 4 * (rng() % 300);
      if (src == dst) x.dst_dtype = x.src_dtype;
      x.src = (const void *)src;
      x.dst = (void *)dst;
      const int ss = x.src_dtype ? 4 : 2, ds = x.dst_dtype ? 4 : 2;
      for (uint64_t k = 0; k < (uint64_t)x.n * ds; ++k) ++writes[dst + k];
      if (src != dst)
        for (uint64_t k = 0; k < (uint64_t)x.n * ss; ++k) ++reads[src + k];
    }
    for (auto &w : writes) bad |= w.second > 1 || reads.count(w.first);
    pf_grads *g = nullptr;
    const pf_status st = pf_grads_create(n, t.data(), &g);
    EXPECT((st == PF_OK) == !bad && (g != nullptr) == !bad);
    if (g) {
      const size_t ws = pf_grads_workspace_bytes(g);
      EXPECT(ws >= sizeof(double));
      EXPECT(pf_grads_clip(g, 1.f, nullptr, AT, ws, nullptr) == PF_ERR_STATE);
      EXPECT(pf_grads_scale(g, 1.f, (double *)AT, nullptr) == PF_ERR_STATE);
      EXPECT(pf_grads_norm(g, (double *)AT, nullptr, AT, ws, nullptr) == PF_ERR_STATE);
      EXPECT(pf_grads_clip(g, 1.f, nullptr, AT, ws - 1, nullptr) == PF_ERR_WORKSPACE);
    }
    pf_grads_destroy(g);
  }
  pf_grads *g = nullptr;
  EXPECT(pf_grads_create(-1, nullptr, &g) == PF_ERR_INVALID_ARG);
  EXPECT(pf_grads_create(1, nullptr, &g) == PF_ERR_INVALID_ARG);
  EXPECT(pf_grads_create(0, nullptr, nullptr) == PF_ERR_INVALID_ARG);
  EXPECT(pf_grads_upload(nullptr, nullptr) == PF_ERR_INVALID_ARG);
  EXPECT(pf_grads_workspace_bytes(nullptr) == 0);
  pf_grads_destroy(nullptr);
}

static void bad_calls() {
  EXPECT(pf_linear_gated_fwd(nullptr, PF_BF16, 1, 0, AT, AT, nullptr, nullptr, nullptr, PF_ACT_SILU, AT, nullptr,
                             nullptr, nullptr, 0, nullptr) == PF_ERR_INVALID_ARG);
  pf_layout *L = nullptr;
  EXPECT(pf_layout_create_gated(256, 128, 64, 2, &L) == PF_OK);
  EXPECT(pf_linear_gated_fwd(L, PF_BF16, 1, 0, AT, AT, nullptr, nullptr, nullptr, PF_ACT_SILU, AT, nullptr, nullptr,
                             nullptr, 0, nullptr) == PF_ERR_STATE);
  EXPECT(pf_linear_gated_fwd(L, PF_BF16, 0, 0, AT, AT, nullptr, nullptr, nullptr, PF_ACT_SILU, AT, nullptr, nullptr,
                             nullptr, 0, nullptr) == PF_ERR_INVALID_ARG);
  EXPECT(pf_linear_gated_fwd_mixed(L, PF_BF16, 1, 0, 0.5f, AT, AT, nullptr, nullptr, AT, PF_ACT_RELU, AT, AT, nullptr,
                                   nullptr, 0, nullptr) == PF_ERR_STATE);
  pf_layout_destroy(L);
}

int main() {
  std::mt19937 rng(5);
  layouts(rng);
  gated_bwd(rng);
  norms(rng);
  lists(rng);
  bad_calls();
  std::printf("%d failed expectations\n", g_fail);
  return g_fail ? 1 : 0;
}
