// Host-only driver of the operators round the matrices for the sanitizer
// build: bucket maps and plans of every shape, the logarithmic maps' thresholds,
// workspaces and launch plans over sequences, heads and layouts, tensors of random
// strides against a count of the elements they cover, the way back's launch plan
// over token and column counts, and every entry point with bad arguments.
// No device is used.  Exits 0 when every expectation holds.
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <random>
#include <set>
#include <vector>

#include "block_stubs.h"
#include "pixelfly.h"
#include "relpos.h"

static int g_fail = 0;
#define EXPECT(cond)                                                            \
  do {                                                                          \
    if (!(cond) && ++g_fail < 40)                                               \
      std::fprintf(stderr, "%s:%d: expectation failed: %s (%s)\n", __FILE__,    \
                   __LINE__, #cond, pf_last_error());                           \
  } while (0)

static void *const AT = (void *)0x100000;

// The plan's block offsets against the map itself.
static void check_plan(const pf_relpos *R) {
  const int32_t *bucket = nullptr;
  int64_t seq = 0;
  int32_t nbk = 0;
  EXPECT(pf_relpos_buckets_get(R, &bucket, &seq, &nbk) == PF_OK);
  EXPECT(pf_relpos_bias_floats(R) == (size_t)seq * 4);
  const int nb = (int)(seq / 64);
  int lo = 1, hi = 0;
  bool any = false;
  std::vector<bool> named(R->order.size() / 64, false);
  for (int d = -(nb - 1); d < nb; ++d) {
    std::set<int32_t> have;
    for (int x = 1; x < 128; ++x) {
      const int64_t i = (int64_t)d * 64 + x - 64 + seq - 1;
      EXPECT(i >= 0 && i < 2 * seq - 1);
      have.insert(bucket[i]);
    }
    const int32_t info = R->info[d + nb - 1];
    if (have.size() == 1) {
      EXPECT(info == *have.begin());
    } else {
      const size_t m = info - pf::kRelposMixed;
      EXPECT(info >= pf::kRelposMixed && m < named.size() && !named[m]);
      if (m >= named.size()) return;
      named[m] = true;
      std::set<uint32_t> pos;
      uint32_t last = 0;
      for (int l = 0; l < 64; ++l) {
        const uint32_t w = R->order[m * 64 + l];
        for (int half = 0; half < 2; ++half) {
          const uint32_t p = w >> (8 * half) & 255, c = w >> (16 + 8 * half) & 255;
          EXPECT(p < 128 && c >= last && (int32_t)c < nbk);
          pos.insert(p);
          last = c;
          const int32_t b = p == 0 ? -1 : bucket[(int64_t)d * 64 + (int64_t)p - 64 + seq - 1];
          EXPECT(c == (uint32_t)(b < 0 ? 0 : b));
        }
      }
      EXPECT(pos.size() == 128);
    }
    if (have.size() > 1 || *have.begin() >= 0) {
      if (!any) lo = d;
      hi = d;
      any = true;
    }
  }
  EXPECT(R->omin == lo && R->omax == hi);
}

static void maps(std::mt19937 &rng) {
  for (int64_t seq : {64, 128, 192, 1024, 4096})
    for (int32_t n : {1, 2, 41, 256})
      for (int kind = 0; kind < 4; ++kind) {
        std::vector<int32_t> b(2 * seq - 1);
        for (int64_t i = 0; i < 2 * seq - 1; ++i) {
          const int64_t d = i - (seq - 1);
          b[i] = kind == 0   ? (int32_t)(rng() % (n + 1)) - 1
                 : kind == 1 ? (d > 0 ? -1 : (int32_t)std::min<int64_t>(-d, n - 1))
                 : kind == 2 ? -1
                             : (int32_t)((d + seq) / 100 % n);
        }
        pf_relpos *R = nullptr;
        EXPECT(pf_relpos_create(seq, n, b.data(), &R) == PF_OK && R);
        if (!R) continue;
        check_plan(R);
        pf_relpos_destroy(R);
      }
  // Logarithmic maps: bucket e + k of distance d as the logarithm says, where
  // it is not within rounding of a threshold.
  for (int both = 0; both < 2; ++both)
    for (int32_t n : {2, 3, 4, 5, 7, 16, 32, 100, 254, 256})
      for (int64_t reach : {(int64_t)129, (int64_t)1000, (int64_t)1 << 20, (int64_t)0x7fffffff}) {
        pf_relpos *R = nullptr;
        const int64_t seq = 2048;
        const pf_status st = pf_relpos_create_log(seq, n, reach, both, &R);
        const int half = both ? n / 2 : n, e = half / 2;
        if (half < 2 || (both && n % 2)) {
          EXPECT(st == PF_ERR_INVALID_ARG && !R);
          continue;
        }
        EXPECT(st == PF_OK && R);
        if (!R) continue;
        check_plan(R);
        const int32_t *b = nullptr;
        pf_relpos_buckets_get(R, &b, nullptr, nullptr);
        for (int64_t i = 0; i < 2 * seq - 1; ++i) {
          const int64_t dist = i - (seq - 1), d = dist < 0 ? -dist : dist;
          const long double x =
              d < e ? 0 : (half - e) * std::log((long double)d / e) / std::log((long double)reach / e);
          const long double near = std::abs(x - std::round(x));
          const int64_t c = d < e ? d : std::min<int64_t>(half - 1, e + (int64_t)std::floor(x));
          const int64_t got = dist > 0 ? (both ? b[i] - half : b[i]) : b[i];
          if (dist > 0 && !both) EXPECT(b[i] == -1);
          else if (d < e || near > 1e-12L) EXPECT(got == c);
          else EXPECT(got == std::min<int64_t>(half - 1, e + (int64_t)std::llround(x)));
        }
        pf_relpos_destroy(R);
      }
  // The largest plan.
  pf_relpos *R = nullptr;
  EXPECT(pf_relpos_create_log(1 << 20, 256, 1 << 19, 1, &R) == PF_OK);
  pf_relpos_destroy(R);
}

struct Call {
  const pf_layout *L;
  const pf_relpos *R;
  int32_t B = 1, H = 1, Hkv = 1, Sq = 1, Skv = 1;
  size_t ws = (size_t)1 << 46;
  pf_attn_tensor t(int64_t heads, int64_t rows) const { return {AT, heads * rows * 64, rows * 64, 64}; }
  pf_status fwd(const pf_attn_tensor *O = nullptr, const int32_t *start = nullptr) const {
    const pf_attn_tensor q = t(H, Sq), k = t(Hkv, Skv), o = O ? *O : q;
    return pf_attn_relpos_fwd(L, R, B, H, Hkv, Sq, Skv, 64, 0.125f, &q, &k, &k, (float *)AT, &o, (float *)AT, start,
                              nullptr, AT, ws, nullptr);
  }
  pf_status bwd(const pf_attn_tensor *dQ = nullptr) const {
    const pf_attn_tensor q = t(H, Sq), k = t(Hkv, Sq), dq = dQ ? *dQ : q;
    return pf_attn_relpos_bwd(L, R, B, H, Hkv, Sq, 64, 0.125f, &q, &k, &k, (float *)AT, &q, (float *)AT, &q, &dq, &k,
                              &k, (float *)AT, nullptr, AT, ws, nullptr);
  }
};

static void plans(std::mt19937 &rng) {
  for (int64_t seq : {64, 128, 832, 4096, 65536}) {
    const int nb = (int)(seq / 64);
    std::vector<pf_layout *> layouts;
    for (int32_t ms : {1, 4, 64})
      for (int32_t g : {0, 1, 2, nb}) {
        if (g > nb || (g == nb && nb > 64)) continue;
        pf_layout *L = nullptr;
        EXPECT(pf_layout_create_attention(seq, 64, ms, g, &L) == PF_OK);
        layouts.push_back(L);
      }
    if (nb <= 64) {
      std::vector<uint8_t> mask((size_t)nb * nb);
      for (auto &x : mask) x = rng() % 4 == 0;
      for (int i = 0; i < nb; ++i) mask[(size_t)i * nb + rng() % nb] = 1;
      pf_layout *L = nullptr;
      EXPECT(pf_layout_create_from_mask(nb, nb, 64, mask.data(), &L) == PF_OK);
      layouts.push_back(L);
    }
    for (int causal = 0; causal < 3; ++causal) {
      pf_relpos *R = nullptr;
      if (causal == 2) {
        std::vector<int32_t> none(2 * seq - 1, -1);
        EXPECT(pf_relpos_create(seq, 1, none.data(), &R) == PF_OK);
      } else {
        EXPECT(pf_relpos_create_log(seq, 32, 128, !causal, &R) == PF_OK);
      }
      for (const pf_layout *L : layouts)
        for (int i = 0; i < 40; ++i) {
          Call c{L, R};
          const int hs[] = {1, 2, 3, 12, 33, 64, 65535}, bs[] = {1, 2, 16, 300, 1 << 20};
          c.H = hs[rng() % 7];
          c.B = bs[rng() % 5];
          do c.Hkv = 1 + rng() % c.H;
          while (c.H % c.Hkv);
          c.Sq = i % 3 == 0 ? 1 : 1 + (int32_t)(rng() % seq);
          c.Skv = 1 + (int32_t)(rng() % seq);
          const size_t need = pf_attn_relpos_workspace_bytes(L, R, c.B, c.H, c.Sq);
          const bool fits = (int64_t)c.B * c.H <= 0x7fffffff / (nb + 1);
          EXPECT(fits || need == 0);
          for (const int32_t *start : {(const int32_t *)nullptr, (const int32_t *)AT}) {
            const pf_status st = c.fwd(nullptr, start);
            EXPECT(st == PF_ERR_STATE || (!fits && st == PF_ERR_INVALID_ARG) || st == PF_ERR_UNSUPPORTED);
            if (st != PF_ERR_STATE) continue;
            Call d = c;  // what the query says is enough
            d.ws = need;
            EXPECT(d.fwd(nullptr, start) == PF_ERR_STATE);
          }
          const pf_status st = c.bwd();
          EXPECT(st == PF_ERR_STATE || (!fits && st == PF_ERR_INVALID_ARG) || st == PF_ERR_UNSUPPORTED);
          if (st == PF_ERR_STATE) {
            Call d = c;
            d.ws = need;
            EXPECT(need >= (size_t)c.B * c.H * c.Sq * 4 && d.bwd() == PF_ERR_STATE);
            d.ws = 0;
            EXPECT(d.bwd() == PF_ERR_WORKSPACE);
          }
        }
      pf_relpos_destroy(R);
    }
    for (pf_layout *L : layouts) pf_layout_destroy(L);
  }
}

// Outputs of random strides: one that is taken has no two rows that meet.
static void strides(std::mt19937 &rng) {
  pf_layout *L = nullptr;
  pf_relpos *R = nullptr;
  EXPECT(pf_layout_create_attention(64, 64, 1, 0, &L) == PF_OK);
  EXPECT(pf_relpos_create_log(64, 8, 20, 1, &R) == PF_OK);
  int taken = 0, refused = 0;
  for (int i = 0; i < 20000; ++i) {
    Call c{L, R};
    c.B = 1 + rng() % 4;
    c.H = 1 + rng() % 4;
    c.Hkv = 1;
    c.Sq = 1 + rng() % 5;
    c.Skv = 1 + rng() % 5;
    auto pick = [&] { return (int64_t)(rng() % 3 == 0 ? rng() % 200 : 8 * (rng() % 60)); };
    pf_attn_tensor o{AT, pick(), pick(), pick()};
    const pf_status st = i % 2 ? c.fwd(&o) : c.bwd(&o);
    if (st != PF_ERR_STATE) {
      EXPECT(st == PF_ERR_INVALID_ARG);
      ++refused;
      continue;
    }
    ++taken;
    EXPECT(o.seq % 8 == 0 && o.head % 8 == 0 && o.token % 8 == 0 && o.token >= 64);
    std::set<int64_t> rows;
    bool meet = false;
    for (int b = 0; b < c.B; ++b)
      for (int h = 0; h < c.H; ++h)
        for (int r = 0; r < c.Sq; ++r) {
          const int64_t at = b * o.seq + h * o.head + r * o.token;
          auto next = rows.lower_bound(at);
          meet = meet || (next != rows.end() && *next < at + 64) || (next != rows.begin() && *std::prev(next) + 64 > at);
          rows.insert(at);
        }
    EXPECT(!meet);
  }
  EXPECT(taken > 1000 && refused > 1000);
  // Extreme strides.
  const int64_t big[] = {INT64_MIN, INT64_MIN + 8, -64, 0, 64, (int64_t)1 << 24, ((int64_t)1 << 24) + 8, (int64_t)1 << 40,
                         (int64_t)1 << 62, INT64_MAX - 7, INT64_MAX};
  for (int64_t s : big)
    for (int64_t h : big)
      for (int64_t t : big) {
        Call c{L, R};
        c.B = 3;
        c.H = 2;
        c.Sq = c.Skv = 60;
        pf_attn_tensor o{AT, s, h, t};
        for (const pf_status st : {c.fwd(&o), c.bwd(&o)})
          EXPECT(st == PF_ERR_STATE || st == PF_ERR_INVALID_ARG || st == PF_ERR_UNSUPPORTED);
      }
  pf_relpos_destroy(R);
  pf_layout_destroy(L);
}

// The way back's launch plan covers every row and column once.
static void way_back(std::mt19937 &rng) {
  for (int i = 0; i < 4000; ++i) {
    const pf_dtype dt = rng() % 2 ? PF_FP32 : PF_BF16;
    const int v = dt == PF_BF16 ? 8 : 4;
    int64_t T = 1 + (int64_t)(std::exp(std::uniform_real_distribution<>(0, 20.7)(rng)));
    int64_t N = 32 * (1 + (int64_t)(std::exp(std::uniform_real_distribution<>(0, 13.1)(rng))));
    T = std::min<int64_t>(T, (int64_t)1 << 30);
    N = std::min<int64_t>(N, (int64_t)1 << 24);
    const bool db = rng() % 2;
    const size_t need = pf_linear_act_workspace_bytes(dt, T, N);
    pf::g_act_launches = pf::g_dbias_launches = 0;
    EXPECT(pf_linear_act_bwd(dt, T, N, PF_ACT_SILU, AT, AT, AT, db ? AT : nullptr, AT, db ? need : 0, nullptr) == PF_OK);
    const pf::ActBwdArgs &a = pf::g_act;
    EXPECT(pf::g_act_launches == 1 && pf::g_dbias_launches == (db && need ? 1 : 0));
    EXPECT(a.T == T && a.N == N && a.cw >= 4 && a.cw <= 64 && 256 % a.cw == 0);
    EXPECT((int64_t)a.groups * a.cw * v >= N && (int64_t)(a.groups - 1) * a.cw * v < N);
    EXPECT(a.rows_per_part > 0 && a.rows_per_part % (256 / a.cw) == 0);
    EXPECT(a.nparts * a.rows_per_part >= T && (a.nparts - 1) * a.rows_per_part < T);
    EXPECT((int64_t)a.groups * a.nparts <= 0x7fffffff);
    EXPECT(!db || (a.nparts > 1) == (a.partials != nullptr));
    EXPECT(!a.partials || need >= (size_t)a.nparts * N * 4);
    if (db && need)
      EXPECT(pf_linear_act_bwd(dt, T, N, PF_ACT_GELU, AT, AT, AT, AT, AT, need - 1, nullptr) == PF_ERR_WORKSPACE);
  }
  const int before = pf::g_act_launches;
  for (int64_t T : {(int64_t)INT64_MIN, (int64_t)-1, (int64_t)0, ((int64_t)1 << 30) + 1, (int64_t)INT64_MAX}) {
    EXPECT(pf_linear_act_workspace_bytes(PF_BF16, T, 64) == 0);
    EXPECT(pf_linear_act_bwd(PF_BF16, T, 64, PF_ACT_GELU, AT, AT, AT, AT, AT, 1 << 30, nullptr) == PF_ERR_INVALID_ARG);
  }
  for (int64_t N : {(int64_t)INT64_MIN, (int64_t)-32, (int64_t)0, (int64_t)40, ((int64_t)1 << 24) + 32, (int64_t)INT64_MAX}) {
    EXPECT(pf_linear_act_workspace_bytes(PF_FP32, 8, N) == 0);
    EXPECT(pf_linear_act_bwd(PF_FP32, 8, N, PF_ACT_RELU, AT, AT, AT, AT, AT, 1 << 30, nullptr) == PF_ERR_INVALID_ARG);
  }
  EXPECT(pf::g_act_launches == before);
}

static void refusals() {
  pf_relpos *R = nullptr;
  const std::vector<int32_t> zero(127, 0);
  for (int64_t seq : {(int64_t)INT64_MIN, (int64_t)-64, (int64_t)0, (int64_t)65, ((int64_t)1 << 20) + 64, (int64_t)INT64_MAX}) {
    EXPECT(pf_relpos_create(seq, 1, zero.data(), &R) == PF_ERR_INVALID_ARG && !R);
    EXPECT(pf_relpos_create_log(seq, 32, 128, 1, &R) == PF_ERR_INVALID_ARG && !R);
  }
  for (int32_t n : {INT32_MIN, -1, 0, 257, INT32_MAX}) {
    EXPECT(pf_relpos_create(64, n, zero.data(), &R) == PF_ERR_INVALID_ARG && !R);
    EXPECT(pf_relpos_create_log(64, n, 128, 0, &R) == PF_ERR_INVALID_ARG && !R);
  }
  for (int64_t reach : {(int64_t)INT64_MIN, (int64_t)0, (int64_t)8, (int64_t)0x80000000, (int64_t)INT64_MAX})
    EXPECT(pf_relpos_create_log(64, 32, reach, 1, &R) == PF_ERR_INVALID_ARG && !R);
  EXPECT(pf_relpos_create(64, 1, nullptr, &R) == PF_ERR_INVALID_ARG && !R);
  EXPECT(pf_relpos_create(64, 1, zero.data(), nullptr) == PF_ERR_INVALID_ARG);
  for (int32_t bad : {INT32_MIN, -2, 1, INT32_MAX}) {
    auto m = zero;
    m[126] = bad;
    EXPECT(pf_relpos_create(64, 1, m.data(), &R) == PF_ERR_INVALID_ARG && !R);
  }
  EXPECT(pf_relpos_buckets_get(nullptr, nullptr, nullptr, nullptr) == PF_ERR_INVALID_ARG);
  EXPECT(pf_relpos_upload(nullptr, nullptr) == PF_ERR_INVALID_ARG);
  EXPECT(pf_relpos_bias_floats(nullptr) == 0);
  EXPECT(pf_relpos_create(64, 1, zero.data(), &R) == PF_OK);
  for (int32_t H : {INT32_MIN, 0, 65536, INT32_MAX})
    EXPECT(pf_relpos_bias(R, H, (float *)AT, (float *)AT, nullptr) == PF_ERR_INVALID_ARG);
  EXPECT(pf_relpos_bias(R, 65535, (float *)AT, (float *)AT, nullptr) == PF_ERR_STATE);
  pf_layout *L = nullptr;
  EXPECT(pf_layout_create_attention(64, 64, 1, 0, &L) == PF_OK);
  for (int32_t x : {INT32_MIN, -1, 0, INT32_MAX}) {
    for (int which = 0; which < 5; ++which) {
      Call c{L, R};
      (which == 0 ? c.B : which == 1 ? c.H : which == 2 ? c.Hkv : which == 3 ? c.Sq : c.Skv) = x;
      EXPECT(c.fwd() != PF_OK);
      if (which < 4) EXPECT(c.bwd() != PF_OK);
      EXPECT(which > 3 || which == 2 || (which == 0 && x > 0) || pf_attn_relpos_workspace_bytes(L, R, c.B, c.H, c.Sq) == 0);
    }
  }
  pf_layout_destroy(L);
  pf_relpos_destroy(R);
  pf_relpos_destroy(nullptr);
}

int main() {
  std::mt19937 rng(7);
  maps(rng);
  plans(rng);
  strides(rng);
  way_back(rng);
  refusals();
  std::printf("block ABI check: %d failed expectations\n", g_fail);
  return g_fail == 0 ? 0 : 1;
}
