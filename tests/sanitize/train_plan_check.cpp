// Host-only driver: every plan of layer normalisation and of the gated product's way
// back, through the entry points, against the kernels there are.  Prints, one a line,
// the normalisation kernels that some call takes ("fwd bf16 8 2 256 0": elements and
// number of a thread's chunks, threads a row, whether the last chunk overlaps), which
// the test compares with those in the library.
#include <cstdint>
#include <cstdio>
#include <set>
#include <string>

#include "pixelfly.h"
#include "train_stubs.h"

static void *const AT = (void *)0x100000;

int main() {
  int fail = 0;
  std::set<std::string> taken;
  for (pf_dtype dt : {PF_BF16, PF_FP32})
    for (int back = 0; back < 2; ++back)
      for (int64_t N = 1; N <= 16384; ++N)
        for (int64_t T : {(int64_t)1, (int64_t)700, (int64_t)1 << 20}) {
          const int vw = dt == PF_BF16 ? 8 : 4;
          const pf_status st =
              back ? pf_layernorm_bwd(dt, T, N, AT, N, AT, N, AT, (float *)AT, (float *)AT, nullptr, 0, AT, N,
                                      nullptr, nullptr, nullptr, 0, nullptr)
                   : pf_layernorm_fwd(dt, T, N, 1e-5f, AT, N, AT, AT, AT, N, nullptr, nullptr, nullptr);
          const pf::NormArgs &a = pf::g_norm;
          const bool single = N < vw;
          const bool ok = st == PF_OK && (single ? a.tpr == 64 && a.chunks == 1
                                                 : (int64_t)a.tpr * a.chunks * vw >= N &&
                                                       pf::norm_plan_exists(vw, back != 0, a.tpr, a.chunks));
          if (!ok && ++fail < 20)
            std::printf("no kernel: dtype %d back %d T %lld N %lld tpr %d chunks %d\n", (int)dt, back, (long long)T,
                        (long long)N, a.tpr, a.chunks);
          char line[64];
          std::snprintf(line, sizeof line, "%s %s %d %d %d %d", back ? "bwd" : "fwd", dt == PF_BF16 ? "bf16" : "fp32",
                        single ? 1 : vw, a.chunks, a.tpr, !single && N % vw != 0);
          taken.insert(line);
        }
  for (const auto &l : taken) std::printf("%s\n", l.c_str());
  for (int64_t N = 32; N <= (1 << 24); N += N < 40000 ? 32 : 99968)
    for (pf_dtype dt : {PF_BF16, PF_FP32}) {
      const pf_status st = pf_linear_gated_bwd(dt, 300, N, 32, PF_ACT_SILU, AT, AT, AT, nullptr, nullptr, 0, nullptr);
      const int cw = pf::g_gated.cw;
      if ((st != PF_OK || cw < 1 || cw > 32 || 256 % cw) && ++fail < 20)
        std::printf("gated way back: N %lld cw %d\n", (long long)N, cw);
    }
  std::printf("%d failed expectations\n", fail);
  return fail ? 1 : 0;
}
