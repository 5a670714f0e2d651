// Stand-ins for the kernel launchers of capi_train.cpp in a host-only build under
// the sanitizers.  The gated product's way back and layer normalisation need nothing
// uploaded, so their calls reach their launches: these keep the arguments for the
// driver.  Those of the gradients never do, as no list is uploaded: reaching one
// aborts.
#include <cstdio>
#include <cstdlib>

#include "train_stubs.h"

namespace pf {

GatedBwdArgs g_gated;
ActBwdArgs g_dbias;
NormArgs g_norm;
int g_launches = 0, g_sums = 0;

hipError_t launch_gated_bwd(int, const GatedBwdArgs &a, hipStream_t) {
  g_gated = a;
  ++g_launches;
  return hipSuccess;
}
hipError_t launch_act_dbias(int, const ActBwdArgs &a, hipStream_t) {
  g_dbias = a;
  ++g_sums;
  return hipSuccess;
}
hipError_t launch_norm_fwd(int, const NormArgs &a, hipStream_t) {
  g_norm = a;
  ++g_launches;
  return hipSuccess;
}
hipError_t launch_norm_bwd(int, const NormArgs &a, hipStream_t) {
  g_norm = a;
  ++g_launches;
  return hipSuccess;
}
hipError_t launch_norm_sum(int, const NormArgs &, hipStream_t) {
  ++g_sums;
  return hipSuccess;
}

[[noreturn]] static void no_kernels(const char *f) {
  std::fprintf(stderr, "kernel launcher %s reached in the host-only build\n", f);
  std::abort();
}
hipError_t launch_grad_sumsq(const GradArgs &, hipStream_t) { no_kernels("grad_sumsq"); }
hipError_t launch_grad_total(const GradArgs &, hipStream_t) { no_kernels("grad_total"); }
hipError_t launch_grad_scale(const GradArgs &, int, hipStream_t) { no_kernels("grad_scale"); }

}  // namespace pf
