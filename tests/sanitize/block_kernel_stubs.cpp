// Stand-ins for the kernel launchers of capi_block.cpp in a host-only build
// under the sanitizers.  The epilogue's way back needs no uploaded layout, so its
// calls reach their launches: these keep the arguments for the driver.  The
// attention's never do, as no plan is uploaded: reaching one aborts.
#include <cstdio>
#include <cstdlib>

#include "block_stubs.h"

namespace pf {

ActBwdArgs g_act;
int g_act_launches = 0, g_dbias_launches = 0;

hipError_t launch_act_bwd(int, const ActBwdArgs &a, hipStream_t) {
  g_act = a;
  ++g_act_launches;
  return hipSuccess;
}
hipError_t launch_act_dbias(int, const ActBwdArgs &, hipStream_t) {
  ++g_dbias_launches;
  return hipSuccess;
}

[[noreturn]] static void no_kernels(const char *f) {
  std::fprintf(stderr, "kernel launcher %s reached in the host-only build\n", f);
  std::abort();
}
hipError_t launch_relpos_bias(const RelposBiasArgs &, int, hipStream_t) { no_kernels("relpos_bias"); }
hipError_t launch_relpos_fwd(const RelposArgs &, hipStream_t) { no_kernels("relpos_fwd"); }
hipError_t launch_relpos_decode(const RelposArgs &, hipStream_t) { no_kernels("relpos_decode"); }
hipError_t launch_relpos_decode_join(const RelposArgs &, hipStream_t) { no_kernels("relpos_decode_join"); }
hipError_t launch_relpos_fwd_join(const RelposArgs &, hipStream_t) { no_kernels("relpos_fwd_join"); }
hipError_t launch_relpos_bwd_dq(const RelposArgs &, hipStream_t) { no_kernels("relpos_bwd_dq"); }
hipError_t launch_relpos_bwd_dkv(const RelposArgs &, hipStream_t) { no_kernels("relpos_bwd_dkv"); }
hipError_t launch_relpos_bwd_join(bool, const RelposArgs &, hipStream_t) { no_kernels("relpos_bwd_join"); }

}  // namespace pf
