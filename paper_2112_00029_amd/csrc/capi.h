// Helpers of the C ABI's source files: error reporting, argument checks and
// the kernel timing hook.
#pragma once

#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <atomic>
#include <mutex>
#include <string>
#include <vector>

#include "layout.h"
#include "pf_internal.h"
#include "pixelfly.h"

namespace pf {
namespace capi {

extern thread_local std::string g_err;  // the calling thread's last error

inline pf_status fail(pf_status s, const std::string &msg) {
  g_err = msg;
  return s;
}

inline bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }

// Kernel timing hook (pf_timing_begin / pf_timing_end): per kernel class,
// event pairs recorded around the next `cap` launches.
struct KernelTimer {
  std::mutex mu;
  std::atomic<int> armed{0};
  int cap = 0;
  std::vector<hipEvent_t> ev[PF_KERNEL_COUNT];  // 2 * cap each: start, end
  int n[PF_KERNEL_COUNT] = {};

  void release() {
    for (auto &v : ev) {
      for (hipEvent_t e : v)
        if (e) (void)hipEventDestroy(e);
      v.clear();
    }
    std::fill(n, n + PF_KERNEL_COUNT, 0);
    cap = 0;
  }
};
extern KernelTimer g_kt;

// Scope around one kernel launch: when the hook is armed and the class has
// room, hands the next launch a pair of events (recorded by the dispatch at
// the kernel's start and end) and counts it if the launch took them.
class Timed {
 public:
  Timed(pf_kernel_class k, hipStream_t) : k_(k) {
    if (!g_kt.armed.load(std::memory_order_acquire) || g_kt.n[k] >= g_kt.cap) return;
    pf::next_launch_events() = {g_kt.ev[k][2 * g_kt.n[k]], g_kt.ev[k][2 * g_kt.n[k] + 1]};
    on_ = true;
  }
  ~Timed() {
    if (!on_) return;
    pf::LaunchEvents &e = pf::next_launch_events();
    if (!e.start) g_kt.n[k_]++;  // consumed by a launch
    e.start = e.stop = nullptr;
  }
  Timed(const Timed &) = delete;
  Timed &operator=(const Timed &) = delete;

 private:
  pf_kernel_class k_;
  bool on_ = false;
};

inline pf_status need_ptr(const void *p, const char *name) {
  if (!p) return fail(PF_ERR_INVALID_ARG, std::string(name) + " is NULL");
  if (!aligned16(p))
    return fail(PF_ERR_INVALID_ARG, std::string(name) + " is not 16-byte aligned");
  return PF_OK;
}

inline bool kernel_block(int32_t b) { return b == 32 || b == 64 || b == 128; }

inline pf_status check_layout_arg(const pf_layout *L) {
  if (!L) return fail(PF_ERR_INVALID_ARG, "layout is NULL");
  if (!kernel_block(L->b))
    return fail(PF_ERR_UNSUPPORTED, "kernels support b in {32, 64, 128}");
  return PF_OK;
}

// Called after all argument checks: the layout must live on this device.
inline pf_status check_state(const pf_layout *L) {
  if (L->device < 0 || !L->dev_mem)
    return fail(PF_ERR_STATE, "layout not uploaded (call pf_layout_upload)");
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess || dev != L->device)
    return fail(PF_ERR_STATE, "layout was uploaded to another device");
  return PF_OK;
}

inline pf_status hip_status(hipError_t e, const char *what) {
  if (e == hipSuccess) return PF_OK;
  return fail(PF_ERR_HIP, std::string(what) + ": " + hipGetErrorString(e));
}

// Workspace of at least `need` bytes (0: none needed).
inline pf_status need_ws(size_t need, const void *ws, size_t ws_bytes) {
  if (need == 0) return PF_OK;
  if (ws_bytes < need)
    return fail(PF_ERR_WORKSPACE, "workspace needs " + std::to_string(need) + " bytes");
  return need_ptr(ws, "workspace");
}

}  // namespace capi
}  // namespace pf
