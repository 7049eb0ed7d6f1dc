// Error reporting of the C ABI, and what the launches of several files need once per device.
#include "ll_common.h"

#include <mutex>
#include <utility>
#include <vector>

namespace ll {

static thread_local int g_last_hip_error = 0;

int hip_failed(hipError_t e) {
  g_last_hip_error = (int)e;
  (void)hipGetLastError();   // clear the sticky error so that later calls start clean
  return LL_EHIP;
}

// A kernel that uses more than 64 KB of dynamic LDS has to be told so once per device; remembered
// here so that the hot path makes no attribute call.
int allow_dynamic_lds(const void* kern, size_t lds) {
  static std::mutex mu;
  static std::vector<std::pair<int, const void*>> done;
  int dev = -1;
  LL_HIP_CHECK(hipGetDevice(&dev));
  std::lock_guard<std::mutex> lock(mu);
  for (const auto& e : done)
    if (e.first == dev && e.second == kern) return LL_OK;
  LL_HIP_CHECK(hipFuncSetAttribute(kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
  done.emplace_back(dev, kern);
  return LL_OK;
}

}  // namespace ll

extern "C" {

const char* ll_error_string(int code) {
  switch (code) {
    case LL_OK: return "success";
    case LL_EINVAL: return "invalid argument (null pointer, bad size or alignment, k out of range, d not a multiple of 8)";
    case LL_EWORKSPACE: return "workspace missing, misaligned or smaller than required";
    case LL_EHIP: return "a HIP call failed (see ll_last_hip_error)";
    case LL_ESCRATCH: return "the shape needs more than the library's static scratch buffer holds (use ll_project with a workspace)";
    default: return "unknown error code";
  }
}

int ll_last_hip_error(void) { return ll::g_last_hip_error; }

}  // extern "C"
