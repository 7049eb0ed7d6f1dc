// Error reporting of the C ABI, and what the launches of several files need once per device.
#include "ll_common.h"

#include <atomic>

namespace ll {

static thread_local int g_last_hip_error = 0;

int hip_failed(hipError_t e) {
  g_last_hip_error = (int)e;
  (void)hipGetLastError();   // clear the sticky error so that later calls start clean
  return LL_EHIP;
}

// A kernel that uses more than 64 KB of dynamic LDS has to be told so once per device; remembered here so that the hot path makes no
// attribute call.  (Places of fixed number, taken in order and never given back: nothing here allocates, throws or waits.  Two threads may both ask for
// a kernel that is new, and past the last place every call asks: the attribute is the same each time.)
int allow_dynamic_lds(const void* kern, size_t lds) {
  constexpr int PLACES = 1024;
  struct Place {
    std::atomic<const void*> kern;
    int dev;
  };
  static Place places[PLACES];
  static std::atomic<int> taken{0};
  int dev = -1;
  LL_HIP_CHECK(hipGetDevice(&dev));
  for (const Place& e : places) {
    const void* k = e.kern.load(std::memory_order_acquire);   // (dev is written before it)
    if (k == kern && e.dev == dev) return LL_OK;
    if (k == nullptr) break;
  }
  LL_HIP_CHECK(hipFuncSetAttribute(kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
  const int at = taken.load(std::memory_order_relaxed) < PLACES ? taken.fetch_add(1, std::memory_order_relaxed) : PLACES;
  if (at < PLACES) {
    places[at].dev = dev;
    places[at].kern.store(kern, std::memory_order_release);
  }
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
