// Dynamic LDS beyond 64 KiB has to be allowed per kernel function, and a function's attributes belong to its copy on the device that is current when they
// are set: once per function and device, not once per process.
#pragma once
#include <atomic>
#include <cstdint>
#ifdef __HIPCC__
#include <hip/hip_runtime.h>
#endif

namespace lc {

// The devices something has been done on.  (Those past the 64th are never remembered: there it is done again every time.)
class DevicesDone {
 public:
  bool has(int device) const { return known(device) && (bits_.load(std::memory_order_acquire) >> device & 1u) != 0; }
  void add(int device) {
    if (known(device)) bits_.fetch_or(uint64_t(1) << device, std::memory_order_release);
  }

 private:
  static bool known(int device) { return device >= 0 && device < 64; }
  std::atomic<uint64_t> bits_{0};
};

#ifdef __HIPCC__
// Allows the kernels all of a CU's LDS on the current device.  `raised`: one per set of functions (a static of their launcher).
template <typename... Kernels>
inline hipError_t raise_lds_limit(DevicesDone* raised, Kernels... kernels) {
  int device = 0;
  hipError_t e = hipGetDevice(&device);
  if (e != hipSuccess || raised->has(device)) return e;
  for (const void* kernel : {reinterpret_cast<const void*>(kernels)...})
    if (e == hipSuccess) e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
  if (e == hipSuccess) raised->add(device);
  return e;
}
#endif

}  // namespace lc
