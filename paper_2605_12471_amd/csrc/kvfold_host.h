// Host-side helpers shared by the translation units that implement the C ABI.
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/kvfold.h"

namespace kvfold {

constexpr int kMaxDevices = 64;

// Records a HIP failure for kvfold_last_hip_error() of the calling thread, clears the runtime's sticky error and
// returns the status to hand back (KVFOLD_ERR_OOM for an allocation failure, KVFOLD_ERR_HIP otherwise).
int hip_fail(hipError_t e);

// Clears device memory and waits for it, on a stream that waits for no other and that none waits for: a cache may be created beside other streams'
// work, or while one of them is being captured.
hipError_t clear_device(void* p, size_t bytes);

// Whether two ranges of memory have no byte in common.
inline bool apart(const void* a, size_t a_bytes, const void* b, size_t b_bytes) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x + a_bytes <= y || y + b_bytes <= x;
}

struct DeviceGuard {
  int prev = -1;
  bool switched = false;
  hipError_t err = hipSuccess;
  explicit DeviceGuard(int dev) {
    err = hipGetDevice(&prev);
    if (err == hipSuccess && prev != dev) {
      err = hipSetDevice(dev);
      switched = (err == hipSuccess);
    }
  }
  ~DeviceGuard() {
    if (switched) (void)hipSetDevice(prev);
  }
};

}  // namespace kvfold
