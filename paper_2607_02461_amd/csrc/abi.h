// What the device entry points share: argument checks, the current device, per-device copies of a handle's tables.
#pragma once

#include <hip/hip_runtime.h>

#include "internal.h"

namespace orbit {

inline bool aligned(const void* p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

struct DeviceInfo {
    int cus = 0;
};

orbit_status hip_fail(hipError_t e, const char* what);
orbit_status current_device(int* dev, DeviceInfo* info);
// The current device, or -1 when no HIP device is visible (handles then stay host-only).
orbit_status device_for_upload(int* dev);

// A copy of `bytes` host bytes on the current device (hipMalloc and a synchronous copy).
orbit_status upload_copy(const char* who, const void* data, size_t bytes, void** out);

// Frees a handle's per-device tables (each on its own device).
template <typename T>
void free_per_device(T* (&ptrs)[kMaxDevices]) {
    for (int dev = 0; dev < kMaxDevices; ++dev) {
        if (ptrs[dev]) {
            int cur = 0;
            (void)hipGetDevice(&cur);
            (void)hipSetDevice(dev);
            (void)hipFree(ptrs[dev]);
            (void)hipSetDevice(cur);
            ptrs[dev] = nullptr;
        }
    }
}

}  // namespace orbit
