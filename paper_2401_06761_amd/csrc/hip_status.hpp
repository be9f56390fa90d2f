// Runtime calls at the C ABI: their errors, and the device that a call's memory lies on.
#pragma once

#include <hip/hip_runtime.h>

#include "apar.h"

namespace apar {

// Keeps what apar_last_hip_error reports if the call failed.
bool hip_ok(hipError_t e, const char* what);

#define HIP_TRY(expr)                                          \
    do {                                                       \
        if (!apar::hip_ok((expr), #expr)) return APAR_ERR_HIP; \
    } while (0)

struct DeviceGuard {
    int prev = 0;
    bool switched = false;
    explicit DeviceGuard(int dev) {
        if (hipGetDevice(&prev) == hipSuccess && prev != dev) switched = (hipSetDevice(dev) == hipSuccess);
    }
    ~DeviceGuard() {
        if (switched) (void)hipSetDevice(prev);
    }
};

// Makes the device that `p` lies on the current one (where there is more than one to ask about).
struct DeviceOf {
    int prev = 0;
    bool switched = false;
    explicit DeviceOf(const void* p) {
        static const int n_devices = [] {
            int n = 0;
            if (hipGetDeviceCount(&n) != hipSuccess) (void)hipGetLastError();
            return n;
        }();
        if (n_devices < 2) return;
        hipPointerAttribute_t attr;
        if (hipPointerGetAttributes(&attr, p) != hipSuccess) {
            (void)hipGetLastError();
            return;
        }
        if (hipGetDevice(&prev) == hipSuccess && prev != attr.device) switched = (hipSetDevice(attr.device) == hipSuccess);
    }
    ~DeviceOf() {
        if (switched) (void)hipSetDevice(prev);
    }
};

}  // namespace apar
