// What the C entry points share: argument checks, error reporting, the current device.
#pragma once

#include <stdint.h>

#include <hip/hip_runtime.h>

#include "cc_join.h"

namespace ccj {

// The hipError_t of the last CC_ERR_DEVICE returned on this thread (cc_last_device_error).
extern thread_local int g_last_device_error;

inline cc_status device_error(hipError_t e) {
    g_last_device_error = (int)e;
    return CC_ERR_DEVICE;
}

inline bool aligned(const void *p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

inline bool mul_ok(int64_t a, int64_t b, int64_t *r) { return !__builtin_mul_overflow(a, b, r); }

inline bool overlaps(const void *a, int64_t na, const void *b, int64_t nb) {
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return na > 0 && nb > 0 && x < y + (uintptr_t)nb && y < x + (uintptr_t)na;
}

// Keeps the store's device current for the duration of a call.
class DeviceGuard {
public:
    explicit DeviceGuard(int dev) {
        err_ = hipGetDevice(&prev_);
        if (err_ == hipSuccess && prev_ != dev) {
            err_ = hipSetDevice(dev);
            switched_ = err_ == hipSuccess;
        }
    }
    ~DeviceGuard() {
        if (switched_)
            (void)hipSetDevice(prev_);
    }
    hipError_t error() const { return err_; }

private:
    int prev_ = 0;
    hipError_t err_ = hipSuccess;
    bool switched_ = false;
};

}  // namespace ccj
