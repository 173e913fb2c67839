// The device that a call works on, while it does.
#pragma once
#include <hip/hip_runtime.h>

namespace {

// Makes `device` the calling thread's current one and leaves the one that was when the call ends: torch and the caller go by it.
class DeviceScope {
public:
    explicit DeviceScope(int device) {
        int count = 0;
        if (hipGetDeviceCount(&count) != hipSuccess || device < 0 || device >= count || hipGetDevice(&before_) != hipSuccess) return;
        if (before_ != device) {
            if (hipSetDevice(device) != hipSuccess) return;
            moved_ = true;
        }
        ok_ = true;
    }
    ~DeviceScope() {
        if (moved_) (void)hipSetDevice(before_);
    }
    DeviceScope(const DeviceScope&) = delete;
    DeviceScope& operator=(const DeviceScope&) = delete;
    bool ok() const { return ok_; }

private:
    int before_ = 0;
    bool moved_ = false, ok_ = false;
};

}  // namespace
