// Helpers of the operators that a program calls on memory of its own: the
// device is made current for the duration of a call and the caller's put back.
#pragma once

#include "common.h"

namespace wmi {

class DeviceScope {
   public:
    explicit DeviceScope(int dev) {
        if (hipGetDevice(&old_) != hipSuccess) old_ = -1;
        if (old_ != dev) WMI_HIP(hipSetDevice(dev));
        else old_ = -1;
    }
    ~DeviceScope() {
        if (old_ >= 0) (void)hipSetDevice(old_);
    }
    DeviceScope(const DeviceScope&) = delete;

   private:
    int old_ = -1;
};

// Whether stream s is recording a graph (calls that move host lists to the
// device refuse then: a replay would not repeat their host side).
inline bool capturing(hipStream_t s) {
    hipStreamCaptureStatus c = hipStreamCaptureStatusNone;
    const hipError_t e = hipStreamIsCapturing(s, &c);
    if (e != hipSuccess) (void)hipGetLastError();
    return e != hipSuccess || c != hipStreamCaptureStatusNone;
}

}  // namespace wmi
