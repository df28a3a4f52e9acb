// What the host sides of the ABI share: error messages and argument checks.
#pragma once

#include <hip/hip_runtime.h>

namespace rheo {

// Sets the calling thread's message (rheo_last_error) and returns `code`.
int fail(int code, const char* fmt, ...);
int hip_fail(hipError_t e, const char* what);
// RHEO_EINVAL for a pointer that is NULL or not 16-byte aligned.
int check_ptr(const void* p, const char* name);

// A handle's device made current for the length of a call: streams and kernels
// belong to it whichever device the calling thread has current.
class OnDevice {
public:
    explicit OnDevice(int device) {
        e_ = hipGetDevice(&before_);
        if (e_ == hipSuccess && before_ != device) {
            e_ = hipSetDevice(device);
            changed_ = e_ == hipSuccess;
        }
    }
    ~OnDevice() {
        if (changed_) (void)hipSetDevice(before_);
    }
    hipError_t error() const { return e_; }

private:
    int before_ = 0;
    bool changed_ = false;
    hipError_t e_ = hipSuccess;
};

}  // namespace rheo
