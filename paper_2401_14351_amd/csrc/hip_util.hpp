// HIP runtime helpers of the loader library.
#pragma once

#include <hip/hip_runtime_api.h>

#include "common.hpp"

namespace sllm {

// The message of a failed HIP call.  HIP keeps the error pending for the thread
// until hipGetLastError, and the next launch check would report it for a good
// launch, so it is taken here, where the failure is.
inline const char* hip_message(hipError_t e) {
    (void)hipGetLastError();
    return hipGetErrorString(e);
}

// Run a HIP call; on failure record the call and the HIP message and return SLLM_E_HIP.
#define SLLM_HIP(call)                                                                      \
    do {                                                                                    \
        hipError_t _e = (call);                                                             \
        if (_e != hipSuccess)                                                               \
            return ::sllm::fail(SLLM_E_HIP, "%s failed: %s", #call, hip_message(_e));       \
    } while (0)

// Make `device` current for the scope and restore the caller's device after.
class DeviceGuard {
  public:
    explicit DeviceGuard(int device) {
        if (hipGetDevice(&prev_) != hipSuccess) prev_ = -1;
        ok_ = (prev_ == device) || hipSetDevice(device) == hipSuccess;
        if (!ok_) (void)hipGetLastError();
    }
    ~DeviceGuard() {
        int cur = -1;
        if (prev_ >= 0 && hipGetDevice(&cur) == hipSuccess && cur != prev_) (void)hipSetDevice(prev_);
    }
    bool ok() const { return ok_; }

  private:
    int prev_ = -1;
    bool ok_ = false;
};

// [p, p + bytes) must be device memory of `device` inside one allocation: a
// kernel or copy that wrote to a host address or past an allocation would
// fault the GPU instead of failing the call.
inline int32_t check_device_range(const void* p, uint64_t bytes, int device, const char* what) {
    if (!bytes) return SLLM_OK;
    hipPointerAttribute_t at{};
    if (hipPointerGetAttributes(&at, p) != hipSuccess) {
        (void)hipGetLastError();  // leave no error behind for later launch checks
        return fail(SLLM_E_INVAL, "%s %p is not device memory", what, p);
    }
    if (at.type != hipMemoryTypeDevice && at.type != hipMemoryTypeManaged)
        return fail(SLLM_E_INVAL, "%s %p is not device memory", what, p);
    if (at.type == hipMemoryTypeDevice && at.device != device)
        return fail(SLLM_E_INVAL, "%s is memory of device %d, not of device %d", what, at.device, device);
    void* base = nullptr;
    size_t size = 0;
    if (hipMemGetAddressRange(&base, &size, const_cast<void*>(p)) != hipSuccess || !base) {
        // no allocation range known (e.g. managed memory): the call cannot
        // show that the whole range is inside one allocation, so refuse it
        (void)hipGetLastError();
        return fail(SLLM_E_INVAL, "%s %p: the runtime reports no allocation range for it; pass memory from hipMalloc",
                    what, p);
    }
    const uint64_t off = (uint64_t)(static_cast<const uint8_t*>(p) - static_cast<const uint8_t*>(base));
    if (bytes > size || off > size - bytes)
        return fail(SLLM_E_RANGE, "%s: %llu bytes from %p run past the end of its allocation", what,
                    (unsigned long long)bytes, p);
    return SLLM_OK;
}

}  // namespace sllm
