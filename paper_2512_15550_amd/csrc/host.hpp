// What the host side of the library's translation units share: error reporting, the current device for a scope, and the device
// memory kept between objects (defined in ctkvr.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>

namespace ctkvr {

// sets the calling thread's message and returns `code`
int fail(int code, const char *fmt, ...);

#define HIP_TRY(expr)                                                                           \
    do {                                                                                        \
        hipError_t e_ = (expr);                                                                 \
        if (e_ != hipSuccess)                                                                   \
            return fail(e_ == hipErrorOutOfMemory ? CTKVR_ENOMEM : CTKVR_EHIP, "%s: %s", #expr, \
                        hipGetErrorString(e_));                                                 \
    } while (0)
#define TRY(expr)                    \
    do {                             \
        int rc_ = (expr);            \
        if (rc_ != CTKVR_OK) return rc_; \
    } while (0)

// Makes a device the calling thread's current one for a scope.  Events, the null stream, function attributes and
// device-wide waits are those of the current device, which need not be the one an index lives on.
struct DeviceScope {
    int before = -1;
    hipError_t err;
    explicit DeviceScope(int dev)
    {
        err = hipGetDevice(&before);
        if (err == hipSuccess && before == dev) before = -1;   // nothing to restore
        else err = hipSetDevice(dev);
    }
    ~DeviceScope()
    {
        if (before >= 0) (void)hipSetDevice(before);
    }
};

struct PoolBlock {
    void *base;
    size_t bytes;
};
// the work on the current device has ended
bool device_idle();
// a block of at least `bytes` on the current device `dev`, and of at most bytes / spare more if it was kept; out->bytes is its
// real size
int pool_get(int dev, size_t bytes, size_t spare, PoolBlock *out);
// gives a block of device `dev` back; idle: its users have been waited for
void pool_put(int dev, PoolBlock b, bool idle);

}  // namespace ctkvr
