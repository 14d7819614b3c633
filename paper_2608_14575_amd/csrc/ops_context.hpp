// What the operators' host sides share (hwr_ops.hip, hwr_train.hip): the context, its errors,
// its device and its work space.
#pragma once

#include <hip/hip_runtime.h>

#include <cstring>
#include <initializer_list>
#include <string>
#include <vector>

#include "c_boundary.hpp"
#include "hwr_ops.h"

struct hwr_ops {
    int dev = 0, cus = 0;
    hipStream_t stream = nullptr;
    void *zeros = nullptr;
    unsigned *arrived = nullptr;       // zeros between calls (launch_probs)
    // Work space: the last block is in use.  Blocks grow by powers of two and stay
    // until hwr_ops_free: captured graphs hold their addresses.
    std::vector<void *> blocks;
    uint64_t size = 0;
    std::string err;
};

namespace hwr {

// The last failed hwr_ops_init of this thread.
std::string &ops_error();

inline hwr_status fail(hwr_ops *c, hwr_status s, const std::string &msg) {
    (c ? c->err : ops_error()) = msg;
    return s;
}
inline hwr_status invalid(hwr_ops *c, const char *msg) { return fail(c, HWR_ERR_INVALID_ARG, msg); }

// (The runtime keeps the error until it is asked for: the next launch would report it again.)
inline hwr_status hip_fail(hwr_ops *c, hipError_t e, const char *what) {
    (void)hipGetLastError();
    std::string m = std::string(what) + ": " + hipGetErrorName(e) + " (" + hipGetErrorString(e) + ")";
    return fail(c, e == hipErrorOutOfMemory ? HWR_ERR_OOM : HWR_ERR_HIP, m);
}

#define OPS_HIP(ctx, call)                                           \
    do {                                                             \
        hipError_t e_ = (call);                                      \
        if (e_ != hipSuccess) return hip_fail((ctx), e_, #call);     \
    } while (0)

// Makes a device current for a scope; the caller's is current again after it.
class OnDevice {
  public:
    explicit OnDevice(int dev) {
        error = hipGetDevice(&before_);
        if (error == hipSuccess && before_ != dev) {
            error = hipSetDevice(dev);
            changed_ = error == hipSuccess;
        }
    }
    ~OnDevice() {
        if (changed_) (void)hipSetDevice(before_);
    }
    OnDevice(const OnDevice &) = delete;
    OnDevice &operator=(const OnDevice &) = delete;
    hipError_t error;

  private:
    int before_ = 0;
    bool changed_ = false;
};

#define OPS_ON_DEVICE(ctx, dev)    \
    const OnDevice on_device(dev); \
    if (on_device.error != hipSuccess) return hip_fail((ctx), on_device.error, "hipSetDevice")

// Whether the context's stream is being captured.
inline hipError_t is_captured(const hwr_ops *c, bool *out) {
    hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
    const hipError_t e = c->stream ? hipStreamIsCapturing(c->stream, &cap) : hipSuccess;
    *out = cap != hipStreamCaptureStatusNone;
    return e;
}

// At least `bytes` of work space at *out.
hwr_status workspace(hwr_ops *c, uint64_t bytes, char **out);

inline bool misaligned(int32_t dtype, std::initializer_list<const void *> ptrs) {
    for (const void *p : ptrs)
        if (reinterpret_cast<uintptr_t>(p) & (dtype == HWR_BF16 ? 1 : 3)) return true;
    return false;
}
inline bool bad_ld(int64_t ld, int32_t width) { return ld != 0 && ld < width; }
inline int64_t dense(int64_t ld, int32_t width) { return ld ? ld : width; }

}  // namespace hwr
