// What the entry points that take rows of tokens have in common: their device,
// their errors, and the rows as kernels take them.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <string>

#include "wf_internal.h"

namespace wf {

struct KvRows {                      // [b][row][head][dim], the channels contiguous
    void* p;
    long long sb, sr, sh;            // strides in elements
};

inline int kv_fail(hipError_t e, const char* what) { return fail(WF_E_HIP, std::string(what) + ": " + hipGetErrorString(e)); }

inline int kv_launched(const char* what) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? WF_OK : kv_fail(e, what);
}

// Rows of a call: the strides are in elements and the channels contiguous.
inline int kv_rows(const wf_rows* r, int precision, const char* name, KvRows* out) {
    if (!r || !r->data) return fail(WF_E_INVALID, std::string(name) + " is NULL");
    if ((uintptr_t)r->data % (precision == WF_BF16 ? 2 : 4)) return fail(WF_E_INVALID, std::string(name) + " is not aligned to its element");
    *out = {r->data, r->stride[0], r->stride[1], r->stride[2]};
    return WF_OK;
}

// Makes a plan's device current for a call.  A default stream is that of the
// current device, and a host thread may have another one current (a new thread
// begins with device 0).
class OnDevice {
public:
    explicit OnDevice(int device) {
        e_ = hipGetDevice(&was_);
        if (e_ == hipSuccess && was_ != device) {
            e_ = hipSetDevice(device);
            changed_ = e_ == hipSuccess;
        }
    }
    ~OnDevice() {
        if (changed_) (void)hipSetDevice(was_);
    }
    OnDevice(const OnDevice&) = delete;
    OnDevice& operator=(const OnDevice&) = delete;
    hipError_t error() const { return e_; }

private:
    int was_ = 0;
    bool changed_ = false;
    hipError_t e_;
};

}  // namespace wf
