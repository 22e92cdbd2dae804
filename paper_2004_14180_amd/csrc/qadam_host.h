// What the host sides of the operators share: checks of arguments, and device memory that lives as long as its handle.
#pragma once

#include <exception>
#include <memory>
#include <vector>

#include "qadam_elements.h"
#include "qadam_internal.h"

namespace qadam {

#define QADAM_HIP(call)                                      \
    do {                                                     \
        hipError_t e_ = (call);                              \
        if (e_ != hipSuccess) return hip_fail(e_, #call);    \
    } while (0)

#define QADAM_CHECK(expr)                 \
    do {                                  \
        const int rc_ = (expr);           \
        if (rc_ != QADAM_OK) return rc_;  \
    } while (0)

// Nothing is thrown through the C boundary: what the standard library throws (no host memory for a table) becomes an error.
template <typename F>
int guarded(F&& f)
{
    try {
        return f();
    } catch (const std::exception& e) {
        return fail(QADAM_EINVAL, e.what());
    }
}

inline bool float_type(int type) { return type == QADAM_F32 || type == QADAM_BF16 || type == QADAM_F16; }

inline int check_address(const void* p, int size, const char* name)
{
    if (!p) return fail(QADAM_EINVAL, name);
    if (reinterpret_cast<uintptr_t>(p) % (uintptr_t)size) return fail(QADAM_EALIGN, name);
    return QADAM_OK;
}

// rows * stride elements are addressed with 64-bit byte offsets
inline int check_matrix(const void* p, int type, int64_t rows, int64_t stride, int64_t least, const char* name)
{
    if (stride < least) return fail(QADAM_EINVAL, "a stride below dim");
    if (stride > (int64_t)1 << 20 && rows > ((int64_t)1 << 60) / stride) return fail(QADAM_ERANGE, "rows * stride beyond 2^60");
    return check_address(p, element_size(type), name);
}

inline int check_device(int device)
{
    int now = -1;
    QADAM_HIP(hipGetDevice(&now));
    return now == device ? QADAM_OK : fail(QADAM_EINVAL, "handle belongs to another device");
}

struct DeviceFree {
    void operator()(void* p) const { (void)hipFree(p); }
};
template <typename T>
using DeviceArray = std::unique_ptr<T, DeviceFree>;

template <typename T>
int allocate(DeviceArray<T>& out, size_t count)
{
    void* p = nullptr;
    QADAM_HIP(hipMalloc(&p, (count ? count : 1) * sizeof(T)));
    out.reset(static_cast<T*>(p));
    return QADAM_OK;
}

template <typename T>
int upload(DeviceArray<T>& out, const std::vector<T>& host)
{
    QADAM_CHECK(allocate(out, host.size()));
    if (!host.empty()) QADAM_HIP(hipMemcpy(out.get(), host.data(), host.size() * sizeof(T), hipMemcpyHostToDevice));
    return QADAM_OK;
}

// a handle's status word; waits for the stream
inline int read_status(uint32_t* status, qadam_status_t* out, int32_t clear, hipStream_t s)
{
    uint32_t flags = 0;
    QADAM_HIP(hipMemcpyAsync(&flags, status, sizeof flags, hipMemcpyDeviceToHost, s));
    if (clear) QADAM_HIP(hipMemsetAsync(status, 0, sizeof flags, s));
    QADAM_HIP(hipStreamSynchronize(s));
    out->flags = flags;
    out->reserved = 0;
    return QADAM_OK;
}

}  // namespace qadam
