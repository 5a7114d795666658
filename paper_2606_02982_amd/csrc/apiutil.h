// Shared by the C entry points: the argument helpers and the two-step run of
// DS_VALIDATE (internal to the library).
#pragma once

#include <string.h>

#include "../../include/driftsched.h"
#include "common.h"
#include "kernels.h"

namespace ds {

constexpr size_t kFlagBytes = 256;   // validation word at the start of every workspace

inline ds_status hip_status(hipError_t e) { return e == hipSuccess ? DS_OK : DS_ERR_HIP; }

inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// Runs the enqueue function twice under DS_VALIDATE: first the data checks
// (with a cleared flag), then, if the stream reports no violation, the work.
template <typename F>
ds_status run(void *ws, uint32_t flags, hipStream_t s, F &&enqueue)
{
    uint32_t *flag = static_cast<uint32_t *>(ws);
    if (flags & DS_VALIDATE) {
        hipError_t e = fill_u32(flag, 0u, 1, s);
        if (e == hipSuccess) e = enqueue(flag);
        uint32_t host = 0;
        if (e == hipSuccess) e = hipMemcpyAsync(&host, flag, 4, hipMemcpyDeviceToHost, s);
        if (e == hipSuccess) e = hipStreamSynchronize(s);
        if (e != hipSuccess) return DS_ERR_HIP;
        if (host) return DS_ERR_DATA;
    }
    return hip_status(enqueue(nullptr));
}

inline void *after_flag(void *ws) { return ws ? static_cast<uint8_t *>(ws) + kFlagBytes : nullptr; }

// The integer a C caller passed for an enum-typed argument. C allows any int
// there; in C++ a value outside the enumeration's range may not be read as
// the enum type, so it is copied out as bytes first.
template <typename E>
int enum_int(const E &e)
{
    static_assert(sizeof(E) == sizeof(int), "the ABI's enums are int-sized");
    int v;
    memcpy(&v, &e, sizeof v);
    return v;
}

inline ds_status check_ws(void *ws, size_t ws_bytes, size_t need)
{
    if (!ws || ws_bytes < need || !aligned(ws, 256)) return DS_ERR_WORKSPACE;
    return DS_OK;
}

}  // namespace ds
