// What the argument checks and launches of the C ABI share (ra_chunk_api.cpp, ra_step_api.cpp).
#pragma once
#include "ra_context.h"

#include <cstdarg>
#include <cstdio>

namespace ra {

// A failed check: its status, and its text in msg.
struct Fail {
    char *msg;
    size_t n;
    __attribute__((format(printf, 3, 4))) ra_status operator()(ra_status st, const char *fmt, ...) const
    {
        if (msg && n) {
            va_list ap;
            va_start(ap, fmt);
            vsnprintf(msg, n, fmt, ap);
            va_end(ap);
        }
        return st;
    }
};

// Runs `launch` on the context's device.
template <typename F> inline ra_status on_device(ra_ctx *c, F launch)
{
    int prev = 0;
    hipError_t e = hipGetDevice(&prev);
    if (e == hipSuccess && prev != c->device) e = hipSetDevice(c->device);
    if (e == hipSuccess) e = launch();
    if (prev != c->device) (void)hipSetDevice(prev);
    if (e != hipSuccess) { set_err(c, "HIP: %s", hipGetErrorString(e)); return RA_ERR_DEVICE; }
    return RA_OK;
}

} // namespace ra
