// Host-side argument checks of the C entry points (api.hip, api_encoder.hip).
#pragma once

#include <stdarg.h>
#include <stdint.h>
#include <stdio.h>

#include "../../include/gpic.h"
#include "common.h"

namespace gpic {
namespace {

inline size_t al(size_t x) { return (x + 255) & ~(size_t)255; }

inline bool aligned(const void *p, size_t a)
{
    return ((uintptr_t)p % a) == 0;
}

gpic_status fail(gpic_status st, const char *fmt, ...)
{
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    set_error("%s", buf);
    return st;
}

gpic_status hip_fail(hipError_t e, const char *where)
{
    return fail(GPIC_ERR_HIP, "%s: %s", where, hipGetErrorString(e));
}

#define CHECK_ARG(cond, ...)                                                   \
    do {                                                                       \
        if (!(cond))                                                           \
            return fail(GPIC_ERR_INVALID_ARG, __VA_ARGS__);                    \
    } while (0)

#define CHECK_HIP(expr, where)                                                 \
    do {                                                                       \
        hipError_t e_ = (expr);                                                \
        if (e_ != hipSuccess)                                                  \
            return hip_fail(e_, where);                                        \
    } while (0)

gpic_status check_ws(void *ws, size_t have, size_t need)
{
    if (need == 0)
        return GPIC_OK;
    if (ws == nullptr || have < need)
        return fail(GPIC_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given",
                    need, ws == nullptr ? (size_t)0 : have);
    if (!aligned(ws, 256))
        return fail(GPIC_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
    return GPIC_OK;
}

} // namespace
} // namespace gpic
