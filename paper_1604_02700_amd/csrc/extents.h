// Checks of the encoder operators' buffers (api_encoder.hip, api_training.hip).
#pragma once

#include "checks.h"

namespace gpic {
namespace {

constexpr int64_t kMaxSide = 1 << 20;      // k, m (2 m), and the sides of an update
constexpr int64_t kMaxPitch = 1 << 22;     // 256 rows of it stay within 32-bit offsets

size_t size_of(int32_t dtype) { return dtype == GPIC_F32 ? 4 : 2; }

gpic_status check_matrix(const void *x, const char *name, int32_t dtype, bool nullable,
                         bool aligned16 = false)
{
    if (x == nullptr) {
        if (nullable)
            return GPIC_OK;
        return fail(GPIC_ERR_INVALID_ARG, "%s is null", name);
    }
    CHECK_ARG(aligned(x, size_of(dtype)), "%s is misaligned", name);
    CHECK_ARG(!aligned16 || aligned(x, 16), "aligned16 is set and %s is not 16-byte aligned",
              name);
    return GPIC_OK;
}

// A matrix in memory: `rows` runs of `width` bytes, `pitch` bytes apart.
struct Extent {
    const char *name;
    const void *p;
    int64_t rows, width, pitch;
};

Extent matrix(const char *name, const void *p, int64_t rows, int64_t cols, int64_t ld, size_t size)
{
    return Extent{name, p, rows, cols * (int64_t)size, ld * (int64_t)size};
}

Extent packed(const char *name, const void *p, int64_t values, size_t size)
{
    return matrix(name, p, 1, values, values, size);
}

// Whether two matrices share a byte.  Columns of one table do not.
bool overlap(Extent a, Extent b)
{
    if (!a.p || !b.p || a.rows <= 0 || b.rows <= 0 || a.width <= 0 || b.width <= 0)
        return false;
    const int64_t at = (int64_t)(uintptr_t)a.p, bt = (int64_t)(uintptr_t)b.p;
    if (at + (a.rows - 1) * a.pitch + a.width <= bt || bt + (b.rows - 1) * b.pitch + b.width <= at)
        return false;
    if (a.rows > 1 && b.rows > 1 && a.pitch == b.pitch) {
        int64_t d = (bt - at) % a.pitch;
        d = d < 0 ? d + a.pitch : d;
        return d < a.width || d + b.width > a.pitch;
    }
    if (a.rows > b.rows)
        return overlap(b, a);
    for (int64_t i = 0; i < a.rows; ++i) {
        // the first row of b that ends beyond this row's start
        const int64_t s = at + i * a.pitch, before = s - bt - b.width;
        const int64_t j = before < 0 ? 0 : (b.rows > 1 ? before / b.pitch + 1 : 1);
        if (j < b.rows && bt + j * b.pitch < s + a.width)
            return true;
    }
    return false;
}

// Results lie apart from what a call reads and from each other.
gpic_status check_apart(const Extent *out, int outs, const Extent *in, int ins)
{
    for (int i = 0; i < outs; ++i) {
        for (int j = 0; j < ins; ++j)
            CHECK_ARG(!overlap(out[i], in[j]), "%s overlaps %s", out[i].name, in[j].name);
        for (int j = 0; j < i; ++j)
            CHECK_ARG(!overlap(out[i], out[j]), "%s overlaps %s", out[i].name, out[j].name);
    }
    return GPIC_OK;
}

#define CHECK(expr)                                                            \
    do {                                                                       \
        gpic_status st_ = (expr);                                              \
        if (st_ != GPIC_OK)                                                    \
            return st_;                                                        \
    } while (0)

} // namespace
} // namespace gpic
