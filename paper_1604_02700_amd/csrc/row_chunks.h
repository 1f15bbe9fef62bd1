// Rows of operands straight from memory into the matrix cores (rows.hip,
// loss.hip).
#pragma once

#include "encoder.h"

namespace gpic {
namespace {

// 16 bytes of a row from value k on; any alignment.  LAST: zeros beyond K.
template <int DT, bool LAST>
__device__ __forceinline__ u32x4 chunk_at(const void *row, int64_t k, int64_t K)
{
    constexpr int kSize = DT == GPIC_F32 ? 4 : 2, kValues = 16 / kSize;
    using loose = u32x4 __attribute__((aligned(2)));
    using loose4 = u32x4 __attribute__((aligned(4)));
    const char *p = static_cast<const char *>(row) + k * kSize;
    if (!LAST || k + kValues <= K) {
        if (DT == GPIC_F32)
            return *reinterpret_cast<const loose4 *>(p);
        return *reinterpret_cast<const loose *>(p);
    }
    u32x4 v = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < kValues; ++i)
        if (k + i < K) {
            if (DT == GPIC_F32)
                v[i] = reinterpret_cast<const uint32_t *>(p)[i];
            else
                v[i / 2] |= (uint32_t)reinterpret_cast<const uint16_t *>(p)[i] << (16 * (i & 1));
        }
    return v;
}

template <int DT>
__device__ __forceinline__ f32x4 mma16(u32x4 w, u32x4 x, f32x4 c)
{
    if (DT == GPIC_F32) {
        // lane group g holds four values of k; the j-th instruction takes the
        // j-th of each
#pragma unroll
        for (int j = 0; j < 4; ++j)
            c = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(f32x4, w)[j],
                                                     __builtin_bit_cast(f32x4, x)[j], c, 0, 0, 0);
        return c;
    }
    if (DT == GPIC_BF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bfrag8, w),
                                                       __builtin_bit_cast(bfrag8, x), c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, w),
                                                  __builtin_bit_cast(half8, x), c, 0, 0, 0);
}

} // namespace
} // namespace gpic
