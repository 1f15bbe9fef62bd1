// Dropout from a counter: Y = R + keep X / (1 - p).  The mask is a function
// of (seed, offset, index) and never stored: value i of the n x m values takes
// half i % 8 of the block that Philox4x32-10 (Salmon, Moraes, Dror and Shaw,
// "Parallel random numbers: as easy as 1, 2, 3", 2011) gives for the counter
// (i / 8, offset) under the key `seed`, and stays where those 16 bits are at
// least the limit round(2^16 p).  Sixteen bits a value instead of a word's 32
// halve the rounds, which would otherwise bound 16-bit matrices; the factor is
// 2^16 / (2^16 - limit), so that what is kept is exact on average.
#include "training.h"

namespace gpic {
namespace {

struct DropArgs {
    const void *X, *R;
    const int64_t *step;
    void *Y;
    int64_t n, m, ldx, ldr, ldy;
    uint64_t seed, offset;
    uint32_t limit;
    float scale;
};

__device__ __forceinline__ void philox_round(uint32_t (&c)[4], uint32_t k0, uint32_t k1)
{
    const uint64_t a = (uint64_t)c[0] * 0xD2511F53u, b = (uint64_t)c[2] * 0xCD9E8D57u;
    c[0] = (uint32_t)(b >> 32) ^ c[1] ^ k0;
    c[1] = (uint32_t)b;
    c[2] = (uint32_t)(a >> 32) ^ c[3] ^ k1;
    c[3] = (uint32_t)a;
}

__device__ __forceinline__ void philox(uint32_t (&c)[4], uint64_t key)
{
    uint32_t k0 = (uint32_t)key, k1 = (uint32_t)(key >> 32);
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        philox_round(c, k0, k1);
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
}

// A thread takes a block's eight values.  Bound by memory, and by the rounds where
// the last-level cache feeds it: 16,384 x 4,096 in bfloat16 with a residual 59 us
// (403 MB, 6.8 TB/s), without one 59 too; 1,003 x 777 in float32 inside a wider
// table 6.9 us, in one run 3.5.  FLAT: rows follow each other
// without a gap in X, R and Y, and the matrix is one run.
template <int DT, bool FLAT>
__global__ __launch_bounds__(256) void dropout_kernel(DropArgs a)
{
    const int64_t total = a.n * a.m, blocks = (total + 7) / 8;
    const uint64_t offset = a.offset + (a.step ? (uint64_t)*a.step : 0);
    for (int64_t b = (int64_t)blockIdx.x * 256 + threadIdx.x; b < blocks;
         b += (int64_t)gridDim.x * 256) {
        uint32_t c[4] = {(uint32_t)b, (uint32_t)((uint64_t)b >> 32), (uint32_t)offset,
                         (uint32_t)(offset >> 32)};
        philox(c, a.seed);
        auto kept = [&](int j) { return ((c[j >> 1] >> (16 * (j & 1))) & 0xffffu) >= a.limit; };
        const int64_t first = b * 8;
        const int valid = total - first < 8 ? (int)(total - first) : 8;
        const int64_t row = FLAT ? 0 : first / a.m, col = first - row * a.m;
        if (FLAT || col + valid <= a.m) {
            const f32x8 x = load8(a.X, row * a.ldx + col, DT, valid);
            f32x8 y = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                y[j] = kept(j) ? x[j] * a.scale : 0.0f;
            if (a.R)
                y = y + load8(a.R, row * a.ldr + col, DT, valid);
            store8(a.Y, row * a.ldy + col, y, DT, valid);
            continue;
        }
        int64_t r = row, k = col;              // the block runs over a row's end
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < valid) {
                float y = kept(j) ? load1(a.X, r * a.ldx + k, DT) * a.scale : 0.0f;
                if (a.R)
                    y += load1(a.R, r * a.ldr + k, DT);
                store1(a.Y, r * a.ldy + k, y, DT);
                if (++k == a.m) {
                    k = 0;
                    ++r;
                }
            }
    }
}

template <int DT>
hipError_t launch(const DropArgs &a, hipStream_t st)
{
    const bool flat = a.n == 1 || (a.ldx == a.m && a.ldy == a.m && (!a.R || a.ldr == a.m));
    int64_t blocks = ((a.n * a.m + 7) / 8 + 255) / 256;
    blocks = blocks > (1 << 20) ? 1 << 20 : blocks;
    if (flat)
        dropout_kernel<DT, true><<<(unsigned)blocks, 256, 0, st>>>(a);
    else
        dropout_kernel<DT, false><<<(unsigned)blocks, 256, 0, st>>>(a);
    return hipGetLastError();
}

} // namespace

hipError_t run_dropout(const Dropout &p, const void *X, const void *R, const int64_t *step,
                       void *Y, hipStream_t st)
{
    if (p.n == 0)
        return hipSuccess;
    const DropArgs a{X, R, step, Y, p.n, p.m, p.ldx, p.ldr, p.ldy, p.seed, p.offset, p.limit,
                     65536.0f / (float)(65536u - p.limit)};
    return p.dtype == GPIC_F32    ? launch<GPIC_F32>(a, st)
           : p.dtype == GPIC_F16 ? launch<GPIC_F16>(a, st)
                                 : launch<GPIC_BF16>(a, st);
}

} // namespace gpic
