// The layers' forward pass for few rows (serving single points): bound by
// reading W once.  A workgroup takes 16 columns of the output (gated: 16 of
// the gate's and the same 16 of the up projection's); its waves share the
// contraction in turns of 128 (float32: 64) values, so that together they
// read long runs of the 16 rows of W, each lane 16 bytes at a time into
// registers and from there into the matrix cores, W's rows as the first
// operand and up to 32 rows of X as the second.  The waves' sums meet in
// LDS and are added in wave order.  float32 uses the float32 matrix
// instruction (the operands are not split: reading them is what counts).
#include <type_traits>

#include "encoder.h"

namespace gpic {

namespace {

struct RowArgs {
    const void *X, *W, *bias, *res;
    void *Y, *Z;
    int64_t ldx, ldw, ldr, ldy, ldz;
    int n;
    int64_t k, m;
    int act;
};

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

template <int DT, bool GATED, int NB, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void few_rows_kernel(RowArgs a)
{
    constexpr int kValues = DT == GPIC_F32 ? 4 : 8;       // of k a lane loads at once
    constexpr int kUnroll = 4, kTurn = 4 * kValues * kUnroll;
    constexpr int kG = GATED ? 2 : 1;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, r = lane & 15;
    const int64_t col0 = (int64_t)blockIdx.x * 16;
    // rows beyond the last are read as the last one and not stored
    const char *w[kG], *x[NB];
    constexpr int kSize = DT == GPIC_F32 ? 4 : 2;
#pragma unroll
    for (int i = 0; i < kG; ++i) {
        const int64_t row = (col0 + r < a.m ? col0 + r : a.m - 1) + i * a.m;
        w[i] = static_cast<const char *>(a.W) + row * a.ldw * kSize;
    }
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        const int row = b * 16 + r < a.n ? b * 16 + r : a.n - 1;
        x[b] = static_cast<const char *>(a.X) + row * a.ldx * kSize;
    }
    f32x4 acc[kG][NB];
#pragma unroll
    for (int i = 0; i < kG; ++i)
#pragma unroll
        for (int b = 0; b < NB; ++b)
            acc[i][b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    u32x4 fw[kG][kUnroll], fx[NB][kUnroll];
    auto load = [&](int64_t k0, auto last) {
        constexpr bool kLast = decltype(last)::value;
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int64_t k = k0 + u * 4 * kValues + g * kValues;
#pragma unroll
            for (int i = 0; i < kG; ++i)
                fw[i][u] = chunk_at<DT, kLast>(w[i], k, a.k);
#pragma unroll
            for (int b = 0; b < NB; ++b)
                fx[b][u] = chunk_at<DT, kLast>(x[b], k, a.k);
        }
    };
    auto multiply = [&]() {
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
#pragma unroll
            for (int i = 0; i < kG; ++i)
#pragma unroll
                for (int b = 0; b < NB; ++b)
                    acc[i][b] = mma16<DT>(fw[i][u], fx[b][u], acc[i][b]);
    };
    int64_t k0 = (int64_t)wave * kTurn;
#pragma unroll 2
    for (; k0 + kTurn <= a.k; k0 += (int64_t)WAVES * kTurn) {
        load(k0, std::false_type{});
        multiply();
    }
    if (k0 < a.k) {                    // the turn that the contraction ends in
        load(k0, std::true_type{});
        multiply();
    }
    __shared__ f32x4 part[WAVES][kG * NB][64];
#pragma unroll
    for (int i = 0; i < kG; ++i)
#pragma unroll
        for (int b = 0; b < NB; ++b)
            part[wave][i * NB + b][lane] = acc[i][b];
    __syncthreads();
    // wave b finishes rows 16 b .. 16 b + 15: a lane four columns of one row
    if (wave >= NB)
        return;
    const int row = wave * 16 + r;
    f32x4 v[kG];
#pragma unroll
    for (int i = 0; i < kG; ++i) {
        v[i] = part[0][i * NB + wave][lane];
#pragma unroll
        for (int s = 1; s < WAVES; ++s)
            v[i] += part[s][i * NB + wave][lane];
    }
    if (row >= a.n)
        return;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int64_t col = col0 + g * 4 + j;
        if (col >= a.m)
            break;
        float z = v[0][j];
        if (GATED) {
            const float u = v[kG - 1][j];
            if (a.Z) {
                static_cast<float *>(a.Z)[row * a.ldz + col] = z;
                static_cast<float *>(a.Z)[row * a.ldz + a.m + col] = u;
            }
            store1(a.Y, row * a.ldy + col, activate(z, a.act) * u, DT);
        } else {
            if (a.bias)
                z += load1(a.bias, col, DT);
            if (a.Z)
                store1(a.Z, row * a.ldz + col, z, DT);
            z = activate(z, a.act);
            if (a.res)
                z += load1(a.res, row * a.ldr + col, DT);
            store1(a.Y, row * a.ldy + col, z, DT);
        }
    }
}

template <int DT, bool GATED, int NB>
hipError_t launch_waves(const RowArgs &a, hipStream_t st)
{
    const int64_t blocks = (a.m + 15) / 16;
    if (blocks > 0x7fffffffll)
        return hipErrorInvalidValue;
    // as many waves as there are turns: then all of W is on its way at once
    const int64_t turns = (a.k + (DT == GPIC_F32 ? 63 : 127)) / (DT == GPIC_F32 ? 64 : 128);
    if (turns <= 4)
        few_rows_kernel<DT, GATED, NB, 4><<<(unsigned)blocks, 256, 0, st>>>(a);
    else if (turns <= 8 || (GATED && NB == 2))
        few_rows_kernel<DT, GATED, NB, 8><<<(unsigned)blocks, 512, 0, st>>>(a);
    else
        few_rows_kernel<DT, GATED, NB, 16><<<(unsigned)blocks, 1024, 0, st>>>(a);
    return hipGetLastError();
}

template <int DT>
hipError_t launch_rows(const RowArgs &a, bool gated, hipStream_t st)
{
    if (gated)
        return a.n <= 16 ? launch_waves<DT, true, 1>(a, st) : launch_waves<DT, true, 2>(a, st);
    return a.n <= 16 ? launch_waves<DT, false, 1>(a, st) : launch_waves<DT, false, 2>(a, st);
}

} // namespace

hipError_t run_few_rows(const Shape &s, bool gated, const void *X, const void *W,
                        const void *bias, const void *res, void *Y, void *Z, hipStream_t st)
{
    RowArgs a{};
    a.X = X;
    a.W = W;
    a.bias = bias;
    a.res = res;
    a.Y = Y;
    a.Z = Z;
    a.ldx = s.ldx;
    a.ldw = s.ldw;
    a.ldr = s.ldr;
    a.ldy = s.ldy;
    a.ldz = s.ldz;
    a.n = (int)s.n;
    a.k = s.k;
    a.m = s.m;
    a.act = s.act;
    if (s.dtype == GPIC_F32)
        return launch_rows<GPIC_F32>(a, gated, st);
    return s.dtype == GPIC_F16 ? launch_rows<GPIC_F16>(a, gated, st)
                               : launch_rows<GPIC_BF16>(a, gated, st);
}

} // namespace gpic
