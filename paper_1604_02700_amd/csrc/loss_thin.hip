// Gradients of up to 64 rows from D (n x v) in float32: dX = D W and dW = D^T X on
// the float32 matrix instruction, W and dW read and written once as they lie.
// float32: the tiled products' split copies of W (two of them, and its columns'
// maxima) are five times its bytes, which is what few rows are bound by.  16 bits:
// D is not rounded.
//
// mfma_f32_16x16x4: a lane (g = lane / 16, r = lane mod 16) holds one value of both
// operands, k = g; of the result rows r of the second operand and columns 4 g +
// q of the first.  A wave takes 64 columns in four instructions c = 0 .. 3.  Where
// the first operand is W its column r is column 4 r + c of the 64, so that a lane
// loads four consecutive values and ends with sixteen: column 16 g + 4 q + c in
// acc[c][q].  X is read once and dW written throughout, so there it is 16 c + r.
//
// With 2,048 -> 32,000 (W 262 MB; D in float32 and all gradients, in us): 1 row 51
// for D, 50 dW, 79 dX and its parts' sum 5; 33 rows 138, 96, 93, 5; 64 rows 164,
// 118, 98, 5.  By the split copies 33 rows took 507.
#include "training.h"

namespace gpic {
namespace {

struct ThinArgs {
    const float *D, *X;        // [n][v], [n][k]
    const void *W;             // [v] of pitch ldw, of the matrices' type, as dX and dW
    void *dX, *dW;
    float *part;               // [parts][n][k]
    int64_t n, k, v, ldw, strips, each, parts;
};

// Columns c .. c + 3 of a row of `cols` that starts at `row`, zeros beyond
template <int DT>
__device__ __forceinline__ f32x4 quad(const void *p, int64_t row, int64_t c, int64_t cols)
{
    if (c + 4 <= cols)
        return load4(p, row + c, DT);
    f32x4 x = 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (c + j < cols)
            x[j] = load1(p, row + c + j, DT);
    return x;
}

// sixteen columns of a row from the four accumulators
__device__ __forceinline__ void put16(float *row, int64_t col, int64_t cols, const f32x4 (&acc)[4])
{
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const f32x4 x = {acc[0][q], acc[1][q], acc[2][q], acc[3][q]};
        const int64_t c = col + 4 * q;
        using any = f32x4 __attribute__((aligned(4)));
        if (c + 4 <= cols) {
            *reinterpret_cast<any *>(row + c) = x;
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (c + j < cols)
                    row[c + j] = x[j];
        }
    }
}

// dW: a wave keeps 64 columns of X (4 STEPS rows) in registers and takes 16 rows
// of dW after another.  Column r = 4 g + q of the first operand is column 16 c + r
// here, of 16 bits 32 (c / 2) + 8 g + 4 (c mod 2) + q, so that four lanes store 64 bytes
// of a row (one row in float32: 98 us with 16 bytes a lane 64 apart, 50 so).  Bound by
// writing dW, from 33 rows on also by its products.
template <int DT, int STEPS>
__global__ __launch_bounds__(256) void thin_weights_kernel(ThinArgs a)
{
    const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
    const int64_t id = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int64_t j0 = id % a.strips * 64, blocks = (a.v + 15) / 16;
    const int64_t b0 = id / a.strips * a.each, b1 = b0 + a.each < blocks ? b0 + a.each : blocks;
    if (b0 >= b1)
        return;
    float x[STEPS][4];
#pragma unroll
    for (int s = 0; s < STEPS; ++s)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int64_t i = 4 * s + g;
            const int64_t j = j0 + (DT == GPIC_F32 ? 16 * c + r
                                                   : 32 * (c / 2) + 8 * (r / 4) + 4 * (c % 2) + r % 4);
            x[s][c] = i < a.n && j < a.k ? a.X[i * a.k + j] : 0.0f;
        }
    // rows beyond the last are computed as the last and not stored
    auto fetch = [&](int64_t b, float (&d)[STEPS]) {
        const int64_t v = b * 16 + r < a.v ? b * 16 + r : a.v - 1;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const int64_t i = 4 * s + g;
            d[s] = i < a.n ? a.D[i * a.v + v] : 0.0f;
        }
    };
    using any = f32x4 __attribute__((aligned(4)));
    float next[STEPS];
    fetch(b0, next);
    for (int64_t b = b0; b < b1; ++b) {
        float d[STEPS];
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
            d[s] = next[s];
        if (b + 1 < b1)
            fetch(b + 1, next);
        f32x4 acc[4];
#pragma unroll
        for (int c = 0; c < 4; ++c)
            acc[c] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
#pragma unroll
            for (int c = 0; c < 4; ++c)
                acc[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[s][c], d[s], acc[c], 0, 0, 0);
        const int64_t v = b * 16 + r;
        if (v >= a.v)
            continue;
        if constexpr (DT != GPIC_F32) {
#pragma unroll
            for (int c = 0; c < 4; c += 2) {
                const int64_t j = j0 + 16 * c + 8 * g, left = a.k - j;
                if (left > 0)
                    store8(a.dW, v * a.k + j,
                           __builtin_shufflevector(acc[c], acc[c + 1], 0, 1, 2, 3, 4, 5, 6, 7), DT,
                           left < 8 ? (int)left : 8);
            }
            continue;
        }
        float *row = static_cast<float *>(a.dW) + v * a.k;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int64_t j = j0 + 16 * c + 4 * g;
            if (j + 4 <= a.k) {
                *reinterpret_cast<any *>(row + j) = acc[c];
            } else {
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (j + q < a.k)
                        row[j + q] = acc[c][q];
            }
        }
    }
}

// Partial dX: 64 columns by 16 NI rows a wave over a run of W's rows, 16 of them
// (row 4 g + s in instruction s) at a time, the next on their way; the four waves
// of a workgroup add up in LDS.  Bound by reading W.
template <int DT, int NI>
__global__ __launch_bounds__(256) void thin_points_kernel(ThinArgs a)
{
    const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15, wave = threadIdx.x >> 6;
    const int64_t j0 = blockIdx.x % a.strips * 64, part = blockIdx.x / a.strips;
    const int64_t blocks = (a.v + 15) / 16, b0 = (part * 4 + wave) * a.each;
    const int64_t b1 = b0 + a.each < blocks ? b0 + a.each : blocks;
    f32x4 acc[NI][4];
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c)
            acc[i][c] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    f32x4 nw[4], nd[NI];
    auto fetch = [&](int64_t b) {
        const int64_t v0 = b * 16 + 4 * g;
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            // (beyond the last row D is zero)
            const int64_t v = v0 + s < a.v ? v0 + s : a.v - 1;
            nw[s] = quad<DT>(a.W, v * a.ldw, j0 + 4 * r, a.k);
        }
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int64_t row = 16 * i + r;
            nd[i] = row < a.n ? quad<GPIC_F32>(a.D, row * a.v, v0, a.v)
                              : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
    };
    if (b0 < b1)
        fetch(b0);
    for (int64_t b = b0; b < b1; ++b) {
        f32x4 w[4], d[NI];
#pragma unroll
        for (int s = 0; s < 4; ++s)
            w[s] = nw[s];
#pragma unroll
        for (int i = 0; i < NI; ++i)
            d[i] = nd[i];
        if (b + 1 < b1)
            fetch(b + 1);
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int i = 0; i < NI; ++i)
                    acc[i][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(w[s][c], d[i][s], acc[i][c], 0,
                                                                     0, 0);
    }
    __shared__ f32x4 all[4][4][64];
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        __syncthreads();
#pragma unroll
        for (int c = 0; c < 4; ++c)
            all[wave][c][lane] = acc[i][c];
        __syncthreads();
        const int64_t row = 16 * i + r;
        if (wave == i && row < a.n) {
            f32x4 sum[4];
#pragma unroll
            for (int c = 0; c < 4; ++c)
                sum[c] = ((all[0][c][lane] + all[1][c][lane]) + all[2][c][lane]) + all[3][c][lane];
            put16(a.part + (part * a.n + row) * a.k, j0 + 16 * g, a.k, sum);
        }
    }
}

// dX from its parts, in float64 in a fixed order
__global__ __launch_bounds__(256) void thin_join_kernel(ThinArgs a, int dtype)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, values = a.n * a.k;
    if (i >= values)
        return;
    double t = 0.0;
#pragma unroll 8
    for (int64_t p = 0; p < a.parts; ++p)
        t += (double)a.part[p * values + i];
    store1(a.dX, i, (float)t, dtype);
}

// db: column sums of D
__global__ __launch_bounds__(256) void thin_bias_kernel(const float *D, int64_t n, int64_t v, void *db,
                                                        int dtype)
{
    const int64_t col = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (col >= v)
        return;
    double t = 0.0;
#pragma unroll 8
    for (int64_t i = 0; i < n; ++i)
        t += (double)D[i * v + col];
    store1(db, col, (float)t, dtype);
}

// about four workgroups a compute unit, none of fewer than four turns a wave
int64_t parts_of(int64_t k, int64_t v)
{
    const int64_t strips = (k + 63) / 64, blocks = (v + 15) / 16;
    int64_t parts = 1024 / strips;
    parts = parts < blocks / 16 ? parts : blocks / 16;
    return parts < 1 ? 1 : parts;
}

} // namespace

size_t thin_ws(int64_t n, int64_t k, int64_t v)
{
    return (size_t)parts_of(k, v) * n * k * 4;
}

namespace {

template <int DT>
hipError_t run(ThinArgs a, void *db, hipStream_t st)
{
    const int64_t n = a.n, blocks = (a.v + 15) / 16;
    hipError_t e = hipSuccess;
    if (a.dW) {
        // about eight waves for each of the card's 1,024 vector units
        a.each = (blocks * a.strips + 8191) / 8192;
        const int64_t waves = (blocks + a.each - 1) / a.each * a.strips;
        const unsigned grid = (unsigned)((waves + 3) / 4);
        if (n <= 16)
            thin_weights_kernel<DT, 4><<<grid, 256, 0, st>>>(a);
        else if (n <= 32)
            thin_weights_kernel<DT, 8><<<grid, 256, 0, st>>>(a);
        else if (n <= 48)
            thin_weights_kernel<DT, 12><<<grid, 256, 0, st>>>(a);
        else
            thin_weights_kernel<DT, 16><<<grid, 256, 0, st>>>(a);
        e = hipGetLastError();
    }
    if (e == hipSuccess && a.dX) {
        a.each = (blocks + 4 * a.parts - 1) / (4 * a.parts);
        const unsigned grid = (unsigned)(a.strips * a.parts);
        if (n <= 16)
            thin_points_kernel<DT, 1><<<grid, 256, 0, st>>>(a);
        else if (n <= 32)
            thin_points_kernel<DT, 2><<<grid, 256, 0, st>>>(a);
        else if (n <= 48)
            thin_points_kernel<DT, 3><<<grid, 256, 0, st>>>(a);
        else
            thin_points_kernel<DT, 4><<<grid, 256, 0, st>>>(a);
        e = hipGetLastError();
        if (e != hipSuccess)
            return e;
        thin_join_kernel<<<(unsigned)((n * a.k + 255) / 256), 256, 0, st>>>(a, DT);
        e = hipGetLastError();
    }
    if (e == hipSuccess && db) {
        thin_bias_kernel<<<(unsigned)((a.v + 255) / 256), 256, 0, st>>>(a.D, n, a.v, db, DT);
        e = hipGetLastError();
    }
    return e;
}

} // namespace

hipError_t run_thin_gradients(const float *D, const float *X, const void *W, int64_t n, int64_t k,
                              int64_t v, int64_t ldw, int dtype, void *dX, void *dW, void *db,
                              float *part, hipStream_t st)
{
    const ThinArgs a{D, X, W, dX, dW, part, n, k, v, ldw, (k + 63) / 64, 0, parts_of(k, v)};
    return dtype == GPIC_F32    ? run<GPIC_F32>(a, db, st)
           : dtype == GPIC_F16 ? run<GPIC_F16>(a, db, st)
                               : run<GPIC_BF16>(a, db, st);
}

} // namespace gpic
