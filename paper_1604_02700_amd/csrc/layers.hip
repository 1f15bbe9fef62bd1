// Layers of an encoder and their gradients: Y = act(X W^T + b) + R, the
// gated projection H = act(X Wg^T) * (X Wu^T), and the passes around their
// matrix products (product.h): packing of operands that the product cannot
// read as they lie, dZ = dY act'(Z), and the column sums of the bias.
//
// float32 operands are multiplied as split halves (encoder.h) under powers
// of two from the largest finite magnitude of what a result's entry sums
// over: forward of each row of X and of W; for dX of each row of dZ and each
// column of W; for dW of each column of dZ and of X.  dZ is written twice
// then, once for each product.
#include "encoder.h"

namespace gpic {

namespace {

constexpr int kSumRows = 64;          // most rows of a partial column sum (below 2^29 in all)

inline size_t up(size_t x) { return (x + 255) & ~(size_t)255; }
__host__ __device__ inline int64_t up64(int64_t x) { return (x + 63) & ~(int64_t)63; }

// Lays a workspace out; with a null base it only counts.
struct Cursor {
    char *base;
    size_t at = 0;
    void *take(size_t bytes)
    {
        void *p = base ? base + at : nullptr;
        at += up(bytes);
        return p;
    }
};

// ---------------------------------------------------------------- maxima
// The largest of `count` values, by a block of 256 threads.
__device__ __forceinline__ float join_max(const float *part, int count)
{
    float best = 0.0f;
#pragma unroll 4
    for (int i = threadIdx.x; i < count; i += 256)
        best = fmaxf(best, part[i]);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
        best = fmaxf(best, __shfl_xor(best, o, 64));
    __shared__ float w[4];
    __syncthreads();
    if ((threadIdx.x & 63) == 0)
        w[threadIdx.x >> 6] = best;
    __syncthreads();
    return fmaxf(fmaxf(w[0], w[1]), fmaxf(w[2], w[3]));
}

// The exponent of the power of two that brings `most` into [2^14, 2^15):
// half-precision parts of the scaled values neither overflow nor, down to
// 2^-17 of the largest, lose bits.  (-113 .. 164: the power itself may be no
// float, so it is applied by ldexp.)
__device__ __forceinline__ int power_for(float most)
{
    if (!(most > 0.0f))
        return 0;
    int e;
    frexpf(most, &e);                 // most = f 2^e, f in [1/2, 1)
    return 15 - e;
}

__device__ __forceinline__ void split2(float x, _Float16 &hi, _Float16 &lo)
{
    hi = (_Float16)x;
    const float r = x - (float)hi;
    lo = fabsf((float)hi) < INFINITY ? (_Float16)r : (_Float16)0.0f;
}

// --------------------------------------------------------------- packing
struct PackJob {
    const void *x;
    int64_t rows, cols, ld;
    void *to;              // split matrix (float32) or rows of up64(cols)
    const int *power;      // float32: of every column
};
struct PackJobs {
    PackJob j[3];
};

// Copies of operands in the form that the product reads (grid.y: which).
// Eight columns a thread.  float32: split parts, every column under its power
// of two; 16 bits: zero-padded rows.
// Bound by memory: 10,007 x 1,000 and 777 x 1,000 in float32, read and
// written (86 MB), 15.8 us, 5.4 TB/s with what the maxima's pass left in the
// caches.  Splitting inside the product instead would do it once per tile
// that reads the operand.
template <bool SPLIT>
__global__ __launch_bounds__(256) void pack_kernel(PackJobs jobs)
{
    const PackJob m = jobs.j[blockIdx.y];
    const int64_t width = SPLIT ? (m.cols + 31) / 32 * 32 : up64(m.cols);
    const int64_t groups = width / 8, total = m.rows * groups;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total;
         i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / groups, c = (i - r * groups) * 8;
        if (SPLIT) {
            const float *x = static_cast<const float *>(m.x) + r * m.ld + c;
            float v[8];
            int power[8];
            if (c + 8 <= m.cols) {
                const f32x4 a = load4(x, 0, GPIC_F32), b = load4(x, 4, GPIC_F32);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    v[k] = a[k];
                    v[4 + k] = b[k];
                }
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    power[k] = m.power[c + k];
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    v[k] = c + k < m.cols ? x[k] : 0.0f;
                    power[k] = c + k < m.cols ? m.power[c + k] : 0;
                }
            }
            half8 h, l;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                _Float16 a, b;
                split2(ldexpf(v[k], power[k]), a, b);
                h[k] = a;
                l[k] = b;
            }
            _Float16 *to = static_cast<_Float16 *>(m.to) + r * 2 * width + split_at(c);
            *reinterpret_cast<half8 *>(to) = h;
            *reinterpret_cast<half8 *>(to + 32) = l;
        } else {
            const unsigned short *x = static_cast<const unsigned short *>(m.x) + r * m.ld + c;
            union {
                unsigned short h[8];
                u32x4 v;
            } u;
            using any = u32x4 __attribute__((aligned(2)));
            if (c + 8 <= m.cols) {
                u.v = *reinterpret_cast<const any *>(x);
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    u.h[k] = c + k < m.cols ? x[k] : (unsigned short)0;
            }
            *reinterpret_cast<u32x4 *>(static_cast<unsigned short *>(m.to) + r * width + c) = u.v;
        }
    }
}

// largest finite |v| and what was there
__device__ __forceinline__ float finite_max(float best, f32x4 v)
{
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const float a = fabsf(v[c]);
        best = a < INFINITY && a > best ? a : best;
    }
    return best;
}

struct RowJob {
    const float *x;
    int64_t rows, cols, ld;
    _Float16 *to;
    int *power;            // [rows]
};
struct RowJobs {
    RowJob j[2];
};

// Split copies of X and W (grid.y) whose rows have a power of two each: LANES
// lanes of a workgroup read a row into registers, find its largest finite
// magnitude and write its parts, so that the matrix is read once; what a row has
// beyond four groups of eight values a lane is read again.  Bound by memory:
// 10,007 x 1,000 and 777 x 1,000, read and written (86 MB), 18 us, 4.8 TB/s.
template <int LANES>
__global__ __launch_bounds__(256) void split_rows_kernel(RowJobs jobs)
{
    constexpr int kRows = 256 / LANES, kHold = 4, kStride = LANES;
    const RowJob m = jobs.j[blockIdx.y];
    const int wave = threadIdx.x >> 6, at = threadIdx.x % LANES;
    const int64_t width = (m.cols + 31) / 32 * 32, groups = width / 8;
    __shared__ float most[4];
    for (int64_t r = (int64_t)blockIdx.x * kRows + threadIdx.x / LANES; r < m.rows;
         r += (int64_t)gridDim.x * kRows) {
        const float *x = m.x + r * m.ld;
        f32x4 v[kHold][2];
        float best = 0.0f;
        auto read = [&](int64_t g, f32x4 (&u)[2]) {
            u[0] = u[1] = 0.0f;
            if (g * 8 + 8 <= m.cols) {
                u[0] = load4(x, g * 8, GPIC_F32);
                u[1] = load4(x, g * 8 + 4, GPIC_F32);
            } else if (g < groups) {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (g * 8 + k < m.cols)
                        u[k / 4][k % 4] = x[g * 8 + k];
            }
        };
#pragma unroll
        for (int h = 0; h < kHold; ++h)
            read(at + h * kStride, v[h]);
#pragma unroll
        for (int h = 0; h < kHold; ++h)
            best = finite_max(finite_max(best, v[h][0]), v[h][1]);
        for (int64_t g = at + kHold * kStride; g < groups; g += kStride) {
            f32x4 u[2];
            read(g, u);
            best = finite_max(finite_max(best, u[0]), u[1]);
        }
#pragma unroll
        for (int o = LANES < 64 ? LANES / 2 : 32; o > 0; o >>= 1)
            best = fmaxf(best, __shfl_xor(best, o, 64));
        if (LANES > 64) {
            __syncthreads();             // the row before has been read
            if ((threadIdx.x & 63) == 0)
                most[wave] = best;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < 4; ++w)
                best = fmaxf(best, most[w]);
        }
        const int power = power_for(best);
        if (at == 0)
            m.power[r] = power;
        auto write = [&](int64_t g, const f32x4 (&u)[2]) {
            if (g >= groups)
                return;
            half8 h, l;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                _Float16 a, b;
                split2(ldexpf(u[k / 4][k % 4], power), a, b);
                h[k] = a;
                l[k] = b;
            }
            _Float16 *to = m.to + r * 2 * width + split_at(g * 8);
            *reinterpret_cast<half8 *>(to) = h;
            *reinterpret_cast<half8 *>(to + 32) = l;
        };
#pragma unroll
        for (int h = 0; h < kHold; ++h)
            write(at + h * kStride, v[h]);
        for (int64_t g = at + kHold * kStride; g < groups; g += kStride) {
            f32x4 u[2];
            read(g, u);
            write(g, u);
        }
    }
}

// ------------------------------------------------------- dZ, column sums
struct GradArgs {
    const void *dY, *Z;
    int64_t ldy, ldz, n, m;
    int act;
    void *dZ;              // as dX's product reads it (16 bits: dW's too), or null
    void *dZ_columns;      // float32: as dW's product reads it, or null
    int64_t ldd;           // row pitch of both in 16-bit values
    int rows;              // of a workgroup
    float *sums;           // [ceil(n / rows)][m] partial column sums, or null
    const float *part;     // float16: partial maxima of dZ
    int parts;
    int *power;            // float16: dZ is stored times two to this; null: 0
    // float32: the powers of dZ's rows and of its columns
    const int *row_power, *column_power;
};

__device__ __forceinline__ f32x4 read4(const void *p, int64_t row_at, int64_t col, int64_t cols,
                                       int dtype)
{
    if (col + 4 <= cols)
        return load4(p, row_at + col, dtype);
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (col + j < cols)
            v[j] = load1(p, row_at + col + j, dtype);
    return v;
}

// four values of dZ from column col on (`end`: no column of this half lies
// at or beyond it), under their powers
template <int DT>
__device__ __forceinline__ void write4(void *dZ, int64_t at, int64_t col, int64_t end, f32x4 v,
                                       i32x4 power)
{
    const bool split = DT == GPIC_F32;
    if (DT != GPIC_BF16) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            v[j] = ldexpf(v[j], power[j]);
    }
    if (split) {
        _Float16 *d = static_cast<_Float16 *>(dZ) + at;
        half4 h, l;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            _Float16 x, y;
            split2(v[j], x, y);
            h[j] = x;
            l[j] = y;
        }
        if ((col & 3) == 0 && col + 4 <= end) {
            *reinterpret_cast<half4 *>(d + split_at(col)) = h;
            *reinterpret_cast<half4 *>(d + split_at(col) + 32) = l;
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (col + j < end) {
                    d[split_at(col + j)] = h[j];
                    d[split_at(col + j) + 32] = l[j];
                }
        }
        return;
    }
    if ((col & 3) == 0 && col + 4 <= end) {
        store4(dZ, at + col, v, DT);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (col + j < end)
                store1(dZ, at + col + j, v[j], DT);
    }
}

// d (gated: and du) of four entries of dZ from dY and Z
template <int ACT, bool GATED>
__device__ __forceinline__ void form4(f32x4 dy, f32x4 g, f32x4 u, f32x4 &d, f32x4 &du)
{
    d = dy;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (GATED || ACT != GPIC_ACT_NONE) {
            float y, dy1;
            activate_grad(g[j], ACT, y, dy1);
            d[j] = GATED ? dy[j] * u[j] * dy1 : dy[j] * dy1;
            du[j] = dy[j] * y;
        }
}

// Partial maxima of a float32 matrix's columns, or of dZ's columns and rows
// (float16: of dZ as a whole): `parts` runs of `each` rows by strips of 4
// `lanes` columns.
struct Maxima {
    const float *x;        // null: dZ
    int64_t rows, cols, ld;
    float *part;           // [parts][cols]
    int64_t strips, parts, each;
    int lanes;             // 16 or 32
    __host__ __device__ int64_t blocks() const { return strips * parts; }
};
struct MaximaArgs {
    Maxima j[3];
    int count;
    // dZ from these; its rows' maxima go to row_part [strips][rows], float16: its
    // own, one a workgroup, to row_part [parts strips]
    const void *dY, *Z;
    int64_t ldy, ldz, m;
    float *row_part;
};

// largest finite magnitudes of four columns of a strip (dZ: and of the up
// projection's) over rows r0 .. r1 - 1; of dZ's rows in row_part, float16: only
// the largest of all, in best
template <int DT, int ACT, bool GATED, bool DZ>
__device__ __forceinline__ void scan_maxima(const MaximaArgs &a, const Maxima &m, int64_t strip,
                                            int64_t r0, int64_t r1, f32x4 &best,
                                            f32x4 &best_u)
{
    constexpr int ZT = GATED ? GPIC_F32 : DT;      // the type of Z
    constexpr int kRows = DZ ? 2 : 4;              // of a lane in flight
    const int lanes = m.lanes, at = threadIdx.x & (lanes - 1), abreast = 256 / lanes;
    const int64_t cols = DZ ? a.m : m.cols, col = (strip * lanes + at) * 4;
    for (int64_t r = r0 + threadIdx.x / lanes; r < r1; r += abreast * kRows) {
        f32x4 x[kRows], g[kRows], u[kRows];
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            x[i] = g[i] = u[i] = 0.0f;
            const int64_t row = r + (int64_t)abreast * i;
            if (row < r1 && col < cols) {
                x[i] = DZ ? read4(a.dY, row * a.ldy, col, cols, DT)
                          : read4(m.x, row * m.ld, col, cols, GPIC_F32);
                if (DZ && (GATED || ACT != GPIC_ACT_NONE))
                    g[i] = read4(a.Z, row * a.ldz, col, cols, ZT);
                if (DZ && GATED)
                    u[i] = read4(a.Z, row * a.ldz + a.m, col, cols, ZT);
            }
        }
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            f32x4 d = x[i], du = 0.0f;
            if (DZ)
                form4<ACT, GATED>(x[i], g[i], u[i], d, du);
            float most = 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float v = fabsf(d[j]), w = fabsf(du[j]);
                const float fv = v < INFINITY ? v : 0.0f, fw = w < INFINITY ? w : 0.0f;
                best[j] = fmaxf(best[j], fv);
                if (DZ && GATED)
                    best_u[j] = fmaxf(best_u[j], fw);
                most = fmaxf(most, DZ && GATED ? fmaxf(fv, fw) : fv);
            }
            if (!DZ || DT == GPIC_F16)
                continue;
            for (int o = lanes / 2; o > 0; o >>= 1)
                most = fmaxf(most, __shfl_xor(most, o, 64));
            const int64_t row = r + (int64_t)abreast * i;
            if (at == 0 && row < r1)
                a.row_part[strip * m.rows + row] = most;
        }
    }
}

// Largest finite magnitudes of the columns of X, W and dZ and of the rows of
// dZ, which is formed for it and not kept: one more pass over dY and Z (the
// second one finds them in the caches where they fit), and no product of
// bounds stands in for a maximum.  Strips are narrow, so that little of the
// last one is beyond the columns.  Bound by memory and by the activation: dY and
// Z of 10,007 x 777 with gelu, X of 10,007 x 1,000 and W (105 MB) 24 us, 4.4 TB/s;
// the powers from the partial maxima 5.5 us.
template <int DT, int ACT, bool GATED>
__global__ __launch_bounds__(256) void maxima_kernel(MaximaArgs a)
{
    int64_t id = blockIdx.x;
    int job = 0;
    while (job + 1 < a.count && id >= a.j[job].blocks())
        id -= a.j[job++].blocks();
    const Maxima m = a.j[job];
    const bool dz = m.x == nullptr;
    const int64_t strip = id % m.strips, part = id / m.strips;
    const int64_t cols = dz ? a.m : m.cols;
    const int64_t r0 = part * m.each, r1 = r0 + m.each < m.rows ? r0 + m.each : m.rows;
    f32x4 best = 0.0f, best_u = 0.0f;
    if (dz)
        scan_maxima<DT, ACT, GATED, true>(a, m, strip, r0, r1, best, best_u);
    else
        scan_maxima<DT, ACT, GATED, false>(a, m, strip, r0, r1, best, best_u);
    if (DT == GPIC_F16) {
        float most = 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            most = fmaxf(most, fmaxf(best[j], best_u[j]));
        __shared__ float each[256];
        each[threadIdx.x] = most;
        __syncthreads();
        most = join_max(each, 256);
        if (threadIdx.x == 0)
            a.row_part[blockIdx.x] = most;
        return;
    }
    __shared__ f32x4 all[2][256];
    all[0][threadIdx.x] = best;
    all[1][threadIdx.x] = best_u;
    __syncthreads();
    // the first `lanes` threads the columns, the next ones the up projection's
    const int lanes = m.lanes, half = threadIdx.x / lanes, at = threadIdx.x & (lanes - 1);
    if (half > (GATED && dz ? 1 : 0))
        return;
    f32x4 v = 0.0f;
    for (int k = at; k < 256; k += lanes)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            v[j] = fmaxf(v[j], all[half][k][j]);
    const int64_t col = (strip * lanes + at) * 4;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (col + j < cols)
            m.part[part * m.cols + (half ? a.m : 0) + col + j] = v[j];
}

// Powers of two from partial maxima [parts][len]: a thread an entry, or
// sixteen where there are many parts.
struct PowerJob {
    const float *part;
    int64_t len, parts;
    int *power;
    __host__ __device__ bool many() const { return parts > 16; }
    __host__ __device__ int64_t blocks() const
    {
        return many() ? (len + 63) / 64 : (len + 1023) / 1024;
    }
};
struct PowerJobs {
    PowerJob j[4];
    int count;
};

__global__ __launch_bounds__(1024) void powers_kernel(PowerJobs a)
{
    int64_t id = blockIdx.x;
    int job = 0;
    while (job + 1 < a.count && id >= a.j[job].blocks())
        id -= a.j[job++].blocks();
    const PowerJob m = a.j[job];
    const bool many = m.many();
    const int first = many ? threadIdx.x >> 6 : 0, step = many ? 16 : 1;
    const int64_t i = many ? id * 64 + (threadIdx.x & 63) : id * 1024 + threadIdx.x;
    float best = 0.0f;
    if (i < m.len) {
#pragma unroll 8
        for (int64_t p = first; p < m.parts; p += step)
            best = fmaxf(best, m.part[p * m.len + i]);
    }
    __shared__ float all[1024];
    if (many) {
        all[threadIdx.x] = best;
        __syncthreads();
        if (threadIdx.x >= 64)
            return;
        for (int w = 1; w < 16; ++w)
            best = fmaxf(best, all[w * 64 + threadIdx.x]);
    }
    if (i < m.len)
        m.power[i] = power_for(best);
}

// dZ of `rows` rows x 256 columns a workgroup (four rows at a time, four
// columns a thread) and their column sums, in float32 in a fixed order.  For
// the products dZ is rounded as their operands are: to the matrices' type
// (float32: to two halves).  In bfloat16 that is what the gradients lose beside
// their own rounding (16,384 x 2,048 -> 8,192: 2.4e-3 off in the 2-norm, 1.7e-3
// if only the result were rounded); two parts of it would double the products.
// Bound by memory: reads dY and Z, writes dZ once.  16,384 x 8,192 in
// bfloat16 with gelu 184 us (805 MB, 4.4 TB/s); gated 8,192 x 5,504 with silu
// 171 us (631 MB, 3.7 TB/s); float32 10,007 x 777 with gelu, both copies, 30 us
// (124 MB, 4.1 TB/s).  Inside the products it would be formed once
// per tile row and column, and twice (dX and dW read it in different orders).
template <int DT, int ACT, bool GATED>
__global__ __launch_bounds__(256) void grad_kernel(GradArgs a)
{
    constexpr int ZT = GATED ? GPIC_F32 : DT;      // the type of Z
    int power = 0;
    if (DT == GPIC_F16 && a.power) {
        power = power_for(join_max(a.part, a.parts));
        if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0)
            *a.power = power;
    }
    const int64_t col = (int64_t)blockIdx.y * 256 + (threadIdx.x & 63) * 4;
    const int64_t r0 = (int64_t)blockIdx.x * a.rows;
    const int64_t r1 = r0 + a.rows < a.n ? r0 + a.rows : a.n;
    f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
    // the padding of dZ's rows (zeros): a layer's columns m .. end, the
    // gated layer's 2 m .. end
    const int64_t all = GATED ? 2 * a.m : a.m;
    const int64_t width = DT == GPIC_F32 ? (all + 31) / 32 * 32 : up64(all);
    const int64_t end = GATED ? a.m : width;
    i32x4 columns = 0, columns_u = 0;
    if (DT == GPIC_F32 && a.dZ_columns) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (col + j < a.m) {
                columns[j] = a.column_power[col + j];
                if (GATED)
                    columns_u[j] = a.column_power[a.m + col + j];
            }
    }
    // dZ from column c on, for the products that read it
    auto put = [&](int64_t r, int64_t c, int64_t last, f32x4 v, i32x4 each) {
        if (a.dZ)
            write4<DT>(a.dZ, r * a.ldd, c, last, v, i32x4{power, power, power, power});
        if (DT == GPIC_F32 && a.dZ_columns)
            write4<DT>(a.dZ_columns, r * a.ldd, c, last, v, each);
    };
    for (int64_t r = r0 + (threadIdx.x >> 6); r < r1; r += 4) {
        if (DT == GPIC_F32 && a.dZ)
            power = a.row_power[r];
        if (col < a.m) {
            const f32x4 dy = read4(a.dY, r * a.ldy, col, a.m, DT);
            f32x4 d = dy;
            if (GATED) {
                const f32x4 g = read4(a.Z, r * a.ldz, col, a.m, ZT);
                const f32x4 u = read4(a.Z, r * a.ldz + a.m, col, a.m, ZT);
                f32x4 du;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float y, dy1;
                    activate_grad(g[j], ACT, y, dy1);
                    d[j] = dy[j] * u[j] * dy1;
                    du[j] = dy[j] * y;
                }
                put(r, col, a.m, d, columns);
                put(r, a.m + col, 2 * a.m, du, columns_u);
            } else {
                if (ACT != GPIC_ACT_NONE) {
                    const f32x4 z = read4(a.Z, r * a.ldz, col, a.m, ZT);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float y, dy1;
                        activate_grad(z[j], ACT, y, dy1);
                        d[j] = dy[j] * dy1;
                    }
                    // beyond the last column z and dy are 0, and d too
                }
                put(r, col, end, d, columns);
                sum += d;
            }
        } else if (!GATED && col < end) {
            put(r, col, end, f32x4{0.0f, 0.0f, 0.0f, 0.0f}, columns);
        }
        // the thread at the gate's last column also writes the padding
        if (GATED && col < a.m && col + 4 >= a.m)
            for (int64_t c = all; c < width; ++c) {
                if (DT == GPIC_F32) {
                    for (void *to : {a.dZ, a.dZ_columns})
                        if (to) {
                            _Float16 *d = static_cast<_Float16 *>(to) + r * a.ldd + split_at(c);
                            d[0] = d[32] = (_Float16)0.0f;
                        }
                } else {
                    store1(a.dZ, r * a.ldd + c, 0.0f, DT);
                }
            }
    }
    if (a.sums == nullptr)
        return;
    __shared__ f32x4 part[256];
    part[threadIdx.x] = sum;
    __syncthreads();
    if (threadIdx.x < 64) {
        sum = ((part[threadIdx.x] + part[threadIdx.x + 64]) + part[threadIdx.x + 128]) +
              part[threadIdx.x + 192];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (col + j < a.m)
                a.sums[(int64_t)blockIdx.x * a.m + col + j] = sum[j];
    }
}

// Column sums from the partial ones, in float64 in a fixed order: 64
// columns a workgroup, sixteen runs of parts.  256 parts of 8,192 columns (8 MB)
// 5 us.
__global__ __launch_bounds__(1024) void sum_parts_kernel(const float *sums, int64_t parts, int64_t m,
                                                         void *db, int dtype)
{
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int64_t col = (int64_t)blockIdx.x * 64 + lane;
    double t = 0.0;
    if (col < m) {
#pragma unroll 8
        for (int64_t p = w; p < parts; p += 16)
            t += (double)sums[p * m + col];
    }
    __shared__ double part[16][64];
    part[w][lane] = t;
    __syncthreads();
    if (w == 0 && col < m) {
        for (int i = 1; i < 16; ++i)
            t += part[i][lane];
        store1(db, col, (float)t, dtype);
    }
}

// ------------------------------------------------------------------- host
unsigned blocks_for(int64_t items)
{
    const int64_t b = (items + 255) / 256;
    return (unsigned)(b < 1 ? 1 : (b > 4096 ? 4096 : b));
}

// A matrix that a product reads: as it lies where it can, else a packed
// copy in the workspace.
struct Source {
    const void *x;
    int64_t rows, cols, ld;
    bool pack;
    void *to = nullptr;
    int *power = nullptr;  // float32: of its rows (backward: columns)
    Operand operand(int dtype) const
    {
        if (!pack)
            return Operand{x, ld, 0, cols};
        const int64_t p = dtype == GPIC_F32 ? split_ld(cols) : up64(cols);
        return Operand{to, p, 0, p};
    }
};

// 16-bit matrices are read as they lie when rows start on 16 bytes and
// hold whole chunks of 8 values; float32 ones are always split.  `aligned16`:
// every matrix starts on 16 bytes.
bool must_pack(int dtype, int64_t cols, int64_t ld, bool aligned16)
{
    return dtype == GPIC_F32 || !aligned16 || cols % 8 || ld % 8;
}

// `powers`: how many powers of two the copy has (float32)
void place(Source &s, int dtype, Cursor &c, int64_t powers)
{
    if (!s.pack)
        return;
    const int64_t p = dtype == GPIC_F32 ? split_ld(s.cols) : up64(s.cols);
    s.to = c.take((size_t)s.rows * p * 2);
    if (dtype == GPIC_F32)
        s.power = static_cast<int *>(c.take((size_t)powers * 4));
}

// X and W of a float32 layer, a power of two for every row
hipError_t launch_split_rows(const Source &x, const Source &w, hipStream_t st)
{
    RowJobs j{};
    const Source *list[2] = {&x, &w};
    for (int i = 0; i < 2; ++i)
        j.j[i] = RowJob{static_cast<const float *>(list[i]->x), list[i]->rows, list[i]->cols,
                        list[i]->ld, static_cast<_Float16 *>(list[i]->to), list[i]->power};
    const int64_t rows = x.rows > w.rows ? x.rows : w.rows;
    // Few lanes a row keep all of them at work and more loads in flight.  us, X's
    // rows by 8, 32, 64 and 256 lanes: 50,000 x 72 13, 24, 42 and 130; 20,000 x 256
    // 14, 15, 20, 54; 10,000 x 512 12, 15, 16, 31; 10,007 x 1,000 25, 14, 17, 30;
    // 10,007 x 2,000 42, 32, 27, 32; 3,200 x 3,000 48, 19, 17, 17; 3,200 x 4,096 58,
    // 26, 23, 20.  Few rows by 64 lanes fill the card better (1,400 x 300 5.4 for
    // 6.8 by 8).
    int lanes = x.cols <= 512 ? 8 : (x.cols <= 1024 ? 32 : (x.cols <= 3000 ? 64 : 256));
    lanes = rows * lanes < 65536 && lanes < 64 ? 64 : lanes;
    int64_t blocks = (rows * lanes + 255) / 256;
    blocks = blocks > (1 << 20) ? 1 << 20 : blocks;
    const dim3 grid((unsigned)blocks, 2);
    if (lanes == 8)
        split_rows_kernel<8><<<grid, 256, 0, st>>>(j);
    else if (lanes == 32)
        split_rows_kernel<32><<<grid, 256, 0, st>>>(j);
    else if (lanes == 64)
        split_rows_kernel<64><<<grid, 256, 0, st>>>(j);
    else
        split_rows_kernel<256><<<grid, 256, 0, st>>>(j);
    return hipGetLastError();
}

hipError_t launch_pack(const Source *const *list, int count, int dtype, hipStream_t st)
{
    PackJobs j{};
    int used = 0;
    int64_t most = 0;
    for (int i = 0; i < count; ++i)
        if (list[i]->pack && list[i]->rows > 0) {
            const Source &s = *list[i];
            j.j[used++] = PackJob{s.x, s.rows, s.cols, s.ld, s.to, s.power};
            const int64_t groups = s.rows * ((s.cols + 63) / 64 * 8);
            most = groups > most ? groups : most;
        }
    if (used == 0)
        return hipSuccess;
    const dim3 grid(blocks_for(most), (unsigned)used);
    if (dtype == GPIC_F32)
        pack_kernel<true><<<grid, 256, 0, st>>>(j);
    else
        pack_kernel<false><<<grid, 256, 0, st>>>(j);
    return hipGetLastError();
}

template <int DT, bool GATED>
hipError_t launch_grad_act(const GradArgs &g, dim3 grid, hipStream_t st)
{
    switch (g.act) {
    case GPIC_ACT_NONE:
        grad_kernel<DT, GPIC_ACT_NONE, GATED><<<grid, 256, 0, st>>>(g);
        break;
    case GPIC_ACT_RELU:
        grad_kernel<DT, GPIC_ACT_RELU, GATED><<<grid, 256, 0, st>>>(g);
        break;
    case GPIC_ACT_GELU:
        grad_kernel<DT, GPIC_ACT_GELU, GATED><<<grid, 256, 0, st>>>(g);
        break;
    default:
        grad_kernel<DT, GPIC_ACT_SILU, GATED><<<grid, 256, 0, st>>>(g);
    }
    return hipGetLastError();
}

template <int DT>
hipError_t launch_grad(const GradArgs &g, bool gated, dim3 grid, hipStream_t st)
{
    return gated ? launch_grad_act<DT, true>(g, grid, st) : launch_grad_act<DT, false>(g, grid, st);
}

int kind_of(int dtype)
{
    return dtype == GPIC_F32 ? kOpSplit : (dtype == GPIC_F16 ? kOpF16 : kOpBf16);
}

// What a forward call keeps in its workspace.
struct Forward {
    Source X{}, W{};
    float *part = nullptr;
    Forward(const Shape &s, bool gated, const void *x, const void *w, Cursor &c)
    {
        if (as_rows(s, gated))
            return;
        const int64_t rows = gated ? 2 * s.m : s.m;
        X = Source{x, s.n, s.k, s.ldx, must_pack(s.dtype, s.k, s.ldx, s.aligned16)};
        W = Source{w, rows, s.k, s.ldw, must_pack(s.dtype, s.k, s.ldw, s.aligned16)};
        place(X, s.dtype, c, X.rows);
        place(W, s.dtype, c, W.rows);
        part = static_cast<float *>(c.take(
            product_plan(s.n, rows, s.k, 1, kind_of(s.dtype), gated ? kEpiGated : kEpiLayer)
                .part_bytes));
    }
};

// Rows of a workgroup of grad_kernel: 64, fewer where that would leave the
// card half empty (1,003 rows of 700: 48 workgroups of 16 turns, 25 us), more
// from 2^29 rows on, where the grid would come to 2^31 threads.
int grad_rows(int64_t n, int64_t m)
{
    int rows = kSumRows;
    while ((n + rows - 1) / rows > (1 << 23))
        rows *= 2;
    while (rows > 8 && (n + rows - 1) / rows * ((m + 255) / 256) < 1024)
        rows /= 2;
    return rows;
}

// How the maxima of a matrix's columns are cut: strips of 128 columns (of 64,
// where that is all: 100,000 x 16 -> 64 14 us instead of 21), about 1,536
// workgroups, none of fewer than 16 rows and no more than 512 runs of rows,
// which the powers are then found from.
Maxima maxima_of(const void *x, int64_t rows, int64_t cols, int64_t ld, int64_t across)
{
    Maxima m{static_cast<const float *>(x), rows, cols, ld, nullptr, 0, 0, 0, across <= 64 ? 16 : 32};
    m.strips = (across + 4 * m.lanes - 1) / (4 * m.lanes);
    int64_t parts = 1536 / m.strips;
    parts = parts < (rows + 15) / 16 ? parts : (rows + 15) / 16;
    parts = parts < 1 ? 1 : (parts > 512 ? 512 : parts);
    m.each = (rows + parts - 1) / parts;
    m.parts = m.each ? (rows + m.each - 1) / m.each : 0;
    return m;
}

// What a backward call keeps in its workspace.
struct Backward {
    Source dZ, X, W;
    void *dZ_columns = nullptr;      // float32: dW's copy of dZ, the powers of its columns
    int *column_power = nullptr;
    Maxima mz{}, mx{}, mw{};         // float32 (mz: float16 too)
    float *row_part = nullptr;       // [mz.strips][n], float16: [mz.blocks()]
    bool form;             // dZ is formed by grad_kernel (else dY is read)
    float *sums;
    int rows_each;         // rows of a workgroup of grad_kernel
    int *power;            // float16: of all of dZ
    float *part;
    int64_t rows;
    Backward(const Shape &s, bool gated, const void *dy, const void *x, const void *w, Cursor &c)
    {
        rows = gated ? 2 * s.m : s.m;
        form = gated || s.act != GPIC_ACT_NONE || s.dtype == GPIC_F32;
        dZ = Source{dy, s.n, rows, s.ldy,
                    form || must_pack(s.dtype, rows, s.ldy, s.aligned16)};
        X = Source{x, s.n, s.k, s.ldx, must_pack(s.dtype, s.k, s.ldx, s.aligned16)};
        W = Source{w, rows, s.k, s.ldw, must_pack(s.dtype, s.k, s.ldw, s.aligned16)};
        place(dZ, s.dtype, c, s.n);
        place(X, s.dtype, c, s.k);
        place(W, s.dtype, c, s.k);
        if (s.dtype == GPIC_F32) {
            dZ_columns = c.take((size_t)s.n * split_ld(rows) * 2);
            column_power = static_cast<int *>(c.take((size_t)rows * 4));
            mz = maxima_of(nullptr, s.n, rows, 0, s.m);
            mx = maxima_of(x, s.n, s.k, s.ldx, s.k);
            mw = maxima_of(w, rows, s.k, s.ldw, s.k);
            for (Maxima *m : {&mz, &mx, &mw})
                m->part = static_cast<float *>(c.take((size_t)(m->parts * m->cols) * 4));
            row_part = static_cast<float *>(c.take((size_t)(mz.strips * s.n) * 4));
        }
        // a dZ that is formed in half precision has a power too, from its own
        // largest magnitude (not gated: dY's): gradients times act' soon fall
        // below 6e-5, where halves lose bits
        power = nullptr;
        if (form && s.dtype == GPIC_F16) {
            mz = maxima_of(nullptr, s.n, rows, 0, s.m);
            row_part = static_cast<float *>(c.take((size_t)mz.blocks() * 4));
            power = static_cast<int *>(c.take(4));
        }
        rows_each = grad_rows(s.n, s.m);
        sums = static_cast<float *>(
            c.take((size_t)((s.n + rows_each - 1) / rows_each) * s.m * 4));
        const int op = kind_of(s.dtype);
        const size_t bx = product_plan(s.n, s.k, rows, 1, op, kEpiLayer).part_bytes;
        const size_t bw = product_plan(rows, s.k, s.n, 1, op, kEpiLayer).part_bytes;
        part = static_cast<float *>(c.take(bx > bw ? bx : bw));
    }
};

#define RUN(expr)                                                              \
    do {                                                                       \
        hipError_t e_ = (expr);                                                \
        if (e_ != hipSuccess)                                                  \
            return e_;                                                         \
    } while (0)

// The powers of two of a float32 backward call: of W's columns and dZ's rows
// for dX, of X's and dZ's columns for dW.  float16: dZ's partial maxima.
template <int DT, bool GATED>
void launch_maxima(const MaximaArgs &a, int act, unsigned blocks, hipStream_t st)
{
    switch (act) {
    case GPIC_ACT_NONE:
        maxima_kernel<DT, GPIC_ACT_NONE, GATED><<<blocks, 256, 0, st>>>(a);
        break;
    case GPIC_ACT_RELU:
        maxima_kernel<DT, GPIC_ACT_RELU, GATED><<<blocks, 256, 0, st>>>(a);
        break;
    case GPIC_ACT_GELU:
        maxima_kernel<DT, GPIC_ACT_GELU, GATED><<<blocks, 256, 0, st>>>(a);
        break;
    default:
        maxima_kernel<DT, GPIC_ACT_SILU, GATED><<<blocks, 256, 0, st>>>(a);
    }
}

hipError_t launch_powers(const Shape &s, bool gated, const Backward &b, const void *dY,
                         const void *Z, bool dX, bool dW, hipStream_t st)
{
    MaximaArgs a{};
    PowerJobs p{};
    const bool f32 = s.dtype == GPIC_F32;
    a.j[a.count++] = b.mz;
    if (dX && f32) {
        a.j[a.count++] = b.mw;
        p.j[p.count++] = PowerJob{b.mw.part, s.k, b.mw.parts, b.W.power};
        p.j[p.count++] = PowerJob{b.row_part, s.n, b.mz.strips, b.dZ.power};
    }
    if (dW && f32) {
        a.j[a.count++] = b.mx;
        p.j[p.count++] = PowerJob{b.mx.part, s.k, b.mx.parts, b.X.power};
        p.j[p.count++] = PowerJob{b.mz.part, b.rows, b.mz.parts, b.column_power};
    }
    a.dY = dY;
    a.Z = Z;
    a.ldy = s.ldy;
    a.ldz = s.ldz;
    a.m = s.m;
    a.row_part = b.row_part;
    int64_t blocks = 0;
    for (int i = 0; i < a.count; ++i)
        blocks += a.j[i].blocks();
    if (f32 && gated)
        launch_maxima<GPIC_F32, true>(a, s.act, (unsigned)blocks, st);
    else if (f32)
        launch_maxima<GPIC_F32, false>(a, s.act, (unsigned)blocks, st);
    else if (gated)
        launch_maxima<GPIC_F16, true>(a, s.act, (unsigned)blocks, st);
    else               // |dZ| <= 1.13 |dY|: the maxima of dY, without reading Z
        maxima_kernel<GPIC_F16, GPIC_ACT_NONE, false><<<(unsigned)blocks, 256, 0, st>>>(a);
    RUN(hipGetLastError());
    if (!f32)
        return hipSuccess;
    blocks = 0;
    for (int i = 0; i < p.count; ++i)
        blocks += p.j[i].blocks();
    powers_kernel<<<(unsigned)blocks, 1024, 0, st>>>(p);
    return hipGetLastError();
}

} // namespace

size_t layer_ws(const Shape &s, bool gated, bool backward)
{
    Cursor c{nullptr};
    if (backward && small_gradients(s, gated))
        return 0;
    if (backward)
        Backward b(s, gated, nullptr, nullptr, nullptr, c);
    else
        Forward f(s, gated, nullptr, nullptr, c);
    return c.at;
}

bool layer_fits(const Shape &s, bool gated, bool backward)
{
    if (s.n == 0 || (backward ? small_gradients(s, gated) : as_rows(s, gated)))
        return true;
    const int64_t rows = gated ? 2 * s.m : s.m;
    const int op = kind_of(s.dtype);
    if (!backward)
        return product_plan(s.n, rows, s.k, 1, op, gated ? kEpiGated : kEpiLayer).fits;
    return product_plan(s.n, s.k, rows, 1, op, kEpiLayer).fits &&
           product_plan(rows, s.k, s.n, 1, op, kEpiLayer).fits;
}

hipError_t run_layer(const Shape &s, bool gated, const void *X, const void *W, const void *bias,
                     const void *res, void *Y, void *Z, void *ws, hipStream_t st)
{
    if (s.n == 0)
        return hipSuccess;
    if (as_rows(s, gated))
        return run_rows(s, gated, X, W, bias, res, Y, Z, st);
    Cursor c{static_cast<char *>(ws)};
    Forward f(s, gated, X, W, c);
    const Source *list[2] = {&f.X, &f.W};
    if (s.dtype == GPIC_F32)
        RUN(launch_split_rows(f.X, f.W, st));
    else
        RUN(launch_pack(list, 2, s.dtype, st));
    ProductArgs a{};
    a.A = f.X.operand(s.dtype);
    a.B = f.W.operand(s.dtype);
    a.M = (int)s.n;
    a.N = (int)f.W.rows;
    a.K = s.k;
    a.batch = 1;
    a.part = f.part;
    Epilogue &e = a.e;
    e.pa = f.X.power;
    e.pb = f.W.power;
    e.bias = bias;
    e.res = res;
    e.out = Y;
    e.pre = Z;
    e.ldr = s.ldr;
    e.ldo = s.ldy;
    e.ldz = s.ldz;
    e.dtype = s.dtype;
    e.act = s.act;
    e.half = s.m;
    return launch_product(kKK, kind_of(s.dtype), gated ? kEpiGated : kEpiLayer, a, st);
}

hipError_t run_layer_backward(const Shape &s, bool gated, const void *dY, const void *X,
                              const void *W, const void *Z, void *dX, void *dW, void *db, void *ws,
                              hipStream_t st)
{
    if (small_gradients(s, gated))
        return run_small_gradients(s, gated, dY, X, W, Z, dX, dW, db, st);
    Cursor c{static_cast<char *>(ws)};
    Backward b(s, gated, dY, X, W, c);
    const int op = kind_of(s.dtype);
    // operands: what the wanted gradients read (of no rows: nothing)
    if (!dW || s.n == 0)
        b.X.pack = false;
    if (!dX || s.n == 0)
        b.W.pack = false;
    const bool need_dz = dX || dW;
    if (need_dz && b.mz.parts > 0)
        RUN(launch_powers(s, gated, b, dY, Z, dX != nullptr, dW != nullptr, st));
    {
        Source plain = b.dZ;
        plain.pack = b.dZ.pack && !b.form && need_dz;
        const Source *list[3] = {&b.X, &b.W, &plain};
        RUN(launch_pack(list, 3, s.dtype, st));
    }
    if (s.n > 0 && ((b.form && need_dz) || db)) {
        GradArgs g{};
        g.dY = dY;
        g.Z = Z;
        g.ldy = s.ldy;
        g.ldz = s.ldz;
        g.n = s.n;
        g.m = s.m;
        g.act = s.act;
        g.dZ = b.form && (dX || (dW && s.dtype != GPIC_F32)) ? b.dZ.to : nullptr;
        g.dZ_columns = dW ? b.dZ_columns : nullptr;
        g.row_power = b.dZ.power;
        g.column_power = b.column_power;
        g.ldd = s.dtype == GPIC_F32 ? split_ld(b.rows) : up64(b.rows);
        g.sums = db ? b.sums : nullptr;
        if (need_dz) {
            g.part = b.row_part;
            g.parts = (int)b.mz.blocks();
            g.power = b.power;
        }
        const int64_t width = gated ? s.m : up64(s.m);
        g.rows = b.rows_each;
        const dim3 grid((unsigned)((s.n + b.rows_each - 1) / b.rows_each),
                        (unsigned)((width + 255) / 256));
        RUN(s.dtype == GPIC_F32    ? launch_grad<GPIC_F32>(g, gated, grid, st)
            : s.dtype == GPIC_F16 ? launch_grad<GPIC_F16>(g, gated, grid, st)
                                  : launch_grad<GPIC_BF16>(g, gated, grid, st));
    }
    if (db) {
        sum_parts_kernel<<<(unsigned)((s.m + 63) / 64), 1024, 0, st>>>(
            b.sums, (s.n + b.rows_each - 1) / b.rows_each, s.m, db, s.dtype);
        RUN(hipGetLastError());
    }
    ProductArgs a{};
    a.batch = 1;
    a.part = b.part;
    a.e.dtype = s.dtype;
    a.e.act = GPIC_ACT_NONE;
    a.e.ldo = s.k;
    const Operand dz = b.dZ.operand(s.dtype);
    if (dX) {
        a.A = dz;
        a.B = b.W.operand(s.dtype);
        a.M = (int)s.n;
        a.N = (int)s.k;
        a.K = b.rows;
        a.e.pa = b.power ? b.power : b.dZ.power;
        a.e.pb = b.W.power;
        a.e.out = dX;
        RUN(launch_product(kKM, op, kEpiLayer, a, st));
    }
    if (dW) {
        a.A = dz;
        if (b.dZ_columns)
            a.A.p = b.dZ_columns;
        a.B = b.X.operand(s.dtype);
        a.M = (int)b.rows;
        a.N = (int)s.k;
        a.K = s.n;
        a.e.pa = b.power ? b.power : b.column_power;
        a.e.pb = b.X.power;
        if (s.n == 0)                              // no rows: dW = 0, no powers
            a.e.pa = a.e.pb = nullptr;
        a.e.out = dW;
        RUN(launch_product(kMM, op, kEpiLayer, a, st));
    }
    return hipSuccess;
}

} // namespace gpic
