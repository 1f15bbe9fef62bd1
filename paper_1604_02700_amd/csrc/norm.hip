// Layer norm and its gradients: y = (x - mean) r w + b with r = 1 / sqrt(var
// + eps); with g = dy w and h = (x - mean) r,
//   dx = r (g - mean(g) - h mean(g h)),  dw = sum_rows dy h,  db = sum_rows dy.
// Sums are float32, over rows float64 at the end, in a fixed order.
#include "training.h"

namespace gpic {
namespace {

struct NormArgs {
    const void *X, *w, *b;
    void *Y;
    float *stats;              // [n][2]: mean, r
    int64_t n, k, ldx, ldy;
    float eps;
};

// The sums over the LANES lanes that share a row, the same in all of them
// (LANES > 64: the whole workgroup; `part` is its scratch, LANES / 64 pairs).
template <int LANES>
__device__ __forceinline__ void row_sums(float &s, float &t, float2 *part)
{
#pragma unroll
    for (int o = (LANES < 64 ? LANES : 64) / 2; o > 0; o >>= 1) {
        s += __shfl_xor(s, o, 64);
        t += __shfl_xor(t, o, 64);
    }
    if (LANES <= 64)
        return;
    __syncthreads();                     // what was here before has been read
    if ((threadIdx.x & 63) == 0)
        part[threadIdx.x >> 6] = make_float2(s, t);
    __syncthreads();
    s = t = 0.0f;
#pragma unroll
    for (int i = 0; i < LANES / 64; ++i) {
        s += part[i].x;
        t += part[i].y;
    }
}

template <int DT>
__device__ __forceinline__ f32x8 read8(const void *p, int64_t row_at, int64_t col, int64_t cols)
{
    const int64_t left = cols - col;
    if (left <= 0)
        return f32x8(0.0f);
    return load8(p, row_at + col, DT, left < 8 ? (int)left : 8);
}

// Eight values of a row as they lie in memory.
template <int DT>
struct Chunk {
    static constexpr int kQuads = DT == GPIC_F32 ? 2 : 1;
    u32x4 q[kQuads];
    __device__ __forceinline__ void load(const void *p, int64_t i, int valid)
    {
        constexpr int kSize = DT == GPIC_F32 ? 4 : 2;
        using loose = u32x4 __attribute__((aligned(kSize)));
        const char *at = static_cast<const char *>(p) + i * kSize;
        if (valid >= 8) {
#pragma unroll
            for (int j = 0; j < kQuads; ++j)
                q[j] = *reinterpret_cast<const loose *>(at + 16 * j);
            return;
        }
#pragma unroll
        for (int j = 0; j < kQuads; ++j)
            q[j] = u32x4{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < valid) {
                if (DT == GPIC_F32)
                    q[j / 4 % kQuads][j % 4] = reinterpret_cast<const uint32_t *>(at)[j];
                else
                    q[0][j / 2] |= (uint32_t)reinterpret_cast<const uint16_t *>(at)[j]
                                   << (16 * (j & 1));
            }
    }
    // keeps the compiler from holding the floats it made of them (16,384 x 2,048 in
    // bfloat16, gradients: 61 us and spilled, 41 so)
    __device__ __forceinline__ void again()
    {
#pragma unroll
        for (int j = 0; j < kQuads; ++j)
            asm volatile("" : "+v"(q[j]));
    }
    __device__ __forceinline__ f32x8 floats() const
    {
        if constexpr (DT == GPIC_F32) {
            const f32x4 a = __builtin_bit_cast(f32x4, q[0]), b = __builtin_bit_cast(f32x4, q[1]);
            return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
        } else if constexpr (DT == GPIC_F16) {
            return __builtin_convertvector(__builtin_bit_cast(half8, q[0]), f32x8);
        } else {
            return __builtin_convertvector(__builtin_bit_cast(bfrag8, q[0]), f32x8);
        }
    }
};

// A row's values count as x c, its deviations as (x c - m) - off, whose
// reciprocal spread is r; the row's own mean, and the reciprocal of its spread.
struct RowStats {
    float c, m, off, r, mean, rs;
};

// (a product of its own: fused into some of the differences from it and not into
// others, it would be two values)
__device__ __forceinline__ float mean_of(float s, float inv)
{
#pragma clang fp contract(off)
    return s * inv;
}

// RowStats from the sums of the deviations from m and of their squares.  The first
// corrects m by `off`, which stays apart: a float32 mean holds little of it where
// a row is far from zero.
__device__ __forceinline__ void settle(RowStats &q, float s, float t, float inv, float eps)
{
    q.off = s * inv;
    const float var = fmaxf(t * inv - q.off * q.off, 0.0f);
    q.r = q.rs = 1.0f / sqrtf((t != t ? t : var) + eps);
    q.mean = q.m + q.off;
}

// Whether that does not hold: a sum or square is no float32, or `off` is so large
// beside the spread that its own rounding shows.
__device__ __forceinline__ bool unsettled(const RowStats &q, float t, float inv)
{
    return !(t < INFINITY && fabsf(q.off) * q.r <= 0x1p-8f && 2.0f * q.off * q.off <= t * inv);
}

// Such rows once more, from memory (a function of its own, which takes none of the
// kernel's registers; 10,007 x 1,000 in float32, every row 1e5 spreads away 58 us for 16,
// of 1e30 71).  Values beyond 1e19 or so are scaled by 2^-100, which leaves
// everything that matters beside the largest.  Rows far from zero are counted again
// from the corrected mean; rows of one value deviate by 0 then.
template <int DT, int LANES>
__device__ __noinline__ void norm_anew(const void *X, const void *w, const void *b, void *Y,
                                       float *stats, int64_t k, float eps, float2 *part)
{
    constexpr float kMost = 0x1.fffffep127f;
    const int at = threadIdx.x % LANES;
    const float inv = 1.0f / (float)k;
    RowStats q;
    q.c = 1.0f;
    bool fresh = true, moved = false;
    for (bool more = true; more;) {
        float s = 0.0f, t = 0.0f;
        if (fresh) {
#pragma unroll 8
            for (int64_t c = at; c < k; c += LANES)
                s += load1(X, c, DT) * q.c;
            row_sums<LANES>(s, t, part);
            q.m = mean_of(s, inv);
        }
        s = t = 0.0f;
#pragma unroll 8
        for (int64_t c = at; c < k; c += LANES) {
            const float d = load1(X, c, DT) * q.c - q.m;
            s += d;
            t += d * d;
        }
        row_sums<LANES>(s, t, part);
        settle(q, s, t, inv, eps * q.c * q.c);
        more = unsettled(q, t, inv) && !moved;
        fresh = q.c == 1.0f && !(t < INFINITY);
        if (fresh)
            q.c = 0x1p-100f;
        moved = more && !fresh;
        q.m = moved ? q.mean : q.m;
    }
    if (q.c != 1.0f) {
        q.rs = q.r * q.c;
        q.mean = q.mean * 0x1p100f;
        if (fabsf(q.mean) == INFINITY)       // of finite values: rounded so
            q.mean = copysignf(kMost, q.mean);
        if (q.r == INFINITY && eps > 0.0f) { // (rows of one value: eps vanishes beside 2^200)
            q.rs = 1.0f / sqrtf(eps);
            q.r = kMost;
        }
    }
    if (stats && at == 0)
        *reinterpret_cast<float2 *>(stats) = make_float2(q.mean, q.rs);
#pragma unroll 4
    for (int64_t c = at; c < k; c += LANES) {
        float y = (load1(X, c, DT) * q.c - q.m - q.off) * q.r;
        if (w)
            y *= load1(w, c, DT);
        if (b)
            y += load1(b, c, DT);
        store1(Y, c, y, DT);
    }
}

template <int DT, int LANES>
__device__ __forceinline__ void norm_anew(const NormArgs &a, int64_t r, float2 *part)
{
    constexpr int kSize = DT == GPIC_F32 ? 4 : 2;
    norm_anew<DT, LANES>(static_cast<const char *>(a.X) + r * a.ldx * kSize, a.w, a.b,
                         static_cast<char *>(a.Y) + r * a.ldy * kSize,
                         a.stats ? a.stats + 2 * r : nullptr, a.k, a.eps, part);
}

// Rows that LANES lanes hold in HOLD groups of eight columns each, with the next
// row on its way while one is finished: the mean, then the deviations from it,
// whose own sum corrects it, so that rows far from zero lose nothing.  Groups of
// lanes take rows in turn over the whole grid, up to 64 each; those that are not
// settled come last (in their turn 26.5 us for 24.7).  Bound by memory: 16,384 x 2,048 in
// bfloat16 24.7 us (5.4 TB/s), 31 with a row a wave and no next one on its way;
// 10,007 x 1,000 in float32 16.0 (5.0); 1,024 workgroups, since 2,048 and more take
// up to 30 % longer (16,384 x 2,048 in float32 46 us, 47, and 59 with 4,096).
template <int DT, int LANES, int HOLD>
__global__ __launch_bounds__(256) void norm_rows_kernel(NormArgs a)
{
    constexpr int kRows = 256 / LANES;
    __shared__ float2 part[LANES > 64 ? LANES / 64 : 1];
    const int at = threadIdx.x % LANES;
    const float inv = 1.0f / (float)a.k;
    int valid[HOLD];
#pragma unroll
    for (int h = 0; h < HOLD; ++h) {
        const int64_t left = a.k - (int64_t)(at + h * LANES) * 8;
        valid[h] = left <= 0 ? 0 : (left < 8 ? (int)left : 8);
    }
    Chunk<DT> w[HOLD], b[HOLD], x[HOLD], next[HOLD];
    auto fetch = [&](int64_t r) {
#pragma unroll
        for (int h = 0; h < HOLD; ++h)
            next[h].load(a.X, r * a.ldx + (at + h * LANES) * 8, valid[h]);
    };
    const int64_t step = (int64_t)gridDim.x * kRows;
    int64_t r = (int64_t)blockIdx.x * kRows + threadIdx.x / LANES;
    const int64_t first = r;
    uint64_t again = 0;                  // which of up to 64 rows are not settled
    if (r < a.n)
        fetch(r);
#pragma unroll
    for (int h = 0; h < HOLD; ++h) {
        if (a.w)
            w[h].load(a.w, (at + h * LANES) * 8, valid[h]);
        if (a.b)
            b[h].load(a.b, (at + h * LANES) * 8, valid[h]);
    }
    for (int turn = 0; r < a.n; ++turn, r += step) {
#pragma unroll
        for (int h = 0; h < HOLD; ++h)
            x[h] = next[h];
        if (r + step < a.n)
            fetch(r + step);
        float s = 0.0f, t = 0.0f;
#pragma unroll
        for (int h = 0; h < HOLD; ++h) {
            const f32x8 v = x[h].floats();
#pragma unroll
            for (int j = 0; j < 8; ++j)
                s += v[j];                   // (zeros beyond the row)
        }
        row_sums<LANES>(s, t, part);
        RowStats q;
        q.m = mean_of(s, inv);
        s = t = 0.0f;
#pragma unroll
        for (int h = 0; h < HOLD; ++h) {
            const f32x8 v = x[h].floats();
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float d = j < valid[h] ? v[j] - q.m : 0.0f;
                s += d;
                t += d * d;
            }
        }
        row_sums<LANES>(s, t, part);
        settle(q, s, t, inv, a.eps);
        const bool open = unsettled(q, t, inv);
        again |= open ? 1ull << turn : 0;
        if (a.stats && at == 0)
            reinterpret_cast<float2 *>(a.stats)[r] = make_float2(q.mean, q.rs);
        const float shift = -q.off * q.r;
#pragma unroll
        for (int h = 0; h < HOLD; ++h) {
            if (!valid[h] || open)           // (Y may be X, which is read again)
                continue;
            f32x8 y = (x[h].floats() - q.m) * q.r + shift;
            if (a.w)
                y = y * w[h].floats();
            if (a.b)
                y = y + b[h].floats();
            store8(a.Y, r * a.ldy + (at + h * LANES) * 8, y, DT, valid[h]);
        }
    }
    for (; again; again &= again - 1)
        norm_anew<DT, LANES>(a, first + __builtin_ctzll(again) * step, part);
}

// Longer rows: a workgroup a row, eight columns at a time a lane; up to kHold
// groups of them stay in registers, what a row has beyond is read again.
template <int DT, int LANES>
__global__ __launch_bounds__(LANES > 256 ? LANES : 256) void norm_kernel(NormArgs a)
{
    constexpr int kHold = 4, kThreads = LANES > 256 ? LANES : 256, kRows = kThreads / LANES;
    __shared__ float2 part[LANES > 64 ? LANES / 64 : 1];
    const int at = threadIdx.x % LANES;
    const int64_t groups = (a.k + 7) / 8;
    const float inv = 1.0f / (float)a.k;
    for (int64_t r = (int64_t)blockIdx.x * kRows + threadIdx.x / LANES; r < a.n;
         r += (int64_t)gridDim.x * kRows) {
        f32x8 v[kHold];
        float s = 0.0f, t = 0.0f;
#pragma unroll
        for (int h = 0; h < kHold; ++h) {
            v[h] = read8<DT>(a.X, r * a.ldx, (int64_t)(at + h * LANES) * 8, a.k);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                s += v[h][j];
        }
        for (int64_t g = at + kHold * LANES; g < groups; g += LANES) {
            const f32x8 u = read8<DT>(a.X, r * a.ldx, g * 8, a.k);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                s += u[j];
        }
        row_sums<LANES>(s, t, part);
        RowStats q;
        q.m = mean_of(s, inv);
        s = t = 0.0f;
        auto deviate = [&](const f32x8 &u, int64_t g) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float d = g * 8 + j < a.k ? u[j] - q.m : 0.0f;
                s += d;
                t += d * d;
            }
        };
#pragma unroll
        for (int h = 0; h < kHold; ++h)
            deviate(v[h], at + h * LANES);
        for (int64_t g = at + kHold * LANES; g < groups; g += LANES)
            deviate(read8<DT>(a.X, r * a.ldx, g * 8, a.k), g);
        row_sums<LANES>(s, t, part);
        settle(q, s, t, inv, a.eps);
        if (unsettled(q, t, inv)) {
            norm_anew<DT, LANES>(a, r, part);
            continue;
        }
        if (a.stats && at == 0)
            reinterpret_cast<float2 *>(a.stats)[r] = make_float2(q.mean, q.rs);
        const float shift = -q.off * q.r;
        auto write = [&](const f32x8 &u, int64_t g) {
            const int64_t left = a.k - g * 8;
            if (left <= 0)
                return;
            const int valid = left < 8 ? (int)left : 8;
            f32x8 y = (u - q.m) * q.r + shift;
            if (a.w)
                y = y * load8(a.w, g * 8, DT, valid);
            if (a.b)
                y = y + load8(a.b, g * 8, DT, valid);
            store8(a.Y, r * a.ldy + g * 8, y, DT, valid);
        };
#pragma unroll
        for (int h = 0; h < kHold; ++h)
            write(v[h], at + h * LANES);
        for (int64_t g = at + kHold * LANES; g < groups; g += LANES)
            write(read8<DT>(a.X, r * a.ldx, g * 8, a.k), g);
    }
}

// h = (x - mean) r - mean of that: the statistics' mean is a float32, off by up to half
// a unit, which is most of a spread where a row is far enough from zero.  What
// is off is the mean of (x - mean) r, found along with the other two.  Rows of the
// largest values deviate by more than a float32 holds, and then r is next to nothing:
// both under a power of two.
struct Deviation {
    float c, m, r;
    __device__ __forceinline__ explicit Deviation(float2 stats)
    {
        c = stats.y < 0x1p-100f ? 0x1p-10f : 1.0f;
        m = stats.x * c;
        r = stats.y < 0x1p-100f ? stats.y * 0x1p10f : stats.y;
    }
    template <class T>
    __device__ __forceinline__ T of(T x) const { return (x * c - m) * r; }
};

// The sums over LANES lanes that share a row within a wave
template <int LANES>
__device__ __forceinline__ void wave_sums(float &s, float &t, float &u)
{
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) {
        s += __shfl_xor(s, o, 64);
        t += __shfl_xor(t, o, 64);
        u += __shfl_xor(u, o, 64);
    }
}

struct NormGradArgs {
    const void *dY, *X, *w;
    const float *stats;
    void *dX;
    float *dots;               // [n][4]: mean(g), mean(g h), mean((x - mean) r)
    float *sums;               // [parts][2][k]: of dy h, of dy
    int64_t n, k, ldx, ldy;
    int64_t strips, each;
};

// mean(g), mean(g h) and what the mean is off by, of every row
template <int DT>
__global__ __launch_bounds__(256) void norm_dots_kernel(NormGradArgs a)
{
    __shared__ float4 part[4];
    const int64_t groups = (a.k + 7) / 8;
    const float inv = 1.0f / (float)a.k;
    for (int64_t r = blockIdx.x; r < a.n; r += gridDim.x) {
        const Deviation dev(reinterpret_cast<const float2 *>(a.stats)[r]);
        float s = 0.0f, t = 0.0f, u = 0.0f;
        for (int64_t g = threadIdx.x; g < groups; g += 256) {
            const int valid = a.k - g * 8 < 8 ? (int)(a.k - g * 8) : 8;
            f32x8 d = load8(a.dY, r * a.ldy + g * 8, DT, valid);
            const f32x8 x = load8(a.X, r * a.ldx + g * 8, DT, valid);
            if (a.w)
                d = d * load8(a.w, g * 8, DT, valid);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < valid) {
                    const float h = dev.of(x[j]);
                    s += d[j];
                    t += d[j] * h;
                    u += h;
                }
        }
        wave_sums<64>(s, t, u);
        __syncthreads();                 // what was here before has been read
        if ((threadIdx.x & 63) == 0)
            part[threadIdx.x >> 6] = make_float4(s, t, u, 0.0f);
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int i = 1; i < 4; ++i) {
                s += part[i].x;
                t += part[i].y;
                u += part[i].z;
            }
            s *= inv;
            u *= inv;
            reinterpret_cast<float4 *>(a.dots)[r] = make_float4(s, t * inv - u * s, u, 0.0f);
        }
    }
}

// Longer rows: mean(g) and mean(g h) first, then dX and the partial sums of a
// strip of 512 columns over `each` rows, four
// rows at a time
template <int DT>
__global__ __launch_bounds__(256) void norm_strip_kernel(NormGradArgs a)
{
    const int64_t strip = blockIdx.x % a.strips, part = blockIdx.x / a.strips;
    const int64_t col = (strip * 64 + (threadIdx.x & 63)) * 8;
    const int64_t r0 = part * a.each, r1 = r0 + a.each < a.n ? r0 + a.each : a.n;
    const int64_t left = a.k - col;
    const int valid = left <= 0 ? 0 : (left < 8 ? (int)left : 8);
    f32x8 sw = 0.0f, sb = 0.0f, w = 1.0f;
    if (a.w && valid)
        w = load8(a.w, col, DT, valid);
    if (valid)
        for (int64_t r = r0 + (threadIdx.x >> 6); r < r1; r += 4) {
            const float2 st = reinterpret_cast<const float2 *>(a.stats)[r];
            const f32x8 d = load8(a.dY, r * a.ldy + col, DT, valid);
            const f32x8 x = load8(a.X, r * a.ldx + col, DT, valid);
            sb += d;
            if (!a.dots)                 // (db alone)
                continue;
            const float4 m = reinterpret_cast<const float4 *>(a.dots)[r];
            const f32x8 h = Deviation(st).of(x) - m.z;
            sw += d * h;
            if (a.dX)
                store8(a.dX, r * a.k + col, (d * w - m.x - h * m.y) * st.y, DT, valid);
        }
    if (!a.sums)
        return;
    __shared__ f32x8 all[2][4][64];
    all[0][threadIdx.x >> 6][threadIdx.x & 63] = sw;
    all[1][threadIdx.x >> 6][threadIdx.x & 63] = sb;
    __syncthreads();
    const int which = threadIdx.x >> 6, l = threadIdx.x & 63;
    if (which < 2 && valid) {
        const f32x8 s = ((all[which][0][l] + all[which][1][l]) + all[which][2][l]) +
                        all[which][3][l];
        store8(a.sums + (part * 2 + which) * a.k, col, s, GPIC_F32, valid);
    }
}

// The same in one pass over X and dY, for rows that LANES lanes hold in HOLD
// groups of eight columns each: the next row is on its way while one is
// finished, and the columns' sums stay in registers until the rows are through,
// then meet in LDS.  Groups of lanes take rows in turn over the whole grid.  Bound
// by memory: 16,384 x 2,048 in bfloat16 41 us with the join (4.9 TB/s), 10,007 x
// 1,000 in float32 26 (4.6); in two passes, rows' means and then strips of
// columns, 63 and 40.
template <int DT, int LANES, int HOLD, int THREADS>
__global__ __launch_bounds__(THREADS) void norm_grad_kernel(NormGradArgs a)
{
    constexpr int kRows = THREADS / LANES, kWaves = THREADS / 64;
    constexpr bool kWide = LANES > 64;
    // sums of rows across waves (two sets in turn), or of columns
    __shared__ float4 part[kWide ? 2 : 1][kWide ? LANES / 64 : 1];
    __shared__ f32x8 cols[kWide ? 1 : kWaves][kWide ? 1 : 64];
    const int at = threadIdx.x % LANES;
    const float inv = 1.0f / (float)a.k;
    int valid[HOLD];
#pragma unroll
    for (int h = 0; h < HOLD; ++h) {
        const int64_t left = a.k - (int64_t)(at + h * LANES) * 8;
        valid[h] = left <= 0 ? 0 : (left < 8 ? (int)left : 8);
    }
    Chunk<DT> w[HOLD], x[HOLD], d[HOLD], nx[HOLD], nd[HOLD];
    f32x8 sw[HOLD], sb[HOLD];
#pragma unroll
    for (int h = 0; h < HOLD; ++h) {
        sw[h] = sb[h] = 0.0f;
        if (a.w)
            w[h].load(a.w, (at + h * LANES) * 8, valid[h]);
    }
    float2 st, nst;
    auto fetch = [&](int64_t r) {
        nst = reinterpret_cast<const float2 *>(a.stats)[r];
#pragma unroll
        for (int h = 0; h < HOLD; ++h) {
            nx[h].load(a.X, r * a.ldx + (at + h * LANES) * 8, valid[h]);
            nd[h].load(a.dY, r * a.ldy + (at + h * LANES) * 8, valid[h]);
        }
    };
    const int64_t step = (int64_t)gridDim.x * kRows;
    int64_t r = (int64_t)blockIdx.x * kRows + threadIdx.x / LANES;
    if (r < a.n)
        fetch(r);
    for (int turn = 0; r < a.n; r += step, turn ^= 1) {
        st = nst;
#pragma unroll
        for (int h = 0; h < HOLD; ++h) {
            x[h] = nx[h];
            d[h] = nd[h];
        }
        if (r + step < a.n)
            fetch(r + step);
        float s = 0.0f, t = 0.0f, u = 0.0f;
        const Deviation dev(st);
#pragma unroll
        for (int h = 0; h < HOLD; ++h) {
            const f32x8 dy = d[h].floats(), hx = dev.of(x[h].floats());
            const f32x8 g = a.w ? dy * w[h].floats() : dy;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < valid[h]) {
                    s += g[j];
                    t += g[j] * hx[j];
                    u += hx[j];
                    sb[h][j] += dy[j];
                }
        }
        wave_sums<(kWide ? 64 : LANES)>(s, t, u);
        if (kWide) {
            if ((threadIdx.x & 63) == 0)
                part[turn & (kWide ? 1 : 0)][threadIdx.x >> 6] = make_float4(s, t, u, 0.0f);
            __syncthreads();
            s = t = u = 0.0f;
#pragma unroll
            for (int i = 0; i < (kWide ? LANES / 64 : 1); ++i) {
                const float4 p = part[turn & (kWide ? 1 : 0)][i];
                s += p.x;
                t += p.y;
                u += p.z;
            }
        }
        s *= inv;
        u *= inv;
        t = t * inv - u * s;
#pragma unroll
        for (int h = 0; HOLD > 2 && h < HOLD; ++h) {
            x[h].again();
            d[h].again();
        }
#pragma unroll
        for (int h = 0; h < HOLD; ++h) {
            if (!valid[h])
                continue;
            const f32x8 dy = d[h].floats(), hx = dev.of(x[h].floats()) - u;
            sw[h] += dy * hx;
            if (a.dX) {
                const f32x8 g = a.w ? dy * w[h].floats() : dy;
                store8(a.dX, r * a.k + (at + h * LANES) * 8, (g - s - hx * t) * st.y, DT,
                       valid[h]);
            }
        }
    }
    if (!a.sums)
        return;
#pragma unroll
    for (int i = 0; i < 2 * HOLD; ++i) {
        const int h = i >> 1;
        f32x8 v = i & 1 ? sb[h] : sw[h];
        float *to = a.sums + ((int64_t)blockIdx.x * 2 + (i & 1)) * a.k;
        if (kWide) {                     // a workgroup's rows are one after another
            if (valid[h])
                store8(to, (at + h * LANES) * 8, v, GPIC_F32, valid[h]);
            continue;
        }
#pragma unroll
        for (int o = LANES; o < 64; o <<= 1)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                v[j] += __shfl_xor(v[j], o, 64);
        __syncthreads();
        cols[kWide ? 0 : threadIdx.x >> 6][kWide ? 0 : threadIdx.x & 63] = v;
        __syncthreads();
        if (threadIdx.x < LANES && valid[h]) {
#pragma unroll
            for (int o = 1; o < kWaves; ++o)
                v += cols[kWide ? 0 : o][kWide ? 0 : threadIdx.x];
            store8(to, (at + h * LANES) * 8, v, GPIC_F32, valid[h]);
        }
    }
}

// dW and db (grid.y) from the partial sums, in float64 in a fixed order: 64
// columns a workgroup, sixteen runs of parts
__global__ __launch_bounds__(1024) void norm_join_kernel(const float *sums, int64_t parts,
                                                         int64_t k, void *dW, void *db, int dtype)
{
    void *out = blockIdx.y ? db : dW;
    if (!out)
        return;
    const int lane = threadIdx.x & 63, run = threadIdx.x >> 6;
    const int64_t col = (int64_t)blockIdx.x * 64 + lane;
    double t = 0.0;
    if (col < k) {
#pragma unroll 8
        for (int64_t p = run; p < parts; p += 16)
            t += (double)sums[(p * 2 + blockIdx.y) * k + col];
    }
    __shared__ double all[16][64];
    all[run][lane] = t;
    __syncthreads();
    if (run == 0 && col < k) {
        for (int i = 1; i < 16; ++i)
            t += all[i][lane];
        store1(out, col, (float)t, dtype);
    }
}

// ------------------------------------------------------------------- host
constexpr int64_t kMostBlocks = 1 << 20;
constexpr int64_t kNormBlocks = 1024;

unsigned capped(int64_t blocks)
{
    return (unsigned)(blocks < 1 ? 1 : (blocks > kMostBlocks ? kMostBlocks : blocks));
}

// How the gradients' rows are cut: one pass by groups of lanes that hold a row
// (up to 8,192 columns), or strips of 512 columns.
struct Cut {
    int lanes, hold;           // 0: strips
    int64_t strips, each, parts;
    explicit Cut(const Norm &p)
    {
        strips = (p.k + 511) / 512;
        lanes = hold = 0;
        each = 0;
        // (float32 rows of 1,025 to 2,048 in a wave take more registers than it has: 16,384 x
        // 2,048 128 us by 64 lanes, 76 by 256; in bfloat16 41 by 64)
        static const int kFit[][2] = {{4, 1},  {8, 1},  {16, 1},  {16, 2}, {64, 1},
                                      {64, 2}, {64, 4}, {256, 1}, {256, 2}, {256, 4}};
        for (auto &f : kFit)
            if (p.k <= f[0] * f[1] * 8 && !(p.dtype == GPIC_F32 && f[0] == 64 && f[1] == 4)) {
                lanes = f[0];
                hold = f[1];
                break;
            }
        if (lanes) {
            // two waves to each of the card's 1,024 vector units, fewer where
            // rows are
            const int rows = lanes > 64 ? 1 : 512 / lanes;
            parts = (p.n + rows - 1) / rows;
            const int64_t most = lanes > 64 ? 512 : 256;
            parts = parts < most ? parts : most;
            return;
        }
        int64_t want = 2048 / strips;
        want = want < (p.n + 15) / 16 ? want : (p.n + 15) / 16;
        want = want < 1 ? 1 : want;
        each = (p.n + want - 1) / want;
        parts = each ? (p.n + each - 1) / each : 0;
    }
};

struct Backward {
    float *dots, *sums;
    Backward(const Norm &p, Cursor &c)
    {
        const Cut s(p);
        dots = s.lanes ? nullptr : static_cast<float *>(c.take((size_t)p.n * 16));
        sums = static_cast<float *>(c.take((size_t)s.parts * 2 * p.k * 4));
    }
};

template <int DT, int LANES, int HOLD>
void launch_rows(const NormArgs &a, hipStream_t st)
{
    constexpr int kSize = DT == GPIC_F32 ? 4 : 2;
    // (64 rows a group of lanes at most)
    constexpr int64_t kRows = 256 / LANES, kMost = kNormBlocks * kRows * 64;
    for (int64_t first = 0; first < a.n; first += kMost) {
        NormArgs p = a;
        p.X = static_cast<const char *>(a.X) + first * a.ldx * kSize;
        p.Y = static_cast<char *>(a.Y) + first * a.ldy * kSize;
        p.stats = a.stats ? a.stats + first * 2 : nullptr;
        p.n = a.n - first < kMost ? a.n - first : kMost;
        const int64_t blocks = (p.n + kRows - 1) / kRows;
        norm_rows_kernel<DT, LANES, HOLD>
            <<<(unsigned)(blocks < kNormBlocks ? blocks : kNormBlocks), 256, 0, st>>>(p);
    }
}

template <int DT>
hipError_t launch_norm(const NormArgs &a, hipStream_t st)
{
    if (a.k > 8192)
        norm_kernel<DT, 1024><<<capped(a.n), 1024, 0, st>>>(a);
    else if (a.k > 4096)
        launch_rows<DT, 256, 4>(a, st);
    else if (a.k > 2048)
        launch_rows<DT, 256, 2>(a, st);
    // Fewer rows than workgroups that stay: one each, in whose lanes more is under way.  us
    // by waves and so: 32 x 2,048 in float32 4.7 and 3.0, 700 x 2,048 5.7 and 4.3, 256 x 1,000
    // in bfloat16 3.6 and 3.2, 1,000 x 1,000 3.8 and 4.0; beyond, 2,000 x 700 4.9 and 6.7.
    else if (a.k > 512 && a.n < 1024)
        launch_rows<DT, 256, 1>(a, st);
    else if (a.k > 1024)
        launch_rows<DT, 64, 4>(a, st);
    else if (a.k > 512)
        launch_rows<DT, 64, 2>(a, st);
    else if (a.k > 256)
        launch_rows<DT, 64, 1>(a, st);
    else if (a.k > 128)
        launch_rows<DT, 16, 2>(a, st);
    else if (a.k > 64)
        launch_rows<DT, 16, 1>(a, st);
    else if (a.k > 32)
        launch_rows<DT, 8, 1>(a, st);
    else                                 // 1,000,000 x 16 in bfloat16: 77 us by 16 lanes, 22 so
        launch_rows<DT, 4, 1>(a, st);
    return hipGetLastError();
}

template <int DT>
hipError_t launch_gradients(const NormGradArgs &a, const Cut &cut, hipStream_t st)
{
    const unsigned blocks = (unsigned)cut.parts;
    switch (cut.lanes * 8 + cut.hold) {
    case 4 * 8 + 1:                      // 1,000,000 x 16 in bfloat16: 129 us by 16 lanes, 37 so
        norm_grad_kernel<DT, 4, 1, 512><<<blocks, 512, 0, st>>>(a);
        return hipGetLastError();
    case 8 * 8 + 1:
        norm_grad_kernel<DT, 8, 1, 512><<<blocks, 512, 0, st>>>(a);
        return hipGetLastError();
    case 16 * 8 + 1:
        norm_grad_kernel<DT, 16, 1, 512><<<blocks, 512, 0, st>>>(a);
        return hipGetLastError();
    case 16 * 8 + 2:
        norm_grad_kernel<DT, 16, 2, 512><<<blocks, 512, 0, st>>>(a);
        return hipGetLastError();
    case 64 * 8 + 1:
        norm_grad_kernel<DT, 64, 1, 512><<<blocks, 512, 0, st>>>(a);
        return hipGetLastError();
    case 64 * 8 + 2:
        norm_grad_kernel<DT, 64, 2, 512><<<blocks, 512, 0, st>>>(a);
        return hipGetLastError();
    case 64 * 8 + 4:
        if constexpr (DT != GPIC_F32)
            norm_grad_kernel<DT, 64, 4, 512><<<blocks, 512, 0, st>>>(a);
        return hipGetLastError();
    case 256 * 8 + 1:
        if constexpr (DT == GPIC_F32)
            norm_grad_kernel<DT, 256, 1, 256><<<blocks, 256, 0, st>>>(a);
        return hipGetLastError();
    case 256 * 8 + 2:
        norm_grad_kernel<DT, 256, 2, 256><<<blocks, 256, 0, st>>>(a);
        return hipGetLastError();
    case 256 * 8 + 4:
        norm_grad_kernel<DT, 256, 4, 256><<<blocks, 256, 0, st>>>(a);
        return hipGetLastError();
    }
    if (a.dots) {
        norm_dots_kernel<DT><<<capped(a.n), 256, 0, st>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
    }
    norm_strip_kernel<DT><<<(unsigned)(cut.parts * a.strips), 256, 0, st>>>(a);
    return hipGetLastError();
}

} // namespace

size_t norm_ws(const Norm &p)
{
    Cursor c{nullptr};
    Backward b(p, c);
    return c.at;
}

hipError_t run_norm(const Norm &p, const void *X, const void *w, const void *b, void *Y,
                    float *stats, hipStream_t st)
{
    if (p.n == 0)
        return hipSuccess;
    const NormArgs a{X, w, b, Y, stats, p.n, p.k, p.ldx, p.ldy, p.eps};
    return p.dtype == GPIC_F32    ? launch_norm<GPIC_F32>(a, st)
           : p.dtype == GPIC_F16 ? launch_norm<GPIC_F16>(a, st)
                                 : launch_norm<GPIC_BF16>(a, st);
}

hipError_t run_norm_backward(const Norm &p, const void *dY, const void *X, const void *w,
                             const float *stats, void *dX, void *dW, void *db, void *ws,
                             hipStream_t st)
{
    Cursor c{static_cast<char *>(ws)};
    const Backward b(p, c);
    const Cut s(p);
    if (p.n > 0 && (dX || dW || db)) {
        const NormGradArgs a{dY, X, w, stats, dX, dX || dW ? b.dots : nullptr,
                             dW || db ? b.sums : nullptr, p.n, p.k,
                             p.ldx, p.ldy, s.strips, s.each};
        const hipError_t e = p.dtype == GPIC_F32    ? launch_gradients<GPIC_F32>(a, s, st)
                             : p.dtype == GPIC_F16 ? launch_gradients<GPIC_F16>(a, s, st)
                                                   : launch_gradients<GPIC_BF16>(a, s, st);
        if (e != hipSuccess)
            return e;
    }
    if (dW || db) {
        norm_join_kernel<<<dim3((unsigned)((p.k + 63) / 64), 2), 1024, 0, st>>>(
            b.sums, s.parts, p.k, dW, db, p.dtype);
        return hipGetLastError();
    }
    return hipSuccess;
}

} // namespace gpic
