// Orthogonalised updates of small matrices in one launch (the larger ones:
// orthogonalize.hip, same formulas, X, A and P in two parts whatever the type): a workgroup holds its
// matrix in LDS as half-precision parts, X [R x LEN] on the smaller side (a
// tall matrix is transposed on the way in and out), and does every step
// there.  Bound by the LDS round trips between the barriers, 5.3 us a step at 64 x
// 256; a launch per product takes three times as long (12 matrices of 64 x 256 in
// float32, five steps: 35 us, 95 in 17 launches).
//
// A = X X^T: the waves share the 32 x 32 blocks and the contraction; sums
// meet in LDS in float32 (in the place of P).  P = b A + c
// A^2 and then X <- a X + P X column block by column block: a wave's new
// columns depend on the same columns of X alone, so X is updated in place.
#include "encoder.h"

namespace gpic {

namespace {

constexpr int kThreads = 512, kWaves = 8;
constexpr float kStore = 1024.0f;          // as in orthogonalize.hip

struct SmallArgs {
    const void *G;
    float *M;
    void *out;                             // O, or the weights (step)
    int m, n, steps;
    float a, b, c;
    double eps;
    float momentum, decay, step;
    int nesterov;
};

__device__ __forceinline__ f32x4 mma_f16(u32x4 a, u32x4 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a),
                                                  __builtin_bit_cast(half8, b), c, 0, 0, 0);
}

// 16 rows of a row-major matrix of halves, 32 values of k from k0 on
__device__ __forceinline__ u32x4 rows_at(const _Float16 *p, int ld, int row, int k0)
{
    const int lane = threadIdx.x & 63;
    return *reinterpret_cast<const u32x4 *>(p + (row + (lane & 15)) * ld + k0 + (lane >> 4) * 8);
}

// 16 columns of it from col on, 32 rows from k0 on, as rows of k
__device__ __forceinline__ u32x4 columns_at(const _Float16 *p, int ld, int col, int k0)
{
    using lds4 = __attribute__((address_space(3))) s16x4;
    const int lane = threadIdx.x & 63, i = lane & 15;
    const _Float16 *q = p + (k0 + 8 * (lane >> 4) + (i >> 2)) * ld + col + (i & 3) * 4;
    union {
        s16x4 h[2];
        u32x4 v;
    } u;
    u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)q);
    u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(q + 4 * ld));
    return u.v;
}

__device__ __forceinline__ f32x4 halves_at(const _Float16 *p)
{
    return __builtin_convertvector(*reinterpret_cast<const half4 *>(p), f32x4);
}

// the parts of v (scaled already)
__device__ __forceinline__ void put_parts(_Float16 *hi, _Float16 *lo, f32x4 v)
{
    const half4 h = __builtin_convertvector(v, half4);
    *reinterpret_cast<half4 *>(hi) = h;
    *reinterpret_cast<half4 *>(lo) =
        __builtin_convertvector(v - __builtin_convertvector(h, f32x4), half4);
}

template <int DT, bool STEP, int R, int LEN>
__global__ __launch_bounds__(kThreads) void polar_small_kernel(SmallArgs a)
{
    constexpr int kLd = LEN + 8, kLdr = R + 8, kTiles = (R / 16) * (R / 16);
    constexpr int kShare = R == 64 ? 2 : 4;      // waves per 32 x 32 block of A
    constexpr int kSumBytes = (kShare - 1) * R * R * 4, kPolyBytes = 2 * R * kLdr * 2;
    __shared__ __attribute__((aligned(16))) _Float16 xh[R * kLd], xl[R * kLd];
    __shared__ __attribute__((aligned(16))) _Float16 ah[R * kLdr], al[R * kLdr];
    __shared__ __attribute__((aligned(16))) char both[kSumBytes > kPolyBytes ? kSumBytes : kPolyBytes];
    __shared__ double norm[kWaves];
    float *sums = reinterpret_cast<float *>(both);
    _Float16 *ph = reinterpret_cast<_Float16 *>(both), *pl = ph + R * kLdr;

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const bool tall = a.m > a.n;
    const int r = tall ? a.n : a.m, len = tall ? a.m : a.n, size = a.m * a.n;
    const int64_t z0 = (int64_t)blockIdx.x * size;
    const int lenp = (len + 31) & ~31;

    // U, held in registers (all loads in flight at once), and its norm
    constexpr int kQuads = R * LEN / (4 * kThreads);
    f32x4 u[kQuads];
#pragma unroll
    for (int q = 0; q < kQuads; ++q) {
        const int i = (q * kThreads + (int)threadIdx.x) * 4;
        u[q] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        if (i + 4 <= size) {
            u[q] = load4(a.G, z0 + i, DT);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (i + j < size)
                    u[q][j] = load1(a.G, z0 + i + j, DT);
        }
    }
    double t = 0.0;
#pragma unroll
    for (int q = 0; q < kQuads; ++q) {
        const int i = (q * kThreads + (int)threadIdx.x) * 4;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (STEP && i + j < size) {
                const float mo = a.M[z0 + i + j] * a.momentum + u[q][j];
                a.M[z0 + i + j] = mo;
                u[q][j] = a.nesterov ? u[q][j] + a.momentum * mo : mo;
            }
            t += (double)u[q][j] * (double)u[q][j];
        }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
        t += __shfl_xor(t, o, 64);
    if (lane == 0)
        norm[wave] = t;
    // zeros where the padding of rows and columns is read
    const u32x4 zero = {0, 0, 0, 0};
    for (int i = threadIdx.x; i < R * (lenp / 8); i += kThreads) {
        const int row = i / (lenp / 8), c = i % (lenp / 8) * 8;
        *reinterpret_cast<u32x4 *>(xh + row * kLd + c) = zero;
        *reinterpret_cast<u32x4 *>(xl + row * kLd + c) = zero;
    }
    __syncthreads();
    t = norm[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w)
        t += norm[w];
    const Wide inv((double)kStore / (sqrt(t) + a.eps));
#pragma unroll
    for (int q = 0; q < kQuads; ++q) {
        const int i = (q * kThreads + (int)threadIdx.x) * 4;
        int i0 = i / a.n, i1 = i - i0 * a.n;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            u[q][j] = inv.times(u[q][j]);
        // four of one row, on their place
        const bool four = !tall && i + 4 <= size && (a.n & 3) == 0;
        if (four)
            put_parts(xh + i0 * kLd + i1, xl + i0 * kLd + i1, u[q]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (i + j < size && !four) {
                const int at = tall ? i1 * kLd + i0 : i0 * kLd + i1;
                const float v = u[q][j];
                const _Float16 h = (_Float16)v;
                xh[at] = h;
                xl[at] = (_Float16)(v - (float)h);
            }
            if (++i1 == a.n) {
                i1 = 0;
                ++i0;
            }
        }
    }
    __syncthreads();

    const float inv2 = 1.0f / (kStore * kStore);
    const int m16 = lane & 15, n4 = (lane >> 4) * 4;       // place in a 16 x 16 result
    for (int k = 0; k < a.steps; ++k) {
        // A = X X^T
        {
            // (R = 32: four waves have no part)
            const int block = wave / kShare, part = wave % kShare;
            const bool mine = block < R / 32 * (R / 32);
            const int ti = block / (R / 32) * 32, tj = block % (R / 32) * 32;
            f32x4 acc[2][2], low[2][2];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                acc[e >> 1][e & 1] = low[e >> 1][e & 1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 2
            for (int c = mine ? part * 32 : lenp; c < lenp; c += 32 * kShare) {
                u32x4 hi[2], hj[2], li[2], lj[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    hi[e] = rows_at(xh, kLd, ti + 16 * e, c);
                    hj[e] = rows_at(xh, kLd, tj + 16 * e, c);
                    li[e] = rows_at(xl, kLd, ti + 16 * e, c);
                    lj[e] = rows_at(xl, kLd, tj + 16 * e, c);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int x = e >> 1, y = e & 1;
                    acc[x][y] = mma_f16(hj[y], hi[x], acc[x][y]);
                    low[x][y] = mma_f16(lj[y], hi[x], low[x][y]);
                    low[x][y] = mma_f16(hj[y], li[x], low[x][y]);
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int x = e >> 1, y = e & 1;
                acc[x][y] += low[x][y];
                if (part > 0 && mine)
                    *reinterpret_cast<f32x4 *>(sums + ((part - 1) * R + ti + 16 * x + m16) * R + tj +
                                               16 * y + n4) = acc[x][y];
            }
            __syncthreads();
            if (part == 0 && mine) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int x = e >> 1, y = e & 1;
                    const int row = ti + 16 * x + m16, col = tj + 16 * y + n4;
#pragma unroll
                    for (int w = 0; w < kShare - 1; ++w)
                        acc[x][y] += *reinterpret_cast<const f32x4 *>(sums + (w * R + row) * R + col);
                    const int at = row * kLdr + col;
                    put_parts(ah + at, al + at, acc[x][y] * (inv2 * kStore));
                }
            }
            __syncthreads();
        }
        // P = b A + c A^2
        for (int tile = wave; tile < kTiles; tile += kWaves) {
            const int ti = tile / (R / 16) * 16, tj = tile % (R / 16) * 16;
            f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int c = 0; c < R; c += 32) {
                const u32x4 bj = rows_at(ah, kLdr, tj, c), bi = rows_at(ah, kLdr, ti, c);
                acc = mma_f16(bj, bi, acc);
                acc = mma_f16(rows_at(al, kLdr, tj, c), bi, acc);
                acc = mma_f16(bj, rows_at(al, kLdr, ti, c), acc);
            }
            const int at = (ti + m16) * kLdr + tj + n4;
            const f32x4 v = halves_at(ah + at) + halves_at(al + at);
            put_parts(ph + at, pl + at, a.b * v + acc * (a.c * inv2 * kStore));
        }
        __syncthreads();
        // X <- a X + P X
        const bool last = k + 1 == a.steps;
        for (int col = wave * 16; col < lenp; col += kWaves * 16) {
            u32x4 bh[R / 32], bl[R / 32];
#pragma unroll
            for (int c = 0; c < R / 32; ++c) {
                bh[c] = columns_at(xh, kLd, col, 32 * c);
                bl[c] = columns_at(xl, kLd, col, 32 * c);
            }
            f32x4 v[R / 16];
#pragma unroll
            for (int i = 0; i < R / 16; ++i) {
                f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int c = 0; c < R / 32; ++c) {
                    const u32x4 p = rows_at(ph, kLdr, 16 * i, 32 * c);
                    acc = mma_f16(bh[c], p, acc);
                    acc = mma_f16(bl[c], p, acc);
                    acc = mma_f16(bh[c], rows_at(pl, kLdr, 16 * i, 32 * c), acc);
                }
                const int at = (16 * i + m16) * kLd + col + n4;
                v[i] = a.a * (halves_at(xh + at) + halves_at(xl + at)) + acc * (inv2 * kStore);
            }
#pragma unroll
            for (int i = 0; i < R / 16; ++i) {
                const int row = 16 * i + m16, at = row * kLd + col + n4;
                if (!last) {
                    put_parts(xh + at, xl + at, v[i]);
                    continue;
                }
                if (row >= r)
                    continue;
                if (DT == GPIC_F32 && !STEP && !tall && col + n4 + 4 <= len) {
                    using any = f32x4 __attribute__((aligned(4)));
                    *reinterpret_cast<any *>(static_cast<float *>(a.out) + z0 +
                                             (int64_t)row * a.n + col + n4) = v[i] * (1.0f / kStore);
                    continue;
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int c = col + n4 + j;
                    if (c >= len)
                        continue;
                    const int64_t o = z0 + (tall ? (int64_t)c * a.n + row : (int64_t)row * a.n + c);
                    float x = v[i][j] * (1.0f / kStore);
                    if (STEP)
                        x = a.decay * load1(a.out, o, DT) - a.step * x;
                    store1(a.out, o, x, DT);
                }
            }
        }
        __syncthreads();
    }
}

template <int DT, bool STEP>
hipError_t launch_small(const SmallArgs &a, int64_t batch, hipStream_t st)
{
    const int r = a.m < a.n ? a.m : a.n, len = a.m < a.n ? a.n : a.m;
    const unsigned grid = (unsigned)batch;
    if (r <= 32 && len <= 256)
        polar_small_kernel<DT, STEP, 32, 256><<<grid, kThreads, 0, st>>>(a);
    else if (r <= 32)
        polar_small_kernel<DT, STEP, 32, 1024><<<grid, kThreads, 0, st>>>(a);
    else
        polar_small_kernel<DT, STEP, 64, 448><<<grid, kThreads, 0, st>>>(a);
    return hipGetLastError();
}

} // namespace

// What fits the 160 KiB of LDS.
bool polar_small(const Polar &p)
{
    const int64_t r = p.m < p.n ? p.m : p.n, len = p.m < p.n ? p.n : p.m;
    return (r <= 32 && len <= 1024) || (r <= 64 && len <= 448);
}

hipError_t run_polar_small(const Polar &p, const MuonStep *h, void *out, const void *G, float *M,
                           hipStream_t st)
{
    SmallArgs a{};
    a.G = G;
    a.M = M;
    a.out = out;
    a.m = (int)p.m;
    a.n = (int)p.n;
    a.steps = p.steps;
    a.a = p.a;
    a.b = p.b;
    a.c = p.c;
    a.eps = p.eps;
    if (h) {
        a.momentum = h->momentum;
        a.nesterov = h->nesterov;
        a.decay = 1.0f - h->lr * h->decay;
        a.step = h->lr * h->scale;
    }
    if (p.dtype == GPIC_F32)
        return h ? launch_small<GPIC_F32, true>(a, p.batch, st)
                 : launch_small<GPIC_F32, false>(a, p.batch, st);
    if (p.dtype == GPIC_F16)
        return h ? launch_small<GPIC_F16, true>(a, p.batch, st)
                 : launch_small<GPIC_F16, false>(a, p.batch, st);
    return h ? launch_small<GPIC_BF16, true>(a, p.batch, st)
             : launch_small<GPIC_BF16, false>(a, p.batch, st);
}

} // namespace gpic
