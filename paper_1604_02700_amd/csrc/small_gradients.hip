// Gradients of a small layer in one launch, straight from the operands as
// they lie: dX = dZ W, dW = dZ^T X and db = the column sums of dZ, with dZ =
// dY act'(Z) (gated: dH Zu act'(Zg) and dH act(Zg)) formed in registers
// where it is used and never rounded.  Products on the float32 matrix cores
// whatever the type: such calls are bound by launches and latency, not by
// operations.
//
// A workgroup owns 16 rows of dX (or of dW, and then their entries of db) by
// 64 columns; its waves share the contraction in turns of 16 values, and
// their sums meet in LDS and are added in wave order.  A turn takes about 0.15
// us of a compute unit, most of it forming dZ; 52 x 512 -> 123 (3.3 million
// products) takes 4.5 us in float32, 200 x 300 -> 700 (42 million) 10.2.
#include "encoder.h"

namespace gpic {

namespace {

constexpr int kTiles = 4;

struct SmallGrad {
    const void *dY, *X, *W, *Z;
    void *dX, *dW, *db;
    int64_t ldy, ldx, ldw, ldz;
    int n, k, m;
    int act;
    int rows_x;        // workgroups down dX (0: not wanted)
};

__device__ __forceinline__ f32x4 mma_f32(f32x4 w, f32x4 x, f32x4 c)
{
    // lane group g holds four values of the contraction; the j-th
    // instruction takes the j-th of each
#pragma unroll
    for (int j = 0; j < 4; ++j)
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(w[j], x[j], c, 0, 0, 0);
    return c;
}

// values at a 32-bit offset (in values)
template <int DT>
__device__ __forceinline__ float load_at(const void *p, uint32_t i)
{
    return load1(static_cast<const char *>(p) + (size_t)(uint32_t)(i * (DT == GPIC_F32 ? 4 : 2)), 0,
                 DT);
}

template <int DT>
__device__ __forceinline__ f32x4 load4_at(const void *p, uint32_t i)
{
    return load4(static_cast<const char *>(p) + (size_t)(uint32_t)(i * (DT == GPIC_F32 ? 4 : 2)), 0,
                 DT);
}

// What a turn reads: four entries of dY and Z each, four by kTiles of the
// other operand.
struct Turn {
    f32x4 dy, z, u, w[kTiles];
};

// act'(z) (da) and act(z) of four values
template <int ACT>
__device__ __forceinline__ void gradients4(f32x4 z, f32x4 &act, f32x4 &da)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float f, d;
        activate_grad(z[i], ACT, f, d);
        act[i] = f;
        da[i] = d;
    }
}

template <int DT, bool GATED, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void small_gradients_kernel(SmallGrad a)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, l = lane & 15;
    constexpr int kHalves = GATED ? 2 : 1;
    const bool of_x = (int)blockIdx.y < a.rows_x;
    const int col0 = (int)blockIdx.x * (16 * kTiles);
    // dX: rows r; dW: rows j of one half, tiles of each half of their own
    const int tiles_m = (a.m + 15) / 16;
    const int tile = of_x ? (int)blockIdx.y : (int)blockIdx.y - a.rows_x;
    const int half0 = of_x ? 0 : tile / tiles_m;
    const int row0 = (of_x ? tile : tile % tiles_m) * 16;
    const bool sums = !of_x && a.db && blockIdx.x == 0;
    const bool products = of_x || a.dW;
    const int turns = of_x ? kHalves * tiles_m : (a.n + 15) / 16;
    const int count = of_x ? a.m : a.n;                  // of the contraction (of one half)
    const void *other = of_x ? a.W : a.X;
    const int64_t ld = of_x ? a.ldw : a.ldx;

    // The lane's entries of a turn: (r, j) of dY and Z, moving along the
    // contraction; entries that do not exist are read as ones that do and
    // taken as zero.  Offsets fit 32 bits (small_gradients).
    auto half_of = [&](int turn) { return of_x && GATED && turn >= tiles_m ? 1 : 0; };
    auto start_of = [&](int turn) { return (turn - half_of(turn) * tiles_m) * 16 + g * 4; };
    const bool row_live = row0 + l < (of_x ? a.n : a.m);
    const uint32_t row = (uint32_t)(row_live ? row0 + l : 0);
    uint32_t col[kTiles];
#pragma unroll
    for (int q = 0; q < kTiles; ++q)
        col[q] = (uint32_t)(col0 + q * 16 + l < a.k ? col0 + q * 16 + l : 0);
    auto load = [&](int turn) {
        Turn t;
        const int c0 = start_of(turn);
        const uint32_t base = half_of(turn) ? (uint32_t)a.m : 0u;
        const bool in4 = c0 + 4 <= count;
        t.z = t.u = 0.0f;
        if (of_x && in4) {
            // a row's four values at once
            t.dy = load4_at<DT>(a.dY, row * (uint32_t)a.ldy + c0);
            if (GATED) {
                t.z = load4_at<GPIC_F32>(a.Z, row * (uint32_t)a.ldz + c0);
                t.u = load4_at<GPIC_F32>(a.Z, row * (uint32_t)a.ldz + a.m + c0);
            } else if (a.act != GPIC_ACT_NONE) {
                t.z = load4_at<DT>(a.Z, row * (uint32_t)a.ldz + c0);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t c = (uint32_t)(c0 + i < count ? c0 + i : 0);
                const uint32_t r = of_x ? row : c, at = of_x ? c : row;
                t.dy[i] = load_at<DT>(a.dY, r * (uint32_t)a.ldy + at);
                if (GATED) {
                    t.z[i] = load_at<GPIC_F32>(a.Z, r * (uint32_t)a.ldz + at);
                    t.u[i] = load_at<GPIC_F32>(a.Z, r * (uint32_t)a.ldz + a.m + at);
                } else if (a.act != GPIC_ACT_NONE) {
                    t.z[i] = load_at<DT>(a.Z, r * (uint32_t)a.ldz + at);
                }
            }
        }
        if (products) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t at = ((c0 + i < count ? c0 + i : 0) + base) * (uint32_t)ld;
#pragma unroll
                for (int q = 0; q < kTiles; ++q)
                    t.w[q][i] = load_at<DT>(other, at + col[q]);
            }
        }
        return t;
    };

    f32x4 acc[kTiles + 1];
#pragma unroll
    for (int q = 0; q <= kTiles; ++q)
        acc[q] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    Turn next;
    if (wave < turns)
        next = load(wave);
    for (int turn = wave; turn < turns; turn += WAVES) {
        const Turn t = next;
        if (turn + WAVES < turns)
            next = load(turn + WAVES);
        f32x4 act = t.z, da = 1.0f;
        if (a.act == GPIC_ACT_RELU)
            gradients4<GPIC_ACT_RELU>(t.z, act, da);
        else if (a.act == GPIC_ACT_GELU)
            gradients4<GPIC_ACT_GELU>(t.z, act, da);
        else if (a.act == GPIC_ACT_SILU)
            gradients4<GPIC_ACT_SILU>(t.z, act, da);
        f32x4 dz = t.dy * da;
        if (GATED)
            dz = half0 || half_of(turn) ? t.dy * act : t.dy * t.u * da;
        const int c0 = start_of(turn);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            dz[i] = row_live && c0 + i < count ? dz[i] : 0.0f;
        if (products) {
#pragma unroll
            for (int q = 0; q < kTiles; ++q) {
                f32x4 w;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    w[i] = c0 + i < count ? t.w[q][i] : 0.0f;
                acc[q] = mma_f32(w, dz, acc[q]);
            }
        }
        if (sums)
            acc[kTiles] = mma_f32(f32x4{1.0f, 1.0f, 1.0f, 1.0f}, dz, acc[kTiles]);
    }
    __shared__ f32x4 part[WAVES][kTiles + 1][64];
#pragma unroll
    for (int q = 0; q <= kTiles; ++q)
        part[wave][q][lane] = acc[q];
    __syncthreads();
    // wave t finishes tile t, the next one the sums: a lane has one row and
    // four columns of it
    if (wave > kTiles)
        return;
    f32x4 v = part[0][wave][lane];
#pragma unroll
    for (int s = 1; s < WAVES; ++s)
        v += part[s][wave][lane];
    if (!row_live)
        return;
    if (wave == kTiles) {
        if (sums && g == 0)
            store1(a.db, row, v[0], DT);
        return;
    }
    if (!products)
        return;
    void *out = of_x ? a.dX : a.dW;
    const int64_t at = ((int64_t)row + (half0 ? a.m : 0)) * a.k;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c = col0 + wave * 16 + g * 4 + i;
        if (c < a.k)
            store1(out, at + c, v[i], DT);
    }
}

template <int DT>
hipError_t launch(const SmallGrad &a, bool gated, bool wide, dim3 grid, hipStream_t st)
{
    if (gated && wide)
        small_gradients_kernel<DT, true, 16><<<grid, 1024, 0, st>>>(a);
    else if (gated)
        small_gradients_kernel<DT, true, 8><<<grid, 512, 0, st>>>(a);
    else if (wide)
        small_gradients_kernel<DT, false, 16><<<grid, 1024, 0, st>>>(a);
    else
        small_gradients_kernel<DT, false, 8><<<grid, 512, 0, st>>>(a);
    return hipGetLastError();
}

int64_t rows_of(const Shape &s, bool gated) { return gated ? 2 * s.m : s.m; }

} // namespace

// Where this beats the tiled products' six to eight launches: short
// contractions (a workgroup goes through all of one) and little work.  us, here
// and tiled, gelu and gated silu: float32 52 x 512 -> 123 4.5 and 26.5, 200 x 300
// -> 700 10.3 and 36, gated 18 and 40, 1,003 x 300 -> 700 33 and 51, gated 54 and
// 52, 100 x 1,000 -> 2 x 1,000 40 and 46, 16 x 2,048 -> 2,048 43 and 46; bfloat16 52 x 512 ->
// 123 5.0 and 13.9, 200 x 300 -> 700 11 and 22, 100 x 1,000 -> 1,000 22 and 21,
// 1,003 x 300 -> 700 33 and 31, 2 x 58 -> 2 x 588 14 and 18, 16 x 2,048 -> 2,048 50 and
// 22 (16 bits: contractions beyond 1,024 for very little work only).
bool small_gradients(const Shape &s, bool gated)
{
    const int64_t rows = rows_of(s, gated), far = (int64_t)1 << 28;
    const int64_t ldz = gated || s.act != GPIC_ACT_NONE ? s.ldz : 0;     // else Z is not read
    if (s.n * s.ldy > far || s.n * s.ldx > far || s.n * ldz > far || rows * s.ldw > far)
        return false;
    if (s.n > 2048 || rows > 2048)
        return false;
    const bool f32 = s.dtype == GPIC_F32, longer = s.n > 1024 || rows > 1024;
    return s.n * rows * s.k <= (int64_t)1 << (f32 ? 28 : (longer ? 22 : 26));
}

hipError_t run_small_gradients(const Shape &s, bool gated, const void *dY, const void *X,
                               const void *W, const void *Z, void *dX, void *dW, void *db,
                               hipStream_t st)
{
    SmallGrad a{dY, X, W, Z, dX, dW, db, s.ldy, s.ldx, s.ldw, s.ldz,
                (int)s.n, (int)s.k, (int)s.m, s.act, 0};
    const int64_t across = (s.k + 16 * kTiles - 1) / (16 * kTiles);
    a.rows_x = dX ? (int)((s.n + 15) / 16) : 0;
    const int64_t rows_w = dW || db ? (gated ? 2 : 1) * ((s.m + 15) / 16) : 0;
    const int64_t down = a.rows_x + rows_w;
    if (down == 0)
        return hipSuccess;
    const dim3 grid((unsigned)(dX || dW ? across : 1), (unsigned)down);
    // by the longer contraction, whatever is wanted: a sum's order is the same
    const int64_t turns = (rows_of(s, gated) > s.n ? rows_of(s, gated) : s.n) / 16;
    if (s.dtype == GPIC_F32)
        return launch<GPIC_F32>(a, gated, turns > 8, grid, st);
    return s.dtype == GPIC_F16 ? launch<GPIC_F16>(a, gated, turns > 8, grid, st)
                               : launch<GPIC_BF16>(a, gated, turns > 8, grid, st);
}

} // namespace gpic
