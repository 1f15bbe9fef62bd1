// Cross entropy over a vocabulary whose logits are never kept: z = X W^T + b,
//   loss_i = log sum_v exp z_iv - z_i,t(i),
//   dZ = g_i (exp(z - lse_i) - [v = t(i)]), dX = dZ W, dW = dZ^T X, db = column sums.
//
// Forward, a tile of logits leaves only each row's largest and sum of
// exponentials (product.h, kEpiLse), the target's logit set aside: from the
// others' lse' = log sum_{v != t} exp z_v the loss is softplus(lse' - z_t),
// which keeps its digits where the target's probability is near one, and the
// gradient of the target's logit is g (exp(-loss) - 1).  Backward, the
// vocabulary goes by in pieces: the piece's logits once more, their gradients
// into one buffer (product.h, kEpiSoft), from there into the sum dX and into
// the piece's rows of dW.
//
// Few rows, or little work, read W once as it lies (few_lse_kernel).
//
// What is rounded to the products' operands is D = exp(z - lse) - [target], at
// most 1, without g: dX_i = g_i sum_v D_iv W_v, and dW_v = G sum_i D_iv (g_i / G x_i)
// with the largest |g| G, so that the usual g, one for all rows, costs nothing;
// float16's (g_i / G) x_i are under a power of two (share_max_kernel).  float32 operands
// are split halves (encoder.h).
#include <type_traits>

#include "row_chunks.h"
#include "training.h"

namespace gpic {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float2 merge(float2 a, float2 b)
{
    const float m = fmaxf(a.x, b.x), at = m == -INFINITY ? 0.0f : m;
    return make_float2(m, a.y * __builtin_amdgcn_exp2f((a.x - at) * kLog2e) +
                              b.y * __builtin_amdgcn_exp2f((b.x - at) * kLog2e));
}

__device__ __forceinline__ int64_t target_at(const void *t, int wide, int64_t row)
{
    return wide ? static_cast<const int64_t *>(t)[row]
                : (int64_t)static_cast<const int32_t *>(t)[row];
}

// ------------------------------------------------------------- few rows
struct FewArgs {
    const void *X, *W, *bias, *targets;
    float2 *strip;             // [blocks of 16 columns][n]
    double *picked;
    int64_t ldx, ldw, n, k, v;
    int wide;
};

// The products of CB blocks of 16 columns and up to 16 NB rows a workgroup, whose
// waves share the contraction in turns; wave w < NB CB ends (true) with rows
// 16 (w mod NB) on and block w / NB, a lane with four columns, from `col` on, of
// `row`.  Bound by reading W: one bfloat16 row, 4,096 -> 65,000, 109 us with the
// join, 4.9 TB/s.  (Workgroups that stay and read a block ahead spilled at 16 waves:
// 45 us where one row of 2,048 -> 32,000 took 38, which two blocks a workgroup now take 34 for.)
template <int DT, int NB, int CB, int WAVES>
__device__ __forceinline__ bool few_logits(const FewArgs &a, double (&v)[4], int64_t &row,
                                           int64_t &col)
{
    constexpr int kValues = DT == GPIC_F32 ? 4 : 8;       // of k a lane loads at once
    constexpr int kSize = DT == GPIC_F32 ? 4 : 2;
    constexpr int kUnroll = 4, kTurn = 4 * kValues * kUnroll;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, r = lane & 15;
    const int64_t col0 = (int64_t)blockIdx.x * (16 * CB), row0 = (int64_t)blockIdx.y * (16 * NB);
    // rows and columns beyond the last are read as the last ones and not kept
    const char *w[CB], *x[NB];
#pragma unroll
    for (int c = 0; c < CB; ++c) {
        const int64_t at = col0 + c * 16 + r < a.v ? col0 + c * 16 + r : a.v - 1;
        w[c] = static_cast<const char *>(a.W) + at * a.ldw * kSize;
    }
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        const int64_t at = row0 + b * 16 + r < a.n ? row0 + b * 16 + r : a.n - 1;
        x[b] = static_cast<const char *>(a.X) + at * a.ldx * kSize;
    }
    f32x4 acc[CB][NB];
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int b = 0; b < NB; ++b)
            acc[c][b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    auto turn = [&](int64_t k0, auto last) {
        constexpr bool kLast = decltype(last)::value;
        u32x4 fw[CB][kUnroll], fx[NB][kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int64_t k = k0 + u * 4 * kValues + g * kValues;
#pragma unroll
            for (int c = 0; c < CB; ++c)
                fw[c][u] = chunk_at<DT, kLast>(w[c], k, a.k);
#pragma unroll
            for (int b = 0; b < NB; ++b)
                fx[b][u] = chunk_at<DT, kLast>(x[b], k, a.k);
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
#pragma unroll
            for (int c = 0; c < CB; ++c)
#pragma unroll
                for (int b = 0; b < NB; ++b)
                    acc[c][b] = mma16<DT>(fw[c][u], fx[b][u], acc[c][b]);
    };
    int64_t k0 = (int64_t)wave * kTurn;
#pragma unroll 2
    for (; k0 + kTurn <= a.k; k0 += (int64_t)WAVES * kTurn)
        turn(k0, std::false_type{});
    if (k0 < a.k)                      // the turn that the contraction ends in
        turn(k0, std::true_type{});
    __shared__ f32x4 part[WAVES][CB * NB][64];
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int b = 0; b < NB; ++b)
            part[wave][c * NB + b][lane] = acc[c][b];
    __syncthreads();
    if (wave >= NB * CB)
        return false;
    row = row0 + wave % NB * 16 + r;
    col = col0 + wave / NB * 16 + g * 4;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        v[j] = 0.0;
#pragma unroll
    for (int s = 0; s < WAVES; ++s)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            v[j] += (double)part[s][wave][lane][j];
    return true;
}

// Each row's largest and sum of exponentials over 16 columns.  The waves' sums of
// a logit meet in float64, and so do the target's and the others' later: a loss
// is the small difference of both, a float32 of 18 is 10^-6 off.
template <int DT, int NB, int CB, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void few_lse_kernel(FewArgs a)
{
    double v[4];
    int64_t row, col0;
    if (!few_logits<DT, NB, CB, WAVES>(a, v, row, col0))
        return;
    const bool live = row < a.n;
    const int64_t t = live ? target_at(a.targets, a.wide, row) : -1;
    float m = -INFINITY, s = 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int64_t col = col0 + j;
        double z = -INFINITY;
        if (col < a.v) {
            const float bias = a.bias ? load1(a.bias, col, DT) : 0.0f;
            z = bias == -INFINITY ? (double)bias : v[j] + (double)bias;
            if (col == t) {
                a.picked[row] = z;
                z = -INFINITY;
            }
        }
        v[j] = z;
        m = fmaxf(m, (float)z);
    }
    m = fmaxf(m, __shfl_xor(m, 16, 64));
    m = fmaxf(m, __shfl_xor(m, 32, 64));
    const double at = m == -INFINITY ? 0.0 : (double)m;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        s += __builtin_amdgcn_exp2f((float)(v[j] - at) * kLog2e);
    s += __shfl_xor(s, 16, 64);
    s += __shfl_xor(s, 32, 64);
    // (the last workgroup's second block may lie beyond the last column)
    if (live && (threadIdx.x & 63) < 16 && col0 < a.v)
        a.strip[(col0 >> 4) * a.n + row] = make_float2(m, s);
}

// lse as at + off.  Where it is so large that a float32 loses its digits (rows
// masked by their type's lowest value everywhere: lse is that value plus log v),
// at is the target's logit and off the loss.
__device__ __forceinline__ void place_lse(float lse, float loss, float &at, float &off)
{
    const bool far = fabsf(lse) > 131072.0f && fabsf(lse) < INFINITY && loss < INFINITY;
    at = far ? lse - loss : lse;
    off = far ? loss : 0.0f;
}

// The same logits to D = g (exp(z - lse) - [target]) in float32, for the gradients
// of a small layer (small_gradients.hip), and a copy of X whose rows without a
// gradient are zeros.
struct SmallArgs {
    FewArgs f;
    const float *dloss, *loss, *lse;
    float *D, *X;              // [n][v], [n][k]
};

template <int DT, int NB, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void small_soft_kernel(SmallArgs s)
{
    const FewArgs &a = s.f;
    double v[4];
    int64_t row, col0;
    {
        // (fewer than 2^31 values: small())
        const uint32_t total = (uint32_t)(a.n * a.k), k = (uint32_t)a.k;
        const uint32_t groups = gridDim.x * gridDim.y, each = (total + groups - 1) / groups;
        const int64_t i0 = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * each;
        const int64_t i1 = i0 + each < total ? i0 + each : total;
#pragma unroll 2
        for (int64_t i = i0 + threadIdx.x; i < i1; i += 64 * WAVES) {
            const int64_t r = (uint32_t)i / k, t = target_at(a.targets, a.wide, r);
            const bool live = t >= 0 && t < a.v && s.dloss[r] != 0.0f;
            s.X[i] = live ? load1(a.X, r * a.ldx + (i - r * a.k), DT) : 0.0f;
        }
    }
    if ((int64_t)blockIdx.y * (16 * NB) >= a.n)      // here for the copy alone
        return;
    if (!few_logits<DT, NB, 1, WAVES>(a, v, row, col0) || row >= a.n)
        return;
    const int64_t t = target_at(a.targets, a.wide, row);
    const float gl = s.dloss[row];
    const bool live = t >= 0 && t < a.v && gl != 0.0f;
    const float loss = s.loss[row];
    float at, off;
    place_lse(s.lse[row], loss, at, off);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int64_t col = col0 + j;
        if (col >= a.v)
            break;
        const float bias = a.bias ? load1(a.bias, col, DT) : 0.0f;
        float d = col == t ? expm1f(-loss)
                           : __builtin_amdgcn_exp2f((float)(v[j] + bias - at - off) * kLog2e);
        d = bias == -INFINITY && col != t ? 0.0f : d;
        s.D[row * a.v + col] = live ? d * gl : 0.0f;
    }
}

// ------------------------------------------------------------------ join
struct JoinArgs {
    const float2 *strip;       // [strips][n]
    const double *picked;
    const void *targets;
    float *loss, *lse;
    int64_t n, strips, v;
    int wide;
};

// The loss of ROWS rows a workgroup from their strips.
template <int ROWS>
__global__ __launch_bounds__(256) void join_kernel(JoinArgs a)
{
    constexpr int kLanes = 256 / ROWS;
    const int r = threadIdx.x % ROWS, l = threadIdx.x / ROWS;
    const int64_t row = (int64_t)blockIdx.x * ROWS + r;
    float2 v = make_float2(-INFINITY, 0.0f);
    if (row < a.n) {
#pragma unroll 8
        for (int64_t s = l; s < a.strips; s += kLanes)
            v = merge(v, a.strip[s * a.n + row]);
    }
#pragma unroll
    for (int o = ROWS; o < 64; o <<= 1)
        v = merge(v, make_float2(__shfl_xor(v.x, o, 64), __shfl_xor(v.y, o, 64)));
    __shared__ float2 all[4][ROWS];
    if ((threadIdx.x & 63) < ROWS)
        all[threadIdx.x >> 6][threadIdx.x & 63] = v;
    __syncthreads();
    if (l > 0 || row >= a.n)
        return;
#pragma unroll
    for (int w = 1; w < 4; ++w)
        v = merge(v, all[w][r]);
    // (no other entry: -inf)
    const double others = (double)v.x + (double)logf(v.y);
    const int64_t t = target_at(a.targets, a.wide, row);
    double loss = 0.0, lse = others;
    if (t >= 0 && t < a.v) {
        // (the logits' difference first: log s may vanish beside a masked row's)
        const double z = a.picked[row], d = ((double)v.x - z) + (double)logf(v.y);
        // softplus(d), the larger of both logits apart; an infinite or NaN
        // logit makes it NaN, a target without probability infinite
        const double tail = (double)log1pf(expf(-fabsf((float)d)));
        loss = z == INFINITY ? NAN : (d > 0.0 ? d + tail : tail);
        lse = z == -INFINITY ? others : fmax(others, z) + tail;
        if (d != d)
            loss = lse = NAN;
    }
    a.loss[row] = (float)loss;
    if (a.lse)
        a.lse[row] = (float)lse;
}

// -------------------------------------------------------------- backward
struct RowsArgs {
    const float *dloss, *loss, *lse;
    const void *targets;
    int wide;
    int64_t n, v;
    LossRow *rows;
    float *most;               // of each workgroup's finite |g|
};

// A row's LossRow; its finite |g|
__device__ __forceinline__ float row_of(const RowsArgs &a, int64_t i, LossRow &r)
{
    const int64_t t = target_at(a.targets, a.wide, i);
    const float g = a.dloss[i];
    r = LossRow{0.0f, 0.0f, 0.0f, 0.0f, -1, {0, 0, 0}};
    if (t >= 0 && t < a.v && g != 0.0f) {
        float at, off;
        place_lse(a.lse[i], a.loss[i], at, off);
        r = LossRow{at, off, g, expm1f(-a.loss[i]), (int)t, {0, 0, 0}};
    }
    return fabsf(r.g) < INFINITY ? fabsf(r.g) : 0.0f;
}

__device__ __forceinline__ float wave_max(float x)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
        x = fmaxf(x, __shfl_xor(x, o, 64));
    return x;
}

__global__ __launch_bounds__(256) void rows_kernel(RowsArgs a)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    float size = 0.0f;
    if (i < a.n) {
        LossRow r;
        size = row_of(a, i, r);
        a.rows[i] = r;
    }
    __shared__ float w[4];
    size = wave_max(size);
    if ((threadIdx.x & 63) == 0)
        w[threadIdx.x >> 6] = size;
    __syncthreads();
    if (threadIdx.x == 0)
        a.most[blockIdx.x] = fmaxf(fmaxf(w[0], w[1]), fmaxf(w[2], w[3]));
}

// G, the largest |g|, and each row's g / G; up to kRowsAtOnce rows' LossRow too, by
// one workgroup.  Else `most` holds `count` workgroups' largest, which each of up
// to 128 goes through (1,000,000 rows: one workgroup 447 us, now 8).
constexpr int64_t kRowsAtOnce = 4096;

__global__ __launch_bounds__(1024) void shares_kernel(RowsArgs a, int64_t count, float *largest,
                                                      float *share)
{
    const bool here = a.n <= kRowsAtOnce;
    float best = 0.0f;
    if (here) {
#pragma unroll 2
        for (int64_t i = threadIdx.x; i < a.n; i += 1024) {
            LossRow r;
            best = fmaxf(best, row_of(a, i, r));
            a.rows[i] = r;
        }
    } else {
        for (int64_t i = threadIdx.x; i < count; i += 1024)
            best = fmaxf(best, a.most[i]);
    }
    __shared__ float w[16];
    best = wave_max(best);
    if ((threadIdx.x & 63) == 0)
        w[threadIdx.x >> 6] = best;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 16; ++i)
        best = fmaxf(best, w[i]);
    best = best > 0.0f ? best : 1.0f;
    if (threadIdx.x == 0 && blockIdx.x == 0)
        *largest = best;
    // (one workgroup: each thread reads the rows that it wrote)
#pragma unroll 4
    for (int64_t i = (int64_t)blockIdx.x * 1024 + threadIdx.x; i < a.n; i += gridDim.x * 1024)
        share[i] = a.rows[i].g / best;
}

// The largest finite |X| times its row's share, a part of every workgroup: halves
// hold shares far below the largest only under a power of two (a row of normal values
// with a share of 2^-20 was off by 1.4e-2, and by no more than its rounding since).
// 5 us of a pass of 107 over 1,003 x 700 -> 10,007, 20 of 4,340 over 8,192 x 2,048 -> 50,000.
// As many lanes a row as it has groups of eight, up to a wave (`lanes`, a power of two).
constexpr int kShareParts = 1024;

__global__ __launch_bounds__(256) void share_max_kernel(const _Float16 *X, const float *share,
                                                        int64_t n, int64_t k, int64_t ldx,
                                                        int lanes, float *part)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int at = threadIdx.x & (lanes - 1), rows = 256 / lanes;
    float best = 0.0f;
#pragma unroll 2
    for (int64_t r = (int64_t)blockIdx.x * rows + threadIdx.x / lanes; r < n;
         r += (int64_t)gridDim.x * rows) {
        const float f = fabsf(share[r]);
#pragma unroll 4
        for (int64_t c = at * 8; c < k; c += lanes * 8) {
            const f32x8 x = load8(X, r * ldx + c, GPIC_F16, k - c < 8 ? (int)(k - c) : 8);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                // (rows without a gradient may hold anything)
                const float v = fabsf(x[j]) * f;
                best = v < INFINITY ? fmaxf(best, v) : best;
            }
        }
    }
    __shared__ float w[4];
    best = wave_max(best);
    if (lane == 0)
        w[wave] = best;
    __syncthreads();
    if (threadIdx.x == 0)
        part[blockIdx.x] = fmaxf(fmaxf(w[0], w[1]), fmaxf(w[2], w[3]));
}

// Partial maxima [parts][cols] of the finite magnitudes of a float32 matrix's
// columns, its rows times a factor each.
struct ColumnArgs {
    const float *x;
    int64_t rows, cols, ld, each, parts;
    const float *row;          // or null
    float *part;
    int *power;
};
struct ColumnJobs {
    ColumnArgs j[2];
};

__global__ __launch_bounds__(256) void column_max_kernel(ColumnJobs jobs)
{
    const ColumnArgs a = jobs.j[blockIdx.z];
    if ((int64_t)blockIdx.y >= a.parts)
        return;
    const int64_t col = ((int64_t)blockIdx.x * 64 + (threadIdx.x & 63)) * 4;
    const int64_t r0 = blockIdx.y * a.each, r1 = r0 + a.each < a.rows ? r0 + a.each : a.rows;
    f32x4 best = 0.0f;
    if (col < a.cols)
#pragma unroll 4
        for (int64_t r = r0 + (threadIdx.x >> 6); r < r1; r += 4) {
            const float f = a.row ? a.row[r] : 1.0f;
            f32x4 x = 0.0f;
            if (col + 4 <= a.cols)
                x = load4(a.x, r * a.ld + col, GPIC_F32);
            else
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (col + j < a.cols)
                        x[j] = a.x[r * a.ld + col + j];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float v = fabsf(x[j] * f);
                best[j] = v < INFINITY ? fmaxf(best[j], v) : best[j];
            }
        }
    __shared__ f32x4 all[4][64];
    all[threadIdx.x >> 6][threadIdx.x & 63] = best;
    __syncthreads();
    if (threadIdx.x >= 64)
        return;
    for (int w = 1; w < 4; ++w)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            best[j] = fmaxf(best[j], all[w][threadIdx.x][j]);
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (col + j < a.cols)
            a.part[blockIdx.y * a.cols + col + j] = best[j];
}

__global__ __launch_bounds__(1024) void column_power_kernel(ColumnJobs jobs)
{
    const ColumnArgs a = jobs.j[blockIdx.y];
    const int lane = threadIdx.x & 63, run = threadIdx.x >> 6;
    const int64_t col = (int64_t)blockIdx.x * 64 + lane;
    float best = 0.0f;
    if (col < a.cols) {
#pragma unroll 8
        for (int64_t p = run; p < a.parts; p += 16)
            best = fmaxf(best, a.part[p * a.cols + col]);
    }
    __shared__ float all[16][64];
    all[run][lane] = best;
    __syncthreads();
    if (run == 0 && col < a.cols) {
        for (int w = 1; w < 16; ++w)
            best = fmaxf(best, all[w][lane]);
        a.power[col] = power_for(best);
    }
}

__global__ __launch_bounds__(256) void zero_kernel(void *p, int64_t values, int dtype)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < values;
         i += (int64_t)gridDim.x * 256)
        store1(p, i, 0.0f, dtype);
}

// ------------------------------------------------------------------- host
#define RUN(expr)                                                              \
    do {                                                                       \
        hipError_t e_ = (expr);                                                \
        if (e_ != hipSuccess)                                                  \
            return e_;                                                         \
    } while (0)

constexpr int kFew = 32;
constexpr int64_t kWideFew = 16384;     // columns that fill the card two blocks at a time

// Few rows (float32's split copies of W cost more for up to 64), or little work,
// where launches count; not many short rows (2,000 x 1 -> 50,000 380 us, 60 tiled).
int64_t few_rows(const Loss &p) { return p.dtype == GPIC_F32 ? kThinRows : kFew; }

bool few(const Loss &p)
{
    const bool f32 = p.dtype == GPIC_F32;
    if (p.n <= few_rows(p))
        return true;
    return p.n <= 2048 && p.n * p.v <= (1 << 23) &&
           p.n * p.v <= ((int64_t)1 << (f32 ? 28 : 27)) / p.k;
}

// The gradients of little work in float32 or of few rows: from D in float32
// (small_gradients.hip, loss_thin.hip).
Shape layer_of(const Loss &p)
{
    Shape s{};
    s.n = p.n;
    s.k = p.k;
    s.m = p.v;
    s.dtype = p.dtype;
    s.act = GPIC_ACT_NONE;
    s.ldx = p.k;
    s.ldw = p.ldw;
    s.ldy = p.v;
    return s;
}

bool little(const Loss &p)
{
    return p.dtype == GPIC_F32 && small_gradients(layer_of(p), false);
}

// 16 bits: up to 8 rows, whose roundings of D do not average out (one row of 39 ->
// 3,840 in float16, dW off by 2.5e-4 in the 2-norm, 1.3e-4 from the result's own), and
// up to 32 over a small W.  us, here and tiled: 1 x 2,048 -> 32,000 109 and 106, 8 rows
// 115 and 107, 32 rows 185 and 108; 32 x 1,000 -> 1,000 24 and 32, 32 x 4,096 -> 100 25 and
// 40, 8 x 65,000 -> 5 64 and 334.
constexpr int kFewSoft = 8;

bool small(const Loss &p)
{
    if (p.n == 0 || little(p))
        return p.n > 0;
    if (p.dtype == GPIC_F32)
        return p.n <= kThinRows;
    return p.n <= kFewSoft || (p.n <= kFew && p.k * p.v <= 1 << 21);
}

int64_t edge_of(const Plan &p) { return p.tile == 0 ? 256 : (p.tile == 1 ? 128 : 64); }

// What a forward call keeps in its workspace.
struct Forward {
    Source X{}, W{};
    int64_t strips;
    float2 *strip;
    double *picked;
    Forward(const Loss &p, const void *x, const void *w, Cursor &c)
    {
        picked = static_cast<double *>(c.take((size_t)p.n * 8));
        if (few(p)) {
            strips = (p.v + 15) / 16;
        } else {
            const Plan plan = product_plan(p.n, p.v, p.k, 1, kind_of(p.dtype), kEpiLse);
            strips = (p.v + edge_of(plan) - 1) / edge_of(plan);
            X = Source{x, p.n, p.k, p.ldx, must_pack(p.dtype, p.k, p.ldx, p.aligned16)};
            W = Source{w, p.v, p.k, p.ldw, must_pack(p.dtype, p.k, p.ldw, p.aligned16)};
            place(X, p.dtype, c, X.rows);
            place(W, p.dtype, c, W.rows);
        }
        strip = static_cast<float2 *>(c.take((size_t)strips * p.n * 8));
    }
};

struct Small {
    float *D, *X, *part;
    Small(const Loss &p, Cursor &c)
    {
        D = static_cast<float *>(c.take((size_t)p.n * p.v * 4));
        X = static_cast<float *>(c.take((size_t)p.n * p.k * 4));
        part = static_cast<float *>(c.take(little(p) ? 0 : thin_ws(p.n, p.k, p.v)));
    }
};

// How the vocabulary is cut: pieces of whole tiles, of which dZ takes up to 512
// MB, of 2,048 columns at least.  Gradients in us with 112, 256, 400, 512 and 1,024
// MB: 8,192 x 2,048 -> 50,000 in bfloat16 4,370, 4,429, 4,244, 4,254 and 4,219 (one
// piece), 8,192 x 512 in float32 4,510, 3,780, 3,614, 3,599 and 3,503.
int64_t piece_of(const Loss &p)
{
    const int64_t size = p.dtype == GPIC_F32 ? 4 : 2, n = p.n < 1 ? 1 : p.n;
    int64_t most = ((int64_t)512 << 20) / (size * n) / 256 * 256;
    most = most < 2048 ? 2048 : most;
    const int64_t pieces = (p.v + most - 1) / most;
    return ((p.v + pieces - 1) / pieces + 255) / 256 * 256;
}

int64_t max_parts(int64_t rows, int64_t cols)
{
    const int64_t strips = (cols + 255) / 256;
    int64_t parts = 1024 / strips;
    parts = parts < (rows + 15) / 16 ? parts : (rows + 15) / 16;
    return parts < 1 ? 1 : (parts > 512 ? 512 : parts);
}

// Lanes that share_max_kernel takes for a row
int share_lanes(int64_t k)
{
    int lanes = 1;
    while (lanes < 64 && lanes * 8 < k)
        lanes *= 2;
    return lanes;
}

// What a backward call keeps in its workspace.
struct Backward {
    int64_t piece, pitch;      // columns of a piece, 16-bit values of a row of dZ
    LossRow *rows;
    float *most, *largest, *share;
    Source X, W;               // as the logits' product reads them (W: a piece)
    Source Xg, Wc{};           // as dW's does, rows times their shares; float32: as dX's
    float *column_part[2] = {nullptr, nullptr};
    float *share_part = nullptr;       // float16: of the largest X times its row's share
    void *dZ;
    float *sum_x, *sum_b;      // dX over the pieces, partial column sums of dZ
    float *part;
    Backward(const Loss &p, const void *x, const void *w, Cursor &c)
    {
        const bool f32 = p.dtype == GPIC_F32;
        piece = piece_of(p);
        const int64_t cols = piece < p.v ? piece : p.v;
        pitch = f32 ? split_ld(up64(cols)) : up64(cols);
        rows = static_cast<LossRow *>(c.take((size_t)p.n * sizeof(LossRow)));
        most = static_cast<float *>(c.take((size_t)((p.n + 255) / 256) * 4));
        largest = static_cast<float *>(c.take(4));
        share = static_cast<float *>(c.take((size_t)p.n * 4));
        X = Source{x, p.n, p.k, p.ldx, must_pack(p.dtype, p.k, p.ldx, p.aligned16)};
        W = Source{w, cols, p.k, p.ldw, must_pack(p.dtype, p.k, p.ldw, p.aligned16)};
        place(X, p.dtype, c, p.n);
        place(W, p.dtype, c, cols);
        Xg = Source{x, p.n, p.k, p.ldx, true};
        Xg.row = share;
        place(Xg, p.dtype, c, p.k);
        if (p.dtype == GPIC_F16) {
            Xg.most = share_part = static_cast<float *>(c.take(kShareParts * 4));
            const int64_t groups = (p.n * share_lanes(p.k) + 255) / 256;
            Xg.count = (int)(groups < kShareParts ? groups : kShareParts);
            Xg.scale = static_cast<int *>(c.take(4));
        }
        if (f32) {
            Wc = Source{w, cols, p.k, p.ldw, true};
            place(Wc, p.dtype, c, p.k);
            for (int i = 0; i < 2; ++i)
                column_part[i] = static_cast<float *>(
                    c.take((size_t)max_parts(i ? p.v : p.n, p.k) * p.k * 4));
        }
        dZ = c.take((size_t)p.n * pitch * 2);
        sum_x = piece < p.v ? static_cast<float *>(c.take((size_t)p.n * p.k * 4)) : nullptr;
        sum_b = static_cast<float *>(c.take((size_t)((p.n + 31) / 32) * cols * 4));
        size_t bytes = 0;
        const int op = kind_of(p.dtype);
        for (int64_t len : {cols, p.v - (p.v - 1) / piece * piece}) {
            const size_t bx = product_plan(p.n, p.k, len, 1, op, kEpiSum).part_bytes;
            const size_t bw = product_plan(len, p.k, p.n, 1, op, kEpiSum).part_bytes;
            bytes = bytes > bx ? bytes : bx;
            bytes = bytes > bw ? bytes : bw;
        }
        part = static_cast<float *>(c.take(bytes));
    }
};

// Turns of a contraction that waves share.
int64_t turns_of(const Loss &p)
{
    const int64_t turn = p.dtype == GPIC_F32 ? 64 : 128;
    return (p.k + turn - 1) / turn;
}

// Fewer workgroups of 32 rows than half the compute units: of 16 rows then
bool thin_grid(const FewArgs &a)
{
    return (a.v + 15) / 16 * ((a.n + 31) / 32) < 128;
}

template <int DT, int NB, int CB>
void launch_waves(const FewArgs &a, int64_t turns, hipStream_t st)
{
    const dim3 blocks((unsigned)((a.v + 16 * CB - 1) / (16 * CB)),
                      (unsigned)((a.n + 16 * NB - 1) / (16 * NB)));
    if (turns <= 4)
        few_lse_kernel<DT, NB, CB, 4><<<blocks, 256, 0, st>>>(a);
    else if (turns <= 8)
        few_lse_kernel<DT, NB, CB, 8><<<blocks, 512, 0, st>>>(a);
    else
        few_lse_kernel<DT, NB, CB, 16><<<blocks, 1024, 0, st>>>(a);
}

template <int DT>
hipError_t launch_few(const FewArgs &a, const Loss &p, hipStream_t st)
{
    // Two blocks of columns a workgroup read X half as often, and where the sixteen
    // waves have one turn each they halve the ends of workgroups; else they leave
    // fewer waves in flight.  us, one and two blocks: 1 x 2,048 -> 32,000 in bfloat16
    // 38.8 and 35.1, 1 x 1,000 17.6 and 20.8, 4 x 4,096 62 and 72, 16 x 4,096 82 and 76,
    // 16 x 2,048 50 and 41, 32 x 2,048 63 and 50, 32 x 1,500 -> 20,000 in float32 65 and 56.
    const int64_t turns = turns_of(p);
    const bool wide = a.v >= kWideFew && (a.n > 8 || (turns > 8 && turns <= 16));
    if (a.n <= 16 && wide)
        launch_waves<DT, 1, 2>(a, turns, st);
    else if (a.n <= 16 || thin_grid(a))
        launch_waves<DT, 1, 1>(a, turns, st);
    else if (wide)
        launch_waves<DT, 2, 2>(a, turns, st);
    else
        launch_waves<DT, 2, 1>(a, turns, st);
    return hipGetLastError();
}

// The powers of the columns of up to two matrices of the same width.
hipError_t launch_columns(const Source *const *list, float *const *part, int count, hipStream_t st)
{
    ColumnJobs jobs{};
    int64_t most = 0;
    for (int i = 0; i < count; ++i) {
        const Source &s = *list[i];
        const int64_t parts = max_parts(s.rows, s.cols), each = (s.rows + parts - 1) / parts;
        const int64_t used = (s.rows + each - 1) / each;
        jobs.j[i] = ColumnArgs{static_cast<const float *>(s.x), s.rows, s.cols, s.ld, each, used,
                               s.row, part[i], s.power};
        most = used > most ? used : most;
    }
    const int64_t cols = list[0]->cols;
    column_max_kernel<<<dim3((unsigned)((cols + 255) / 256), (unsigned)most, (unsigned)count), 256,
                        0, st>>>(jobs);
    RUN(hipGetLastError());
    column_power_kernel<<<dim3((unsigned)((cols + 63) / 64), (unsigned)count), 1024, 0, st>>>(jobs);
    return hipGetLastError();
}

} // namespace

size_t loss_ws(const Loss &p, bool backward)
{
    Cursor c{nullptr};
    if (p.n == 0)                        // (results of zeros at the most)
        return 0;
    if (backward && small(p))
        Small m(p, c);
    else if (backward)
        Backward b(p, nullptr, nullptr, c);
    else
        Forward f(p, nullptr, nullptr, c);
    return c.at;
}

bool loss_fits(const Loss &p, bool backward)
{
    if (p.n == 0 || (backward ? small(p) : few(p)))
        return true;
    const int op = kind_of(p.dtype);
    if (!backward)
        return product_plan(p.n, p.v, p.k, 1, op, kEpiLse).fits;
    const int64_t piece = piece_of(p) < p.v ? piece_of(p) : p.v;
    return product_plan(p.n, piece, p.k, 1, op, kEpiSoft).fits &&
           product_plan(p.n, p.k, piece, 1, op, kEpiSum).fits &&
           product_plan(piece, p.k, p.n, 1, op, kEpiSum).fits;
}

hipError_t run_loss(const Loss &p, const void *X, const void *W, const void *bias,
                    const void *targets, float *loss, float *lse, void *ws, hipStream_t st)
{
    if (p.n == 0)
        return hipSuccess;
    Cursor c{static_cast<char *>(ws)};
    Forward f(p, X, W, c);
    if (few(p)) {
        const FewArgs a{X, W, bias, targets, f.strip, f.picked, p.ldx, p.ldw, p.n, p.k, p.v, p.wide};
        RUN(p.dtype == GPIC_F32    ? launch_few<GPIC_F32>(a, p, st)
            : p.dtype == GPIC_F16 ? launch_few<GPIC_F16>(a, p, st)
                                  : launch_few<GPIC_BF16>(a, p, st));
    } else {
        const Source *list[2] = {&f.X, &f.W};
        if (p.dtype == GPIC_F32)
            RUN(launch_split_rows(f.X, f.W, st));
        else
            RUN(launch_pack(list, 2, p.dtype, st));
        ProductArgs a{};
        a.A = f.X.operand(p.dtype);
        a.B = f.W.operand(p.dtype);
        a.M = (int)p.n;
        a.N = (int)p.v;
        a.K = p.k;
        a.batch = 1;
        a.e.pa = f.X.power;
        a.e.pb = f.W.power;
        a.e.bias = bias;
        a.e.targets = targets;
        a.e.wide = p.wide;
        a.e.strip = f.strip;
        a.e.picked = f.picked;
        RUN(launch_product(kKK, kind_of(p.dtype), kEpiLse, a, st));
    }
    const JoinArgs j{f.strip, f.picked, targets, loss, lse, p.n, f.strips, p.v, p.wide};
    if (p.n < 64)
        join_kernel<1><<<(unsigned)p.n, 256, 0, st>>>(j);
    else
        join_kernel<16><<<(unsigned)((p.n + 15) / 16), 256, 0, st>>>(j);
    return hipGetLastError();
}

template <int DT, int NB>
hipError_t launch_small_of(const SmallArgs &a, int64_t turns, hipStream_t st)
{
    const FewArgs &f = a.f;
    const int64_t x = (f.v + 15) / 16, y = (f.n + 16 * NB - 1) / (16 * NB);
    const int64_t threads = turns <= 4 ? 256 : (turns <= 8 ? 512 : 1024);
    // X's copy: up to eight values a thread on up to 1,024 workgroups
    int64_t more = (f.n * f.k + 8 * threads - 1) / (8 * threads);
    more = ((more < 1024 ? more : 1024) + x - 1) / x;
    const dim3 blocks((unsigned)x, (unsigned)(y > more ? y : more));
    if (turns <= 4)
        small_soft_kernel<DT, NB, 4><<<blocks, 256, 0, st>>>(a);
    else if (turns <= 8)
        small_soft_kernel<DT, NB, 8><<<blocks, 512, 0, st>>>(a);
    else
        small_soft_kernel<DT, NB, 16><<<blocks, 1024, 0, st>>>(a);
    return hipGetLastError();
}

template <int DT>
hipError_t launch_small(const SmallArgs &a, const Loss &p, hipStream_t st)
{
    const int64_t turns = turns_of(p);
    if (p.n <= 16 || thin_grid(a.f))
        return launch_small_of<DT, 1>(a, turns, st);
    // W once for all rows up to 64 (64 rows over 2,048 -> 32,000: 185 us with it
    // read twice, 164 so; the forward kernel 133 and 160, which reads it twice)
    if constexpr (DT == GPIC_F32)
        if (p.n > 32 && p.n <= kThinRows && p.v >= kWideFew / 4)
            return launch_small_of<DT, 4>(a, turns, st);
    return launch_small_of<DT, 2>(a, turns, st);
}

hipError_t run_loss_backward(const Loss &p, const float *dloss, const void *X, const void *W,
                             const void *bias, const void *targets, const float *loss,
                             const float *lse, void *dX, void *dW, void *db, void *ws,
                             hipStream_t st)
{
    const size_t size = p.dtype == GPIC_F32 ? 4 : 2;
    if (p.n == 0) {
        if (dW)
            zero_kernel<<<4096, 256, 0, st>>>(dW, p.v * p.k, p.dtype);
        if (db)
            zero_kernel<<<64, 256, 0, st>>>(db, p.v, p.dtype);
        return hipGetLastError();
    }
    if (!dX && !dW && !db)
        return hipSuccess;
    Cursor c{static_cast<char *>(ws)};
    if (small(p)) {
        const Small m(p, c);
        SmallArgs a{};
        a.f = FewArgs{X, W, bias, targets, nullptr, nullptr, p.ldx, p.ldw, p.n, p.k, p.v, p.wide};
        a.dloss = dloss;
        a.loss = loss;
        a.lse = lse;
        a.D = m.D;
        a.X = m.X;
        RUN(p.dtype == GPIC_F32    ? launch_small<GPIC_F32>(a, p, st)
            : p.dtype == GPIC_F16 ? launch_small<GPIC_F16>(a, p, st)
                                  : launch_small<GPIC_BF16>(a, p, st));
        if (little(p))
            return run_small_gradients(layer_of(p), false, m.D, m.X, W, nullptr, dX, dW, db, st);
        return run_thin_gradients(m.D, m.X, W, p.n, p.k, p.v, p.ldw, p.dtype, dX, dW, db, m.part, st);
    }
    Backward b(p, X, W, c);
    const bool f32 = p.dtype == GPIC_F32;
    const int op = kind_of(p.dtype);
    {
        const RowsArgs a{dloss, loss, lse, targets, p.wide, p.n, p.v, b.rows, b.most};
        const int64_t blocks = (p.n + 255) / 256;
        unsigned groups = 1;
        if (p.n > kRowsAtOnce) {
            rows_kernel<<<(unsigned)blocks, 256, 0, st>>>(a);
            RUN(hipGetLastError());
            groups = (unsigned)(p.n < 128 * 4096 ? (p.n + 4095) / 4096 : 128);
        }
        shares_kernel<<<groups, 1024, 0, st>>>(a, blocks, b.largest, b.share);
        RUN(hipGetLastError());
    }
    if (b.share_part && dW) {
        share_max_kernel<<<(unsigned)b.Xg.count, 256, 0, st>>>(
            static_cast<const _Float16 *>(X), b.share, p.n, p.k, p.ldx, share_lanes(p.k),
            b.share_part);
        RUN(hipGetLastError());
    }
    if (f32 && (dX || dW)) {
        Source all = b.Wc;
        all.rows = p.v;
        const Source *list[2];
        float *part[2];
        int count = 0;
        if (dW) {
            list[count] = &b.Xg;
            part[count++] = b.column_part[0];
        }
        if (dX) {
            list[count] = &all;
            part[count++] = b.column_part[1];
        }
        RUN(launch_columns(list, part, count, st));
    }
    for (int64_t first = 0; first < p.v; first += b.piece) {
        const int64_t len = p.v - first < b.piece ? p.v - first : b.piece;
        const void *w = static_cast<const char *>(W) + (size_t)first * p.ldw * size;
        b.W.x = b.Wc.x = w;
        b.W.rows = b.Wc.rows = len;
        // X is packed with the first piece
        Source x = b.X, xg = b.Xg, wc = b.Wc;
        if (first > 0)
            x.rows = xg.rows = 0;
        xg.pack = dW != nullptr;
        wc.pack = f32 && dX;
        const Source *list[3] = {&xg, f32 ? &wc : &x, &b.W};
        if (f32)
            RUN(launch_split_rows(x, b.W, st));
        RUN(launch_pack(list, f32 ? 2 : 3, p.dtype, st));
        ProductArgs a{};
        a.A = b.X.operand(p.dtype);
        a.B = b.W.operand(p.dtype);
        a.M = (int)p.n;
        a.N = (int)len;
        a.K = p.k;
        a.batch = 1;
        a.part = b.part;
        a.e.pa = f32 ? b.X.power : nullptr;
        a.e.pb = b.W.power;
        a.e.bias = bias;
        a.e.rows = b.rows;
        a.e.first = first;
        a.e.p_hi = b.dZ;
        a.e.ldp = b.pitch;
        a.e.sums = db ? b.sum_b : nullptr;
        RUN(launch_product(kKK, op, kEpiSoft, a, st));
        if (db) {
            const Plan plan = product_plan(p.n, len, p.k, 1, op, kEpiSoft);
            const int64_t each = edge_of(plan) / 2;      // rows of a wave
            RUN(launch_sum_parts(b.sum_b, (p.n + each - 1) / each, len,
                                 static_cast<char *>(db) + (size_t)first * size, p.dtype, st));
        }
        const int64_t width = f32 ? split_ld(up64(len)) : up64(len);
        if (dX) {
            ProductArgs x{};
            x.A = Operand{b.dZ, b.pitch, 0, width};
            x.B = f32 ? b.Wc.operand(p.dtype) : b.W.operand(p.dtype);
            x.M = (int)p.n;
            x.N = (int)p.k;
            x.K = len;
            x.batch = 1;
            x.part = b.part;
            x.e.dtype = p.dtype;
            x.e.pb = b.Wc.power;
            x.e.factor = &b.rows->g;
            x.e.factor_step = sizeof(LossRow) / sizeof(float);
            x.e.res = first > 0 ? b.sum_x : nullptr;
            x.e.ldr = x.e.ldo = p.k;
            x.e.last = first + len >= p.v;
            x.e.out = x.e.last ? dX : b.sum_x;
            RUN(launch_product(kKM, op, kEpiSum, x, st));
        }
        if (dW) {
            ProductArgs d{};
            d.A = Operand{b.dZ, b.pitch, 0, width};
            d.B = b.Xg.operand(p.dtype);
            d.M = (int)len;
            d.N = (int)p.k;
            d.K = p.n;
            d.batch = 1;
            d.part = b.part;
            d.e.dtype = p.dtype;
            d.e.pb = b.Xg.power;
            d.e.pa = b.Xg.scale;
            d.e.factor = b.largest;
            d.e.factor_step = 0;
            d.e.ldo = p.k;
            d.e.last = 1;
            d.e.out = static_cast<char *>(dW) + (size_t)first * p.k * size;
            RUN(launch_product(kMM, op, kEpiSum, d, st));
        }
    }
    return hipSuccess;
}

} // namespace gpic
