// The layers' forward pass where a tiled product would not pay: few rows
// (few_rows_kernel; small layers too), and many rows of a short contraction
// (short_kernel).
//
// Few rows (serving single points) are bound by reading W once.  A workgroup takes 16 columns of the output (gated: 16 of
// the gate's and the same 16 of the up projection's); its waves share the
// contraction in turns of 128 (float32: 64) values, so that together they
// read long runs of the 16 rows of W, each lane 16 bytes at a time into
// registers and from there into the matrix cores, W's rows as the first
// operand and up to 32 rows of X as the second.  The waves' sums meet in
// LDS and are added in wave order.  float32 uses the float32 matrix
// instruction (the operands are not split: reading them is what counts).
// One bfloat16 row, 2,048 -> 8,192: 8.7 us, 3.9 TB/s of W; four float16
// rows, 2,048 -> 2 x 5,504: 14 us, 3.2 TB/s; seven float32 rows, 1,000 -> 777:
// 6.4 us, most of it latency.
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
    int strips;            // short_kernel: strips of columns, row tiles a wave
    int64_t each;
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
    const int64_t col0 = (int64_t)blockIdx.x * 16, row0 = (int64_t)blockIdx.y * (16 * NB);
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
        const int64_t row = row0 + b * 16 + r < a.n ? row0 + b * 16 + r : a.n - 1;
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
    const int64_t row = row0 + wave * 16 + r;
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
    const dim3 blocks((unsigned)((a.m + 15) / 16), (unsigned)((a.n + 16 * NB - 1) / (16 * NB)));
    // as many waves as there are turns: then all of W is on its way at once
    const int64_t turns = (a.k + (DT == GPIC_F32 ? 63 : 127)) / (DT == GPIC_F32 ? 64 : 128);
    if (turns <= 4)
        few_rows_kernel<DT, GATED, NB, 4><<<blocks, 256, 0, st>>>(a);
    else if (turns <= 8 || (GATED && NB == 2))
        few_rows_kernel<DT, GATED, NB, 8><<<blocks, 512, 0, st>>>(a);
    else
        few_rows_kernel<DT, GATED, NB, 16><<<blocks, 1024, 0, st>>>(a);
    return hipGetLastError();
}

template <int DT>
hipError_t launch_rows(const RowArgs &a, bool gated, hipStream_t st)
{
    if (gated)
        return a.n <= 16 ? launch_waves<DT, true, 1>(a, st) : launch_waves<DT, true, 2>(a, st);
    return a.n <= 16 ? launch_waves<DT, false, 1>(a, st) : launch_waves<DT, false, 2>(a, st);
}

// ------------------------------------------------------ short contraction
// N consecutive values of a type at any alignment, `valid` of which exist.
template <int DT, int N>
struct Run {
    using Values = float __attribute__((ext_vector_type(N)));
    using F = float __attribute__((ext_vector_type(N), aligned(4)));
    using H = _Float16 __attribute__((ext_vector_type(N), aligned(2)));
    using B = __bf16 __attribute__((ext_vector_type(N), aligned(2)));
    static __device__ __forceinline__ Values load(const void *p, int64_t i, int valid)
    {
        if (valid >= N) {
            if (DT == GPIC_F32)
                return *reinterpret_cast<const F *>(static_cast<const float *>(p) + i);
            if (DT == GPIC_F16)
                return __builtin_convertvector(
                    *reinterpret_cast<const H *>(static_cast<const _Float16 *>(p) + i), Values);
            return __builtin_convertvector(
                *reinterpret_cast<const B *>(static_cast<const __bf16 *>(p) + i), Values);
        }
        Values v = 0.0f;
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (j < valid)
                v[j] = load1(p, i + j, DT);
        return v;
    }
    static __device__ __forceinline__ void store(void *p, int64_t i, Values v, int valid)
    {
        if (valid >= N) {
            if (DT == GPIC_F32)
                *reinterpret_cast<F *>(static_cast<float *>(p) + i) = v;
            else if (DT == GPIC_F16)
                *reinterpret_cast<H *>(static_cast<_Float16 *>(p) + i) =
                    __builtin_convertvector(v, H);
            else
                *reinterpret_cast<B *>(static_cast<__bf16 *>(p) + i) =
                    __builtin_convertvector(v, B);
            return;
        }
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (j < valid)
                store1(p, i + j, v[j], DT);
    }
};

template <int ACT, class V, int N>
__device__ __forceinline__ void activate_run(V &v)
{
#pragma unroll
    for (int j = 0; j < N; ++j)
        v[j] = activate(v[j], ACT);
}

template <class V, int N>
__device__ __forceinline__ V activated(V v, int act)
{
    if (act == GPIC_ACT_RELU)
        activate_run<GPIC_ACT_RELU, V, N>(v);
    else if (act == GPIC_ACT_GELU)
        activate_run<GPIC_ACT_GELU, V, N>(v);
    else if (act == GPIC_ACT_SILU)
        activate_run<GPIC_ACT_SILU, V, N>(v);
    return v;
}

// A wave holds a strip of W (64 of its rows, all of k) as fragments in
// registers and takes 16 rows of X after another past it, the next 16 on
// their way.  KC: fragments that cover k.  A lane's results are N
// consecutive columns of one row, so that four lanes write 64 bytes of it
// (the 16-bit types: two matrix instructions' columns are interleaved).
// Bound by writing the results and, for gelu, by its arithmetic: 50,000 x 16
// -> 256 in float32 15.4 us without an activation (55 MB, 3.6 TB/s), 19.0 with
// gelu; 33 as a tiled product after two packing launches.  16,384 x 16 -> 8,192
// in bfloat16 61 us (4.4 TB/s), gelu 94 (150 tiled).  Waves: about eight for
// each of the card's 1,024 vector units, a few row tiles each; 2 or 64 of them
// take 10 % longer.
template <int DT, bool GATED, int KC>
__global__ __launch_bounds__(256) void short_kernel(RowArgs a)
{
    constexpr int kSize = DT == GPIC_F32 ? 4 : 2, kValues = 16 / kSize;
    constexpr int kG = GATED ? 2 : 1, N = DT == GPIC_F32 ? 4 : 8, kPer = N / 4;
    constexpr int kGroups = 4 / (kG * kPer);             // groups of 4 N columns
    constexpr int kCols = kGroups * 4 * N;               // of a strip (gated: of one half)
    using R = Run<DT, N>;
    using Values = typename R::Values;
    const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
    const int64_t id = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int64_t col0 = id % a.strips * kCols, tiles = ((int64_t)a.n + 15) / 16;
    const int64_t first = id / a.strips * a.each;
    const int64_t end = first + a.each < tiles ? first + a.each : tiles;
    if (first >= end)
        return;

    // Where this lane's last 16 bytes lie.  A fragment that runs past k is
    // read from k's last 16 bytes instead, in W as in X, and what the lanes
    // before it hold already is masked off.
    const bool tiny = a.k < kValues;
    const int64_t at = ((KC - 1) * 4 + g) * kValues;
    const int64_t last = at < a.k - kValues ? at : (tiny ? 0 : a.k - kValues);
    const int64_t skip = at - last;                      // values held already
    u32x4 keep;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (DT == GPIC_F32)
            keep[j] = j >= skip ? 0xffffffffu : 0u;
        else
            keep[j] = (2 * j >= skip ? 0xffffu : 0u) | (2 * j + 1 >= skip ? 0xffff0000u : 0u);
    }
    auto fetch = [&](const char *row, u32x4 (&f)[KC]) {
#pragma unroll
        for (int c = 0; c < KC - 1; ++c)
            f[c] = chunk_at<DT, false>(row, (c * 4 + g) * kValues, a.k);
        f[KC - 1] = tiny ? chunk_at<DT, true>(row, at, a.k)
                         : chunk_at<DT, false>(row, last, a.k);
    };
    auto clip = [&](u32x4 (&f)[KC]) {
        if (!tiny)
            f[KC - 1] &= keep;
    };

    u32x4 fw[kG][kGroups][kPer][KC];
    Values bias[kGroups];
    int valid[kGroups];
    int64_t col[kGroups];
#pragma unroll
    for (int q = 0; q < kGroups; ++q) {
        const int64_t base = col0 + q * 4 * N;
        col[q] = base + g * N;
        valid[q] = a.m - col[q] < N ? (int)(a.m - col[q]) : N;
        bias[q] = 0.0f;
        if (!GATED && a.bias && valid[q] > 0)
            bias[q] = R::load(a.bias, col[q], valid[q]);
#pragma unroll
        for (int i = 0; i < kG; ++i)
#pragma unroll
            for (int p = 0; p < kPer; ++p) {
                // columns beyond the last are computed as the last, not stored
                int64_t row = base + (r >> 2) * N + p * 4 + (r & 3);
                row = (row < a.m ? row : a.m - 1) + i * a.m;
                fetch(static_cast<const char *>(a.W) + row * a.ldw * kSize, fw[i][q][p]);
                clip(fw[i][q][p]);
            }
    }

    auto row_of = [&](int64_t tile) {
        const int64_t row = tile * 16 + r;
        return static_cast<const char *>(a.X) + (row < a.n ? row : a.n - 1) * a.ldx * kSize;
    };
    u32x4 next[KC];
    fetch(row_of(first), next);
    for (int64_t t = first; t < end; ++t) {
        u32x4 fx[KC];
#pragma unroll
        for (int c = 0; c < KC; ++c)
            fx[c] = next[c];
        clip(fx);
        fetch(row_of(t + 1 < end ? t + 1 : t), next);
        const int64_t row = t * 16 + r;
        // the products first, so that none waits for another's sum
        f32x4 acc[kGroups][kG][kPer];
#pragma unroll
        for (int c = 0; c < KC; ++c)
#pragma unroll
            for (int q = 0; q < kGroups; ++q)
#pragma unroll
                for (int i = 0; i < kG; ++i)
#pragma unroll
                    for (int p = 0; p < kPer; ++p)
                        acc[q][i][p] = mma16<DT>(fw[i][q][p][c], fx[c],
                                                 c == 0 ? f32x4{0.0f, 0.0f, 0.0f, 0.0f}
                                                        : acc[q][i][p]);
#pragma unroll
        for (int q = 0; q < kGroups; ++q) {
            Values v[kG];
#pragma unroll
            for (int i = 0; i < kG; ++i)
#pragma unroll
                for (int j = 0; j < N; ++j)
                    v[i][j] = acc[q][i][j / 4][j % 4];
            if (row >= a.n || valid[q] <= 0)
                continue;
            if (GATED) {
                if (a.Z) {
                    Run<GPIC_F32, N>::store(a.Z, row * a.ldz + col[q], v[0], valid[q]);
                    Run<GPIC_F32, N>::store(a.Z, row * a.ldz + a.m + col[q], v[kG - 1], valid[q]);
                }
                R::store(a.Y, row * a.ldy + col[q],
                         activated<Values, N>(v[0], a.act) * v[kG - 1], valid[q]);
                continue;
            }
            Values z = v[0];
            if (a.bias)
                z = z + bias[q];
            if (a.Z)
                R::store(a.Z, row * a.ldz + col[q], z, valid[q]);
            z = activated<Values, N>(z, a.act);
            if (a.res)
                z = z + R::load(a.res, row * a.ldr + col[q], valid[q]);
            R::store(a.Y, row * a.ldy + col[q], z, valid[q]);
        }
    }
}

template <int DT, bool GATED>
hipError_t launch_short(RowArgs a, hipStream_t st)
{
    constexpr int kCols = GATED ? 32 : 64;
    const int64_t tiles = ((int64_t)a.n + 15) / 16, strips = (a.m + kCols - 1) / kCols;
    // about eight waves for each of the card's 1,024 vector units
    a.strips = (int)strips;
    a.each = (tiles * strips + 8191) / 8192;
    const int64_t waves = (tiles + a.each - 1) / a.each * strips;
    const dim3 grid((unsigned)((waves + 3) / 4));
    const int chunks = (int)((a.k * (DT == GPIC_F32 ? 4 : 2) + 63) / 64);
    if (chunks == 1)
        short_kernel<DT, GATED, 1><<<grid, 256, 0, st>>>(a);
    else if (chunks == 2)
        short_kernel<DT, GATED, 2><<<grid, 256, 0, st>>>(a);
    else if (DT != GPIC_F32)
        return hipErrorInvalidValue;
    else if (chunks == 3)
        short_kernel<GPIC_F32, GATED, 3><<<grid, 256, 0, st>>>(a);
    else if (chunks == 4)
        short_kernel<GPIC_F32, GATED, 4><<<grid, 256, 0, st>>>(a);
    else
        return hipErrorInvalidValue;
    return hipGetLastError();
}

template <int DT>
hipError_t launch_either(const RowArgs &a, bool gated, hipStream_t st)
{
    if (a.n > kFewRows && a.k <= 64)
        return gated ? launch_short<DT, true>(a, st) : launch_short<DT, false>(a, st);
    return launch_rows<DT>(a, gated, st);
}

} // namespace

// Few rows, or up to 64 values of k, where a layer's results outweigh its
// products, or little work, where launches do (32 rows at a time then).
// float32 beyond 32 values of k only for small results: the float32 matrix
// instruction then costs more than packed operands' two launches.  gelu, us,
// here and as a tiled product: 1,003 x 64 -> 700 6.9 and 9.7, 50,000 x 64 -> 256 42
// and 40, 16,384 x 64 -> 8,192 251 and 192, 16,384 x 32 -> 8,192 179 and 170 (bfloat16
// 107 and 150); 52 x 512 -> 123 5.5 and 15, 200 x 300 -> 700 5.8 and 14.5 (bfloat16 5.9
// and 9.7), 100 x 1,000 -> 1,000 7.9 and 19 (4.9 and 10), 1,003 x 300 -> 700 14 and 16
// (12.4 and 10.3), 2,000 x 700 -> 700 48 and 26 (34 and 16).
bool as_rows(const Shape &s, bool gated)
{
    const bool f32 = s.dtype == GPIC_F32;
    const int64_t rows = gated ? 2 * s.m : s.m;
    if (s.n <= kFewRows || s.k <= 32 || (s.k <= 64 && (!f32 || s.n * rows <= (1 << 23))))
        return true;
    return s.n <= 2048 && s.n * rows <= ((int64_t)1 << (f32 ? 28 : 27)) / s.k;
}

hipError_t run_rows(const Shape &s, bool gated, const void *X, const void *W,
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
        return launch_either<GPIC_F32>(a, gated, st);
    return s.dtype == GPIC_F16 ? launch_either<GPIC_F16>(a, gated, st)
                               : launch_either<GPIC_BF16>(a, gated, st);
}

} // namespace gpic
