// Internal declarations of the encoder operators (layers, their gradients,
// the orthogonalised update): operand and epilogue descriptions of the
// tiled matrix product, activations, and the host launchers.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/gpic.h"

namespace gpic {

using half8 = _Float16 __attribute__((ext_vector_type(8)));
using bfrag8 = __bf16 __attribute__((ext_vector_type(8)));
using half4 = _Float16 __attribute__((ext_vector_type(4)));
using bf4 = __bf16 __attribute__((ext_vector_type(4)));
using f32x4 = float __attribute__((ext_vector_type(4)));
using f32x8 = float __attribute__((ext_vector_type(8), aligned(16)));
using i32x4 = int __attribute__((ext_vector_type(4)));
using u32x4 = unsigned int __attribute__((ext_vector_type(4)));
using s16x4 = short __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------ activations
// Phi(z) and phi(z) of the normal distribution.  erfc(x) for x = |z| /
// sqrt(2) by Abramowitz and Stegun 7.1.26 (t = 1 / (1 + p x), a quintic in t
// times exp(-x^2); absolute error 1.5e-7, half of that in Phi, about a
// float32 rounding of Phi near 1), taken on the side where nothing cancels:
// one exponential, one reciprocal and seven multiply-adds, where the
// library's erff costs about forty instructions and would take a quarter
// of the time of a large layer's product.
__device__ __forceinline__ void normal_tail(float z, float &tail, float &e)
{
    e = __builtin_amdgcn_exp2f(z * z * -0.72134752044448170f);
    const float t = __builtin_amdgcn_rcpf(1.0f + 0.23164189f * fabsf(z));
    float q = 0.53070271f;                      // half of the table's a_5 .. a_1
    q = q * t - 0.72657601f;
    q = q * t + 0.71070687f;
    q = q * t - 0.14224837f;
    q = q * t + 0.12741480f;
    tail = q * t * e;                           // Phi(-|z|)
}

__device__ __forceinline__ void normal_cdf_pdf(float z, float &cdf, float &pdf)
{
    float tail, e;
    normal_tail(z, tail, e);
    cdf = z > 0.0f ? 1.0f - tail : tail;
    pdf = 0.39894228040143268f * e;
}

__device__ __forceinline__ float sigmoidf(float z)
{
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.4426950408889634f));
}

// act(z).  Infinities go where the function's limit is (silu and gelu of
// -inf are 0), NaN stays NaN.
__device__ __forceinline__ float activate(float z, int act)
{
    if (act == GPIC_ACT_RELU)
        return z > 0.0f || z != z ? z : 0.0f;
    if (act == GPIC_ACT_GELU) {
        // z Phi(z) = max(z, 0) - |z| Phi(-|z|); the bound keeps infinity times
        // the tail's zero out, and is past where the tail is one
        float tail, e;
        normal_tail(z, tail, e);
        return fmaxf(z, 0.0f) - fminf(fabsf(z), 14.5f) * tail;
    }
    if (act == GPIC_ACT_SILU)
        return fmaxf(z, -104.0f) * sigmoidf(z);
    return z;
}

// act(z) and act'(z); act' is 0 at z = 0 for the rectifier
__device__ __forceinline__ void activate_grad(float z, int act, float &a, float &da)
{
    a = z;
    da = 1.0f;
    if (act == GPIC_ACT_RELU) {
        a = z > 0.0f || z != z ? z : 0.0f;
        da = z > 0.0f ? 1.0f : (z != z ? z : 0.0f);
    } else if (act == GPIC_ACT_GELU) {
        float c, p;
        normal_cdf_pdf(z, c, p);
        a = z < -14.0f ? 0.0f : z * c;
        da = fabsf(z) > 14.0f ? c : c + z * p;
    } else if (act == GPIC_ACT_SILU) {
        const float s = sigmoidf(z);
        a = z < -104.0f ? 0.0f : z * s;
        da = fabsf(z) > 104.0f ? s : s * (1.0f + z * (1.0f - s));
    }
}

// eight values at once: one choice of the function for all of them
__device__ __forceinline__ f32x8 activate8(f32x8 z, int act)
{
    if (act == GPIC_ACT_RELU) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            z[j] = activate(z[j], GPIC_ACT_RELU);
    } else if (act == GPIC_ACT_GELU) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            z[j] = activate(z[j], GPIC_ACT_GELU);
    } else if (act == GPIC_ACT_SILU) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            z[j] = activate(z[j], GPIC_ACT_SILU);
    }
    return z;
}

// ------------------------------------------------- typed loads and stores
__device__ __forceinline__ float load1(const void *p, int64_t i, int dtype)
{
    if (dtype == GPIC_F32)
        return static_cast<const float *>(p)[i];
    if (dtype == GPIC_F16)
        return (float)static_cast<const _Float16 *>(p)[i];
    return (float)static_cast<const __bf16 *>(p)[i];
}

__device__ __forceinline__ void store1(void *p, int64_t i, float v, int dtype)
{
    if (dtype == GPIC_F32)
        static_cast<float *>(p)[i] = v;
    else if (dtype == GPIC_F16)
        static_cast<_Float16 *>(p)[i] = (_Float16)v;
    else
        static_cast<__bf16 *>(p)[i] = (__bf16)v;
}

// four consecutive values at any alignment (the card's 16-byte accesses
// need none)
__device__ __forceinline__ f32x4 load4(const void *p, int64_t i, int dtype)
{
    using f = float __attribute__((ext_vector_type(4), aligned(4)));
    using h = _Float16 __attribute__((ext_vector_type(4), aligned(2)));
    using b = __bf16 __attribute__((ext_vector_type(4), aligned(2)));
    if (dtype == GPIC_F32)
        return *reinterpret_cast<const f *>(static_cast<const float *>(p) + i);
    if (dtype == GPIC_F16)
        return __builtin_convertvector(
            *reinterpret_cast<const h *>(static_cast<const _Float16 *>(p) + i), f32x4);
    return __builtin_convertvector(
        *reinterpret_cast<const b *>(static_cast<const __bf16 *>(p) + i), f32x4);
}

// the same, stored; p + i aligned to four values
__device__ __forceinline__ void store4(void *p, int64_t i, f32x4 v, int dtype)
{
    if (dtype == GPIC_F32)
        *reinterpret_cast<f32x4 *>(static_cast<float *>(p) + i) = v;
    else if (dtype == GPIC_F16)
        *reinterpret_cast<half4 *>(static_cast<_Float16 *>(p) + i) =
            __builtin_convertvector(v, half4);
    else
        *reinterpret_cast<bf4 *>(static_cast<__bf16 *>(p) + i) =
            __builtin_convertvector(v, bf4);
}

// Eight values p[i .. i + 7], of which `valid` exist, at any alignment (the
// card's 16-byte accesses need none; where a row starts on 16 bytes they
// cover whole lines).
using f32x8_any = float __attribute__((ext_vector_type(8), aligned(4)));
using half8_any = _Float16 __attribute__((ext_vector_type(8), aligned(2)));
using bfrag8_any = __bf16 __attribute__((ext_vector_type(8), aligned(2)));

__device__ __forceinline__ f32x8 load8(const void *p, int64_t i, int dtype, int valid)
{
    if (valid >= 8) {
        if (dtype == GPIC_F32)
            return *reinterpret_cast<const f32x8_any *>(static_cast<const float *>(p) + i);
        if (dtype == GPIC_F16)
            return __builtin_convertvector(
                *reinterpret_cast<const half8_any *>(static_cast<const _Float16 *>(p) + i), f32x8);
        return __builtin_convertvector(
            *reinterpret_cast<const bfrag8_any *>(static_cast<const __bf16 *>(p) + i), f32x8);
    }
    f32x8 v = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < valid)
            v[j] = load1(p, i + j, dtype);
    return v;
}

__device__ __forceinline__ void store8(void *p, int64_t i, f32x8 v, int dtype, int valid)
{
    if (valid >= 8) {
        if (dtype == GPIC_F32)
            *reinterpret_cast<f32x8_any *>(static_cast<float *>(p) + i) = v;
        else if (dtype == GPIC_F16)
            *reinterpret_cast<half8_any *>(static_cast<_Float16 *>(p) + i) =
                __builtin_convertvector(v, half8);
        else
            *reinterpret_cast<bfrag8_any *>(static_cast<__bf16 *>(p) + i) =
                __builtin_convertvector(v, bfrag8);
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < valid)
            store1(p, i + j, v[j], dtype);
}

// ---------------------------------------------------------- split matrices
// A float32 matrix as 16-bit parts: x = (hi + lo) / s, s a power of two,
// hi = half(s x), lo = half(s x - hi), 22 significant bits together for
// entries down to 2^-17 of the largest under the same s (below it, to 2^-39 of
// that largest).  s belongs to what the product does not sum over, a row of
// its operand, so that no row's bits depend on another row.  The
// columns come in groups of 32, each as 32 hi and then 32 lo values, so a
// matrix of c columns has rows of 2 * ceil(c / 32) * 32 halves (zeros
// beyond c) and any 128-byte line holds both parts of its 32 values.
__host__ __device__ __forceinline__ int64_t split_ld(int64_t cols)
{
    return (cols + 31) / 32 * 64;
}
__host__ __device__ __forceinline__ int64_t split_at(int64_t col)
{
    return (col >> 5) * 64 + (col & 31);
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

// ----------------------------------------------------- workspaces' layout
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

// -------------------------------------------------------- matrix product
// out[M x N] = epilogue(sum_k A(i, k) B(j, k)) over 16-bit operands on the
// matrix cores, float32 accumulation, an optional batch in the grid.
// An operand is either k-contiguous (rows i, row pitch ld) or k-strided
// (rows k, row pitch ld, i contiguous).  Rows are 16-byte aligned, ld % 8
// == 0 and the contiguous extent % 8 == 0.
struct Operand {
    const void *p;
    int64_t ld;        // row pitch in 16-bit values
    int64_t batch;     // pitch between matrices of a batch, 16-bit values
    int64_t cols;      // 16-bit values of a row that may be read
};

// kEpiGram: P = acc; kEpiPoly: P = beta C + acc, both over the upper triangle
// of tiles and mirrored, C and P symmetric; kEpiUpdate: X' = beta X + acc;
// kEpiResult: the same as a result (or, is_step, weights moved by it);
// kEpiLse: logits z = acc + bias, of which each row's largest and sum of
// exponentials over the tile's columns are kept (but the target's, which is
// kept itself); kEpiSoft: exp(z - lse) - [target] as an operand of further
// products; kEpiSum: acc times a factor (of its row), added to float32 sums
enum {
    kEpiLayer = 0, kEpiGated = 1, kEpiGram = 2, kEpiPoly = 3, kEpiUpdate = 4, kEpiResult = 5,
    kEpiLse = 6, kEpiSoft = 7, kEpiSum = 8
};
__host__ __device__ constexpr bool symmetric(int epi) { return epi == kEpiGram || epi == kEpiPoly; }
// whose operands may be under powers of two
__host__ __device__ constexpr bool powered(int epi)
{
    return epi == kEpiLayer || epi == kEpiGated || epi >= kEpiLse;
}
// whose tiles are not cut along the contraction
__host__ __device__ constexpr bool uncut(int epi) { return epi == kEpiLse || epi == kEpiSoft; }

// Brings exp(z - lse) - [target], at most 1, next to the largest half.
constexpr int kSoftPower = 15;

// What kEpiSoft knows of a row.
struct LossRow {
    float at, off;     // their sum is lse; off is 0 but where |lse| leaves it no digits
    float g;           // the loss's gradient
    float picked;      // exp(z - lse) - 1 of the target
    int target;        // its column; -1: none, no gradient
    int unused[3];
};

struct Epilogue {
    // layers: the powers of two that the operands were multiplied by, their
    // exponents (device pointers, null = 0): of split operands one for every
    // row i of A and every row j of B, of float16 ones one for all of A; the
    // others multiply acc by alpha
    const int *pa, *pb;
    float alpha;
    // kEpiLayer, kEpiGated: z = acc (+ bias); y = act(z) (+ residual)
    const void *bias, *res;
    void *out, *pre;
    int64_t ldr, ldo, ldz;
    int dtype, act;
    int64_t half;      // gated: columns of one half
    // C, P, X, X' as 16-bit parts: split matrices, or for single operands
    // a matrix of high halves and (X, X') one of low halves of the same pitch
    float beta;
    const void *c_hi, *c_lo;
    void *p_hi, *p_lo;
    int64_t ldp, batch_p;      // of C, P, X, X' (16-bit values)
    float store_scale;         // P, X' are stored times this
    float load_scale;          // C, X are multiplied by this when read
    // kEpiResult: out = beta X + acc, or out = decay out - step (beta X + acc)
    int is_step;
    float decay, step;
    int64_t batch_o;
    // kEpiLse: targets (32 or 64 bits), [tiles across][M] largest logit and
    // sum of exponentials, [M] target's logit
    const void *targets;
    int wide;
    float2 *strip;
    double *picked;
    // kEpiSoft: rows, the column that the piece starts at, where exp(z - lse) -
    // [target] goes (p_hi, ldp; times 2^kSoftPower but in bfloat16), [row blocks][N]
    // column sums of it times g, or null
    const LossRow *rows;
    int64_t first;
    float *sums;
    // kEpiSum: operand A is under 2^kSoftPower (but in bfloat16), float16 both
    // together under 2^*pa more (if not null); factors, one a
    // row or (factor_step 0) for all; sums so far (float32, res and ldr) or null;
    // out is float32, or (last) of the operands' type
    const float *factor;
    int factor_step;
    int last;
};

struct ProductArgs {
    Operand A, B;
    int M, N;          // output rows, columns
    int64_t K;         // contraction length
    int batch;
    float *part;       // the parts of split tiles: [splits][tail][tile]
    int whole, splits; // set by the launch, from the plan
    Epilogue e;
};

enum { kOpF16 = 0, kOpBf16 = 1, kOpSplit = 2 };    // operand kinds
enum { kKK = 0, kKM = 1, kMM = 2 };                // A, B k-contiguous (K) or k-strided (M)

// How a product is cut: `whole` tiles over the full contraction, then
// `tail` tiles in `splits` parts each, joined by a second launch.
struct Plan {
    bool fits;         // false: more threads than a launch takes with every tile
    int tile;          // 0: 256 x 256, 1: 128 x 128, 2: 64 x 64
    int tm, tn;        // tiles down and across
    int64_t whole, tail;
    int splits;
    size_t part_bytes;
};
// N: columns of the tiled product (gated: both halves)
Plan product_plan(int64_t M, int64_t N, int64_t K, int64_t batch, int op, int epi);

// One product (and the join of its split tiles).
hipError_t launch_product(int modes, int op, int epi, const ProductArgs &a, hipStream_t s);

// instantiations, one translation unit per pair of operand orders
hipError_t launch_product_kk(int op, int epi, const Plan &p, const ProductArgs &a, hipStream_t s);
hipError_t launch_product_km(int op, int epi, const Plan &p, const ProductArgs &a, hipStream_t s);
hipError_t launch_product_mm(int op, int epi, const Plan &p, const ProductArgs &a, hipStream_t s);
hipError_t launch_product_loss(int modes, int op, int epi, const Plan &p, const ProductArgs &a,
                               hipStream_t s);

// ---------------------------------------------------- operands' copies (layers.hip)
inline int kind_of(int dtype)
{
    return dtype == GPIC_F32 ? kOpSplit : (dtype == GPIC_F16 ? kOpF16 : kOpBf16);
}

// A matrix that a product reads: as it lies where it can, else a packed
// copy in the workspace.
struct Source {
    const void *x;
    int64_t rows, cols, ld;
    bool pack;
    void *to = nullptr;
    int *power = nullptr;  // float32: of its rows (backward: columns)
    const float *row = nullptr;    // packed times this, by row (0: zeros)
    const float *most = nullptr;   // float16: `count` parts of the largest of that, for
    int count = 0;                 // the power of two that goes to *scale
    int *scale = nullptr;
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
inline bool must_pack(int dtype, int64_t cols, int64_t ld, bool aligned16)
{
    return dtype == GPIC_F32 || !aligned16 || cols % 8 || ld % 8;
}

// `powers`: how many powers of two the copy has (float32)
inline void place(Source &s, int dtype, Cursor &c, int64_t powers)
{
    if (!s.pack)
        return;
    const int64_t p = dtype == GPIC_F32 ? split_ld(s.cols) : up64(s.cols);
    s.to = c.take((size_t)s.rows * p * 2);
    if (dtype == GPIC_F32)
        s.power = static_cast<int *>(c.take((size_t)powers * 4));
}

// X and W of a float32 layer, split under a power of two for every row
hipError_t launch_split_rows(const Source &x, const Source &w, hipStream_t st);
// copies of up to three operands (those to be packed); float32: split under a
// power of two for every column
hipError_t launch_pack(const Source *const *list, int count, int dtype, hipStream_t st);
// db [m] = sums of `parts` partial column sums [parts][m]
hipError_t launch_sum_parts(const float *sums, int64_t parts, int64_t m, void *db, int dtype,
                            hipStream_t st);

// ------------------------------------------------------------- layers.hip
struct Shape {         // a layer: n rows, k inputs, m outputs
    int64_t n, k, m;
    int dtype, act;
    int64_t ldx, ldw, ldr, ldy, ldz;
    bool aligned16;    // every matrix starts on 16 bytes
};
size_t layer_ws(const Shape &s, bool gated, bool backward);
// Whether every launch of a call stays below a grid's 2^32 threads.
bool layer_fits(const Shape &s, bool gated, bool backward);
hipError_t run_layer(const Shape &s, bool gated, const void *X, const void *W,
                     const void *bias, const void *res, void *Y, void *Z, void *ws,
                     hipStream_t st);
hipError_t run_layer_backward(const Shape &s, bool gated, const void *dY, const void *X,
                              const void *W, const void *Z, void *dX, void *dW, void *db,
                              void *ws, hipStream_t st);

// ---------------------------------------------------------------- rows.hip
// The forward layer of few rows, a short contraction or little work (as_rows), straight
// from the operands as they lie (any pitch and alignment, no workspace).
constexpr int kFewRows = 32;
bool as_rows(const Shape &s, bool gated);
hipError_t run_rows(const Shape &s, bool gated, const void *X, const void *W,
                        const void *bias, const void *res, void *Y, void *Z, hipStream_t st);

// ------------------------------------------------------ small_gradients.hip
// The gradients of a small layer (small_gradients) in one launch, straight
// from the operands as they lie, without a workspace.
bool small_gradients(const Shape &s, bool gated);
hipError_t run_small_gradients(const Shape &s, bool gated, const void *dY, const void *X,
                               const void *W, const void *Z, void *dX, void *dW, void *db,
                               hipStream_t st);

// ------------------------------------------------------ orthogonalize.hip
// x times a positive factor whose float may overflow or vanish (1 / norm over
// float32's range of matrices): as a mantissa in [1/2, 1) and a power of two
struct Wide {
    float mantissa;
    int power;
    __device__ __forceinline__ Wide(double factor)
    {
        mantissa = (float)frexp(factor, &power);
    }
    __device__ __forceinline__ float times(float x) const { return ldexpf(x, power) * mantissa; }
};
struct Polar {
    int64_t batch, m, n;
    int dtype, steps;
    float a, b, c;
    double eps;
};
// the optimiser step around it
struct MuonStep {
    float lr, momentum, decay, scale;
    int nesterov;
};
size_t polar_ws(const Polar &p);           // 0 for what polar_small.hip takes
bool polar_small(const Polar &p);
hipError_t run_polar_small(const Polar &p, const MuonStep *h, void *out, const void *G, float *M,
                           hipStream_t st);
hipError_t run_orthogonalize(const Polar &p, const void *G, void *O, void *ws, hipStream_t st);
hipError_t run_muon(const Polar &p, const MuonStep &h, void *W, const void *G, float *M,
                    void *ws, hipStream_t st);

} // namespace gpic
