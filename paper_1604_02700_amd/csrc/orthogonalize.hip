// Orthogonalised updates: Newton-Schulz iterates of a matrix on its
// smaller side,
//   X_0 = U / (|U|_F + eps),  A = X X^T (X^T X for a tall X),
//   X <- a X + (b A + c A^2) X  (on the right for a tall X),
// and the optimiser step W <- decay W - step X around them.  Per step two
// symmetric products (the upper triangle of tiles, mirrored) and one full
// one (product.h), all on the half-precision matrix cores.  4,096 squared in
// bfloat16: a step 89 + 11 us (A, its join), 91 + 12 (b A + c A^2), 135 (X); 2,048 x
// 8,192 in float32: 120 + 10, 49, 172.
//
// Precision.  The quintic has slope a at 0 (3.4 for the usual
// coefficients) and is applied `steps` times, so what is rounded off X in
// its small singular directions grows by a^steps against them.
//   float32 and float16 matrices: X, A and b A + c A^2 are split halves, 22
//   bits, all products of split operands (error as float32's own).
//   bfloat16 matrices: the products read half-precision X, A, b A + c A^2
//   (11 bits; the values are bounded, so halves lose nothing to bfloat16's
//   range and carry 3 more bits), and X keeps the low half beside it for the
//   term a X, which carries the small directions: with X rounded to 11 bits
//   there too, a gradient of low rank over noise comes out 1.4e-2 off, with
//   8 bits 1.1e-1, so 1.1e-4 (512 x 2048, float64 reference).  The final
//   rounding (1.7e-3) apart, Gaussian matrices are 1.9e-3 off at 160 x 700, 1.7e-3
//   at 512 x 2,048, 1.3e-3 at 1,024 x 4,096, 1.2e-3 at 2,048 squared, gradients of
//   a decaying spectrum 1.4e-3 to 0.6e-3: the fewer directions, the less the
//   roundings average out.  Up to 128 rows (columns) they are split as the others
//   are (2.1e-3 off in halves at 65 x 300, 1.9e-3 at 128 x 300, 1e-6 split), for
//   99 us instead of 84 and 105 instead of 87; at 512 x 2,048 it would be 192
//   instead of 156, at 1,024 x 4,096 434 instead of 281.
// The norm is summed in float64.
#include "encoder.h"

namespace gpic {

namespace {

constexpr int kParts = 1024;           // partial sums of squares per matrix
constexpr int64_t kSplitSide = 128;    // bfloat16: split operands up to this smaller side
constexpr float kStore = 1024.0f;      // X, A, P are stored times this: entries of
                                       // each are at most 60 for the coefficients and
                                       // steps that the entry points accept (1.3 and
                                       // 2.8 for the usual ones)

inline size_t up(size_t x) { return (x + 255) & ~(size_t)255; }
__host__ __device__ inline int64_t up64(int64_t x) { return (x + 63) & ~(int64_t)63; }

struct Input {
    const void *G;
    float *M;              // null: U = G
    float momentum;
    int nesterov;
    int64_t m, n;
};

using loose4 = f32x4 __attribute__((aligned(4)));

// U of one entry, M advanced already
__device__ __forceinline__ float u_of(float g, float mom, const Input &in)
{
    return in.nesterov ? g + in.momentum * mom : mom;
}

// Sum of squares of U (float64, partial per workgroup); with a momentum
// also M <- momentum M + G, in place.  Bound by memory: 16-byte accesses at
// whatever alignment the matrix of the stack has.  4,096 squared in bfloat16
// (34 MB, from the caches) 11 us; 2,048 x 8,192 in float32 with a momentum (201
// MB) 35 us, 5.7 TB/s.
template <int DT, bool STEP>
__global__ __launch_bounds__(256) void norm_kernel(Input in, double *part)
{
    const int64_t size = in.m * in.n, z0 = (int64_t)blockIdx.y * size;
    const int64_t stride = (int64_t)gridDim.x * 1024;
    double t = 0.0;
    int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
#pragma unroll 4
    for (; i + 4 <= size; i += stride) {
        f32x4 u = load4(in.G, z0 + i, DT);
        if (STEP) {
            loose4 *pm = reinterpret_cast<loose4 *>(in.M + z0 + i);
            const f32x4 mo = *pm * in.momentum + u;
            *pm = mo;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                u[j] = u_of(u[j], mo[j], in);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            t += (double)u[j] * (double)u[j];
    }
    for (; i < size; i = size) {                      // the last one to three entries
        for (int64_t k = i; k < size; ++k) {
            float u = load1(in.G, z0 + k, DT);
            if (STEP) {
                const float mo = in.M[z0 + k] * in.momentum + u;
                in.M[z0 + k] = mo;
                u = u_of(u, mo, in);
            }
            t += (double)u * (double)u;
        }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
        t += __shfl_xor(t, o, 64);
    __shared__ double w[4];
    if ((threadIdx.x & 63) == 0)
        w[threadIdx.x >> 6] = t;
    __syncthreads();
    if (threadIdx.x == 0)
        part[(int64_t)blockIdx.y * kParts + blockIdx.x] = ((w[0] + w[1]) + w[2]) + w[3];
}

struct Planes {
    _Float16 *hi, *lo;     // lo null: split matrix
    int64_t ld, batch;
};

// X_0 = U / (|U|_F + eps) in 16-bit parts, zeros in the padding of both
// buffers' rows.  Four columns a thread.  Bound by memory: 2,048 x 8,192 in
// float32 with a momentum (201 MB) 33 us, 6.1 TB/s.
template <int DT, bool STEP>
__global__ __launch_bounds__(256) void start_kernel(Input in, const double *part, int parts,
                                                    double eps, Planes x0, Planes x1)
{
    __shared__ double w[4];
    double t = 0.0;
    for (int i = threadIdx.x; i < parts; i += 256)
        t += part[(int64_t)blockIdx.y * kParts + i];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
        t += __shfl_xor(t, o, 64);
    if ((threadIdx.x & 63) == 0)
        w[threadIdx.x >> 6] = t;
    __syncthreads();
    const Wide inv((double)kStore / (sqrt(((w[0] + w[1]) + w[2]) + w[3]) + eps));
    const int64_t z = blockIdx.y, z0 = z * in.m * in.n;
    const int64_t quads = up64(in.n) / 4, total = in.m * quads;
    const bool split = x0.lo == nullptr;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total;
         i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / quads, c = (i - r * quads) * 4;
        f32x4 u = {0.0f, 0.0f, 0.0f, 0.0f};
        const int64_t at = z0 + r * in.n + c;
        if (c + 4 <= in.n) {
            u = load4(in.G, at, DT);
            if (STEP) {
                const f32x4 mo = *reinterpret_cast<const loose4 *>(in.M + at);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    u[j] = u_of(u[j], mo[j], in);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (c + j < in.n) {
                    u[j] = load1(in.G, at + j, DT);
                    if (STEP)
                        u[j] = u_of(u[j], in.M[at + j], in);
                }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            u[j] = inv.times(u[j]);
        const half4 h = __builtin_convertvector(u, half4);
        const half4 l = __builtin_convertvector(u - __builtin_convertvector(h, f32x4), half4);
        const int64_t o = z * x0.batch + r * x0.ld + (split ? split_at(c) : c);
        *reinterpret_cast<half4 *>(x0.hi + o) = h;
        *reinterpret_cast<half4 *>((split ? x0.hi + 32 : x0.lo) + o) = l;
        if (c + 4 > in.n) {            // padding of the other buffer (its rest is written later)
            const half4 zero = {0, 0, 0, 0};
            *reinterpret_cast<half4 *>(x1.hi + o) = zero;
            *reinterpret_cast<half4 *>((split ? x1.hi + 32 : x1.lo) + o) = zero;
        }
    }
}

struct Layout {
    bool split, tall;
    int64_t r, len;        // smaller and larger side
    int64_t ldx, lds;      // pitches of X and of the r x r matrices
    Planes x[2], gram, poly;
    double *part;
    float *sums;
    size_t bytes;

    Layout(const Polar &p, char *base)
    {
        size_t at = 0;
        auto take = [&](size_t b) {
            char *q = base ? base + at : nullptr;
            at += up(b);
            return q;
        };
        split = p.dtype != GPIC_BF16 || p.m <= kSplitSide || p.n <= kSplitSide;
        tall = p.m > p.n;
        r = tall ? p.n : p.m;
        len = tall ? p.m : p.n;
        ldx = up64(p.n) * (split ? 2 : 1);
        lds = up64(r) * (split ? 2 : 1);
        part = reinterpret_cast<double *>(take((size_t)p.batch * kParts * 8));
        for (Planes &q : x) {
            q.ld = ldx;
            q.batch = p.m * ldx;
            q.hi = reinterpret_cast<_Float16 *>(take((size_t)(p.batch * q.batch) * 2));
            q.lo = split ? nullptr : reinterpret_cast<_Float16 *>(take((size_t)(p.batch * q.batch) * 2));
        }
        for (Planes *q : {&gram, &poly}) {
            q->ld = lds;
            q->batch = r * lds;
            q->hi = reinterpret_cast<_Float16 *>(take((size_t)(p.batch * q->batch) * 2));
            q->lo = nullptr;
        }
        const int op = split ? kOpSplit : kOpF16;
        const int64_t b = p.batch;
        size_t most = product_plan(r, r, len, b, op, kEpiGram).part_bytes;
        const size_t s1 = product_plan(r, r, r, b, op, kEpiGram).part_bytes;
        const size_t s2 = product_plan(p.m, p.n, r, b, op, kEpiUpdate).part_bytes;
        most = s1 > most ? s1 : most;
        most = s2 > most ? s2 : most;
        sums = reinterpret_cast<float *>(take(most));
        bytes = at;
    }
};

Operand operand(const Planes &p) { return Operand{p.hi, p.ld, p.batch, p.ld}; }

#define RUN(expr)                                                              \
    do {                                                                       \
        hipError_t e_ = (expr);                                                \
        if (e_ != hipSuccess)                                                  \
            return e_;                                                         \
    } while (0)

template <int DT, bool STEP>
hipError_t launch_start(const Polar &p, const Input &in, const Layout &L, hipStream_t st)
{
    int64_t parts = (p.m * p.n + 4095) / 4096;
    parts = parts > kParts ? kParts : parts;
    norm_kernel<DT, STEP><<<dim3((unsigned)parts, (unsigned)p.batch), 256, 0, st>>>(in, L.part);
    RUN(hipGetLastError());
    int64_t blocks = (p.m * (up64(p.n) / 4) + 255) / 256;
    blocks = blocks > 4096 ? 4096 : blocks;
    start_kernel<DT, STEP><<<dim3((unsigned)blocks, (unsigned)p.batch), 256, 0, st>>>(
        in, L.part, (int)parts, p.eps, L.x[0], L.x[1]);
    return hipGetLastError();
}

template <int DT>
hipError_t launch_start(const Polar &p, const Input &in, const Layout &L, hipStream_t st)
{
    return in.M ? launch_start<DT, true>(p, in, L, st) : launch_start<DT, false>(p, in, L, st);
}

hipError_t iterate(const Polar &p, const Input &in, void *out, const MuonStep *h, void *ws,
                   hipStream_t st)
{
    if (p.batch == 0)
        return hipSuccess;
    Layout L(p, static_cast<char *>(ws));
    const int op = L.split ? kOpSplit : kOpF16;
    const int64_t size = p.m * p.n;
    RUN(p.dtype == GPIC_F32    ? launch_start<GPIC_F32>(p, in, L, st)
        : p.dtype == GPIC_F16 ? launch_start<GPIC_F16>(p, in, L, st)
                              : launch_start<GPIC_BF16>(p, in, L, st));
    const float inv2 = 1.0f / (kStore * kStore);
    for (int k = 0; k < p.steps; ++k) {
        const Planes &x = L.x[k & 1], &y = L.x[(k + 1) & 1];
        const bool last = k + 1 == p.steps;
        ProductArgs a{};
        a.batch = (int)p.batch;
        a.part = L.sums;
        a.e.store_scale = kStore;
        a.e.load_scale = 1.0f / kStore;
        // A = X X^T (X^T X)
        a.A = a.B = operand(x);
        a.M = a.N = (int)L.r;
        a.K = L.len;
        a.e.alpha = inv2;
        a.e.p_hi = L.gram.hi;
        a.e.ldp = L.lds;
        a.e.batch_p = L.gram.batch;
        RUN(launch_product(L.tall ? kMM : kKK, op, kEpiGram, a, st));
        // P = b A + c A A
        a.A = a.B = operand(L.gram);
        a.K = L.r;
        a.e.alpha = p.c * inv2;
        a.e.beta = p.b;
        a.e.c_hi = L.gram.hi;
        a.e.p_hi = L.poly.hi;
        RUN(launch_product(kKK, op, kEpiPoly, a, st));
        // X' = a X + P X (a X + X P)
        a.A = operand(L.tall ? x : L.poly);
        a.B = operand(L.tall ? L.poly : x);
        a.M = (int)p.m;
        a.N = (int)p.n;
        a.e.alpha = inv2;
        a.e.beta = p.a;
        a.e.c_hi = x.hi;
        a.e.c_lo = x.lo;
        a.e.p_hi = y.hi;
        a.e.p_lo = y.lo;
        a.e.ldp = L.ldx;
        a.e.batch_p = x.batch;
        if (last) {
            a.e.out = out;
            a.e.dtype = p.dtype;
            a.e.ldo = p.n;
            a.e.batch_o = size;
            if (h) {
                a.e.is_step = 1;
                a.e.decay = 1.0f - h->lr * h->decay;
                a.e.step = h->lr * h->scale;
            }
        }
        RUN(launch_product(L.tall ? kKK : kKM, op, last ? kEpiResult : kEpiUpdate, a, st));
    }
    return hipSuccess;
}

} // namespace

size_t polar_ws(const Polar &p)
{
    return polar_small(p) ? 0 : Layout(p, nullptr).bytes;
}

hipError_t run_orthogonalize(const Polar &p, const void *G, void *O, void *ws, hipStream_t st)
{
    if (polar_small(p))
        return p.batch ? run_polar_small(p, nullptr, O, G, nullptr, st) : hipSuccess;
    Input in{};
    in.G = G;
    in.m = p.m;
    in.n = p.n;
    return iterate(p, in, O, nullptr, ws, st);
}

hipError_t run_muon(const Polar &p, const MuonStep &h, void *W, const void *G, float *M, void *ws,
                    hipStream_t st)
{
    if (polar_small(p))
        return p.batch ? run_polar_small(p, &h, W, G, M, st) : hipSuccess;
    Input in{};
    in.G = G;
    in.M = M;
    in.momentum = h.momentum;
    in.nesterov = h.nesterov;
    in.m = p.m;
    in.n = p.n;
    return iterate(p, in, W, &h, ws, st);
}

} // namespace gpic
