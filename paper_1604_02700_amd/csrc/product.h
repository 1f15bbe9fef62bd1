// The tiled matrix product of the encoder operators (device code, one
// instantiation per tile, operand order, operand kind and epilogue).
//
// out[i][j] = epilogue(sum_k A(i, k) B(j, k)).  A workgroup owns a BM x BN
// tile; per step of the contraction it copies 64 x (BM + BN) 16-bit values
// straight from memory into LDS (16 bytes a lane, no registers in between)
// into one of two buffers while the waves multiply out of the other: one
// barrier a step.  A step is two slabs of 32 values of k.  For split
// operands (float32 values as hi + lo halves) the slabs are the hi and the
// lo parts of the same 32 values, and three of the four slab products are
// summed (lo lo is below 2^-22 of the product); otherwise they are 64
// values of k and two slab products are.
//
// LDS layouts (16-byte chunks; the copies write lane after lane, so the
// permutation is applied to the addresses that the lanes read):
//   k-contiguous operand: a row of the tile is 128 bytes (its 64 values of
//     the step); chunk c of row r lies at chunk c ^ ((r >> 1) & 7): the 16
//     rows that a fragment read touches fall on 16 different chunks of the
//     256 bytes that the banks span.
//   k-strided operand: a slab's row is one k, BM (BN) values wide; pairs of
//     chunks are permuted by bits of k so that the eight rows that half a
//     wave reads at once fall on different 32-byte pieces; fragments are
//     formed by the transposing LDS read.
// The B side is the first operand of the matrix instruction, so that a lane
// holds four consecutive columns j of one row i.
#pragma once

#include "encoder.h"

namespace gpic {
namespace {

__device__ __forceinline__ uint32_t uniform(uint32_t x)
{
    return (uint32_t)__builtin_amdgcn_readfirstlane((int)x);
}

// 64 lanes x 16 bytes from rsrc + voff (zero beyond its end) to LDS at
// lds + 16 * lane.  Asynchronous: counted by vmcnt, waited for by
// `copies_done`; no destination register.
__device__ __forceinline__ void copy_to_lds(u32x4 rsrc, uint32_t voff, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %0\n\t"
                 "s_nop 0\n\t"
                 "buffer_load_dwordx4 %1, %2, 0 offen lds"
                 :
                 : "s"(lds), "v"(voff), "s"(rsrc)
                 : "memory", "m0");
}

// this wave's copies have landed, and its LDS reads have returned
__device__ __forceinline__ void copies_done()
{
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
}

__device__ __forceinline__ uint32_t lds_address(const void *p)
{
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char *)p;
}

__device__ __forceinline__ u32x4 make_rsrc(const char *base, int64_t bytes)
{
    const uint64_t b = (uint64_t)base;
    const int64_t n = bytes < 0 ? 0 : (bytes > 0xfffffff0ll ? 0xfffffff0ll : bytes);
    u32x4 r;
    r[0] = uniform((uint32_t)b);
    r[1] = uniform((uint32_t)(b >> 32) & 0xffffu);
    r[2] = uniform((uint32_t)n);
    r[3] = 0x00020000u;
    return r;
}

constexpr uint32_t kOutside = 0xfffffff0u;      // an offset beyond any buffer

// bits of k that permute the chunk pairs of a k-strided row of `width`
template <int width>
__device__ __forceinline__ int pair_swizzle(int k)
{
    if (width >= 128)
        return (k & 3) | ((k >> 1) & 4);
    return ((k >> 1) & 1) | ((k >> 2) & 2);
}

// One operand's side of a tile: EXT rows (or columns) of it.
template <int EXT, bool STRIDED, bool SPLIT, int NT>
struct Side {
    static constexpr int kBytes = EXT * 128;              // LDS bytes of one step
    static constexpr int kCopies = kBytes / (NT * 16);    // copies a wave issues
    uint32_t voff[kCopies];
    const char *base;
    int64_t left;             // bytes from base to the end of the operand
    int64_t advance;          // bytes of one step

    // row0: first row of the tile; rows: of the whole operand.  row_of(r):
    // the operand's row of the tile's row r (k-contiguous only).
    template <class RowOf>
    __device__ void init(const Operand &o, int64_t z, int64_t row0, int64_t rows, int64_t K,
                         int64_t k0, RowOf row_of)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        const char *p = static_cast<const char *>(o.p) + z * o.batch * 2;
        if (!STRIDED) {
            // k0: first value of the contraction; split rows hold 2 values each
            const int64_t at = SPLIT ? 2 * k0 : k0;
            base = p + at * 2;
            left = ((rows - 1) * o.ld + o.cols - at) * 2;
            advance = 128;
#pragma unroll
            for (int c = 0; c < kCopies; ++c) {
                const int r = (wave * kCopies + c) * 8 + (lane >> 3);
                const int chunk = (lane & 7) ^ ((r >> 1) & 7);
                const int64_t row = row_of(row0, r);
                voff[c] = row < rows ? (uint32_t)((row - row_of(row0, 0)) * o.ld * 2 + chunk * 16)
                                     : kOutside;
            }
            const int64_t first = row_of(row0, 0) * o.ld * 2;
            base += first;
            left -= first;
        } else {
            base = p + (k0 * o.ld + (SPLIT ? split_at(row0) : row0)) * 2;
            left = ((K - 1 - k0) * o.ld + o.cols - (SPLIT ? split_at(row0) : row0)) * 2;
            advance = (SPLIT ? 32 : 64) * o.ld * 2;
            constexpr int kChunks = EXT / 8;              // chunks of a slab's row
            constexpr int kRows = 64 / kChunks;           // rows a copy covers
#pragma unroll
            for (int c = 0; c < kCopies; ++c) {
                const int r = (wave * kCopies + c) * kRows + lane / kChunks;    // 0 .. 63
                const int k = r & 31, slab = r >> 5;
                const int pos = lane % kChunks;
                const int chunk = (((pos >> 1) ^ pair_swizzle<EXT>(k)) << 1) | (pos & 1);
                uint32_t v;
                int64_t col;              // first value of the chunk in the row
                if (SPLIT) {
                    v = (uint32_t)(k * o.ld * 2) + ((chunk >> 2) * 8 + slab * 4 + (chunk & 3)) * 16;
                    col = split_at(row0) + ((chunk >> 2) * 8 + slab * 4 + (chunk & 3)) * 8;
                } else {
                    v = (uint32_t)((slab * 32 + k) * o.ld * 2) + chunk * 16;
                    col = row0 + chunk * 8;
                }
                // beyond the row: the next row's values, never used, but
                // kept out so that nothing outside the operand is read
                voff[c] = col < o.cols ? v : kOutside;
            }
        }
    }

    // issue the copies of one step; kleft: values of k that are left
    __device__ __forceinline__ void copy(uint32_t lds, int64_t kleft) const
    {
        const u32x4 rsrc = make_rsrc(base, left);
        const int wave = threadIdx.x >> 6;
        const uint32_t at = lds + (uint32_t)wave * (kCopies * 1024);
        if (!STRIDED && !SPLIT && kleft < 64) {
            const int lane = threadIdx.x & 63;
#pragma unroll
            for (int c = 0; c < kCopies; ++c) {
                const int r = (wave * kCopies + c) * 8 + (lane >> 3);
                const int chunk = (lane & 7) ^ ((r >> 1) & 7);
                copy_to_lds(rsrc, chunk * 8 < kleft ? voff[c] : kOutside, uniform(at + c * 1024));
            }
        } else {
#pragma unroll
            for (int c = 0; c < kCopies; ++c)
                copy_to_lds(rsrc, voff[c], uniform(at + c * 1024));
        }
    }
    __device__ __forceinline__ void step()
    {
        base += advance;
        left -= advance;
    }
};

// Fragment of 16 rows at `row` (a multiple of 16 within the tile) of slab s.
template <int EXT, bool STRIDED>
__device__ __forceinline__ u32x4 fragment(const char *tile, int s, int row)
{
    const int lane = threadIdx.x & 63, g = lane >> 4, i = lane & 15;
    if (!STRIDED) {
        const int chunk = (s * 4 + g) ^ ((i >> 1) & 7);
        return *reinterpret_cast<const u32x4 *>(tile + (row + i) * 128 + chunk * 16);
    }
    using lds4 = __attribute__((address_space(3))) s16x4;
    const int k = 8 * g + (i >> 2);
    const int pair = (row >> 4) ^ pair_swizzle<EXT>(k);
    const char *p = tile + s * (EXT * 64) + k * (EXT * 2) + pair * 32 + (i & 3) * 8;
    // pair_swizzle does not look at bit 2 of k, so the second four rows of k
    // lie 4 rows further at the same place
    union {
        s16x4 h[2];
        u32x4 v;
    } u;
    u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(p));
    u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(p + 4 * EXT * 2));
    return u.v;
}

template <int OP>
__device__ __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c)
{
    if (OP == kOpBf16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bfrag8, a),
                                                       __builtin_bit_cast(bfrag8, b), c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a),
                                                  __builtin_bit_cast(half8, b), c, 0, 0, 0);
}

// --------------------------------------------------------------- epilogue
__device__ __forceinline__ int64_t part_at(const Epilogue &e, int64_t row, int64_t col)
{
    return row * e.ldp + (e.is_split ? split_at(col) : col);
}

__device__ __forceinline__ void store_parts(const Epilogue &e, int64_t z, int64_t row, int64_t col,
                                            f32x4 v)
{
    const int64_t at = z * e.batch_p + part_at(e, row, col);
    _Float16 *hi = static_cast<_Float16 *>(e.p_hi) + at;
    v *= e.store_scale;
    const half4 h = __builtin_convertvector(v, half4);
    *reinterpret_cast<half4 *>(hi) = h;
    if (e.is_split || e.p_lo) {
        const half4 l = __builtin_convertvector(v - __builtin_convertvector(h, f32x4), half4);
        _Float16 *lo = e.is_split ? hi + 32 : static_cast<_Float16 *>(e.p_lo) + at;
        *reinterpret_cast<half4 *>(lo) = l;
    }
}

__device__ __forceinline__ f32x4 load_parts(const Epilogue &e, int64_t z, int64_t row, int64_t col)
{
    const int64_t at = z * e.batch_p + part_at(e, row, col);
    const _Float16 *hi = static_cast<const _Float16 *>(e.c_hi) + at;
    f32x4 v = __builtin_convertvector(*reinterpret_cast<const half4 *>(hi), f32x4);
    if (e.is_split || e.c_lo) {
        const _Float16 *lo = e.is_split ? hi + 32 : static_cast<const _Float16 *>(e.c_lo) + at;
        v += __builtin_convertvector(*reinterpret_cast<const half4 *>(lo), f32x4);
    }
    return v * e.load_scale;
}

__device__ __forceinline__ void scaled(const Epilogue &e, f32x4 &v)
{
    if (e.sa)
        v *= 1.0f / *e.sa;                // powers of two: exact
    if (e.sb)
        v *= 1.0f / *e.sb;
    v *= e.alpha;
}

// Four consecutive columns col .. col + 3 (col % 4 == 0) of one row.
// mirror (kEpiSym): also the transposed four.
template <int EPI>
__device__ __forceinline__ void finish4(const Epilogue &e, int64_t z, int64_t row, int64_t col,
                                        int M, int N, f32x4 v, bool mirror)
{
    // the vector and the scalar paths round alike
#pragma clang fp contract(off)
    scaled(e, v);
    if (EPI == kEpiLayer) {
        const bool whole = e.vec && col + 4 <= N;
        if (whole) {
            if (e.bias)
                v += load4(e.bias, col, e.dtype);
            if (e.pre)
                store4(e.pre, row * e.ldz + col, v, e.dtype);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                v[j] = activate(v[j], e.act);
            if (e.res)
                v += load4(e.res, row * e.ldr + col, e.dtype);
            store4(e.out, row * e.ldo + col, v, e.dtype);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int64_t c = col + j;
                if (c >= N)
                    continue;
                float x = v[j];
                if (e.bias)
                    x += load1(e.bias, c, e.dtype);
                if (e.pre)
                    store1(e.pre, row * e.ldz + c, x, e.dtype);
                x = activate(x, e.act);
                if (e.res)
                    x += load1(e.res, row * e.ldr + c, e.dtype);
                store1(e.out, row * e.ldo + c, x, e.dtype);
            }
        }
    } else if (EPI == kEpiSym) {
        // columns N .. up to a multiple of 64 hold zeros: the products
        // over this matrix read whole steps of k
        if (e.c_hi)
            v = e.beta * load_parts(e, z, row, col) + v;
        store_parts(e, z, row, col, v);
        if (mirror) {
            v *= e.store_scale;
            const int64_t at = z * e.batch_p;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (col + j >= N)
                    continue;
                const int64_t p = at + part_at(e, col + j, row);
                const _Float16 h = (_Float16)v[j];
                static_cast<_Float16 *>(e.p_hi)[p] = h;
                if (e.is_split)
                    static_cast<_Float16 *>(e.p_hi)[p + 32] = (_Float16)(v[j] - (float)h);
            }
        }
    } else if (EPI == kEpiUpdate) {
        v += e.beta * load_parts(e, z, row, col);
        if (!e.to_out) {
            store_parts(e, z, row, col, v);
            return;
        }
        const int64_t o = z * e.batch_o + row * e.ldo + col;
        if (e.vec && col + 4 <= N) {
            if (e.is_step)
                v = e.decay * load4(e.out, o, e.dtype) - e.step * v;
            store4(e.out, o, v, e.dtype);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (col + j >= N)
                    continue;
                float x = v[j];
                if (e.is_step)
                    x = e.decay * load1(e.out, o + j, e.dtype) - e.step * x;
                store1(e.out, o + j, x, e.dtype);
            }
        }
    }
}

// Four columns of the gated layer: gate g and up u of the same columns.
__device__ __forceinline__ void finish4_gated(const Epilogue &e, int64_t row, int64_t col, f32x4 g,
                                              f32x4 u)
{
#pragma clang fp contract(off)
    scaled(e, g);
    scaled(e, u);
    if (e.vec && col + 4 <= e.half) {
        if (e.pre) {
            store4(e.pre, row * e.ldz + col, g, GPIC_F32);
            store4(e.pre, row * e.ldz + e.half + col, u, GPIC_F32);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            g[j] = activate(g[j], e.act) * u[j];
        store4(e.out, row * e.ldo + col, g, e.dtype);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t c = col + j;
            if (c >= e.half)
                continue;
            if (e.pre) {
                store1(e.pre, row * e.ldz + c, g[j], GPIC_F32);
                store1(e.pre, row * e.ldz + e.half + c, u[j], GPIC_F32);
            }
            store1(e.out, row * e.ldo + c, activate(g[j], e.act) * u[j], e.dtype);
        }
    }
}

// ----------------------------------------------------------------- kernel
// Tile of 16 WM RM x 16 WN RN (WM x WN waves of RM x RN fragments each).
template <int WM, int WN, int RM, int RN>
struct Tile {
    static constexpr int kWM = WM, kWN = WN, kRM = RM, kRN = RN;
    static constexpr int kBM = 16 * WM * RM, kBN = 16 * WN * RN;
    static constexpr int kThreads = 64 * WM * WN;
};

// Which tile a workgroup takes: consecutive ids go round the 8 compute
// dies, so each die gets one contiguous run of tiles, walked in bands of 8
// tile rows (its second-level cache then holds the band's A and a few
// columns of B).  Symmetric products count the upper triangle's tiles by rows.
__device__ __forceinline__ void which_tile(int id, int count, int tm, int tn, bool sym, int &ti,
                                           int &tj)
{
    const int per = count / 8, extra = count % 8, die = id % 8, k = id / 8;
    id = die * per + (die < extra ? die : extra) + k;
    if (sym) {
        // rows of tn, tn - 1, .. tiles: row i starts at i tn - i (i - 1) / 2
        const float b = 2.0f * tn + 1.0f;
        int i = (int)((b - sqrtf(b * b - 8.0f * id)) * 0.5f);
        i = i < 0 ? 0 : (i >= tn ? tn - 1 : i);
        while (i > 0 && i * tn - i * (i - 1) / 2 > id)
            --i;
        while (i + 1 < tn && (i + 1) * tn - (i + 1) * i / 2 <= id)
            ++i;
        ti = i;
        tj = i + (id - (i * tn - i * (i - 1) / 2));
        return;
    }
    const int band = id / (8 * tn), first = band * 8;
    const int rows = tm - first < 8 ? tm - first : 8;
    const int in = id - band * 8 * tn;
    ti = first + in % rows;
    tj = in / rows;
}

template <class T, bool ASTR, bool BSTR, int OP, int EPI>
__global__ __launch_bounds__(T::kThreads) void product_kernel(ProductArgs a, int tm, int tn)
{
    constexpr bool SPLIT = OP == kOpSplit;
    constexpr int kStep = SPLIT ? 32 : 64;           // values of k per step
    using SideA = Side<T::kBM, ASTR, SPLIT, T::kThreads>;
    using SideB = Side<T::kBN, BSTR, SPLIT, T::kThreads>;
    constexpr int kBuf = SideA::kBytes + SideB::kBytes;
    __shared__ __attribute__((aligned(1024))) char lds[2 * kBuf];

    int ti, tj;
    which_tile(blockIdx.x, gridDim.x, tm, tn, EPI == kEpiSym, ti, tj);
    const int64_t z = blockIdx.y;
    const int64_t row0 = (int64_t)ti * T::kBM;
    const int64_t col0 = (int64_t)tj * T::kBN;
    const int split = blockIdx.z;
    // this part's steps of the contraction
    const int64_t steps = (a.K + kStep - 1) / kStep;
    const int64_t s0 = steps * split / a.splits, s1 = steps * (split + 1) / a.splits;

    SideA sa;
    SideB sb;
    sa.init(a.A, z, row0, a.M, a.K, s0 * kStep, [](int64_t r0, int r) { return r0 + r; });
    if (EPI == kEpiGated) {
        // rows of B in turn 16 of the gate's and the up projection's 16 of
        // the same columns, so that both meet in one lane.  Rows at or
        // beyond `half` in the gate's half are not wanted: outside.
        const int64_t half = a.e.half, j0 = col0 / 2, all = a.N;
        sb.init(a.B, z, j0, all, a.K, s0 * kStep, [half, all](int64_t r0, int r) {
            const int64_t c = r0 + (r >> 5) * 16 + (r & 15);
            return c >= half ? all : ((r & 16) ? half + c : c);
        });
    } else {
        sb.init(a.B, z, col0, a.N, a.K, s0 * kStep, [](int64_t r0, int r) { return r0 + r; });
    }

    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int wm = (wave / T::kWN) * (16 * T::kRM), wn = (wave % T::kWN) * (16 * T::kRN);
    f32x4 acc[T::kRM][T::kRN];
#pragma unroll
    for (int i = 0; i < T::kRM; ++i)
#pragma unroll
        for (int j = 0; j < T::kRN; ++j)
            acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    const uint32_t lds0 = lds_address(lds);
    int64_t kleft = a.K - s0 * kStep;
    if (s1 > s0) {
        sa.copy(lds0, kleft);
        sb.copy(lds0 + SideA::kBytes, kleft);
    }
    for (int64_t s = s0; s < s1; ++s) {
        const int cur = (int)(s - s0) & 1;
        // this step's copies have landed in every wave's view, and nobody
        // reads the other buffer any more
        copies_done();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (s + 1 < s1) {
            sa.step();
            sb.step();
            kleft -= kStep;
            const uint32_t to = lds0 + (uint32_t)(cur ^ 1) * kBuf;
            sa.copy(to, kleft);
            sb.copy(to + SideA::kBytes, kleft);
        }
        const char *ta = lds + cur * kBuf, *tb = ta + SideA::kBytes;
        u32x4 fa[2][T::kRM], fb[2][T::kRN];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int j = 0; j < T::kRN; ++j)
                fb[h][j] = fragment<T::kBN, BSTR>(tb, h, wn + 16 * j);
#pragma unroll
            for (int i = 0; i < T::kRM; ++i)
                fa[h][i] = fragment<T::kBM, ASTR>(ta, h, wm + 16 * i);
        }
#pragma unroll
        for (int i = 0; i < T::kRM; ++i)
#pragma unroll
            for (int j = 0; j < T::kRN; ++j) {
                acc[i][j] = mma<OP>(fb[0][j], fa[0][i], acc[i][j]);
                if (SPLIT)
                    acc[i][j] = mma<OP>(fb[1][j], fa[0][i], acc[i][j]);
            }
#pragma unroll
        for (int i = 0; i < T::kRM; ++i)
#pragma unroll
            for (int j = 0; j < T::kRN; ++j)
                acc[i][j] = mma<OP>(fb[SPLIT ? 0 : 1][j], fa[1][i], acc[i][j]);
        asm volatile("" ::: "memory");
    }

    // lane: row i of each fragment, columns 4 g .. 4 g + 3
    const int g4 = (lane >> 4) * 4;
#pragma unroll
    for (int i = 0; i < T::kRM; ++i) {
        const int64_t row = row0 + wm + 16 * i + (lane & 15);
        if (row >= a.M)
            continue;
        if (EPI == kEpiGated) {
#pragma unroll
            for (int j = 0; j < T::kRN; j += 2) {
                const int64_t col = col0 / 2 + (wn + 16 * j) / 2 + g4;
                if (col < a.e.half)
                    finish4_gated(a.e, row, col, acc[i][j], acc[i][j + 1]);
            }
            continue;
        }
#pragma unroll
        for (int j = 0; j < T::kRN; ++j) {
            const int64_t col = col0 + wn + 16 * j + g4;
            const int64_t end = EPI == kEpiSym ? (a.N + 63) / 64 * 64 : a.N;
            if (col >= end)
                continue;
            if (a.splits > 1) {
                const int64_t n4 = (a.N + 63) / 64 * 64;
                float *p = a.part + ((split * a.batch + z) * (int64_t)a.M + row) * n4 + col;
                *reinterpret_cast<f32x4 *>(p) = acc[i][j];
            } else {
                finish4<EPI>(a.e, z, row, col, a.M, a.N, acc[i][j],
                             EPI == kEpiSym && ti != tj);
            }
        }
    }
}

// The parts of a split contraction in order, then the epilogue.  Four
// columns a thread.
template <int EPI>
__global__ __launch_bounds__(256) void product_join_kernel(ProductArgs a, int tile)
{
    const int64_t n4 = (a.N + 63) / 64 * 64, quads = n4 / 4;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t z = blockIdx.y;
    if (id >= a.M * quads)
        return;
    const int64_t row = id / quads, col = (id % quads) * 4;
    const bool lower = EPI == kEpiSym && row / tile > col / tile;
    if (lower || (EPI != kEpiSym && col >= a.N))
        return;                     // symmetric: written by the mirrored tile
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int s = 0; s < a.splits; ++s)
        v += *reinterpret_cast<const f32x4 *>(
            a.part + ((s * a.batch + z) * (int64_t)a.M + row) * n4 + col);
    finish4<EPI>(a.e, z, row, col, a.M, a.N, v,
                 EPI == kEpiSym && row / tile != col / tile);
}

// ------------------------------------------------------------------- host
using TileL = Tile<2, 4, 8, 4>;      // 256 x 256, 8 waves
using TileM = Tile<2, 2, 4, 4>;      // 128 x 128, 4 waves
using TileS = Tile<2, 2, 2, 2>;      // 64 x 64, 4 waves

template <class T, bool ASTR, bool BSTR, int OP, int EPI>
hipError_t launch_tile(const ProductArgs &a, hipStream_t s)
{
    const int64_t tm = ((int64_t)a.M + T::kBM - 1) / T::kBM;
    const int64_t tn = ((int64_t)(EPI == kEpiGated ? 2 * a.e.half : a.N) + T::kBN - 1) / T::kBN;
    const int64_t tiles = EPI == kEpiSym ? tn * (tn + 1) / 2 : tm * tn;
    if (tiles > 0x7fffffffll || a.batch > 65535 || a.splits > 65535)
        return hipErrorInvalidValue;
    product_kernel<T, ASTR, BSTR, OP, EPI>
        <<<dim3((unsigned)tiles, (unsigned)a.batch, (unsigned)a.splits), T::kThreads, 0, s>>>(
            a, (int)tm, (int)tn);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && a.splits > 1) {
        const int64_t quads = (int64_t)a.M * ((a.N + 63) / 64 * 64) / 4;
        product_join_kernel<EPI><<<dim3((unsigned)((quads + 255) / 256), (unsigned)a.batch),
                                   256, 0, s>>>(a, T::kBN);
        e = hipGetLastError();
    }
    return e;
}

} // namespace

// product.hip: the tile for a product (0 = large, 1 = middle, 2 = small)
int product_tile(int M, int N, int64_t K, int batch, int op, bool sym);

namespace {

template <bool ASTR, bool BSTR, int OP, int EPI>
hipError_t launch_any_tile(const ProductArgs &a, hipStream_t s)
{
    const int N = EPI == kEpiGated ? (int)(2 * a.e.half) : a.N;
    switch (product_tile(a.M, N, a.K, a.batch, OP, EPI == kEpiSym)) {
    case 0:
        return launch_tile<TileL, ASTR, BSTR, OP, EPI>(a, s);
    case 1:
        return launch_tile<TileM, ASTR, BSTR, OP, EPI>(a, s);
    default:
        return launch_tile<TileS, ASTR, BSTR, OP, EPI>(a, s);
    }
}

} // namespace
} // namespace gpic
