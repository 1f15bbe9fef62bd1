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

#include <type_traits>

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

// EXT rows (or columns) of one operand, as a tile or a part of one reads
// them.  NT: threads that share the copies.  `row_of(r)`: the operand's row
// of the part's row r, for r a multiple of 8 plus what is added to both
// (k-strided: chunks of 8 stay together).
template <int EXT, bool STRIDED, bool SPLIT, int NT>
struct Side {
    static constexpr int kBytes = EXT * 128;              // LDS bytes of one step
    static constexpr int kCopies = kBytes / (NT * 16);    // copies a wave issues
    uint32_t voff[kCopies];

    template <class RowOf>
    __device__ void init(const Operand &o, int64_t first, int64_t rows, RowOf row_of)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        if (!STRIDED) {
#pragma unroll
            for (int c = 0; c < kCopies; ++c) {
                const int r = (wave * kCopies + c) * 8 + (lane >> 3);
                const int chunk = (lane & 7) ^ ((r >> 1) & 7);
                const int64_t row = row_of(r);
                voff[c] = row < rows ? (uint32_t)((row - first) * o.ld * 2 + chunk * 16) : kOutside;
            }
        } else {
            constexpr int kChunks = EXT / 8;              // chunks of a slab's row
            constexpr int kRows = 64 / kChunks;           // rows a copy covers
#pragma unroll
            for (int c = 0; c < kCopies; ++c) {
                const int r = (wave * kCopies + c) * kRows + lane / kChunks;    // 0 .. 63
                const int k = r & 31, slab = r >> 5;
                const int pos = lane % kChunks;
                const int chunk = (((pos >> 1) ^ pair_swizzle<EXT>(k)) << 1) | (pos & 1);
                const int64_t row = row_of(chunk * 8);
                // 16-bit values from the start of the operand's row k
                const int64_t at = SPLIT ? split_at(row) + slab * 32 : row;
                const int64_t start = SPLIT ? split_at(first) : first;
                // beyond the row: never used, kept inside the operand
                voff[c] = at < o.cols
                              ? (uint32_t)(((SPLIT ? k : slab * 32 + k) * o.ld + at - start) * 2)
                              : kOutside;
            }
        }
    }

    // issue the copies of one step; kleft: values of k that are left
    __device__ __forceinline__ void copy(u32x4 rsrc, uint32_t lds, int64_t kleft) const
    {
        const int wave = threadIdx.x >> 6;
        const uint32_t at = lds + (uint32_t)wave * (kCopies * 1024);
#pragma unroll
        for (int c = 0; c < kCopies; ++c)
            copy_one(rsrc, at, c, kleft);
    }
    __device__ __forceinline__ void copy_one(u32x4 rsrc, uint32_t at, int c, int64_t kleft) const
    {
        uint32_t v = voff[c];
        if (!STRIDED && !SPLIT) {         // the last step may end inside a row's 64 values
            const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
            const int r = (wave * kCopies + c) * 8 + (lane >> 3);
            const int chunk = (lane & 7) ^ ((r >> 1) & 7);
            const int valid = kleft < 64 ? (int)kleft : 64;
            v = chunk * 8 < valid ? v : kOutside;
        }
        copy_to_lds(rsrc, v, uniform(at + c * 1024));
    }
};

// Where one operand's copies of a step start, and what is left of it.
template <bool STRIDED, bool SPLIT>
struct Stream {
    const char *base;
    int64_t left, advance;
    // first: the operand's row (column) that offsets count from; k0: first k
    __device__ void init(const Operand &o, int64_t z, int64_t first, int64_t rows, int64_t K,
                         int64_t k0)
    {
        int64_t at, end;
        if (!STRIDED) {
            at = first * o.ld + (SPLIT ? 2 * k0 : k0);
            end = (rows - 1) * o.ld + o.cols;
            advance = 128;
        } else {
            at = k0 * o.ld + (SPLIT ? split_at(first) : first);
            end = (K - 1) * o.ld + o.cols;
            advance = (SPLIT ? 32 : 64) * o.ld * 2;
        }
        base = static_cast<const char *>(o.p) + (z * o.batch + at) * 2;
        left = (end - at) * 2;
    }
    __device__ __forceinline__ u32x4 rsrc() const { return make_rsrc(base, left); }
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
// A wave's accumulators go through LDS (its own piece, no barrier) so that
// a lane finishes eight consecutive columns of a row: 16-byte loads and
// stores that cover whole lines.
// 16-bit parts of iterates: of split operands one split matrix; of single
// ones a matrix of high halves and, for X (kEpiUpdate, kEpiResult), one of low
// halves beside it.
template <int OP, int EPI>
struct Parts {
    static constexpr bool kSplit = OP == kOpSplit;
    static constexpr bool kLow = !kSplit && (EPI == kEpiUpdate || EPI == kEpiResult);

    static __device__ __forceinline__ int64_t at(const Epilogue &e, int64_t z, int64_t row,
                                                 int64_t col)
    {
        return z * e.batch_p + row * e.ldp + (kSplit ? split_at(col) : col);
    }
    // v (times store_scale already), eight columns
    static __device__ __forceinline__ void store(const Epilogue &e, int64_t at, f32x8 v)
    {
        _Float16 *hi = static_cast<_Float16 *>(e.p_hi) + at;
        const half8 h = __builtin_convertvector(v, half8);
        *reinterpret_cast<half8 *>(hi) = h;
        if (kSplit || kLow) {
            _Float16 *lo = kSplit ? hi + 32 : static_cast<_Float16 *>(e.p_lo) + at;
            *reinterpret_cast<half8 *>(lo) =
                __builtin_convertvector(v - __builtin_convertvector(h, f32x8), half8);
        }
    }
    static __device__ __forceinline__ f32x8 load(const Epilogue &e, int64_t at)
    {
        const _Float16 *hi = static_cast<const _Float16 *>(e.c_hi) + at;
        f32x8 v = __builtin_convertvector(*reinterpret_cast<const half8 *>(hi), f32x8);
        if (kSplit || kLow) {
            const _Float16 *lo = kSplit ? hi + 32 : static_cast<const _Float16 *>(e.c_lo) + at;
            v += __builtin_convertvector(*reinterpret_cast<const half8 *>(lo), f32x8);
        }
        return v * e.load_scale;
    }
};

// What the accumulators are multiplied by: in layers 2^-(row's power +
// column's), both operands' powers of two taken off at once (one after the
// other could overflow or underflow on the way to a result that does
// neither), elsewhere alpha.
using i32x8 = int __attribute__((ext_vector_type(8), aligned(4)));

// the powers of ROWS rows from row0 on, one a lane
template <int ROWS, int OP, int EPI>
__device__ __forceinline__ int row_powers(const Epilogue &e, int64_t row0, int64_t M)
{
    if (OP != kOpBf16 && EPI == kEpiSum)
        return kSoftPower + (OP == kOpF16 && e.pa ? e.pa[0] : 0);
    if (OP == kOpBf16 || !powered(EPI) || !e.pa)
        return 0;
    static_assert(ROWS <= 64, "a row a lane");
    const int64_t row = row0 + (threadIdx.x & 63);
    return e.pa[OP == kOpSplit ? (row < M ? row : M - 1) : 0];
}

// the powers of eight columns, of which `valid` exist
template <int OP, int EPI>
__device__ __forceinline__ i32x8 column_powers(const Epilogue &e, int64_t col, int valid)
{
    i32x8 p = 0;
    if (OP != kOpSplit || !powered(EPI) || !e.pb || valid <= 0)
        return p;
    if (valid >= 8)
        return *reinterpret_cast<const i32x8 *>(e.pb + col);
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < valid)
            p[j] = e.pb[col + j];
    return p;
}

template <int OP, int EPI>
__device__ __forceinline__ f32x8 staged(const float *p, const Epilogue &e, int row, i32x8 columns)
{
    f32x8 v = *reinterpret_cast<const f32x8 *>(p);
    if (!powered(EPI))
        return v * e.alpha;
    if (OP != kOpBf16) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            v[j] = ldexpf(v[j], -(row + columns[j]));
    }
    return v;
}

// The type of what an epilogue reads and writes, known from the operands
// where it can be (orthogonalised matrices of half-precision operands are
// bfloat16, those of split ones float32 or float16).
template <int OP, int EPI>
__device__ __forceinline__ int out_type(const Epilogue &e)
{
    if (EPI == kEpiResult)
        return OP == kOpF16 ? GPIC_BF16
                            : (e.dtype == GPIC_F32 ? GPIC_F32
                                                   : (e.dtype == GPIC_F16 ? GPIC_F16 : GPIC_BF16));
    return OP == kOpSplit ? GPIC_F32 : (OP == kOpF16 ? GPIC_F16 : GPIC_BF16);
}

// Finishes `ROWS` x `COLS` accumulators that the wave has staged at `st`
// (pitch COLS + 4 floats), the output's rows from row0, columns from col0
// (gated: columns from col0 / 2).  mirror (symmetric): the transposed block too.
template <int ROWS, int COLS, int OP, int EPI>
__device__ __forceinline__ void finish_block(const Epilogue &e, int64_t z, int64_t row0,
                                             int64_t col0, int64_t M, int64_t N, float *st,
                                             bool mirror)
{
    // the whole and the partial accesses round alike
#pragma clang fp contract(off)
    const int dtype = out_type<OP, EPI>(e);
    using P = Parts<OP, EPI>;
    constexpr bool kSym = symmetric(EPI);
    constexpr int kPitch = COLS + 4;
    constexpr int kOut = EPI == kEpiGated ? COLS / 2 : COLS;     // output columns
    constexpr int kLanes = kOut / 8, kRowsPass = 64 / kLanes < ROWS ? 64 / kLanes : ROWS;
    constexpr int kPasses = ROWS / kRowsPass;            // lanes beyond the rows do nothing
    constexpr int kGroup = kPasses < 4 ? 1 : 2;                  // rows in flight a lane
    static_assert(kPasses * kRowsPass == ROWS && kPasses % kGroup == 0, "passes");
    const int lane = threadIdx.x & 63, q = lane % kLanes, r0 = lane / kLanes;
    const bool idle = kLanes * kRowsPass < 64 && r0 >= kRowsPass;
    const int powers = row_powers<ROWS, OP, EPI>(e, row0, M);
    if (EPI == kEpiGated) {
        const int64_t col = col0 / 2 + q * 8, half = e.half;
        const int valid = half - col < 8 ? (int)(half - col) : 8;
        const float *src = st + (q >> 1) * 32 + (q & 1) * 8;
        const i32x8 pg = column_powers<OP, EPI>(e, col, valid);
        const i32x8 pu = column_powers<OP, EPI>(e, half + col, valid);
        for (int p = 0; p < kPasses; ++p) {
            const int r = p * kRowsPass + r0;
            const int64_t row = row0 + r;
            const int pr = OP == kOpBf16 ? 0 : __shfl(powers, r & 63, 64);
            if (valid <= 0 || row >= M || idle)
                continue;
            f32x8 g = staged<OP, EPI>(src + r * kPitch, e, pr, pg);
            const f32x8 u = staged<OP, EPI>(src + r * kPitch + 16, e, pr, pu);
            if (e.pre) {
                store8(e.pre, row * e.ldz + col, g, GPIC_F32, valid);
                store8(e.pre, row * e.ldz + half + col, u, GPIC_F32, valid);
            }
            store8(e.out, row * e.ldo + col, activate8(g, e.act) * u, dtype, valid);
        }
        return;
    }
    const int64_t col = col0 + q * 8;
    // 16-bit parts: the padding up to a multiple of 64 columns is written too
    const int64_t end = symmetric(EPI) ? (N + 63) / 64 * 64 : N;
    const int64_t here = end - col;
    const int valid = here < 0 ? 0 : (here < 8 ? (int)here : 8);
    const i32x8 pc = column_powers<OP, EPI>(e, col, valid);
    f32x8 bias = 0.0f;
    if (EPI == kEpiLayer && e.bias && valid > 0)
        bias = load8(e.bias, col, dtype, valid);
    for (int p0 = 0; p0 < kPasses; p0 += kGroup) {
        f32x8 v[kGroup], c[kGroup];
#pragma unroll
        for (int p = 0; p < kGroup; ++p) {
            const int r = (p0 + p) * kRowsPass + r0;
            const int64_t row = row0 + r;
            const int pr = OP == kOpBf16 || !powered(EPI) ? 0 : __shfl(powers, r & 63, 64);
            v[p] = staged<OP, EPI>(st + (idle ? 0 : r) * kPitch + q * 8, e, pr, pc);
            c[p] = 0.0f;
            if (EPI == kEpiPoly || EPI == kEpiUpdate || EPI == kEpiResult) {
                // lanes that finish nothing load the first entry
                const bool live = valid > 0 && row < M && !idle;
                c[p] = P::load(e, live ? P::at(e, z, row, col) : z * e.batch_p) * e.beta;
            }
            if (valid <= 0 || row >= M || idle)
                continue;
            if (EPI == kEpiLayer && e.res)
                c[p] = load8(e.res, row * e.ldr + col, dtype, valid);
            if (EPI == kEpiSum) {
                v[p] = v[p] * e.factor[row * e.factor_step];
                if (e.res)
                    c[p] = load8(e.res, row * e.ldr + col, GPIC_F32, valid);
            }
            if (EPI == kEpiResult && e.is_step) {
                // decay W - step (beta X + acc)
                const f32x8 old = load8(e.out, z * e.batch_o + row * e.ldo + col, dtype, valid);
                c[p] = old * e.decay - c[p] * e.step;
                v[p] = v[p] * -e.step;
            }
        }
#pragma unroll
        for (int p = 0; p < kGroup; ++p) {
            const int r = (p0 + p) * kRowsPass + r0;
            const int64_t row = row0 + r;
            if (valid <= 0 || row >= M || idle)
                continue;
            f32x8 x = v[p];
            if (EPI == kEpiLayer) {
                if (e.bias)
                    x = x + bias;
                if (e.pre)
                    store8(e.pre, row * e.ldz + col, x, dtype, valid);
                x = activate8(x, e.act);
                if (e.res)
                    x = x + c[p];
                store8(e.out, row * e.ldo + col, x, dtype, valid);
            } else if (EPI == kEpiSum) {
                x = x + c[p];
                if (e.last)
                    store8(e.out, row * e.ldo + col, x, dtype, valid);
                else
                    store8(e.out, row * e.ldo + col, x, GPIC_F32, valid);
            } else if (kSym) {
                x = (EPI == kEpiPoly ? x + c[p] : x) * e.store_scale;
                P::store(e, P::at(e, z, row, col), x);
                if (mirror)
                    *reinterpret_cast<f32x8 *>(st + r * kPitch + q * 8) = x;
            } else {
                x = x + c[p];
                if (EPI == kEpiUpdate)
                    P::store(e, P::at(e, z, row, col), x * e.store_scale);
                else
                    store8(e.out, z * e.batch_o + row * e.ldo + col, x, dtype, valid);
            }
        }
    }
}

// The transposed block of what finish_block has left at `st` (times
// store_scale), a lane eight rows of a column; wave `first` of `waves`.  Only
// whole tiles above the diagonal are mirrored, so the rows all exist;
// columns beyond N are padding.
template <int ROWS, int COLS, int OP, int EPI>
__device__ __forceinline__ void mirror_block(const Epilogue &e, int64_t z, int64_t row0,
                                             int64_t col0, int64_t N, const float *st, int first,
                                             int waves)
{
    constexpr int kL = ROWS / 8, kC = 64 / kL, kPitch = COLS + 4;
    static_assert(COLS % kC == 0, "columns");
    const int lane = threadIdx.x & 63, rq = (lane % kL) * 8;
    for (int p = first; p < COLS / kC; p += waves) {
        const int c = p * kC + lane / kL;
        f32x8 x;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            x[j] = st[(rq + j) * kPitch + c];
        if (col0 + c < N)
            Parts<OP, EPI>::store(e, Parts<OP, EPI>::at(e, z, col0 + c, row0 + rq), x);
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

using TileL = Tile<2, 4, 8, 4>;      // 256 x 256, 8 waves
using TileM = Tile<2, 2, 4, 4>;      // 128 x 128, 4 waves
using TileS = Tile<2, 2, 2, 2>;      // 64 x 64, 4 waves

// Where tile `id` of `count` lies.  Consecutive ids go round the 8 compute
// dies, so each die gets one contiguous run of tiles, walked in bands of 8
// tile rows (its second-level cache then holds the band's A and a few
// columns of B).  Symmetric products count the upper triangle's tiles by rows.
__device__ __forceinline__ int die_order(int id, int count)
{
    const int per = count / 8, extra = count % 8, die = id % 8, k = id / 8;
    return die * per + (die < extra ? die : extra) + k;
}

__device__ __forceinline__ void which_tile(int id, int tm, int tn, bool sym, int &ti, int &tj)
{
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

// What a workgroup does: whole tiles first, then the parts of the tiles
// whose contraction is split.
struct Work {
    int tile, split, parts, ti, tj;
    int64_t z, s0, s1;         // matrix of the batch, steps of the contraction
    __device__ Work(const ProductArgs &a, int tm, int tn, bool sym, int step)
    {
        split = 0;
        parts = 1;
        if ((int)blockIdx.x < a.whole) {
            tile = die_order(blockIdx.x, a.whole);
        } else {
            const int t = (int)blockIdx.x - a.whole, tail = ((int)gridDim.x - a.whole) / a.splits;
            parts = a.splits;
            split = t / tail;
            tile = a.whole + t % tail;
        }
        const int each = sym ? tn * (tn + 1) / 2 : tm * tn;
        z = tile / each;
        which_tile(tile % each, tm, tn, sym, ti, tj);
        const int64_t steps = (a.K + step - 1) / step;
        s0 = steps * split / parts;
        s1 = steps * (split + 1) / parts;
    }
};

// The operand row of row r of B's tile.  Gated: in turn 16 rows of the
// gate's projection and the 16 of the up projection for the same columns, so
// that both meet in one lane; rows whose column is at or beyond `half` are
// outside.
template <int EPI>
__device__ __forceinline__ int64_t row_of_b(const ProductArgs &a, int64_t col0, int r)
{
    if (EPI != kEpiGated)
        return col0 + r;
    const int64_t c = col0 / 2 + (r >> 5) * 16 + (r & 15);
    return c >= a.e.half ? (int64_t)a.N : ((r & 16) ? a.e.half + c : c);
}

// The accumulators of a tile are staged a few fragment rows at a time.
template <class T>
struct Staging {
    static constexpr int kCols = 16 * T::kRN, kPitch = kCols + 4;
    static constexpr int kFrags = T::kRM < 4 ? T::kRM : 4;           // fragment rows at once
    static constexpr int kRows = 16 * kFrags;
    static constexpr int kFloats = kRows * kPitch;                   // a wave's piece
    static constexpr int kBytes = kFloats * 4 * (T::kThreads / 64);
};

// ------------------------------------------------- epilogues of the loss
constexpr float kLog2e = 1.4426950408889634f;

// (largest, sum of exponentials) of two sets together; no members: (-inf, 0).
// A NaN or an infinite logit makes the sum NaN.
__device__ __forceinline__ float2 merge_lse(float2 a, float2 b)
{
    const float m = fmaxf(a.x, b.x), at = m == -INFINITY ? 0.0f : m;
    return make_float2(m, a.y * __builtin_amdgcn_exp2f((a.x - at) * kLog2e) +
                              b.y * __builtin_amdgcn_exp2f((b.x - at) * kLog2e));
}

__device__ __forceinline__ int64_t target_of(const void *t, int wide, int64_t row)
{
    return wide ? static_cast<const int64_t *>(t)[row]
                : (int64_t)static_cast<const int32_t *>(t)[row];
}

// Each row's (largest, sum of exponentials) over the tile's columns, straight
// from the accumulators: a lane holds 4 RN of a row's logits, four lanes the
// wave's share of it, and the waves side by side meet in LDS.
template <class T, int OP>
__device__ __forceinline__ void finish_lse(const ProductArgs &a, const Work &w,
                                           f32x4 (&acc)[T::kRM][T::kRN], char *lds)
{
    constexpr int kDt = OP == kOpSplit ? GPIC_F32 : (OP == kOpF16 ? GPIC_F16 : GPIC_BF16);
    const Epilogue &e = a.e;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, g = lane >> 4;
    const int wm = (wave / T::kWN) * (16 * T::kRM), wn = wave % T::kWN;
    const int64_t col0 = (int64_t)w.tj * T::kBN + wn * (16 * T::kRN) + 4 * g;
    float bias[T::kRN][4];
    int pc[T::kRN][4];
#pragma unroll
    for (int j = 0; j < T::kRN; ++j)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int64_t col = col0 + 16 * j + c;
            // columns beyond the last are no logits
            bias[j][c] = col < a.N ? (e.bias ? load1(e.bias, col, kDt) : 0.0f) : -INFINITY;
            pc[j][c] = OP == kOpSplit && col < a.N ? e.pb[col] : 0;
        }
    float2 *all = reinterpret_cast<float2 *>(lds);             // [WN][BM]
#pragma unroll
    for (int i = 0; i < T::kRM; ++i) {
        const int r = wm + 16 * i + (lane & 15);
        const int64_t row = (int64_t)w.ti * T::kBM + r;
        const bool live = row < a.M;
        const int pr = OP == kOpSplit && live ? e.pa[row] : 0;
        float z[T::kRN][4];
#pragma unroll
        for (int j = 0; j < T::kRN; ++j)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                float v = acc[i][j][c];
                if (OP == kOpSplit)
                    v = ldexpf(v, -(pr + pc[j][c]));
                z[j][c] = bias[j][c] == -INFINITY ? -INFINITY : v + bias[j][c];
            }
        const int64_t t = live ? target_of(e.targets, e.wide, row) : -1;
        const int64_t at = t - col0;
        const bool mine = t >= 0 && t < a.N && at >= 0 && at < 16 * T::kRN && (at & 15) < 4;
        if (__any(mine)) {
#pragma unroll
            for (int j = 0; j < T::kRN; ++j)
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (mine && at == 16 * j + c) {
                        e.picked[row] = z[j][c];
                        z[j][c] = -INFINITY;
                    }
        }
        float m = -INFINITY;
#pragma unroll
        for (int j = 0; j < T::kRN; ++j)
#pragma unroll
            for (int c = 0; c < 4; ++c)
                m = fmaxf(m, z[j][c]);
        m = fmaxf(m, __shfl_xor(m, 16, 64));
        m = fmaxf(m, __shfl_xor(m, 32, 64));
        const float base = m == -INFINITY ? 0.0f : m;
        float s = 0.0f;
#pragma unroll
        for (int j = 0; j < T::kRN; ++j)
#pragma unroll
            for (int c = 0; c < 4; ++c)
                s += __builtin_amdgcn_exp2f((z[j][c] - base) * kLog2e);
        s += __shfl_xor(s, 16, 64);
        s += __shfl_xor(s, 32, 64);
        if (g == 0)
            all[wn * T::kBM + r] = make_float2(m, s);
    }
    __syncthreads();
    for (int r = threadIdx.x; r < T::kBM; r += T::kThreads) {
        const int64_t row = (int64_t)w.ti * T::kBM + r;
        if (row >= a.M)
            break;
        float2 v = all[r];
#pragma unroll
        for (int n = 1; n < T::kWN; ++n)
            v = merge_lse(v, all[n * T::kBM + r]);
        e.strip[(int64_t)w.tj * a.M + row] = v;
    }
}

// D = exp(z - lse) - [target] straight from the accumulators, rounded as the
// products that follow read it and only then staged in LDS (its own piece, no
// barrier), so that whole lines go out (a row's padding up to 64 columns zeros);
// and its column sums times g, unrounded.  The loss's gradient g is left out of
// what is rounded: it is the same for every row as a rule (1 / n), and its own
// rounding to 16 bits would be every entry's, up to 2^-8 of the gradients.
// 8,192 x 2,048 -> 25,088 in bfloat16 775 to 791 us (1.07 PFLOP/s, matrix pipe busy
// 52 %); with logits staged in float32 and finished from there 844.
template <class T, int OP>
__device__ __forceinline__ void finish_soft(const ProductArgs &a, const Work &w,
                                            f32x4 (&acc)[T::kRM][T::kRN], char *lds)
{
    constexpr bool kSplit = OP == kOpSplit;
    constexpr int kDt = kSplit ? GPIC_F32 : (OP == kOpF16 ? GPIC_F16 : GPIC_BF16);
    constexpr int kFrags = Staging<T>::kFrags, kRows = Staging<T>::kRows;
    constexpr int kWidth = 16 * T::kRN * (kSplit ? 4 : 2);       // bytes of a row
    constexpr int kPitch = kWidth + 16, kLanes = kWidth / 16, kRowsPass = 64 / kLanes;
    static_assert(kRows * kPitch <= Staging<T>::kFloats * 4, "a wave's piece");
    static_assert(kRows % kRowsPass == 0, "passes");
    const Epilogue &e = a.e;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, g = lane >> 4;
    const int64_t row0 = (int64_t)w.ti * T::kBM + (wave / T::kWN) * (16 * T::kRM);
    const int64_t col0 = (int64_t)w.tj * T::kBN + (wave % T::kWN) * (16 * T::kRN);
    const int64_t end = ((int64_t)a.N + 63) / 64 * 64;
    char *st = lds + wave * (Staging<T>::kFloats * 4);
    float bias[T::kRN][4], sum[T::kRN][4];
    int pc[T::kRN][4];
#pragma unroll
    for (int j = 0; j < T::kRN; ++j)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int64_t col = col0 + 16 * j + 4 * g + c;
            // columns beyond the last, as those that the bias takes out, are zeros
            bias[j][c] = col < a.N ? (e.bias ? load1(e.bias, e.first + col, kDt) : 0.0f)
                                   : -INFINITY;
            pc[j][c] = kSplit && col < a.N ? e.pb[col] : 0;
            sum[j][c] = 0.0f;
        }
#pragma unroll
    for (int i0 = 0; i0 < T::kRM; i0 += kFrags) {
#pragma unroll
        for (int i = 0; i < kFrags; ++i) {
            const int64_t row = row0 + 16 * (i0 + i) + (lane & 15);
            LossRow info{0.0f, 0.0f, 0.0f, 0.0f, -1, {0, 0, 0}};
            if (row < a.M)
                info = e.rows[row];
            const int pr = kSplit && row < a.M ? e.pa[row] : 0;
            float d[T::kRN][4];
#pragma unroll
            for (int j = 0; j < T::kRN; ++j)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    float z = acc[i0 + i][j][c];
                    if (kSplit)
                        z = ldexpf(z, -(pr + pc[j][c]));
                    z = __builtin_amdgcn_exp2f((z + bias[j][c] - info.at - info.off) * kLog2e);
                    d[j][c] = info.target < 0 || bias[j][c] == -INFINITY ? 0.0f : z;
                }
            const int at = info.target < 0 ? -1 : info.target - (int)(e.first + col0) - 4 * g;
            const bool mine = at >= 0 && at < 16 * T::kRN && (at & 15) < 4;
            if (__any(mine)) {
#pragma unroll
                for (int j = 0; j < T::kRN; ++j)
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        if (mine && at == 16 * j + c)
                            d[j][c] = info.picked;
            }
            char *to = st + (16 * i + (lane & 15)) * kPitch;
#pragma unroll
            for (int j = 0; j < T::kRN; ++j) {
                f32x4 v;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    sum[j][c] += d[j][c] * info.g;
                    v[c] = OP == kOpBf16 ? d[j][c] : d[j][c] * (float)(1 << kSoftPower);
                }
                if (kSplit) {
                    half4 hi, lo;
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        _Float16 x, y;
                        split2(v[c], x, y);
                        hi[c] = x;
                        lo[c] = y;
                    }
                    char *p = to + (j >> 1) * 128 + (j & 1) * 32 + g * 8;
                    *reinterpret_cast<half4 *>(p) = hi;
                    *reinterpret_cast<half4 *>(p + 64) = lo;
                } else if (OP == kOpF16) {
                    *reinterpret_cast<half4 *>(to + j * 32 + g * 8) =
                        __builtin_convertvector(v, half4);
                } else {
                    *reinterpret_cast<bf4 *>(to + j * 32 + g * 8) = __builtin_convertvector(v, bf4);
                }
            }
        }
        const int q = lane % kLanes, r0 = lane / kLanes;
        const int64_t col = col0 + (kSplit ? (q >> 3) * 32 + (q & 3) * 8 : q * 8);
#pragma unroll 4
        for (int r = r0; r < kRows; r += kRowsPass) {
            const int64_t row = row0 + 16 * i0 + r;
            if (row < a.M && col < end)
                *reinterpret_cast<u32x4 *>(static_cast<char *>(e.p_hi) +
                                           (row * e.ldp + (kSplit ? 2 : 1) * col0) * 2 + q * 16) =
                    *reinterpret_cast<const u32x4 *>(st + r * kPitch + q * 16);
        }
    }
    if (!e.sums || row0 >= a.M)
        return;
    float *to = e.sums + row0 / (16 * T::kRM) * a.N;
#pragma unroll
    for (int j = 0; j < T::kRN; ++j)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            float s = sum[j][c];
#pragma unroll
            for (int o = 1; o < 16; o <<= 1)
                s += __shfl_xor(s, o, 64);
            const int64_t col = col0 + 16 * j + 4 * g + c;
            if ((lane & 15) == 0 && col < a.N)
                to[col] = s;
        }
}

// A wave's accumulators to their place: the epilogue, or the partial sums.
template <class T, int OP, int EPI>
__device__ __forceinline__ void finish_tile(const ProductArgs &a, const Work &w,
                                            f32x4 (&acc)[T::kRM][T::kRN], char *lds)
{
    using St = Staging<T>;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int wm = (wave / T::kWN) * (16 * T::kRM), wn = (wave % T::kWN) * (16 * T::kRN);
    // every wave is done with the buffers
    copies_done();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if constexpr (EPI == kEpiLse) {
        finish_lse<T, OP>(a, w, acc, lds);
        return;
    }
    if constexpr (EPI == kEpiSoft) {
        finish_soft<T, OP>(a, w, acc, lds);
        return;
    }
    float *st = reinterpret_cast<float *>(lds) + wave * St::kFloats;
    float *to = st + (lane & 15) * St::kPitch + (lane >> 4) * 4;
    float *part = a.part + ((int64_t)w.split * (((int)gridDim.x - a.whole) / w.parts) +
                            (w.tile - a.whole)) * ((int64_t)T::kBM * T::kBN) +
                  wm * T::kBN + wn;
#pragma unroll
    for (int i0 = 0; i0 < T::kRM; i0 += St::kFrags) {
#pragma unroll
        for (int i = 0; i < St::kFrags; ++i)
#pragma unroll
            for (int j = 0; j < T::kRN; ++j)
                *reinterpret_cast<f32x4 *>(to + 16 * i * St::kPitch + 16 * j) = acc[i0 + i][j];
        if (w.parts > 1) {
            for (int r = lane / (St::kCols / 4); r < St::kRows; r += 64 / (St::kCols / 4)) {
                const int c = lane % (St::kCols / 4) * 4;
                *reinterpret_cast<f32x4 *>(part + (16 * i0 + r) * T::kBN + c) =
                    *reinterpret_cast<const f32x4 *>(st + r * St::kPitch + c);
            }
        } else {
            const int64_t r0 = (int64_t)w.ti * T::kBM + wm + 16 * i0, c0 = (int64_t)w.tj * T::kBN + wn;
            const bool mirror = symmetric(EPI) && w.ti != w.tj;
            finish_block<St::kRows, St::kCols, OP, EPI>(a.e, w.z, r0, c0, a.M, a.N, st, mirror);
            if (mirror)
                mirror_block<St::kRows, St::kCols, OP, EPI>(a.e, w.z, r0, c0, a.N, st, 0, 1);
        }
    }
}

// The middle and the small tile.  Several workgroups share a compute unit (2
// of the middle, 5 of the small), so that one's barriers and epilogue lie
// under another's products.  Middle: 4,096 squared times its transpose, upper
// triangle (528 tiles, 71 GFLOP), 89 us, matrix pipe busy 35 %, a quarter of
// the waves' cycles spent waiting; small: 10,007 x 1,000 -> 777 in float32 (2,041
// tiles, 47 GFLOP of half products) 81 us, pipe busy 28 %: bound by the reads
// of fragments (a fragment feeds 4 instructions, 2 in the small tile) and by
// the last round's idle units.
template <class T, bool ASTR, bool BSTR, int OP, int EPI>
__global__ __launch_bounds__(T::kThreads) void product_kernel(ProductArgs a, int tm, int tn)
{
    constexpr bool SPLIT = OP == kOpSplit;
    constexpr int kStep = SPLIT ? 32 : 64;           // values of k per step
    using SideA = Side<T::kBM, ASTR, SPLIT, T::kThreads>;
    using SideB = Side<T::kBN, BSTR, SPLIT, T::kThreads>;
    constexpr int kBuf = SideA::kBytes + SideB::kBytes;
    using St = Staging<T>;
    constexpr int kLds = 2 * kBuf > St::kBytes ? 2 * kBuf : St::kBytes;
    __shared__ __attribute__((aligned(1024))) char lds[kLds];

    const Work w(a, tm, tn, symmetric(EPI), kStep);
    const int64_t z = w.z, s0 = w.s0, s1 = w.s1;
    const int64_t row0 = (int64_t)w.ti * T::kBM, col0 = (int64_t)w.tj * T::kBN;

    SideA sa;
    SideB sb;
    Stream<ASTR, SPLIT> pa;
    Stream<BSTR, SPLIT> pb;
    const int64_t first_b = EPI == kEpiGated ? col0 / 2 : col0;
    sa.init(a.A, row0, a.M, [&](int r) { return row0 + r; });
    sb.init(a.B, first_b, a.N, [&](int r) { return row_of_b<EPI>(a, col0, r); });
    pa.init(a.A, z, row0, a.M, a.K, s0 * kStep);
    pb.init(a.B, z, first_b, a.N, a.K, s0 * kStep);

    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int wm = (wave / T::kWN) * (16 * T::kRM), wn = (wave % T::kWN) * (16 * T::kRN);
    f32x4 acc[T::kRM][T::kRN];
#pragma unroll
    for (int i = 0; i < T::kRM; ++i)
#pragma unroll
        for (int j = 0; j < T::kRN; ++j)
            acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    // Two steps of copies ahead, one slab of fragments ahead: while the
    // waves multiply one slab's fragments they read the next slab's.  The
    // barrier lies between the slabs of a step: by then every wave holds
    // the step's second slab in registers, so its buffer takes the copies
    // of the step after next.
    const uint32_t lds0 = lds_address(lds);
    int64_t kleft = a.K - s0 * kStep;
    auto copy_next = [&](int buf) {
        const uint32_t to = lds0 + (uint32_t)buf * kBuf;
        sa.copy(pa.rsrc(), to, kleft);
        sb.copy(pb.rsrc(), to + SideA::kBytes, kleft);
        pa.step();
        pb.step();
        kleft -= kStep;
    };
    u32x4 fa[2][T::kRM], fb[2][T::kRN];
    auto read = [&](int buf, int slab) {
        const char *ta = lds + buf * kBuf, *tb = ta + SideA::kBytes;
#pragma unroll
        for (int j = 0; j < T::kRN; ++j)
            fb[slab][j] = fragment<T::kBN, BSTR>(tb, slab, wn + 16 * j);
#pragma unroll
        for (int i = 0; i < T::kRM; ++i)
            fa[slab][i] = fragment<T::kBM, ASTR>(ta, slab, wm + 16 * i);
    };
    auto multiply = [&](int pa, int pb) {
#pragma unroll
        for (int i = 0; i < T::kRM; ++i)
#pragma unroll
            for (int j = 0; j < T::kRN; ++j)
                acc[i][j] = mma<OP>(fb[pb][j], fa[pa][i], acc[i][j]);
    };
    // one LDS read, then the share of `products` that goes with it
    constexpr int kReads = T::kRM * (ASTR ? 2 : 1) + T::kRN * (BSTR ? 2 : 1);
    constexpr int kPerRead = T::kRM * T::kRN / kReads > 0 ? T::kRM * T::kRN / kReads : 1;
    auto interleave = [&]() {
#pragma unroll
        for (int r = 0; r < kReads; ++r) {
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, kPerRead, 0);
        }
    };
    if (s1 > s0) {
        copy_next(0);
        copies_done();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (s0 + 1 < s1)
            copy_next(1);
        read(0, 0);
    }
    // The small tile's copies go out one by one between its few products (64
    // to 512 tiles 10 % faster, K = 2,048); the middle tile's at once (spread,
    // they cost it 7 %).
    constexpr int kMma = T::kRM * T::kRN;
    constexpr bool kSpread = kMma == SideA::kCopies + SideB::kCopies;
    const uint32_t lds_wave = (uint32_t)wave * 1024;
    for (int64_t s = s0; s < s1; ++s) {
        const int cur = (int)(s - s0) & 1;
        read(cur, 1);
        multiply(0, 0);
        interleave();
        copies_done();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (kSpread) {
            // copies between the products; beyond the contraction they fill
            // the buffer with what no product takes
            const uint32_t to = lds0 + (uint32_t)cur * kBuf;
            const u32x4 ra = pa.rsrc(), rb = pb.rsrc();
            if (!SPLIT)
                read(cur ^ 1, 0);
#pragma unroll
            for (int n = 0; n < kMma * (SPLIT ? 2 : 1); ++n) {
                const int q = n / kMma, i = n % kMma / T::kRN, j = n % T::kRN;
                const int ha = SPLIT ? q : 1, hb = SPLIT ? 1 - q : 1;
                acc[i][j] = mma<OP>(fb[hb][j], fa[ha][i], acc[i][j]);
                if (n < SideA::kCopies)
                    sa.copy_one(ra, to + lds_wave * SideA::kCopies, n, kleft);
                else if (n < SideA::kCopies + SideB::kCopies)
                    sb.copy_one(rb, to + SideA::kBytes + lds_wave * SideB::kCopies,
                                n - SideA::kCopies, kleft);
            }
            if (SPLIT)
                read(cur ^ 1, 0);
            pa.step();
            pb.step();
            kleft -= kStep;
            continue;
        }
        if (s + 2 < s1)
            copy_next(cur);
        if (SPLIT) {
            multiply(0, 1);
            multiply(1, 0);
            read(cur ^ 1, 0);
        } else {
            read(cur ^ 1, 0);
            multiply(1, 1);
            interleave();
        }
    }
    finish_tile<T, OP, EPI>(a, w, acc, lds);
}

// The 256 x 256 tile: 8 waves of 128 x 64, two to a SIMD.  A step is four
// phases, each 16 (split: 24) matrix instructions on one quarter of a wave's
// tile: rows A0, A1 (64 each) by columns B0, B1 (32 each) in the order A0 B0,
// A0 B1, A1 B1, A1 B0.  Between its matrix instructions a phase reads the
// fragments that a later phase needs and issues two copies, so that the two
// waves of a SIMD fill each other's gaps.  A phase begins with a barrier,
// before which a wave has waited for all but its last phase's reads and all
// but its last ten copies.  Hence what a phase reads (its copies are older
// than ten) has landed for every wave, and what was read two phases before
// has been read by every wave: copies run two steps ahead, into that place.
// 8,192 cubed in bfloat16: 930 to 1,020 us, box to box (1.08 to 1.18
// PFLOP/s), matrix pipe busy 64 % at the 1.6 to 1.85 GHz that the card's power
// leaves; the copies and the fragment reads cost about 20 % each (timed by
// what is left without them).  16,384 x 8,192 -> 2,048 (the gradient of a layer's
// inputs) 433 to 480 us, 1.15 to 1.27 PFLOP/s; 16,384 x 2,048 -> 8,192 with bias, gelu
// and both results written 530 to 630 us, of which a tile's epilogue, during
// which the unit's matrix pipe idles, is a quarter.  Four waves of 128 x 128 gave 956, waves
// one barrier apart with reads before the products 1.06, one buffer step ahead
// with all copies at its start 1.04.
//   phase     multiplies   reads        copies (step t + 2)
//   1         A0 B0        B1           A0
//   2         A0 B1        A1           B0
//   3         A1 B1        A0 (t + 1)   B1
//   4         A1 B0        B0 (t + 1)   A1
template <bool ASTR, bool BSTR, int OP, int EPI>
__global__ __launch_bounds__(512) void product_large_kernel(ProductArgs a, int tm, int tn)
{
    using T = TileL;
    constexpr bool SPLIT = OP == kOpSplit;
    constexpr int kStep = SPLIT ? 32 : 64;           // values of k per step
    using SideA = Side<128, ASTR, SPLIT, T::kThreads>;
    using SideB = Side<128, BSTR, SPLIT, T::kThreads>;
    constexpr int kPart = 128 * 128;                 // LDS bytes of A0, A1, B0 or B1
    constexpr int kBuf = 4 * kPart;
    constexpr int kLds = 2 * kBuf > Staging<T>::kBytes ? 2 * kBuf : Staging<T>::kBytes;
    __shared__ __attribute__((aligned(1024))) char lds[kLds];

    const Work w(a, tm, tn, symmetric(EPI), kStep);
    const int64_t z = w.z;
    const int64_t row0 = (int64_t)w.ti * T::kBM, col0 = (int64_t)w.tj * T::kBN;
    SideA sa[2];
    SideB sb[2];
    Stream<ASTR, SPLIT> pa;
    Stream<BSTR, SPLIT> pb;
    const int64_t first_b = EPI == kEpiGated ? col0 / 2 : col0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        sa[h].init(a.A, row0, a.M,
                   [&](int r) { return row0 + (r >> 6) * 128 + h * 64 + (r & 63); });
        sb[h].init(a.B, first_b, a.N, [&](int r) {
            return row_of_b<EPI>(a, col0, (r >> 5) * 64 + h * 32 + (r & 31));
        });
    }
    pa.init(a.A, z, row0, a.M, a.K, w.s0 * kStep);
    pb.init(a.B, z, first_b, a.N, a.K, w.s0 * kStep);

    const int wave = threadIdx.x >> 6;
    const int ra = (wave / T::kWN) * 64, rb = (wave % T::kWN) * 32;   // within a group
    f32x4 acc[T::kRM][T::kRN];
#pragma unroll
    for (int i = 0; i < T::kRM; ++i)
#pragma unroll
        for (int j = 0; j < T::kRN; ++j)
            acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    u32x4 fa[2][2][4], fb[2][2][2];                  // [half][slab][fragment]

    const uint32_t lds0 = lds_address(lds);
    int64_t kleft_a = a.K - w.s0 * kStep, kleft_b = kleft_a;
    // LDS: A0, A1, B0, B1 of buffer 0, then of buffer 1
    const uint32_t lds_wave = lds0 + (uint32_t)wave * (SideA::kCopies * 1024);
    // copy c of A (B) half h into its place in buffer buf
    auto copy_a = [&](int buf, int h, int c) {
        sa[h].copy_one(pa.rsrc(), lds_wave + (uint32_t)(buf * kBuf + h * kPart), c, kleft_a);
    };
    auto copy_b = [&](int buf, int h, int c) {
        sb[h].copy_one(pb.rsrc(), lds_wave + (uint32_t)(buf * kBuf + (2 + h) * kPart), c, kleft_b);
    };
    auto next_a = [&]() {
        pa.step();
        kleft_a -= kStep;
    };
    auto next_b = [&]() {
        pb.step();
        kleft_b -= kStep;
    };
    auto read_a = [&](int buf, int h, int s, int i) {
        fa[h][s][i] = fragment<128, ASTR>(lds + buf * kBuf + h * kPart, s, ra + 16 * i);
    };
    auto read_b = [&](int buf, int h, int s, int j) {
        fb[h][s][j] = fragment<128, BSTR>(lds + buf * kBuf + (2 + h) * kPart, s, rb + 16 * j);
    };
    auto barrier = [&]() {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    // one phase: quarter (ha, hb); `what` reads fragment n of the next
    // group (8 of A if reads_a, else 4 of B), `copy` issues copy c;
    // read_a_before: the phase before read 8 of A
    auto phase = [&](int ha, int hb, bool reads_a, bool read_a_before, auto what, auto copy) {
        constexpr int kA = ASTR ? 15 : 8, kB = BSTR ? 8 : 4;
        if (read_a_before)        // lgkmcnt counts to 15
            asm volatile("s_waitcnt vmcnt(10) lgkmcnt(%0)" ::"n"(kA) : "memory");
        else
            asm volatile("s_waitcnt vmcnt(10) lgkmcnt(%0)" ::"n"(kB) : "memory");
        __builtin_amdgcn_sched_barrier(0);
        barrier();
        constexpr int kMma = SPLIT ? 24 : 16;
#pragma unroll
        for (int n = 0; n < kMma; ++n) {
            const int q = n / 8, i = n % 8 / 2, j = n % 2;
            const int qa = SPLIT ? q == 1 : q, qb = SPLIT ? q == 2 : q;
            acc[4 * ha + i][2 * hb + j] =
                mma<OP>(fb[hb][qb][j], fa[ha][qa][i], acc[4 * ha + i][2 * hb + j]);
            // B's fragments may replace the ones this phase uses: slab 0 from
            // the last eight instructions on, slab 1 after them
            if (reads_a ? n < 8 : n == kMma - 8 || n == kMma - 7) {
                __builtin_amdgcn_sched_barrier(0);
                what(reads_a ? n : n - (kMma - 8));
                __builtin_amdgcn_sched_barrier(0);
            }
            if (n == kMma - 6 || n == kMma - 3) {
                __builtin_amdgcn_sched_barrier(0);
                copy(n == kMma - 6 ? 0 : 1);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        if (!reads_a) {
            what(2);
            what(3);
        }
        __builtin_amdgcn_sched_barrier(0);
    };

    // the first two steps; copies beyond the contraction fill LDS with
    // zeros or values that no product takes
    static_assert(SideA::kCopies == 2 && SideB::kCopies == 2, "two copies a phase");
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int c = 0; c < 2; ++c)
            copy_a(t, 0, c);
#pragma unroll
        for (int c = 0; c < 4; ++c)
            copy_b(t, c >> 1, c & 1);
        next_b();
#pragma unroll
        for (int c = 0; c < 2; ++c)
            copy_a(t, 1, c);
        next_a();
    }
    asm volatile("s_waitcnt vmcnt(10)" ::: "memory");
    barrier();
#pragma unroll
    for (int n = 0; n < 8; ++n)
        read_a(0, 0, n >> 2, n & 3);
#pragma unroll
    for (int n = 0; n < 4; ++n)
        read_b(0, 0, n >> 1, n & 1);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    barrier();
    for (int64_t s = w.s0; s < w.s1; ++s) {
        const int cur = (int)(s - w.s0) & 1;
        phase(0, 0, false, false, [&](int n) { read_b(cur, 1, n >> 1, n & 1); },
              [&](int c) { copy_a(cur, 0, c); });
        phase(0, 1, true, false, [&](int n) { read_a(cur, 1, n >> 2, n & 3); },
              [&](int c) { copy_b(cur, 0, c); });
        phase(1, 1, true, true, [&](int n) { read_a(cur ^ 1, 0, n >> 2, n & 3); },
              [&](int c) { copy_b(cur, 1, c); });
        next_b();
        phase(1, 0, false, true, [&](int n) { read_b(cur ^ 1, 0, n >> 1, n & 1); },
              [&](int c) { copy_a(cur, 1, c); });
        next_a();
    }
    finish_tile<T, OP, EPI>(a, w, acc, lds);
}

// The parts of the split tiles, added in order, then the epilogue.  A
// workgroup takes the rows and columns that a wave stages; eight parts'
// loads are in flight (few tiles have many parts).  The mirrored block goes
// out by rows of at least 64 bytes: with 32 the dies' caches write parts of
// each other's lines, and a join of 136 tiles takes 18 us for 6.
template <class T, int OP, int EPI>
__global__ __launch_bounds__(256) void product_join_kernel(ProductArgs a, int tm, int tn, int tail)
{
    using St = Staging<T>;
    constexpr int kCols = St::kCols, kPitch = St::kPitch, kRows = St::kRows;
    __shared__ __attribute__((aligned(16))) float st[kRows * kPitch];
    constexpr int kAcross = T::kBN / kCols, kPieces = T::kBM / kRows * kAcross;
    const int tile = a.whole + blockIdx.x / kPieces, piece = blockIdx.x % kPieces;
    const int pr = piece / kAcross * kRows, pc = piece % kAcross * kCols;
    int ti, tj;
    const int each = symmetric(EPI) ? tn * (tn + 1) / 2 : tm * tn;
    const int64_t z = tile / each;
    which_tile(tile % each, tm, tn, symmetric(EPI), ti, tj);
    const int64_t row0 = (int64_t)ti * T::kBM + pr, col0 = (int64_t)tj * T::kBN + pc;
    if (row0 >= a.M || col0 >= (symmetric(EPI) ? ((int64_t)a.N + 63) / 64 * 64 : a.N))
        return;
    const int64_t pitch = (int64_t)tail * T::kBM * T::kBN;         // between parts
    const float *part = a.part + (int64_t)(tile - a.whole) * T::kBM * T::kBN + pr * T::kBN + pc;
    constexpr int kQuads = kCols / 4;
    for (int i = threadIdx.x; i < kRows * kQuads; i += 256) {
        const int r = i / kQuads, c = i % kQuads * 4;
        const float *p = part + r * T::kBN + c;
        f32x4 v = *reinterpret_cast<const f32x4 *>(p);
#pragma unroll 8
        for (int s = 1; s < a.splits; ++s)
            v += *reinterpret_cast<const f32x4 *>(p + s * pitch);
        *reinterpret_cast<f32x4 *>(st + r * kPitch + c) = v;
    }
    __syncthreads();
    const int wave = threadIdx.x >> 6;
    const bool mirror = symmetric(EPI) && ti != tj;
    constexpr int kWaveRows = kRows / 4;
    finish_block<kWaveRows, kCols, OP, EPI>(a.e, z, row0 + wave * kWaveRows, col0, a.M, a.N,
                                            st + wave * kWaveRows * kPitch, mirror);
    if (mirror) {
        __syncthreads();
        mirror_block<kRows, kCols, OP, EPI>(a.e, z, row0, col0, a.N, st, wave, 4);
    }
}

// ------------------------------------------------------------------- host
template <class T, bool ASTR, bool BSTR, int OP, int EPI>
hipError_t launch_tile(const Plan &p, ProductArgs a, hipStream_t s)
{
    a.whole = (int)p.whole;
    a.splits = p.splits;
    const int64_t blocks = p.whole + p.tail * p.splits;
    if constexpr (std::is_same<T, TileL>::value)
        product_large_kernel<ASTR, BSTR, OP, EPI>
            <<<(unsigned)blocks, T::kThreads, 0, s>>>(a, p.tm, p.tn);
    else
        product_kernel<T, ASTR, BSTR, OP, EPI>
            <<<(unsigned)blocks, T::kThreads, 0, s>>>(a, p.tm, p.tn);
    hipError_t e = hipGetLastError();
    if constexpr (uncut(EPI)) {
        return e;
    } else {
        if (e == hipSuccess && p.tail > 0) {
            using St = Staging<T>;
            constexpr int kPieces = T::kBM / St::kRows * (T::kBN / St::kCols);
            product_join_kernel<T, OP, EPI>
                <<<(unsigned)(p.tail * kPieces), 256, 0, s>>>(a, p.tm, p.tn, (int)p.tail);
            e = hipGetLastError();
        }
        return e;
    }
}

template <bool ASTR, bool BSTR, int OP, int EPI>
hipError_t launch_any_tile(const Plan &p, const ProductArgs &a, hipStream_t s)
{
    switch (p.tile) {
    case 0:
        return launch_tile<TileL, ASTR, BSTR, OP, EPI>(p, a, s);
    case 1:
        return launch_tile<TileM, ASTR, BSTR, OP, EPI>(p, a, s);
    default:
        return launch_tile<TileS, ASTR, BSTR, OP, EPI>(p, a, s);
    }
}

} // namespace
} // namespace gpic
