// The embedding table: Y_i = s T[id_i], and its gradient dT_v = s sum over
// the i with id_i = v of dY_i.  Ids outside the table are padding: rows of
// zeros, no gradient.
//
// The gradient adds in float32 in a fixed order: the ids are sorted with
// their positions (stable), every row of the table finds its run, and a wave
// adds a run of up to 64 rows of dY, eight columns a lane.  Longer runs
// (tokens as frequent as words are) are cut where the sorted positions pass
// multiples of 64; the cuts' sums are added by a workgroup in a second launch.
// A few ids are not sorted: each position compares itself with all of them.
#include "common.h"
#include "training.h"

namespace gpic {
namespace {

constexpr int kRun = 64;               // longest run that one wave adds
constexpr int64_t kFewIds = 1024;      // compared one by one

struct TableArgs {
    const void *ids, *T, *dY;
    void *Y, *dT;
    int64_t n, k, rows, ldt, ldy;
    float scale;
    int accumulate;
    // sorted: keys, positions, where each row's run starts, cut runs' sums
    const uint64_t *key;
    const int32_t *pos;
    uint32_t *start;
    float *part;
    int64_t strips;
};

// id i, or -1 where it is outside the table
template <bool WIDE>
__device__ __forceinline__ int64_t id_at(const void *ids, int64_t i, int64_t rows)
{
    const int64_t id = WIDE ? static_cast<const int64_t *>(ids)[i]
                            : (int64_t)static_cast<const int32_t *>(ids)[i];
    return id >= 0 && id < rows ? id : -1;
}

__device__ __forceinline__ int valid8(int64_t col, int64_t cols)
{
    const int64_t left = cols - col;
    return left <= 0 ? 0 : (left < 8 ? (int)left : 8);
}

template <int DT, bool WIDE>
__global__ __launch_bounds__(256) void lookup_kernel(TableArgs a)
{
    const int64_t groups = (a.k + 7) / 8, total = a.n * groups;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total;
         i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / groups, col = (i - row * groups) * 8;
        const int64_t id = id_at<WIDE>(a.ids, row, a.rows);
        const int valid = valid8(col, a.k);
        f32x8 v = 0.0f;
        if (id >= 0)
            v = load8(a.T, id * a.ldt + col, DT, valid) * a.scale;
        store8(a.Y, row * a.ldy + col, v, DT, valid);
    }
}

template <int DT>
__global__ __launch_bounds__(256) void zero_rows_kernel(TableArgs a)
{
    const int64_t groups = (a.k + 7) / 8, total = a.rows * groups;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total;
         i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / groups, col = (i - row * groups) * 8;
        store8(a.dT, row * a.ldt + col, f32x8(0.0f), DT, valid8(col, a.k));
    }
}

// dT's row v from column col on, or what it held and that
template <int DT>
__device__ __forceinline__ void put(const TableArgs &a, int64_t v, int64_t col, f32x8 sum,
                                    int valid)
{
    sum = sum * a.scale;
    if (a.accumulate)
        sum = sum + load8(a.dT, v * a.ldt + col, DT, valid);
    store8(a.dT, v * a.ldt + col, sum, DT, valid);
}

// A workgroup for every position and strip of 512 columns: where no earlier
// position has the same id, the waves add a quarter each of the ones that do.
template <int DT, bool WIDE>
__global__ __launch_bounds__(256) void few_ids_kernel(TableArgs a)
{
    const int64_t i = blockIdx.x / a.strips, strip = blockIdx.x % a.strips;
    const int64_t id = id_at<WIDE>(a.ids, i, a.rows);
    if (id < 0)
        return;
    int earlier = 0;
    for (int64_t j = threadIdx.x; j < i; j += 256)
        earlier |= id_at<WIDE>(a.ids, j, a.rows) == id;
    if (__syncthreads_or(earlier))
        return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t col = (strip * 64 + lane) * 8;
    const int valid = valid8(col, a.k);
    const int64_t each = (a.n - i + 255) / 256 * 64;
    const int64_t j0 = i + wave * each, j1 = j0 + each < a.n ? j0 + each : a.n;
    f32x8 sum = 0.0f;
    for (int64_t j = j0; j < j1; j += 64) {
        uint64_t same = __ballot(j + lane < j1 && id_at<WIDE>(a.ids, j + lane, a.rows) == id);
        while (same) {
            const int64_t row = j + __builtin_ctzll(same);
            same &= same - 1;
            if (valid)
                sum += load8(a.dY, row * a.ldy + col, DT, valid);
        }
    }
    __shared__ f32x8 part[4][64];
    part[wave][lane] = sum;
    __syncthreads();
    if (wave == 0 && valid)
        put<DT>(a, id, col, ((part[0][lane] + part[1][lane]) + part[2][lane]) + part[3][lane],
                valid);
}

template <bool WIDE>
__global__ __launch_bounds__(256) void keys_kernel(const void *ids, int64_t n, int64_t rows,
                                                   uint64_t *key, int32_t *pos)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n;
         i += (int64_t)gridDim.x * 256) {
        const int64_t id = id_at<WIDE>(ids, i, rows);
        key[i] = (uint64_t)(id < 0 ? rows : id);       // padding sorts last
        pos[i] = (int32_t)i;
    }
}

// start[v]: the first sorted position whose id is at least v
__global__ __launch_bounds__(256) void starts_kernel(TableArgs a)
{
    for (int64_t v = (int64_t)blockIdx.x * 256 + threadIdx.x; v <= a.rows;
         v += (int64_t)gridDim.x * 256) {
        int64_t lo = 0, hi = a.n;
        while (lo < hi) {
            const int64_t mid = (lo + hi) / 2;
            if ((int64_t)a.key[mid] < v)
                lo = mid + 1;
            else
                hi = mid;
        }
        a.start[v] = (uint32_t)lo;
    }
}

// the sum of dY's rows at sorted positions j0 .. j1 - 1
template <int DT>
__device__ __forceinline__ f32x8 add_rows(const TableArgs &a, int64_t j0, int64_t j1, int64_t col,
                                          int valid)
{
    f32x8 sum = 0.0f;
    if (valid) {
#pragma unroll 8
        for (int64_t j = j0; j < j1; ++j)
            sum += load8(a.dY, (int64_t)a.pos[j] * a.ldy + col, DT, valid);
    }
    return sum;
}

// A wave for every row of the table and strip of 512 columns.
template <int DT>
__global__ __launch_bounds__(256) void rows_kernel(TableArgs a)
{
    const int64_t tasks = a.rows * a.strips;
    for (int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); t < tasks;
         t += (int64_t)gridDim.x * 4) {
        const int64_t v = t / a.strips, col = (t % a.strips * 64 + (threadIdx.x & 63)) * 8;
        const int64_t j0 = a.start[v], j1 = a.start[v + 1];
        const int valid = valid8(col, a.k);
        if (!valid || j1 - j0 > kRun || (a.accumulate && j0 == j1))
            continue;
        put<DT>(a, v, col, add_rows<DT>(a, j0, j1, col, valid), valid);
    }
}

// Of the runs longer than 64, what lies in a chunk of 64 sorted positions:
// the run that the chunk begins in (slot 0) and the one that it ends in
// (slot 1).
template <int DT>
__global__ __launch_bounds__(256) void cuts_kernel(TableArgs a)
{
    const int64_t chunks = (a.n + kRun - 1) / kRun, tasks = chunks * a.strips;
    for (int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); t < tasks;
         t += (int64_t)gridDim.x * 4) {
        const int64_t c = t / a.strips, col = (t % a.strips * 64 + (threadIdx.x & 63)) * 8;
        const int64_t first = c * kRun, end = first + kRun < a.n ? first + kRun : a.n;
        const int valid = valid8(col, a.k);
        const int64_t head = (int64_t)a.key[first], tail = (int64_t)a.key[end - 1];
        if (head >= a.rows)
            continue;
        float *to = a.part + c * 2 * a.k + col;
        if (a.start[head + 1] - a.start[head] > kRun) {
            const int64_t j1 = a.start[head + 1] < end ? a.start[head + 1] : end;
            store8(to, 0, add_rows<DT>(a, first, j1, col, valid), GPIC_F32, valid);
        }
        if (tail != head && tail < a.rows && a.start[tail + 1] - a.start[tail] > kRun)
            store8(to, a.k, add_rows<DT>(a, a.start[tail], end, col, valid), GPIC_F32, valid);
    }
}

// The cuts' sums of the run that starts in a chunk, by the sixteen waves of a
// workgroup.
template <int DT>
__global__ __launch_bounds__(1024) void join_cuts_kernel(TableArgs a)
{
    __shared__ f32x8 all[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t tasks = (a.n + kRun - 1) / kRun * a.strips;
    for (int64_t t = blockIdx.x; t < tasks; t += gridDim.x) {
        const int64_t c = t / a.strips, first = c * kRun;
        const int64_t end = first + kRun < a.n ? first + kRun : a.n;
        const int64_t v = (int64_t)a.key[end - 1];
        if (v >= a.rows)
            continue;
        const int64_t j0 = a.start[v], j1 = a.start[v + 1];
        if (j0 < first || j1 - j0 <= kRun)
            continue;
        const int64_t col = (t % a.strips * 64 + lane) * 8;
        const int valid = valid8(col, a.k);
        const int64_t cuts = (j1 - 1) / kRun - c + 1, each = (cuts + 15) / 16;
        const int64_t c0 = c + wave * each, c1 = c0 + each < c + cuts ? c0 + each : c + cuts;
        f32x8 sum = 0.0f;
        if (valid) {
#pragma unroll 4
            for (int64_t i = c0; i < c1; ++i)
                sum += load8(a.part, (i * 2 + (i == c && j0 > first)) * a.k + col, GPIC_F32, valid);
        }
        all[wave][lane] = sum;
        __syncthreads();
        if (wave == 0 && valid) {
            for (int i = 1; i < 16; ++i)
                sum += all[i][lane];
            put<DT>(a, v, col, sum, valid);
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------- host
unsigned capped(int64_t blocks)
{
    return (unsigned)(blocks < 1 ? 1 : (blocks > (1 << 20) ? 1 << 20 : blocks));
}

struct Sorted {
    uint64_t *key[2];
    int32_t *pos[2];
    uint32_t *hist, *hsum, *start;
    float *part;
    Sorted(const Embedding &p, Cursor &c)
    {
        const size_t n = (size_t)p.n, most = n > 4096 ? n : 4096;
        auto larger = [&](size_t bytes) { return bytes > 2 * most ? bytes : 2 * most; };
        for (int i = 0; i < 2; ++i) {
            key[i] = static_cast<uint64_t *>(c.take(n * 8));
            pos[i] = static_cast<int32_t *>(c.take(n * 4));
        }
        hist = static_cast<uint32_t *>(c.take(larger(radix_hist_bytes(p.n))));
        hsum = static_cast<uint32_t *>(c.take(larger(radix_hsum_bytes(p.n))));
        start = static_cast<uint32_t *>(c.take(((size_t)p.rows + 1) * 4));
        part = static_cast<float *>(c.take((n + kRun - 1) / kRun * 2 * (size_t)p.k * 4));
    }
};

#define RUN(expr)                                                              \
    do {                                                                       \
        hipError_t e_ = (expr);                                                \
        if (e_ != hipSuccess)                                                  \
            return e_;                                                         \
    } while (0)

template <int DT>
hipError_t few_ids(const Embedding &p, const TableArgs &a, hipStream_t st)
{
    if (!p.accumulate) {
        zero_rows_kernel<DT><<<capped((p.rows * ((p.k + 7) / 8) + 255) / 256), 256, 0, st>>>(a);
        RUN(hipGetLastError());
    }
    if (p.n == 0)
        return hipSuccess;
    const unsigned blocks = (unsigned)(p.n * a.strips);
    if (p.wide)
        few_ids_kernel<DT, true><<<blocks, 256, 0, st>>>(a);
    else
        few_ids_kernel<DT, false><<<blocks, 256, 0, st>>>(a);
    return hipGetLastError();
}

template <int DT>
hipError_t sorted_ids(const Embedding &p, TableArgs a, void *ws, hipStream_t st)
{
    Cursor c{static_cast<char *>(ws)};
    Sorted s(p, c);
    const unsigned blocks = capped((p.n + 255) / 256);
    if (p.wide)
        keys_kernel<true><<<blocks, 256, 0, st>>>(a.ids, p.n, p.rows, s.key[0], s.pos[0]);
    else
        keys_kernel<false><<<blocks, 256, 0, st>>>(a.ids, p.n, p.rows, s.key[0], s.pos[0]);
    RUN(hipGetLastError());
    int bits = 8;
    while (bits < 32 && (p.rows >> bits) != 0)
        bits += 8;
    RUN(radix_sort_u64(s.key[0], s.pos[0], s.key[1], s.pos[1], p.n, bits, s.hist, s.hsum, st,
                       true));
    a.key = s.key[0];
    a.pos = s.pos[0];
    a.start = s.start;
    a.part = s.part;
    starts_kernel<<<capped((p.rows + 256) / 256), 256, 0, st>>>(a);
    RUN(hipGetLastError());
    const int64_t chunks = (p.n + kRun - 1) / kRun;
    rows_kernel<DT><<<capped((p.rows * a.strips + 3) / 4), 256, 0, st>>>(a);
    RUN(hipGetLastError());
    cuts_kernel<DT><<<capped((chunks * a.strips + 3) / 4), 256, 0, st>>>(a);
    RUN(hipGetLastError());
    join_cuts_kernel<DT><<<capped(chunks * a.strips), 1024, 0, st>>>(a);
    return hipGetLastError();
}

template <int DT>
hipError_t lookup(const Embedding &p, const TableArgs &a, hipStream_t st)
{
    const unsigned blocks = capped((p.n * ((p.k + 7) / 8) + 255) / 256);
    if (p.wide)
        lookup_kernel<DT, true><<<blocks, 256, 0, st>>>(a);
    else
        lookup_kernel<DT, false><<<blocks, 256, 0, st>>>(a);
    return hipGetLastError();
}

template <int DT>
hipError_t gradient(const Embedding &p, const TableArgs &a, void *ws, hipStream_t st)
{
    return p.n <= kFewIds ? few_ids<DT>(p, a, st) : sorted_ids<DT>(p, a, ws, st);
}

TableArgs args_of(const Embedding &p, const void *ids)
{
    TableArgs a{};
    a.ids = ids;
    a.n = p.n;
    a.k = p.k;
    a.rows = p.rows;
    a.ldt = p.ldt;
    a.ldy = p.ldy;
    a.scale = p.scale;
    a.accumulate = p.accumulate;
    a.strips = (p.k + 511) / 512;
    return a;
}

} // namespace

size_t embedding_ws(const Embedding &p)
{
    if (p.n <= kFewIds)
        return 0;
    Cursor c{nullptr};
    Sorted s(p, c);
    return c.at;
}

hipError_t run_embedding(const Embedding &p, const void *ids, const void *T, void *Y,
                         hipStream_t st)
{
    if (p.n == 0)
        return hipSuccess;
    TableArgs a = args_of(p, ids);
    a.T = T;
    a.Y = Y;
    return p.dtype == GPIC_F32    ? lookup<GPIC_F32>(p, a, st)
           : p.dtype == GPIC_F16 ? lookup<GPIC_F16>(p, a, st)
                                 : lookup<GPIC_BF16>(p, a, st);
}

hipError_t run_embedding_backward(const Embedding &p, const void *dY, const void *ids, void *dT,
                                  void *ws, hipStream_t st)
{
    TableArgs a = args_of(p, ids);
    a.dY = dY;
    a.dT = dT;
    return p.dtype == GPIC_F32    ? gradient<GPIC_F32>(p, a, ws, st)
           : p.dtype == GPIC_F16 ? gradient<GPIC_F16>(p, a, ws, st)
                                 : gradient<GPIC_BF16>(p, a, ws, st);
}

} // namespace gpic
