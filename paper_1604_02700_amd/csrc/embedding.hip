// The embedding table: Y_i = s T[id_i], and its gradient dT_v = s sum over
// the i with id_i = v of dY_i.  Ids outside the table are padding: rows of
// zeros, no gradient.
//
// The gradient adds in float32 in a fixed order: the ids are sorted with
// their positions (stable), every row of the table finds its run, and a wave
// adds a run of up to 16 rows of dY, eight columns a lane.  Longer runs
// (tokens as frequent as words are) are cut where the sorted positions pass
// multiples of 16; the cuts' sums are added by a second launch.
// A few ids are not sorted: each position compares itself with all of them.
#include "training.h"

namespace gpic {
namespace {

constexpr int kRun = 16;               // longest run that one wave adds
constexpr int64_t kFewIds = 1024;      // compared one by one

struct TableArgs {
    const void *ids, *T, *dY;
    void *Y, *dT;
    int64_t n, k, rows, ldt, ldy;
    float scale;
    int accumulate;
    // sorted: keys, positions, where each row's run starts, cut runs' sums
    const uint32_t *key;
    const int32_t *pos;
    uint32_t *start;
    float *part;
    struct CutRun *run;
    int64_t strips;
};

// The run longer than 16 that starts in a chunk: its row of the table, the chunk
// after its last (the chunk itself: there is none), its first sum's slot.
struct CutRun {
    uint32_t row, end, slot, unused;
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

// Eight columns that a lane adds: its own, or, where a row ends within them, the
// row's last eight, of which it keeps those from `skip` on; beyond the row the
// first eight, of which it keeps none.  So no load of a run depends on a branch.
// TINY: rows of fewer than eight columns.
template <int DT, bool TINY>
struct Window {
    int64_t col;
    int skip, tiny;
    __device__ __forceinline__ Window(int64_t c, int64_t k)
    {
        tiny = TINY ? (int)k : 8;
        skip = c >= k ? 8 : 0;
        col = c >= k ? 0 : c;
        if (!TINY && c < k && c + 8 > k) {
            col = k - 8;
            skip = (int)(c - col);
        }
    }
    __device__ __forceinline__ f32x8 load(const void *p, int64_t row_at) const
    {
        return load8(p, row_at + col, DT, TINY ? tiny : 8);
    }
    __device__ __forceinline__ f32x8 load_sum(const float *p, int64_t row_at) const
    {
        return load8(p, row_at + col, GPIC_F32, TINY ? tiny : 8);
    }
    __device__ __forceinline__ void store(void *p, int64_t row_at, f32x8 v, int dtype) const
    {
        if (skip == 0) {
            store8(p, row_at + col, v, dtype, TINY ? tiny : 8);
            return;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j >= skip)
                store1(p, row_at + col + j, v[j], dtype);
    }
};

// Eight columns a thread.  Bound by memory: 32,768 rows of 1,024 of 50,000 in
// bfloat16, as frequent as words are, 18 to 22 us (67 MB written and the rows that
// occur read: 4.4 to 4.9 TB/s).
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

// dT's row v, or what it held and that
template <int DT, bool TINY>
__device__ __forceinline__ void put(const TableArgs &a, int64_t v, const Window<DT, TINY> &w,
                                    f32x8 sum)
{
    if (w.skip == 8)
        return;
    sum = sum * a.scale;
    if (a.accumulate)
        sum = sum + w.load(a.dT, v * a.ldt);
    w.store(a.dT, v * a.ldt, sum, DT);
}

// What earlier launches wrote, at an index that the wave shares: through the
// scalar cache, whose loads return sooner than a vector's.
template <class T>
__device__ __forceinline__ T shared_load(const T *p, int64_t i)
{
    return *(const __attribute__((address_space(4))) T *)(uintptr_t)(p + i);
}
__device__ __forceinline__ int64_t wave_index()
{
    return (int64_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
}

// sum[h] += load(item, h) for item = get(j0 .. j1 - 1), in order.  A batch's loads
// are all under way before the first is added; the last one loads its last item
// again in place of what it lacks.
template <int COUNT, int HOLD, class Get, class Load>
__device__ __forceinline__ void add_batch(int64_t j, int64_t j1, Get get, Load load,
                                          f32x8 (&sum)[HOLD])
{
    f32x8 v[COUNT][HOLD];
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
        const int64_t item = get(j + i < j1 ? j + i : j1 - 1);
#pragma unroll
        for (int h = 0; h < HOLD; ++h)
            v[i][h] = load(item, h);
    }
#pragma unroll
    for (int i = 0; i < COUNT; ++i)
        if (j + i < j1)
#pragma unroll
            for (int h = 0; h < HOLD; ++h)
                sum[h] += v[i][h];
}

template <int HOLD, class Get, class Load>
__device__ __forceinline__ void add_batches(int64_t j0, int64_t j1, Get get, Load load,
                                            f32x8 (&sum)[HOLD])
{
    constexpr int kMost = HOLD > 1 ? 4 : 8;
    int64_t j = j0;
    for (; j1 - j > 2; j += kMost)
        add_batch<kMost>(j, j1, get, load, sum);
    if (j1 - j == 2)
        add_batch<2>(j, j1, get, load, sum);
    else if (j1 - j == 1)
        add_batch<1>(j, j1, get, load, sum);
}

// A workgroup for every position and strip of 512 columns: where no earlier
// position has the same id, its waves list the ones that do and add an eighth
// each.
constexpr int kFewWaves = 8;

template <int DT, bool WIDE, bool TINY>
__global__ __launch_bounds__(64 * kFewWaves) void few_ids_kernel(TableArgs a)
{
    const int64_t i = blockIdx.x / a.strips, strip = blockIdx.x % a.strips;
    const int64_t id = id_at<WIDE>(a.ids, i, a.rows);
    if (id < 0)
        return;
    int earlier = 0;
    for (int64_t j = threadIdx.x; j < i; j += 64 * kFewWaves)
        earlier |= id_at<WIDE>(a.ids, j, a.rows) == id;
    if (__syncthreads_or(earlier))
        return;
    // each wave lists its run of positions; together they are in order
    __shared__ int list[kFewWaves][kFewIds / kFewWaves + 64], found[kFewWaves];
    const int lane = threadIdx.x & 63, wave = (int)wave_index();
    const int64_t each = (a.n - i + 64 * kFewWaves - 1) / (64 * kFewWaves) * 64;
    const int64_t j0 = i + wave * each, j1 = j0 + each < a.n ? j0 + each : a.n;
    int count = 0;
    for (int64_t j = j0; j < j1; j += 64) {
        const bool same = j + lane < j1 && id_at<WIDE>(a.ids, j + lane, a.rows) == id;
        const uint64_t all = __ballot(same);
        if (same)
            list[wave][count + __popcll(all & ~(~0ull << lane))] = (int)(j + lane);
        count += __popcll(all);
    }
    if (lane == 0)
        found[wave] = count;
    __syncthreads();
    int end[kFewWaves];
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w)
        end[w] = found[w] + (w ? end[w - 1] : 0);
    const int total = end[kFewWaves - 1];
    const Window<DT, TINY> window((strip * 64 + lane) * 8, a.k);
    f32x8 sum[1];
    sum[0] = 0.0f;
    add_batches(total * wave / kFewWaves, total * (wave + 1) / kFewWaves,
                [&](int64_t e) {
                    int w = 0, before = 0;
#pragma unroll
                    for (int k = 0; k + 1 < kFewWaves; ++k)
                        if (e >= end[k]) {
                            w = k + 1;
                            before = end[k];
                        }
                    return (int64_t)list[w][e - before];
                },
                [&](int64_t row, int) { return window.load(a.dY, row * a.ldy); }, sum);
    __shared__ f32x8 part[kFewWaves][64];
    part[wave][lane] = sum[0];
    __syncthreads();
    if (wave > 0)
        return;
#pragma unroll
    for (int w = 1; w < kFewWaves; ++w)
        sum[0] += part[w][lane];
    put(a, id, window, sum[0]);
}

// ------------------------------------------------------------------- sort
// Stable sort of (id, position) by 8-bit digits, two launches a digit: a
// workgroup counts its tile's digits; then every workgroup finds its tile's
// places from all tiles' counts (at most 256, so no launch scans them) and
// scatters, its keys ranked within their wave by ballots over the digit's bits.
// 32,768 ids below 50,000: 2 x (3.6 + 4.8) us, latency; with the counts scanned by
// launches of their own 2 x 22.
constexpr int kMostTiles = 256;

struct SortArgs {
    const void *ids;           // of the first digit's pass, else null
    int64_t n, rows;
    const uint32_t *key_in;
    const int32_t *pos_in;
    uint32_t *key;
    int32_t *pos;
    uint32_t *counts;          // [tiles][256]
    int64_t tile;              // keys, a multiple of 1,024
    int shift;
};

template <bool WIDE>
__device__ __forceinline__ uint32_t key_at(const SortArgs &a, int64_t i)
{
    if (!a.ids)
        return a.key_in[i];
    const int64_t id = id_at<WIDE>(a.ids, i, a.rows);
    return (uint32_t)(id < 0 ? a.rows : id);             // padding sorts last
}

template <bool WIDE>
__global__ __launch_bounds__(256) void count_digits_kernel(SortArgs a)
{
    __shared__ uint32_t count[256];
    count[threadIdx.x] = 0;
    __syncthreads();
    const int64_t i0 = blockIdx.x * a.tile, i1 = i0 + a.tile < a.n ? i0 + a.tile : a.n;
#pragma unroll 4
    for (int64_t i = i0 + threadIdx.x; i < i1; i += 256)
        atomicAdd(&count[(key_at<WIDE>(a, i) >> a.shift) & 255u], 1u);
    __syncthreads();
    a.counts[(int64_t)blockIdx.x * 256 + threadIdx.x] = count[threadIdx.x];
}

template <bool WIDE>
__global__ __launch_bounds__(1024) void scatter_digits_kernel(SortArgs a)
{
    __shared__ uint32_t base[256], part[2][4][256], in_wave[16][256], wave_sum[4];
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    uint32_t before = 0, all = 0;
    const int tiles = (int)gridDim.x;
#pragma unroll 8
    for (int i = t >> 8; i < tiles; i += 4) {
        const uint32_t c = a.counts[(int64_t)i * 256 + (t & 255)];
        before += i < (int)blockIdx.x ? c : 0;
        all += c;
    }
    part[0][t >> 8][t & 255] = before;
    part[1][t >> 8][t & 255] = all;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        in_wave[4 * i + (t >> 8)][t & 255] = 0;
    __syncthreads();
    uint32_t sum = 0;
    if (t < 256) {
        before = all = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            before += part[0][i][t];
            all += part[1][i][t];
        }
        sum = all;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const uint32_t x = __shfl_up(sum, o, 64);
            sum += lane >= o ? x : 0;
        }
        if (lane == 63)
            wave_sum[wave] = sum;
    }
    __syncthreads();
    if (t < 256) {
        for (int w = 0; w < wave; ++w)
            sum += wave_sum[w];
        base[t] = sum - all + before;
    }
    const int64_t i0 = blockIdx.x * a.tile, i1 = i0 + a.tile < a.n ? i0 + a.tile : a.n;
    const uint64_t lower = lane == 0 ? 0 : ~0ull >> (64 - lane);
    for (int64_t first = i0; first < i1; first += 1024) {
        const int64_t i = first + t;
        const bool live = i < i1;
        uint32_t key = 0;
        int32_t pos = 0;
        if (live) {
            key = key_at<WIDE>(a, i);
            pos = a.ids ? (int32_t)i : a.pos_in[i];
        }
        const uint32_t digit = (key >> a.shift) & 255u;
        uint64_t peers = __ballot(live);
#pragma unroll
        for (int bit = 0; bit < 8; ++bit) {
            const uint64_t set = __ballot((digit >> bit) & 1u);
            peers &= (digit >> bit) & 1u ? set : ~set;
        }
        if (live && (peers & lower) == 0)
            in_wave[wave][digit] = (uint32_t)__popcll(peers);
        __syncthreads();
        // each wave's first place for a digit
        if (t < 256) {
            uint32_t at = base[t];
#pragma unroll
            for (int w = 0; w < 16; ++w) {
                const uint32_t c = in_wave[w][t];
                in_wave[w][t] = at;
                at += c;
            }
            base[t] = at;
        }
        __syncthreads();
        if (live) {
            const uint32_t to = in_wave[wave][digit] + (uint32_t)__popcll(peers & lower);
            a.key[to] = key;
            a.pos[to] = pos;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 4; ++k)
            in_wave[4 * k + (t >> 8)][t & 255] = 0;
        __syncthreads();
    }
}

// start[v]: the first sorted position whose id is at least v (50,000 rows among
// 32,768 ids 6 us: fifteen dependent loads)
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

// ------------------------------------------------------------ sums of runs
// the sum of dY's rows at sorted positions j0 .. j1 - 1
template <int DT, bool TINY, int HOLD>
__device__ __forceinline__ void add_rows(const TableArgs &a, int64_t j0, int64_t j1,
                                         const Window<DT, TINY> (&w)[HOLD], f32x8 (&sum)[HOLD])
{
#pragma unroll
    for (int h = 0; h < HOLD; ++h)
        sum[h] = 0.0f;
    add_batches(j0, j1, [&](int64_t j) { return (int64_t)shared_load(a.pos, j); },
                [&](int64_t row, int h) { return w[h].load(a.dY, row * a.ldy); }, sum);
}

// Of the runs longer than 16, what lies in a chunk of 16 sorted positions: the
// run that the chunk begins in (slot 0) and the one that it ends in (slot 1); and
// which of them starts here.
template <int DT, bool TINY>
__device__ __forceinline__ void cut_runs(const TableArgs &a, int64_t t)
{
    const int64_t c = a.strips == 1 ? t : t / a.strips, strip = t - c * a.strips;
    const Window<DT, TINY> w[1] = {Window<DT, TINY>((strip * 64 + (threadIdx.x & 63)) * 8, a.k)};
    const int64_t first = c * kRun, end = first + kRun < a.n ? first + kRun : a.n;
    const int64_t head = shared_load(a.key, first), tail = shared_load(a.key, end - 1);
    CutRun run{0, (uint32_t)c, 0, 0};
    // (not unrolled: one copy of the sums' code)
#pragma unroll 1
    for (int slot = 0; slot < 2; ++slot) {
        const int64_t v = slot ? tail : head;
        if (v >= a.rows || (slot && tail == head))
            break;
        const int64_t s0 = shared_load(a.start, v), s1 = shared_load(a.start, v + 1);
        if (s1 - s0 <= kRun)
            continue;
        if (s0 >= first)
            run = CutRun{(uint32_t)v, (uint32_t)((s1 - 1) / kRun + 1), (uint32_t)slot, 0};
        f32x8 sum[1];
        add_rows(a, s0 > first ? s0 : first, s1 < end ? s1 : end, w, sum);
        if (w[0].skip < 8)
            w[0].store(a.part, (c * 2 + slot) * a.k, sum[0], GPIC_F32);
    }
    if (strip == 0 && (threadIdx.x & 63) == 0)
        a.run[c] = run;
}

// The cuts' sums of the runs that start in sixteen chunks, a wave a chunk; of a
// run of more than sixteen cuts (no two can start within sixteen chunks) by all
// waves of the workgroup, a narrow row by as many groups of lanes as fit (300,000 x
// 64 of two ids 150 us with one, 38 so).  Bound by latency, where a run is and then its cuts' sums:
// 6 us (18 where ids and starts are read to find it).
constexpr int kJoinWaves = 16;

template <int DT, bool TINY>
__global__ __launch_bounds__(64 * kJoinWaves) void join_cuts_kernel(TableArgs a)
{
    __shared__ f32x8 all[kJoinWaves][64];
    const int lane = threadIdx.x & 63;
    const int64_t wave = wave_index(), chunks = (a.n + kRun - 1) / kRun;
    const int64_t block = a.strips == 1 ? (int64_t)blockIdx.x : blockIdx.x / a.strips;
    const int64_t strip = blockIdx.x - block * a.strips;
    const Window<DT, TINY> w((strip * 64 + lane) * 8, a.k);
    // the runs of the workgroup's chunks, one a lane
    const int64_t c0 = block * kJoinWaves, its = c0 + (lane < kJoinWaves ? lane : 0);
    CutRun run{0, (uint32_t)its, 0, 0};
    if (lane < kJoinWaves && its < chunks)
        run = a.run[its];
    const int cuts = (int)((int64_t)run.end - its);
    const uint64_t large = __ballot(lane < kJoinWaves && cuts > kJoinWaves);
    // lanes that a narrow row takes, of as many groups as fit into a wave
    int span = 64;
    if (a.strips == 1)
        while (span > 1 && span * 4 >= a.k)
            span >>= 1;
    // first this wave's own run, if it is short, then its share of the long one
    for (int pass = 0; pass < 2; ++pass) {
        const int which = pass == 0 ? (int)wave : (large ? __builtin_ctzll(large) : 0);
        const int64_t c = c0 + which;
        const int64_t count = __builtin_amdgcn_readlane(cuts, which);
        const int64_t v = (uint32_t)__builtin_amdgcn_readlane((int)run.row, which);
        const int slot = __builtin_amdgcn_readlane((int)run.slot, which);
        f32x8 sum[1];
        sum[0] = 0.0f;
        auto item = [&](int64_t i) { return i * 2 + (i == c ? slot : 0); };
        if (pass == 0) {
            if (count > kJoinWaves || count <= 0)
                continue;
            add_batches(c, c + count, item,
                        [&](int64_t at, int) { return w.load_sum(a.part, at * a.k); }, sum);
            put(a, v, w, sum[0]);
            continue;
        }
        if (!large)
            break;
        // its groups of lanes take a run of cuts each
        const int groups = kJoinWaves * (64 / span), group = (int)wave * (64 / span) + lane / span;
        const Window<DT, TINY> own((strip * 64 + (lane & (span - 1))) * 8, a.k);
        add_batches(c + count * group / groups, c + count * (group + 1) / groups, item,
                    [&](int64_t at, int) { return own.load_sum(a.part, at * a.k); }, sum);
        for (int o = span; o < 64; o <<= 1)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                sum[0][j] += __shfl_xor(sum[0][j], o, 64);
        all[wave][lane] = sum[0];
        __syncthreads();
        if (wave > 0)
            break;
        for (int i = 1; i < kJoinWaves; ++i)
            sum[0] += all[i][lane];
        put(a, v, w, sum[0]);
    }
}

// The first workgroups cut the long runs, whose chain of loads is hidden behind
// the others, whose waves take a row of the table and 1,024 (ONE: 512) columns
// each.  Bound by memory: 32,768 x 1,024 -> 50,000 in bfloat16, ids as frequent as
// words are, 30 us for both (67 MB read, 102 written), 24 + 10 one after the other.
// With runs of 64 rows a wave 58 us: the longest runs end last.
template <int DT, bool TINY, bool ONE>
__global__ __launch_bounds__(256) void rows_kernel(TableArgs a, int64_t cuts)
{
    if ((int64_t)blockIdx.x < cuts) {
        const int64_t chunks = (a.n + kRun - 1) / kRun;
        for (int64_t t = (int64_t)blockIdx.x * 4 + wave_index(); t < chunks * a.strips; t += cuts * 4)
            cut_runs<DT, TINY>(a, t);
        return;
    }
    using W = Window<DT, TINY>;
    constexpr int kHold = ONE ? 1 : 2;
    const int64_t strips = (a.strips + kHold - 1) / kHold, tasks = a.rows * strips;
    for (int64_t t = ((int64_t)blockIdx.x - cuts) * 4 + wave_index(); t < tasks;
         t += ((int64_t)gridDim.x - cuts) * 4) {
        const int64_t v = strips == 1 ? t : t / strips;
        const int64_t col = ((t - v * strips) * kHold * 64 + (threadIdx.x & 63)) * 8;
        const int64_t j0 = shared_load(a.start, v), j1 = shared_load(a.start, v + 1);
        if (j1 - j0 > kRun || (a.accumulate && j0 == j1))
            continue;
        if constexpr (ONE) {
            const W w[1] = {W(col, a.k)};
            f32x8 sum[1];
            add_rows(a, j0, j1, w, sum);
            put(a, v, w[0], sum[0]);
        } else {
            const W w[2] = {W(col, a.k), W(col + 512, a.k)};
            f32x8 sum[2];
            add_rows(a, j0, j1, w, sum);
            put(a, v, w[0], sum[0]);
            put(a, v, w[1], sum[1]);
        }
    }
}

// ------------------------------------------------------------------- host
unsigned capped(int64_t blocks)
{
    return (unsigned)(blocks < 1 ? 1 : (blocks > (1 << 20) ? 1 << 20 : blocks));
}

struct Sorted {
    uint32_t *key[2], *counts, *start;
    int32_t *pos[2];
    float *part;
    CutRun *run;
    Sorted(const Embedding &p, Cursor &c)
    {
        const size_t n = (size_t)p.n;
        for (int i = 0; i < 2; ++i) {
            key[i] = static_cast<uint32_t *>(c.take(n * 4));
            pos[i] = static_cast<int32_t *>(c.take(n * 4));
        }
        counts = static_cast<uint32_t *>(c.take((size_t)kMostTiles * 256 * 4));
        start = static_cast<uint32_t *>(c.take(((size_t)p.rows + 1) * 4));
        part = static_cast<float *>(c.take((n + kRun - 1) / kRun * 2 * (size_t)p.k * 4));
        run = static_cast<CutRun *>(c.take((n + kRun - 1) / kRun * sizeof(CutRun)));
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
    if (p.k < 8 && p.wide)
        few_ids_kernel<DT, true, true><<<blocks, 64 * kFewWaves, 0, st>>>(a);
    else if (p.k < 8)
        few_ids_kernel<DT, false, true><<<blocks, 64 * kFewWaves, 0, st>>>(a);
    else if (p.wide)
        few_ids_kernel<DT, true, false><<<blocks, 64 * kFewWaves, 0, st>>>(a);
    else
        few_ids_kernel<DT, false, false><<<blocks, 64 * kFewWaves, 0, st>>>(a);
    return hipGetLastError();
}

template <bool WIDE>
hipError_t sort_ids(const Embedding &p, const void *ids, const Sorted &s, int &at, hipStream_t st)
{
    SortArgs a{};
    a.ids = ids;
    a.n = p.n;
    a.rows = p.rows;
    a.counts = s.counts;
    a.tile = (p.n + kMostTiles - 1) / kMostTiles;
    a.tile = (a.tile + 1023) / 1024 * 1024;
    const unsigned tiles = (unsigned)((p.n + a.tile - 1) / a.tile);
    at = 0;
    for (int shift = 0; shift < 32 && (shift == 0 || (p.rows >> shift) != 0); shift += 8) {
        a.shift = shift;
        a.key = s.key[at];
        a.pos = s.pos[at];
        count_digits_kernel<WIDE><<<tiles, 256, 0, st>>>(a);
        RUN(hipGetLastError());
        scatter_digits_kernel<WIDE><<<tiles, 1024, 0, st>>>(a);
        RUN(hipGetLastError());
        a.ids = nullptr;
        a.key_in = s.key[at];
        a.pos_in = s.pos[at];
        at ^= 1;
    }
    at ^= 1;
    return hipSuccess;
}

template <int DT, bool TINY>
hipError_t add_runs(const Embedding &p, const TableArgs &a, hipStream_t st)
{
    const int64_t chunks = (p.n + kRun - 1) / kRun;
    const int64_t joins = (chunks + kJoinWaves - 1) / kJoinWaves * a.strips;
    const int64_t pairs = (a.strips + 1) / 2, cuts = capped((chunks * a.strips + 3) / 4);
    const unsigned rows = capped((p.rows * (a.strips == 1 ? 1 : pairs) + 3) / 4);
    if (a.strips == 1)
        rows_kernel<DT, TINY, true><<<(unsigned)cuts + rows, 256, 0, st>>>(a, cuts);
    else
        rows_kernel<DT, TINY, false><<<(unsigned)cuts + rows, 256, 0, st>>>(a, cuts);
    RUN(hipGetLastError());
    join_cuts_kernel<DT, TINY><<<(unsigned)joins, 64 * kJoinWaves, 0, st>>>(a);
    return hipGetLastError();
}

template <int DT>
hipError_t sorted_ids(const Embedding &p, TableArgs a, void *ws, hipStream_t st)
{
    Cursor c{static_cast<char *>(ws)};
    const Sorted s(p, c);
    int at = 0;
    RUN(p.wide ? sort_ids<true>(p, a.ids, s, at, st) : sort_ids<false>(p, a.ids, s, at, st));
    a.key = s.key[at];
    a.pos = s.pos[at];
    a.start = s.start;
    a.part = s.part;
    a.run = s.run;
    starts_kernel<<<capped((p.rows + 256) / 256), 256, 0, st>>>(a);
    RUN(hipGetLastError());
    return p.k < 8 ? add_runs<DT, true>(p, a, st) : add_runs<DT, false>(p, a, st);
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

bool embedding_fits(const Embedding &p)
{
    const int64_t chunks = (p.n + kRun - 1) / kRun, strips = (p.k + 511) / 512;
    return p.n <= kFewIds || (chunks / kJoinWaves + 1) * strips <= (int64_t)3 << 20;
}

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
