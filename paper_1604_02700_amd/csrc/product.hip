// Matrix products of the encoder operators: how a product is cut into
// tiles, and the dispatch over operand orders (kernels: product.h).
#include "encoder.h"

namespace gpic {

namespace {

// Measured times in us that the choice of a plan goes by (bfloat16, K = 512
// and 2,048, 64 to 2,560 tiles; an MI355X of 256 compute units).
struct TileCost {
    int edge, resident;        // tiles a compute unit holds at once
    double fixed;              // of a tile: first copies, epilogue
    double step[5];            // of 64 values of k with 1 .. resident tiles on the unit
    double split;              // times this for split operands (32 values of k),
                               // whose results have twice the bytes: 1.8 times `fixed`
};
constexpr TileCost kCost[3] = {
    {256, 1, 10.0, {1.50}, 1.39},
    {128, 2, 5.0, {0.74, 1.06}, 1.25},
    {64, 5, 3.0, {0.38, 0.47, 0.63, 0.77, 1.03}, 1.1},
};
constexpr int kUnits = 256;
constexpr double kJoin = 4.0;              // the join's launch
constexpr double kJoinBytes = 3.0e6;       // partial sums written and read, bytes per us

// `n` workgroups of `steps` steps each
double time_of(const TileCost &c, bool split, int64_t n, double steps)
{
    if (n <= 0)
        return 0.0;
    const int64_t slots = (int64_t)kUnits * c.resident, full = n / slots, rest = n % slots;
    const double f = split ? c.split : 1.0, fixed = c.fixed * (split ? 1.8 : 1.0);
    double t = (double)full * (fixed + steps * c.step[c.resident - 1] * f);
    if (rest)
        t += fixed + steps * c.step[(rest - 1) / kUnits] * f;
    return t;
}

} // namespace

// Every tile size; all tiles whole, or the last round's tiles (or all of
// them) in parts, whichever the measured times say is shortest.
Plan product_plan(int64_t M, int64_t N, int64_t K, int64_t batch, int op, int epi)
{
    Plan best{};
    best.splits = 1;
    best.fits = M <= 0 || N <= 0 || batch <= 0;
    if (best.fits)
        return best;
    const bool sym = symmetric(epi), split = op == kOpSplit;
    const int64_t step = split ? 32 : 64, steps = (K + step - 1) / step;
    static const int kParts[] = {2, 3, 4, 6, 8, 12, 16, 24, 32};
    double least = 0.0;
    for (int t = 0; t < 3; ++t) {
        const TileCost &c = kCost[t];
        const int64_t tm = (M + c.edge - 1) / c.edge, tn = (N + c.edge - 1) / c.edge;
        const int64_t tiles = (sym ? tn * (tn + 1) / 2 : tm * tn) * batch;
        auto consider = [&](int64_t whole, int parts) {
            const int64_t tail = tiles - whole;
            // a grid of 2^32 threads or more is refused (2^30 rows of a narrow matrix)
            if ((whole + tail * parts) * (c.edge == 256 ? 512 : 256) >= (int64_t)1 << 32)
                return;
            double time = time_of(c, split, whole, (double)steps);
            size_t bytes = 0;
            if (tail) {
                bytes = (size_t)parts * tail * c.edge * c.edge * sizeof(float);
                time += time_of(c, split, tail * parts, (double)((steps + parts - 1) / parts)) +
                        kJoin + 2.0 * (double)bytes / kJoinBytes;
            }
            if (least != 0.0 && time >= least)
                return;
            least = time;
            best = Plan{true, t, (int)tm, (int)tn, whole, tail, tail ? parts : 1, bytes};
        };
        consider(tiles, 1);
        const int64_t slots = (int64_t)kUnits * c.resident, round = tiles / slots * slots;
        for (int parts : kParts)
            if (parts * 2 <= steps) {
                if (round < tiles)
                    consider(round, parts);
                if (round > 0 && tiles < 2 * slots)
                    consider(0, parts);
            }
    }
    return best;
}

hipError_t launch_product(int modes, int op, int epi, const ProductArgs &a, hipStream_t s)
{
    const Plan p = product_plan(a.M, epi == kEpiGated ? 2 * a.e.half : a.N, a.K, a.batch, op, epi);
    if (!p.fits)
        return hipErrorInvalidValue;
    if (p.whole + p.tail == 0)
        return hipSuccess;
    if (modes == kKK)
        return launch_product_kk(op, epi, p, a, s);
    if (modes == kKM)
        return launch_product_km(op, epi, p, a, s);
    return launch_product_mm(op, epi, p, a, s);
}

} // namespace gpic
