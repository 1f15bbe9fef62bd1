// Matrix products of the encoder operators: how a product is cut into
// tiles, and the dispatch over operand orders (kernels: product.h).
#include "encoder.h"

namespace gpic {

Plan product_plan(int64_t M, int64_t N, int64_t K, int64_t batch, int op, int epi)
{
    Plan p{};
    p.splits = 1;
    if (M <= 0 || N <= 0 || batch <= 0)
        return p;
    const bool sym = epi == kEpiSym;
    int64_t tiles = 0;
    for (int t = 0; t < 3; ++t) {
        const int edge = 256 >> t;
        const int64_t tm = (M + edge - 1) / edge, tn = (N + edge - 1) / edge;
        tiles = (sym ? tn * (tn + 1) / 2 : tm * tn) * batch;
        p.tile = t;
        p.tm = (int)tm;
        p.tn = (int)tn;
        if (tiles >= 192)
            break;
    }
    p.whole = tiles;
    const int64_t step = op == kOpSplit ? 32 : 64, steps = (K + step - 1) / step;
    if (tiles < 192 && steps >= 16) {
        int64_t parts = 512 / tiles;
        parts = parts > steps / 8 ? steps / 8 : parts;
        parts = parts > 32 ? 32 : parts;
        if (parts >= 2) {
            p.whole = 0;
            p.tail = tiles;
            p.splits = (int)parts;
            const int64_t edge = 256 >> p.tile;
            p.part_bytes = (size_t)(parts * tiles * edge * edge) * sizeof(float);
        }
    }
    return p;
}

hipError_t launch_product(int modes, int op, int epi, const ProductArgs &a, hipStream_t s)
{
    const Plan p = product_plan(a.M, epi == kEpiGated ? 2 * a.e.half : a.N, a.K, a.batch, op, epi);
    if (p.whole + p.tail == 0)
        return hipSuccess;
    if (p.whole + p.tail * p.splits > 0x7fffffffll)
        return hipErrorInvalidValue;
    if (modes == kKK)
        return launch_product_kk(op, epi, p, a, s);
    if (modes == kKM)
        return launch_product_km(op, epi, p, a, s);
    return launch_product_mm(op, epi, p, a, s);
}

} // namespace gpic
