// Matrix products of the encoder operators: which tile, how many parts of
// the contraction, and the dispatch over operand orders (kernels:
// product.h).
#include "encoder.h"

namespace gpic {

namespace {

constexpr int kSize[3] = {256, 128, 64};         // tile edges

int64_t tiles_of(int M, int N, int edge, int batch, bool sym)
{
    const int64_t tm = (M + edge - 1) / edge, tn = (N + edge - 1) / edge;
    return (sym ? tn * (tn + 1) / 2 : tm * tn) * batch;
}

} // namespace

int product_tile(int M, int N, int64_t K, int batch, int op, bool sym);

int product_tile(int M, int N, int64_t, int batch, int, bool sym)
{
    for (int t = 0; t < 2; ++t)
        if (tiles_of(M, N, kSize[t], batch, sym) >= 192)
            return t;
    return 2;
}

int product_splits(int M, int N, int64_t K, int batch, int op, bool sym)
{
    const int t = product_tile(M, N, K, batch, op, sym);
    const int64_t tiles = tiles_of(M, N, kSize[t], batch, sym);
    const int64_t steps = (K + (op == kOpSplit ? 31 : 63)) / (op == kOpSplit ? 32 : 64);
    if (tiles <= 0 || tiles >= 192 || steps < 16)
        return 1;
    int64_t parts = 512 / tiles;
    if (parts > steps / 8)
        parts = steps / 8;
    if (parts > 32)
        parts = 32;
    return parts < 2 ? 1 : (int)parts;
}

size_t product_part_bytes(int M, int N, int batch, int splits)
{
    if (splits < 2)
        return 0;
    return (size_t)splits * batch * M * (((size_t)N + 63) / 64 * 64) * sizeof(float);
}

hipError_t launch_product(int modes, int op, int epi, const ProductArgs &a, hipStream_t s)
{
    if (a.M <= 0 || a.N <= 0 || a.batch <= 0)
        return hipSuccess;
    if (modes == kKK)
        return launch_product_kk(op, epi, a, s);
    if (modes == kKM)
        return launch_product_km(op, epi, a, s);
    return launch_product_mm(op, epi, a, s);
}

} // namespace gpic
