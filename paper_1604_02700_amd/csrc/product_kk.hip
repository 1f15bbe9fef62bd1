// Matrix products with both operands k-contiguous (product.h): layers
// forward, Gram matrices of wide matrices and the polynomial's square.
#include "product.h"

namespace gpic {

hipError_t launch_product_kk(int op, int epi, const Plan &p, const ProductArgs &a,
                             hipStream_t s)
{
    if (epi == kEpiLayer) {
        if (op == kOpBf16)
            return launch_any_tile<false, false, kOpBf16, kEpiLayer>(p, a, s);
        if (op == kOpF16)
            return launch_any_tile<false, false, kOpF16, kEpiLayer>(p, a, s);
        return launch_any_tile<false, false, kOpSplit, kEpiLayer>(p, a, s);
    }
    if (epi == kEpiGated) {
        if (op == kOpBf16)
            return launch_any_tile<false, false, kOpBf16, kEpiGated>(p, a, s);
        if (op == kOpF16)
            return launch_any_tile<false, false, kOpF16, kEpiGated>(p, a, s);
        return launch_any_tile<false, false, kOpSplit, kEpiGated>(p, a, s);
    }
    if (epi == kEpiGram)
        return op == kOpF16 ? launch_any_tile<false, false, kOpF16, kEpiGram>(p, a, s)
                            : launch_any_tile<false, false, kOpSplit, kEpiGram>(p, a, s);
    if (epi == kEpiPoly)
        return op == kOpF16 ? launch_any_tile<false, false, kOpF16, kEpiPoly>(p, a, s)
                            : launch_any_tile<false, false, kOpSplit, kEpiPoly>(p, a, s);
    if (epi == kEpiUpdate)
        return op == kOpF16 ? launch_any_tile<false, false, kOpF16, kEpiUpdate>(p, a, s)
                            : launch_any_tile<false, false, kOpSplit, kEpiUpdate>(p, a, s);
    return op == kOpF16 ? launch_any_tile<false, false, kOpF16, kEpiResult>(p, a, s)
                        : launch_any_tile<false, false, kOpSplit, kEpiResult>(p, a, s);
}

} // namespace gpic
