// Matrix products with A k-contiguous and B k-strided (product.h): the
// gradient of a layer's input and the update of a wide orthogonalisation.
#include "product.h"

namespace gpic {

hipError_t launch_product_km(int op, int epi, const Plan &p, const ProductArgs &a,
                             hipStream_t s)
{
    if (epi == kEpiLayer) {
        if (op == kOpBf16)
            return launch_any_tile<false, true, kOpBf16, kEpiLayer>(p, a, s);
        if (op == kOpF16)
            return launch_any_tile<false, true, kOpF16, kEpiLayer>(p, a, s);
        return launch_any_tile<false, true, kOpSplit, kEpiLayer>(p, a, s);
    }
    if (epi == kEpiUpdate)
        return op == kOpF16 ? launch_any_tile<false, true, kOpF16, kEpiUpdate>(p, a, s)
                            : launch_any_tile<false, true, kOpSplit, kEpiUpdate>(p, a, s);
    return op == kOpF16 ? launch_any_tile<false, true, kOpF16, kEpiResult>(p, a, s)
                        : launch_any_tile<false, true, kOpSplit, kEpiResult>(p, a, s);
}

} // namespace gpic
