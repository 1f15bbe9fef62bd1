// Matrix products with both operands k-strided (product.h): the gradient
// of a layer's weights and the Gram matrix of a tall orthogonalisation.
#include "product.h"

namespace gpic {

hipError_t launch_product_mm(int op, int epi, const Plan &p, const ProductArgs &a,
                             hipStream_t s)
{
    if (epi == kEpiLayer) {
        if (op == kOpBf16)
            return launch_any_tile<true, true, kOpBf16, kEpiLayer>(p, a, s);
        if (op == kOpF16)
            return launch_any_tile<true, true, kOpF16, kEpiLayer>(p, a, s);
        return launch_any_tile<true, true, kOpSplit, kEpiLayer>(p, a, s);
    }
    return op == kOpF16 ? launch_any_tile<true, true, kOpF16, kEpiGram>(p, a, s)
                        : launch_any_tile<true, true, kOpSplit, kEpiGram>(p, a, s);
}

} // namespace gpic
