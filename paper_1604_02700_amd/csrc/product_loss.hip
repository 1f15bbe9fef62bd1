// Matrix products of the loss (product.h): logits to their rows' sums of
// exponentials, logits to their gradients (both operands k-contiguous), and
// the sum over the pieces of the vocabulary of the gradient of the points (A
// k-contiguous, B k-strided).
#include "product.h"

namespace gpic {

namespace {

template <bool BSTR, int EPI>
hipError_t launch_kind(int op, const Plan &p, const ProductArgs &a, hipStream_t s)
{
    if (op == kOpBf16)
        return launch_any_tile<false, BSTR, kOpBf16, EPI>(p, a, s);
    if (op == kOpF16)
        return launch_any_tile<false, BSTR, kOpF16, EPI>(p, a, s);
    return launch_any_tile<false, BSTR, kOpSplit, EPI>(p, a, s);
}

} // namespace

hipError_t launch_product_loss(int op, int epi, const Plan &p, const ProductArgs &a,
                               hipStream_t s)
{
    if (epi == kEpiLse)
        return launch_kind<false, kEpiLse>(op, p, a, s);
    if (epi == kEpiSoft)
        return launch_kind<false, kEpiSoft>(op, p, a, s);
    return launch_kind<true, kEpiSum>(op, p, a, s);
}

} // namespace gpic
