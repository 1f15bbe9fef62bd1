// Matrix products of the loss (product.h): logits to their rows' sums of
// exponentials, logits to their gradients (both operands k-contiguous), and
// the gradients (B k-strided): of the points, summed over the pieces of the
// vocabulary (A k-contiguous), and of the weights (A k-strided).
#include "product.h"

namespace gpic {

namespace {

template <bool ASTR, bool BSTR, int EPI>
hipError_t launch_kind(int op, const Plan &p, const ProductArgs &a, hipStream_t s)
{
    if (op == kOpBf16)
        return launch_any_tile<ASTR, BSTR, kOpBf16, EPI>(p, a, s);
    if (op == kOpF16)
        return launch_any_tile<ASTR, BSTR, kOpF16, EPI>(p, a, s);
    return launch_any_tile<ASTR, BSTR, kOpSplit, EPI>(p, a, s);
}

} // namespace

hipError_t launch_product_loss(int modes, int op, int epi, const Plan &p, const ProductArgs &a,
                               hipStream_t s)
{
    if (epi == kEpiLse)
        return launch_kind<false, false, kEpiLse>(op, p, a, s);
    if (epi == kEpiSoft)
        return launch_kind<false, false, kEpiSoft>(op, p, a, s);
    return modes == kKM ? launch_kind<false, true, kEpiSum>(op, p, a, s)
                        : launch_kind<true, true, kEpiSum>(op, p, a, s);
}

} // namespace gpic
