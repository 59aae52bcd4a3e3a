// The kernels of product.h for bf16 rows.
#include "product_launch.h"
#include "product_narrow.h"

namespace slicegcn {

int launch_product_bf16(int layouts, int epilogue, const ProductPlan &plan, ProductArgs &a, hipStream_t stream)
{
    return launch_product<bf16>(layouts, epilogue, plan, a, stream);
}

int launch_narrow_bf16(const NarrowArgs &a, ProductArgs &join, int act, bool gated, unsigned blocks, hipStream_t stream)
{
    if (int rc = launch_narrow<bf16>(a, act, gated, blocks, stream)) return rc;
    return a.want_w ? launch_join<bf16, EPI_STORE>(join, stream) : SLICEGCN_OK;
}

int launch_pair_bf16(ProductArgs *x, ProductArgs *w, const BiasSums &bias, hipStream_t stream) { return launch_pair<bf16>(x, w, bias, stream); }

} // namespace slicegcn
