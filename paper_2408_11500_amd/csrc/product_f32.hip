// The kernels of product.h for f32 rows.
#include "product_launch.h"

namespace slicegcn {

int launch_product_f32(int layouts, int epilogue, const ProductPlan &plan, ProductArgs &a, hipStream_t stream)
{
    return launch_product<float>(layouts, epilogue, plan, a, stream);
}

int launch_pair_f32(ProductArgs *x, ProductArgs *w, const BiasSums &bias, hipStream_t stream) { return launch_pair<float>(x, w, bias, stream); }

} // namespace slicegcn
