// The kernels of product.h for f16 rows.
#include "product_launch.h"

namespace slicegcn {

int launch_product_f16(int layouts, int epilogue, const ProductPlan &plan, ProductArgs &a, hipStream_t stream)
{
    return launch_product<f16>(layouts, epilogue, plan, a, stream);
}

} // namespace slicegcn
