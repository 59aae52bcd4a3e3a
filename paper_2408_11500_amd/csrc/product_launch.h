// Which kernel a product of one element type takes.
#pragma once

#include "product_rows.h"

namespace slicegcn {
namespace {

template <class T, int LM, int LN, int EPI, bool SPLIT> int launch_sums(const ProductPlan &plan, ProductArgs &a, hipStream_t stream)
{
    if constexpr (sizeof(T) == 2) {
        if (plan.kernel == BY_TILES) {
            if constexpr (SPLIT) return launch_direct<T, LM, LN, EPI, PARTS>(a, stream);
            else return launch_whole<T, LM, LN, EPI>(plan, a, stream);
        }
        if constexpr (LM == LAYOUT_KC && !SPLIT)
            if (plan.kernel == BY_ROWS) return launch_rows<T, LN, EPI>(a, stream);
    }
    if constexpr (sizeof(T) == 4)
        if (plan.tile == 0) return launch_tile<T, LM, LN, EPI, 0, SPLIT>(a, stream);
    switch (plan.tile) {
    case 1: return launch_tile<T, LM, LN, EPI, 1, SPLIT>(a, stream);
    default: return launch_tile<T, LM, LN, EPI, 2, SPLIT>(a, stream);
    }
}

template <class T, int LM, int LN, int EPI> int launch_layouts(const ProductPlan &plan, ProductArgs &a, hipStream_t stream)
{
    a.splits = plan.splits;
    a.steps_per_split = plan.steps_per_split;
    if constexpr (EPI == EPI_STORE) {
        if (plan.stage == SUMS_ALONE) return launch_sums<T, LM, LN, EPI_STORE, true>(plan, a, stream);
        if (plan.stage == JOIN_ALONE) return launch_join<T, EPI_STORE>(a, stream);
    }
    if (plan.splits == 1) return launch_sums<T, LM, LN, EPI, false>(plan, a, stream);
    const int32_t sets = a.sets;
    if (EPI == EPI_GATED) { // each product by itself, and both joined
        a.sets = 2;
        a.a[1] = a.a[0];
    }
    const int rc = launch_sums<T, LM, LN, EPI_STORE, true>(plan, a, stream);
    a.sets = sets;
    if (rc) return rc;
    return launch_join<T, EPI>(a, stream);
}

template <class T> int launch_product(int layouts, int epilogue, const ProductPlan &plan, ProductArgs &a, hipStream_t stream)
{
    switch (layouts) {
    case PRODUCT_XW:
        return epilogue == EPI_GATED ? launch_layouts<T, LAYOUT_KC, LAYOUT_OC, EPI_GATED>(plan, a, stream)
                                     : launch_layouts<T, LAYOUT_KC, LAYOUT_OC, EPI_FORWARD>(plan, a, stream);
    case PRODUCT_GWT: return launch_layouts<T, LAYOUT_KC, LAYOUT_KC, EPI_STORE>(plan, a, stream);
    default: return launch_layouts<T, LAYOUT_OC, LAYOUT_OC, EPI_STORE>(plan, a, stream);
    }
}

} // namespace
} // namespace slicegcn
