// Norms around a block on fp32 rows.
#include "resnorm_kernels.h"

namespace slicegcn {
namespace resnorm {

template void launch_fwd<float>(const Args &, const Shape &, int64_t, hipStream_t);
template void launch_bwd<float>(const Args &, const Shape &, int64_t, hipStream_t);

} // namespace resnorm
} // namespace slicegcn
