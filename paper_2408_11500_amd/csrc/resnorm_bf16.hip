// Norms around a block on bf16 rows.
#include "resnorm_kernels.h"

namespace slicegcn {
namespace resnorm {

template void launch_fwd<bf16>(const Args &, const Shape &, int64_t, hipStream_t);
template void launch_bwd<bf16>(const Args &, const Shape &, int64_t, hipStream_t);

} // namespace resnorm
} // namespace slicegcn
