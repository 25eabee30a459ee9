// The linear layer's kernels for f16 and 8-bit weights.
#include "lm_matmul_impl.h"

namespace qnn_lm {
hipError_t launch_matmul_f16_w8(const MatmulArgs &a, void *ws, hipStream_t s)
{
    return launch_matmul_one<F16, 8>(a, ws, s);
}
}  // namespace qnn_lm
