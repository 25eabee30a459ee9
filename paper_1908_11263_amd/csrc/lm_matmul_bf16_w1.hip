// The linear layer's kernels for bf16 and 1-bit weights.
#include "lm_matmul_impl.h"

namespace qnn_lm {
hipError_t launch_matmul_bf16_w1(const MatmulArgs &a, void *ws, hipStream_t s)
{
    return launch_matmul_one<Bf16, 1>(a, ws, s);
}
}  // namespace qnn_lm
