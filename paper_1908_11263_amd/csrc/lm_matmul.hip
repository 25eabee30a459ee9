// The linear layer: kernel by size (qnn_lm_matmul).
#include "lm_matmul_rows.h"

namespace qnn_lm {

template <class N>
static hipError_t launch_typed(const MatmulArgs &a, int bits, hipStream_t s)
{
    switch (bits) {
    case 16: return launch_rows_bits<N, 16>(a, s);
    case 8: return launch_rows_bits<N, 8>(a, s);
    case 4: return launch_rows_bits<N, 4>(a, s);
    case 2: return launch_rows_bits<N, 2>(a, s);
    case 1: return launch_rows_bits<N, 1>(a, s);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_matmul(const MatmulArgs &a, int type, int bits, void *ws, hipStream_t s)
{
    (void)ws;
    return type == QNN_LM_BF16 ? launch_typed<Bf16>(a, bits, s) : launch_typed<F16>(a, bits, s);
}

size_t matmul_workspace(const MatmulArgs &, int, int) { return 0; }

}  // namespace qnn_lm
