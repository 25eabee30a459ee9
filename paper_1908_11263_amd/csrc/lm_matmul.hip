// The linear layer: instances by type and width of weights.
#include "lm_internal.h"

namespace qnn_lm {

hipError_t launch_matmul_bf16_w16(const MatmulArgs &a, hipStream_t s);
hipError_t launch_matmul_bf16_w8(const MatmulArgs &a, hipStream_t s);
hipError_t launch_matmul_bf16_w4(const MatmulArgs &a, hipStream_t s);
hipError_t launch_matmul_bf16_w2(const MatmulArgs &a, hipStream_t s);
hipError_t launch_matmul_bf16_w1(const MatmulArgs &a, hipStream_t s);
hipError_t launch_matmul_f16_w16(const MatmulArgs &a, hipStream_t s);
hipError_t launch_matmul_f16_w8(const MatmulArgs &a, hipStream_t s);
hipError_t launch_matmul_f16_w4(const MatmulArgs &a, hipStream_t s);
hipError_t launch_matmul_f16_w2(const MatmulArgs &a, hipStream_t s);
hipError_t launch_matmul_f16_w1(const MatmulArgs &a, hipStream_t s);

static hipError_t launch_bf16(const MatmulArgs &a, int bits, hipStream_t s)
{
    switch (bits) {
    case 16: return launch_matmul_bf16_w16(a, s);
    case 8: return launch_matmul_bf16_w8(a, s);
    case 4: return launch_matmul_bf16_w4(a, s);
    case 2: return launch_matmul_bf16_w2(a, s);
    case 1: return launch_matmul_bf16_w1(a, s);
    }
    return hipErrorInvalidValue;
}

static hipError_t launch_f16(const MatmulArgs &a, int bits, hipStream_t s)
{
    switch (bits) {
    case 16: return launch_matmul_f16_w16(a, s);
    case 8: return launch_matmul_f16_w8(a, s);
    case 4: return launch_matmul_f16_w4(a, s);
    case 2: return launch_matmul_f16_w2(a, s);
    case 1: return launch_matmul_f16_w1(a, s);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_matmul(const MatmulArgs &a, int type, int bits, void *ws, hipStream_t s)
{
    (void)ws;
    return type == QNN_LM_BF16 ? launch_bf16(a, bits, s) : launch_f16(a, bits, s);
}

size_t matmul_workspace(const MatmulArgs &, int, int) { return 0; }

}  // namespace qnn_lm
