// The linear layer: instances by type and width of weights.
#include "lm_internal.h"

namespace qnn_lm {

hipError_t launch_matmul_bf16_w16(const MatmulArgs &a, void *ws, hipStream_t s);
hipError_t launch_matmul_bf16_w8(const MatmulArgs &a, void *ws, hipStream_t s);
hipError_t launch_matmul_bf16_w4(const MatmulArgs &a, void *ws, hipStream_t s);
hipError_t launch_matmul_bf16_w2(const MatmulArgs &a, void *ws, hipStream_t s);
hipError_t launch_matmul_bf16_w1(const MatmulArgs &a, void *ws, hipStream_t s);
hipError_t launch_matmul_f16_w16(const MatmulArgs &a, void *ws, hipStream_t s);
hipError_t launch_matmul_f16_w8(const MatmulArgs &a, void *ws, hipStream_t s);
hipError_t launch_matmul_f16_w4(const MatmulArgs &a, void *ws, hipStream_t s);
hipError_t launch_matmul_f16_w2(const MatmulArgs &a, void *ws, hipStream_t s);
hipError_t launch_matmul_f16_w1(const MatmulArgs &a, void *ws, hipStream_t s);

static hipError_t launch_bf16(const MatmulArgs &a, int bits, void *ws, hipStream_t s)
{
    switch (bits) {
    case 16: return launch_matmul_bf16_w16(a, ws, s);
    case 8: return launch_matmul_bf16_w8(a, ws, s);
    case 4: return launch_matmul_bf16_w4(a, ws, s);
    case 2: return launch_matmul_bf16_w2(a, ws, s);
    case 1: return launch_matmul_bf16_w1(a, ws, s);
    }
    return hipErrorInvalidValue;
}

static hipError_t launch_f16(const MatmulArgs &a, int bits, void *ws, hipStream_t s)
{
    switch (bits) {
    case 16: return launch_matmul_f16_w16(a, ws, s);
    case 8: return launch_matmul_f16_w8(a, ws, s);
    case 4: return launch_matmul_f16_w4(a, ws, s);
    case 2: return launch_matmul_f16_w2(a, ws, s);
    case 1: return launch_matmul_f16_w1(a, ws, s);
    }
    return hipErrorInvalidValue;
}

// Measured rules (see the kernels' heads):
//   up to 16 rows the weights go straight to registers; above, x is worth
//   sharing through local memory.
//   Tiles of 128 x 256 where they fill the 256 compute units twice over; else
//   tiles of 64 rows of x, and of 128 rows of weights, and pieces of k, until
//   there are workgroups enough.
TilePlan plan_matmul(const MatmulArgs &a, int bits)
{
    TilePlan p = {0, 0, 1, (a.k + 127) / 128 * 128};
    // (the tile kernel's offsets within a tile are 32 bits)
    // (and it copies four scales at a time)
    if (a.r <= 16 || a.x_pitch >= 1 << 23 || a.w_row >= 1 << 23 ||
        (a.groups > 1 && (a.gated ? 2 : 1) * (int64_t)a.m * a.groups < 4))
        return p;
    const int64_t rows = a.gated ? 2 * (int64_t)a.m : a.m;
    const bool near = rows * a.w_row < (int64_t)1 << 31;  // a gated tile of 128 rows reaches both halves
    auto count = [&](int tf, int wf) { return ((int64_t)a.r + 32 * tf - 1) / (32 * tf) * ((rows + 128 * wf - 1) / (128 * wf)); };
    p.tf = 4;
    p.wf = 2;
    if (a.r <= 32 && bits != 16 && (!a.gated || near)) {
        p.tf = p.wf = 1;
    } else if (a.r <= 64 || count(4, 2) < 512) {
        p.tf = 2;
        if (count(2, 2) < 512 && (!a.gated || near))
            p.wf = 1;
    }
    if (p.tf == 4)
        return p;
    const int64_t groups = count(p.tf, p.wf);
    const int32_t blocks = (a.k + 127) / 128;
    int32_t splits = (int32_t)(512 / groups);
    if (splits > blocks / 4)
        splits = blocks / 4;
    if (splits > 8)
        splits = 8;
    if (splits > 1) {
        p.columns = (blocks + splits - 1) / splits * 128;
        p.splits = (a.k + p.columns - 1) / p.columns;
    }
    return p;
}

hipError_t launch_matmul(const MatmulArgs &a, int type, int bits, void *ws, hipStream_t s)
{
    return type == QNN_LM_BF16 ? launch_bf16(a, bits, ws, s) : launch_f16(a, bits, ws, s);
}

size_t matmul_workspace(const MatmulArgs &a, int, int bits)
{
    const TilePlan p = plan_matmul(a, bits);
    return p.splits > 1 ? (size_t)p.splits * a.r * a.m * (a.gated ? 8 : 4) : 0;
}

}  // namespace qnn_lm
