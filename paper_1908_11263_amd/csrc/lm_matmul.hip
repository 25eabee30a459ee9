// The linear layer: instances by type and width of weights.
#include <algorithm>
#include <cmath>

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

// Rules, with what was measured on both sides (us; bf16, 4-bit weights in groups
// of 128 unless said; x rows by columns to outputs):
//   Up to 16 rows the weights go straight to registers; above, x is worth
//   sharing through local memory.
//   Tiles of 128 x 256 where they fill the 256 compute units twice over (4096 x
//   11264 to 4096), else tiles of 64 rows of x (1024 x 4096 to 8192, 8 bits: 79
//   against 90), and of 128 rows of weights where those of 256 do not fill them
//   either (256 x 4096 to 14336: 51 against 64); 32 rows of x where there are
//   no more (32 x 4096 to 22528: 25 against 28).
//   Pieces of k shorten a workgroup's chain of steps, which bounds small grids,
//   and cost their sums' way through memory: about the square root of the chain
//   over the sums, and one more where that asks no compute unit for another
//   workgroup.  128 x 4096 to 4096: 20.9 in 4 pieces, 26 in 2, 39 whole; 256 x
//   4096 to 4096: 26 in 4, 29 in 2, 39 whole; 512 x 4096 to 4096: 37 in 2, 40
//   whole, 41 in 4; 128 x 4096 to 14336: 35.6 in 2, 39.6 whole, 39.4 in 4; 1024 x
//   4096 to 4096: 53 whole, 62 in 2; 16-bit weights, 256 x 4096 to 4096: 23 in 2,
//   29.5 whole, 26 in 4; 128 x 4096 to 14336: 31 whole, 37 in 2; gated, 64 x 4096
//   to 11264: 34.6 in 4, 36 in 3, 37 in 2, 43 whole.
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
    const float chain = bits == 16 ? 1000.f : bits == 8 ? 1900.f : 2500.f;
    int64_t splits = (int64_t)(sqrtf(chain * (float)a.k / ((float)a.r * (float)rows)) + 0.5f);
    if (splits > 0 && (groups * (splits + 1) + 255) / 256 == (groups * splits + 255) / 256)
        ++splits;
    splits = std::min({splits, 768 / groups, (int64_t)blocks / 4, (int64_t)8});
    if (splits > 1) {
        p.columns = (int32_t)((blocks + splits - 1) / splits * 128);
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
