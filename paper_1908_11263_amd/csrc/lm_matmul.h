// Shared by the linear layer's kernels.
#pragma once

#include "lm_common.h"
#include "lm_internal.h"

namespace qnn_lm {

// In fp32.  erff and tanhf are the device library's; the exponentials go
// through exp2 (a relative error of about 2^-24 |t|, far below the result's
// rounding to 16 bits).
__device__ __forceinline__ float activate(float t, int act)
{
    switch (act) {
    case QNN_LM_ACT_RELU: return t < 0.f ? 0.f : t;  // (NaN stays)
    case QNN_LM_ACT_SILU: return t / (1.f + __builtin_amdgcn_exp2f(-1.44269504088896f * t));
    case QNN_LM_ACT_GELU: return 0.5f * t * (1.f + erff(0.707106781186548f * t));
    case QNN_LM_ACT_GELU_TANH: return 0.5f * t * (1.f + tanhf(0.797884560802865f * (t + 0.044715f * t * t * t)));
    default: return t;
    }
}

// y[row][col] from its sums (`up`: the second half's, gated layers).
template <class N>
__device__ __forceinline__ void finish(const MatmulArgs &a, int64_t row, int64_t col, float t, float up)
{
    if (a.bias) {
        t += a.bias[col];
        if (a.gated)
            up += a.bias[a.m + col];
    }
    t = activate(t, a.act);
    if (a.gated)
        t *= up;
    if (a.residual)
        t += load1<N>(a.residual, row * a.residual_pitch + col);
    store1<N>(a.y, row * a.y_pitch + col, t);
}

// Bytes of a lane's piece of NF eights of codes.
template <int BITS, int NF>
constexpr int kRaw = NF * BITS;

// Loads NB bytes (1, 2, 4, 8 or 16 of them, at their own alignment).
template <int NB>
__device__ __forceinline__ void load_raw(const uint8_t *p, uint32_t *r)
{
    if constexpr (NB >= 8) {
        load_words<NB / 4>(p, r);
    } else if constexpr (NB == 4) {
        r[0] = *(const uint32_t *)p;
    } else if constexpr (NB == 2) {
        r[0] = *(const uint16_t *)p;
    } else {
        r[0] = *p;
    }
}

}  // namespace qnn_lm
