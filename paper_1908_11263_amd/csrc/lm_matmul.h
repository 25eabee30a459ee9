// Shared by the linear layer's kernels.
#pragma once

#include "lm_common.h"
#include "lm_internal.h"

namespace qnn_lm {

// t Phi(t) from erfc x = p(u) exp(-x^2), u = 1 / (1 + 0.425 x), x = |t| / sqrt 2:
// p without a constant, of degree 8, is fitted to erfc's scaled form so that its
// largest relative error over 0 .. 9.6 is least (1.3e-7, found by weighted least
// squares).  Nothing cancels below 0: the result is within 3e-6 of itself for |t|
// < 5 and 1e-5 for |t| < 9, where the exponential's argument rounds, far below its
// own rounding to 16 bits.  (t / 2 (1 + erf) in 32 bits is off by 3e-4 at -3.5.)
__device__ __forceinline__ float gelu(float t)
{
    const float x = __builtin_fabsf(t) * 0.707106781186548f;
    const float u = __builtin_amdgcn_rcpf(__builtin_fmaf(0.425f, x, 1.f));
    float p = __builtin_fmaf(0.0720406324f, u, -0.315499127f);
    p = __builtin_fmaf(p, u, 0.41165176f);
    p = __builtin_fmaf(p, u, -0.106962503f);
    p = __builtin_fmaf(p, u, 0.25704947f);
    p = __builtin_fmaf(p, u, 0.200111344f);
    p = __builtin_fmaf(p, u, 0.241935894f);
    p = __builtin_fmaf(p, u, 0.239672408f);
    const float q = 0.5f * p * u * __builtin_amdgcn_exp2f(x * x * -1.44269504088896f);  // Phi(-|t|)
    return t * (t > 0.f ? 1.f - q : q);
}

// In fp32.  tanhf is the device library's; the exponentials go through exp2 (a
// relative error of about 2^-24 |t|, far below the result's rounding to 16 bits).
__device__ __forceinline__ float activate(float t, int act)
{
    switch (act) {
    case QNN_LM_ACT_RELU: return t < 0.f ? 0.f : t;  // (NaN stays)
    case QNN_LM_ACT_SILU: return t / (1.f + __builtin_amdgcn_exp2f(-1.44269504088896f * t));
    case QNN_LM_ACT_GELU: return gelu(t);
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
