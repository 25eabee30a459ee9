// Norm after a block, gate, residual scale and norm before the next block
// (qnn_lm_norm_residual), one pass over the data:
//   h' = alpha h + beta gate N_post(y),  x = N_pre(h').
// Bound by memory: a row is read once into registers, normed there twice, and
// written once.  Statistics are taken about the mean, in fp32, from registers
// (mean first, then the squares), so that a large mean costs no digits.
//   8192 rows of 5120 (layer norms, gates, fp32 h): 116 us, 4.35 TB/s, where a
//   copy reaches 5.5; one row of 4096: 5.7 us, of which 3.5 are the kernel (a
//   sum over the workgroup a norm, two a layer norm, one after the other).
#include "lm_common.h"
#include "lm_internal.h"

namespace qnn_lm {

// Sum over the threads of a row: a wave (WAVES = 1) or the workgroup.
template <int WAVES>
__device__ __forceinline__ float row_sum(float v, float *red)
{
#pragma unroll
    for (int o = 32; o; o >>= 1)
        v += __shfl_xor(v, o, 64);
    if constexpr (WAVES > 1) {
        __syncthreads();  // the last sum has been read
        if ((threadIdx.x & 63) == 0)
            red[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0;
#pragma unroll
        for (int i = 0; i < WAVES; ++i)
            v += red[i];
    }
    return v;
}

// Element of the i-th vector of 8 (or, with VEC = 1, the i-th single element)
// of this thread.
template <int WAVES, int VEC>
__device__ __forceinline__ int32_t elem(int i)
{
    const int t = WAVES == 1 ? (threadIdx.x & 63) : threadIdx.x;
    return (i * (WAVES * 64) + t) * VEC;
}

// v <- (v - mean) * rstd * weight + bias over the d elements of the row
template <int WAVES, int VEC, int NV>
__device__ __forceinline__ void norm_row(float (&v)[NV][VEC], int32_t d, bool layer, float eps, const float *weight,
                                         const float *bias, float *red)
{
    if (layer) {
        float s = 0;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                s += v[i][e];  // (zero past the row's end)
        const float mean = row_sum<WAVES>(s, red) / (float)d;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                v[i][e] = elem<WAVES, VEC>(i) < d ? v[i][e] - mean : 0.f;
    }
    float q = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            q += v[i][e] * v[i][e];
    const float rstd = 1.f / sqrtf(row_sum<WAVES>(q, red) / (float)d + eps);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int32_t at = elem<WAVES, VEC>(i);
        if (at >= d)
            continue;
        float w[VEC], b[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            w[e] = 1.f;
            b[e] = 0.f;
        }
        if constexpr (VEC == 8) {
            if (weight)
                load8<F32>(weight, at, w);
            if (bias)
                load8<F32>(bias, at, b);
        } else {
            if (weight)
                w[0] = weight[at];
            if (bias)
                b[0] = bias[at];
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            v[i][e] = v[i][e] * rstd * w[e] + b[e];
    }
}

template <class N, int VEC>
__device__ __forceinline__ void load_vec(const void *p, int64_t at, float (&v)[VEC])
{
    if constexpr (VEC == 8)
        load8<N>(p, at, v);
    else
        v[0] = load1<N>(p, at);
}

template <class N, int VEC>
__device__ __forceinline__ void store_vec(void *p, int64_t at, const float (&v)[VEC])
{
    if constexpr (VEC == 8)
        store8<N>(p, at, v);
    else
        store1<N>(p, at, v[0]);
}

// WAVES waves a row (WAVES = 1: four rows a workgroup), NV vectors of VEC
// elements a thread.
template <class N, class H, int WAVES, int VEC, int NV>
__global__ void __launch_bounds__(WAVES == 1 ? 256 : WAVES * 64) norm_kernel(NormArgs a)
{
    __shared__ float red[WAVES];
    const int64_t row = WAVES == 1 ? (int64_t)workgroup() * 4 + (threadIdx.x >> 6) : workgroup();
    if (row >= a.r)
        return;
    float h[NV][VEC], z[NV][VEC];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int32_t at = elem<WAVES, VEC>(i);
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            h[i][e] = z[i][e] = 0.f;
        if (at < a.d) {
            load_vec<H, VEC>(a.h, row * a.h_pitch + at, h[i]);
            if (a.y)
                load_vec<N, VEC>(a.y, row * a.y_pitch + at, z[i]);
        }
    }
    if (a.y) {
        if (a.post)
            norm_row<WAVES, VEC, NV>(z, a.d, a.layer, a.eps, a.post_weight, a.post_bias, red);
        const int64_t grow = a.gates ? row / a.gate_rows * a.d : 0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int32_t at = elem<WAVES, VEC>(i);
            if (at >= a.d)
                continue;
            if (a.gates) {
                float g[VEC];
                load_vec<N, VEC>(a.gate, grow + at, g);
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    z[i][e] *= g[e];
            }
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                h[i][e] = a.alpha * h[i][e] + a.beta * z[i][e];
            store_vec<H, VEC>(a.h_out, row * a.d + at, h[i]);
        }
    }
    norm_row<WAVES, VEC, NV>(h, a.d, a.layer, a.eps, a.pre_weight, a.pre_bias, red);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int32_t at = elem<WAVES, VEC>(i);
        if (at < a.d)
            store_vec<N, VEC>(a.x, row * a.d + at, h[i]);
    }
}

template <class N, class H, int VEC>
hipError_t launch_sized(const NormArgs &a, hipStream_t s)
{
    // A wave a row up to 1024 elements (16-byte accesses), a workgroup a row
    // above: the fewest registers that hold the row.  One element an access: 8
    // or 32 a thread, the 32 of sixteen waves only (four waves with 32 went to
    // scratch memory: 4000 rows of 7287 4657 us, with sixteen and 8 126; of 7288
    // 79).
    const int64_t vecs = (a.d + VEC - 1) / VEC;  // of a row
#define QNN_LM_NORM(WAVES, NV)                                                                                     \
    if (vecs <= (WAVES) * 64 * (NV)) {                                                                             \
        const dim3 grid = grid_of((WAVES) == 1 ? ((int64_t)a.r + 3) / 4 : a.r);                                    \
        hipLaunchKernelGGL((norm_kernel<N, H, WAVES, VEC, NV>), grid, dim3((WAVES) == 1 ? 256 : (WAVES) * 64),       \
                           0, s, a);                                                                               \
        return hipGetLastError();                                                                                  \
    }
    if constexpr (VEC == 8) {
        QNN_LM_NORM(1, 2)
        QNN_LM_NORM(4, 1)
        QNN_LM_NORM(4, 2)
        QNN_LM_NORM(4, 3)
        QNN_LM_NORM(4, 4)
        QNN_LM_NORM(16, 4)
    } else {
        QNN_LM_NORM(4, 8)
        QNN_LM_NORM(16, 8)
        QNN_LM_NORM(16, 32)
    }
#undef QNN_LM_NORM
    return hipErrorInvalidValue;
}

template <class N, class H>
hipError_t launch_typed(const NormArgs &a, hipStream_t s)
{
    // 16-byte accesses where every row starts on 8 elements
    const bool vec = a.d % 8 == 0 && a.h_pitch % 8 == 0 && (!a.y || a.y_pitch % 8 == 0);
    return vec ? launch_sized<N, H, 8>(a, s) : launch_sized<N, H, 1>(a, s);
}

hipError_t launch_norm(const NormArgs &a, int type, int h_type, hipStream_t s)
{
    if (type == QNN_LM_F32)
        return launch_typed<F32, F32>(a, s);
    if (type == QNN_LM_BF16)
        return h_type == QNN_LM_F32 ? launch_typed<Bf16, F32>(a, s) : launch_typed<Bf16, Bf16>(a, s);
    return h_type == QNN_LM_F32 ? launch_typed<F16, F32>(a, s) : launch_typed<F16, F16>(a, s);
}

}  // namespace qnn_lm
