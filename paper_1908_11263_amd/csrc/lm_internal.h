// Launchers of the kernels of include/qnn_lm.h (arguments already checked).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "qnn_internal.h"
#include "qnn_lm.h"

namespace qnn_lm {

// A launch may have fewer than 2^32 threads along an axis: more than 2^20
// workgroups are laid out in rows of so many, and a kernel takes its number from
// workgroup().  The last row's may lie past the end.
inline dim3 grid_of(int64_t groups)
{
    const int64_t row = 1 << 20;
    return groups <= row ? dim3((unsigned)groups) : dim3((unsigned)row, (unsigned)((groups + row - 1) / row));
}
__device__ __forceinline__ uint32_t workgroup() { return blockIdx.y * gridDim.x + blockIdx.x; }

struct MatmulArgs {
    const void *x, *w, *residual;
    const float *scale, *bias;
    void *y;
    int32_t r, k, m, group;      // group: weights of a scale (k itself for one scale a row)
    int32_t groups;              // scales of a row
    int32_t act, gated;
    int64_t x_pitch, residual_pitch, y_pitch;
    int64_t w_row;               // bytes of a row of weights
};
// How the linear layer is cut: rows of x in tiles of 32 tf, rows of weights in
// tiles of 128 wf, k in pieces of `columns`; tf = 0: the kernel for few rows.
struct TilePlan {
    int32_t tf, wf, splits, columns;
};
TilePlan plan_matmul(const MatmulArgs &a, int bits);
hipError_t launch_matmul(const MatmulArgs &a, int type, int bits, void *ws, hipStream_t s);
size_t matmul_workspace(const MatmulArgs &a, int type, int bits);

struct NormArgs {
    const void *h, *y, *gate;
    const float *post_weight, *post_bias, *pre_weight, *pre_bias;
    void *h_out, *x;
    int32_t r, d, layer, post, gates, gate_rows;  // gate_rows: rows that share a row of gate
    float eps, alpha, beta;
    int64_t h_pitch, y_pitch;
};
hipError_t launch_norm(const NormArgs &a, int type, int h_type, hipStream_t s);

struct CacheArgs {
    uint8_t *k, *v;
    float *k_scale, *v_scale;
    const int32_t *table;
    int32_t pages, heads, page, b, width;
    int64_t k_page, k_head, k_slot, v_page, v_head, v_slot;
    qnn::FastDiv page_div;
};
hipError_t launch_append(const CacheArgs &c, int bits, int dim, int type, const void *k, const void *v,
                         const int64_t *k_stride, const int64_t *v_stride, int t, const int32_t *lens,
                         const int32_t *counts, hipStream_t s);
hipError_t launch_keep(const CacheArgs &c, int bits, int dim, int t, const int32_t *lens, const int32_t *path,
                       const int32_t *kept, hipStream_t s);
hipError_t launch_read(const CacheArgs &c, int bits, int dim, int type, int cache_type, int t, const int32_t *start,
                       void *k, void *v, hipStream_t s);

struct AttendArgs {
    const void *q;
    const int32_t *lens, *counts;
    const uint64_t *mask;
    void *out;
    float *lse;
    int32_t t, heads;
    float scale;
    int64_t q_b, q_t, q_h;
};
hipError_t launch_attend(const AttendArgs &a, const CacheArgs &c, int bits, int dim, int type, void *ws, hipStream_t s);
size_t attend_workspace(const AttendArgs &a, const CacheArgs &c, int dim);

}  // namespace qnn_lm
