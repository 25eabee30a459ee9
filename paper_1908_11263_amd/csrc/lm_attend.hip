// Plan of the attention and the kernel that joins the pieces of its positions.
#include "lm_attend.h"

namespace qnn_lm {

// One wave a row of outputs.
template <class N, int DIM>
__global__ void __launch_bounds__(256) join_kernel(const float *part, void *out, float *lse, int64_t all, int32_t splits)
{
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (row >= all)
        return;
    const float *ml = part + splits * all * DIM;
    float m = -INFINITY;
    for (int s = lane; s < splits; s += 64)
        m = fmaxf(m, ml[(s * all + row) * 2]);
#pragma unroll
    for (int o = 32; o; o >>= 1)
        m = fmaxf(m, __shfl_xor(m, o, 64));
    constexpr int E = DIM / 64;
    float l = 0.f, v[E] = {};
    if (m != -INFINITY)
        for (int s = 0; s < splits; ++s) {
            const int64_t at = s * all + row;
            const float ms = ml[at * 2];
            if (ms == -INFINITY)
                continue;
            const float f = __builtin_amdgcn_exp2f(ms - m);
            l += ml[at * 2 + 1] * f;
#pragma unroll
            for (int e = 0; e < E; ++e)
                v[e] += part[at * DIM + lane * E + e] * f;
        }
    const float inv = m == -INFINITY ? 0.f : 1.f / l;
#pragma unroll
    for (int e = 0; e < E; ++e)
        store1<N>(out, row * DIM + lane * E + e, v[e] * inv);
    if (lse && lane == 0)
        lse[row] = m == -INFINITY ? -INFINITY : 0.693147180559945f * (m + log2f(l));
}

// Rows a workgroup and pieces of the positions.  Up to 32 rows (16 of 256
// channels, whose outputs fill the registers) go to the kernel whose waves share
// out the positions.  Positions are split until there are two
// workgroups for each of the 256 compute units, in pieces of at least 128
// positions.  Lengths live on the device: the plan goes by what the table can
// reach, the kernels share out the positions that there are.
static AttendPlan plan_attend(const AttendArgs &a, const CacheArgs &c, int dim)
{
    AttendPlan p;
    p.g = a.heads / c.heads;
    p.rows = a.t * p.g;
    p.many = p.rows > (dim == 256 ? 16 : 32);
    p.nr = p.many ? (p.rows <= 64 || dim == 256 ? 1 : 2) : (p.rows <= 16 ? 1 : 2);
    const int32_t tile = (p.many ? 64 : 16) * p.nr;
    p.row_tiles = (p.rows + tile - 1) / tile;
    const int64_t groups = (int64_t)p.row_tiles * c.heads * c.b;
    const int64_t most = ((int64_t)c.width * c.page + 127) / 128;
    int64_t splits = (512 + groups - 1) / groups;
    splits = splits < most ? splits : most;
    p.splits = (int32_t)(splits < 1 ? 1 : splits);
    p.part = nullptr;
    return p;
}

size_t attend_workspace(const AttendArgs &a, const CacheArgs &c, int dim)
{
    const AttendPlan p = plan_attend(a, c, dim);
    if (p.splits == 1)
        return 0;
    return (size_t)p.splits * c.b * a.t * a.heads * (dim + 2) * sizeof(float);
}

template <class N>
static hipError_t launch_join(const AttendArgs &a, const AttendPlan &p, int64_t all, int dim, hipStream_t s)
{
    const dim3 grid((unsigned)((all + 3) / 4));
    if (dim == 64)
        hipLaunchKernelGGL((join_kernel<N, 64>), grid, dim3(256), 0, s, p.part, a.out, a.lse, all, p.splits);
    else if (dim == 128)
        hipLaunchKernelGGL((join_kernel<N, 128>), grid, dim3(256), 0, s, p.part, a.out, a.lse, all, p.splits);
    else
        hipLaunchKernelGGL((join_kernel<N, 256>), grid, dim3(256), 0, s, p.part, a.out, a.lse, all, p.splits);
    return hipGetLastError();
}

hipError_t launch_attend(const AttendArgs &a, const CacheArgs &c, int bits, int dim, int type, void *ws, hipStream_t s)
{
    AttendPlan p = plan_attend(a, c, dim);
    p.part = (float *)ws;
    const hipError_t e = type == QNN_LM_BF16 ? launch_attend_bf16(a, c, p, bits, dim, s)
                                             : launch_attend_f16(a, c, p, bits, dim, s);
    if (e != hipSuccess || p.splits == 1)
        return e;
    const int64_t all = (int64_t)c.b * a.t * a.heads;
    return type == QNN_LM_BF16 ? launch_join<Bf16>(a, p, all, dim, s) : launch_join<F16>(a, p, all, dim, s);
}

}  // namespace qnn_lm
