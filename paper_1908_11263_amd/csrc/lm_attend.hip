// Plan of the attention and the kernel that joins the pieces of its positions.
#include "lm_attend.h"

namespace qnn_lm {

constexpr int kMostSplits = 512;

// Joins the pieces of a row's positions: a workgroup a row (with a wave a row,
// whose pieces wait for each other, one token over 32768 positions takes 63 us
// in all instead of 25).  The pieces' maxima
// are read at once and turned into factors; then DIM / 4 threads own four
// channels each of every (1024 / DIM)-th piece (their loads do not wait for each
// other), and the sums of those are added in order.
template <class N, int DIM>
__global__ void __launch_bounds__(256) join_kernel(const float *part, void *out, float *lse, int64_t all, int32_t splits)
{
    constexpr int LANES = DIM / 4, SETS = 256 / LANES;
    __shared__ float factor[kMostSplits], red[8];
    __shared__ f4 sums[SETS][LANES];
    const int64_t row = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const float *ml = part + splits * all * DIM;
    float m[2], l[2], top = -INFINITY;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int s = i * 256 + tid;
        m[i] = s < splits ? ml[(s * all + row) * 2] : -INFINITY;
        l[i] = s < splits ? ml[(s * all + row) * 2 + 1] : 0.f;
        top = fmaxf(top, m[i]);
    }
#pragma unroll
    for (int o = 32; o; o >>= 1)
        top = fmaxf(top, __shfl_xor(top, o, 64));
    if (lane == 0)
        red[wave] = top;
    __syncthreads();
    top = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int s = i * 256 + tid;
        // (a piece that has seen nothing counts for nothing, whatever it holds)
        const float f = m[i] == -INFINITY ? 0.f : fmaxf(__builtin_amdgcn_exp2f(m[i] - top), kLeast);
        if (s < splits)
            factor[s] = f;
        sum += m[i] == -INFINITY ? 0.f : l[i] * f;
    }
#pragma unroll
    for (int o = 32; o; o >>= 1)
        sum += __shfl_xor(sum, o, 64);
    if (lane == 0)
        red[4 + wave] = sum;
    __syncthreads();
    sum = (red[4] + red[5]) + (red[6] + red[7]);
    const int c = tid % LANES, set = tid / LANES;
    f4 v = {0, 0, 0, 0};
#pragma unroll 4
    for (int s = set; s < splits; s += SETS)
        v += *(const f4 *)(part + (s * all + row) * DIM + 4 * c) * factor[s];
    sums[set][c] = v;
    __syncthreads();
    if (tid < LANES) {
        v = sums[0][c];
#pragma unroll
        for (int i = 1; i < SETS; ++i)
            v += sums[i][c];
        const float inv = top == -INFINITY ? 0.f : 1.f / sum;
        const u2 r = {pack2<N>(v[0] * inv, v[1] * inv), pack2<N>(v[2] * inv, v[3] * inv)};
        *(u2 *)((typename N::T *)out + row * DIM + 4 * c) = r;
    }
    if (lse && tid == 0)
        lse[row] = top == -INFINITY ? -INFINITY : 0.693147180559945f * (top + log2f(sum));
}

// Rows a workgroup and pieces of the positions.  Up to 32 rows (16 of 256
// channels, whose outputs fill the registers) go to the kernel whose waves share
// out the positions.  Positions are split until there are two
// workgroups for each of the 256 compute units, in pieces of at least 128
// positions (trees of 16 over 8 sequences of 8192, 8 bits: 63 us so, 76 and 72 us
// with three and four workgroups a unit).  Above 64 rows a wave takes 32: 227
// against 333 us for trees of 61 over 32768 positions at 4 bits.  Lengths live on the device: the plan goes by what the table can
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
    int64_t splits = (kMostSplits + groups - 1) / groups;
    splits = splits < most ? splits : most;  // (at most kMostSplits)
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
    const dim3 grid((unsigned)all);
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
