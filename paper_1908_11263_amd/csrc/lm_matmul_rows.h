// The linear layer for up to 16 rows (a token, a small tree of drafts): bound
// by reading the weights once.
//
// y = x w^T on the 16x16x32 matrix instruction, A = 16 rows of x, B = 16 rows
// of weights.  A lane holds NF eights of consecutive codes of one row of
// weights, loaded straight from memory into registers (16 bytes where the
// codes allow it) and expanded there: nothing is staged, nothing is shared, no
// barrier in the loop.  The four lanes of a row take consecutive pieces, so a
// step covers 32 NF columns of k in an order of its own; x is read at the same
// columns.  A step lies inside one group, so a group's scale multiplies the
// step's sums (exact products, fp32 sums), one scale a lane.
// A workgroup owns 16 WR rows of weights (16 WR / 2 outputs where gated: gate
// and up rows side by side) and 16 NC rows of x; its waves split k and are
// joined through local memory in a fixed order.
//   One row of bf16, 8192 to 16384: 16-bit weights 39 us (6.8 TB/s), 8 bits 27 us
//   (5.0), 4 bits in groups of 128 21 us (3.4: expanding the codes); 4096 to 4096
//   at 4 bits: 5.3 us, the launch and one chain of loads.  16 rows, 4096 to 16384
//   at 4 bits: 19 us.
#pragma once

#include "lm_matmul.h"

namespace qnn_lm {

template <class N, int BITS, int NF, int WR, int NC, bool GATED, bool XL>
struct RowsTile {
    static constexpr int kStep = 32 * NF;
    uint32_t w[WR][kRaw<BITS, NF> < 4 ? 1 : kRaw<BITS, NF> / 4];
    typename N::V8 x[XL ? 1 : NC][XL ? 1 : NF];  // XL: x lies in local memory
    float scale[WR];

    // (Never skipped: behind a branch that may skip a load, a wait for an older
    // one has to be a wait for all.  Pieces past k are read from the row's start
    // and cleared in add().)
    __device__ __forceinline__ void load(const MatmulArgs &a, const uint8_t *const (&wp)[WR],
                                         const typename N::T *const (&xp)[NC], const float *const (&sp)[WR],
                                         int32_t k0, int kq)
    {
        int32_t k = k0 + kq * 8 * NF;  // this lane's piece
        k = k < a.k ? k : 0;
#pragma unroll
        for (int r = 0; r < WR; ++r) {
            load_raw<kRaw<BITS, NF>>(wp[r] + (int64_t)k * BITS / 8, w[r]);
            if constexpr (BITS != 16)
                scale[r] = sp[r][a.groups > 1 ? k0 >> __builtin_ctz(a.group) : 0];
        }
        if constexpr (!XL)
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int f = 0; f < NF; ++f)
                    x[c][f] = *(const typename N::V8 *)(xp[c] + k + 8 * f);
    }

    // xl: this lane's row of x in local memory (XL), zero past k.
    __device__ __forceinline__ void add(f4 (&acc)[WR][NC], const MatmulArgs &a, int32_t k0, int kq,
                                        const typename N::T *xl)
    {
        const bool grouped = BITS != 16 && a.groups > 1;
        if (k0 + kStep > a.k && k0 + kq * 8 * NF >= a.k) {
            // (a code is finite whatever its bits, a 16-bit weight need not be)
            if constexpr (!XL) {
                const u4 zero = {0, 0, 0, 0};
#pragma unroll
                for (int c = 0; c < NC; ++c)
#pragma unroll
                    for (int f = 0; f < NF; ++f)
                        x[c][f] = __builtin_bit_cast(typename N::V8, zero);
            }
            if constexpr (BITS == 16)
#pragma unroll
                for (int r = 0; r < WR; ++r)
#pragma unroll
                    for (uint32_t &v : w[r])
                        v = 0;
        }
#pragma unroll
        for (int r = 0; r < WR; ++r) {
            f4 part[NC];
#pragma unroll
            for (int c = 0; c < NC; ++c)
                part[c] = grouped ? (f4){0, 0, 0, 0} : acc[r][c];
            steps<0>(r, part, xl + k0 + kq * 8 * NF);
#pragma unroll
            for (int c = 0; c < NC; ++c)
                acc[r][c] = grouped ? acc[r][c] + scale[r] * part[c] : part[c];
        }
    }

    template <int F>
    __device__ __forceinline__ void steps(int r, f4 (&part)[NC], const typename N::T *xl) const
    {
        if constexpr (F < NF) {
            const typename N::V8 b = expand<N, BITS, F>(w[r]);
            if constexpr (XL) {
                part[0] = mfma16(*(const typename N::V8 *)(xl + 8 * F), b, part[0]);
            } else {
#pragma unroll
                for (int c = 0; c < NC; ++c)
                    part[c] = mfma16(x[c][F], b, part[c]);
            }
            steps<F + 1>(r, part, xl);
        }
    }
};

// Bytes of x in local memory.
template <int NF>
size_t rows_x_bytes(const MatmulArgs &a)
{
    constexpr int64_t step = 32 * NF;
    return (size_t)a.r * (size_t)(((a.k + step - 1) / step * step + 8) * 2);
}

template <class N, int BITS, int NF, int WR, int NC, bool GATED, bool XL, int WAVES>
__global__ void __launch_bounds__(64 * WAVES) matmul_rows_kernel(MatmulArgs a)
{
    using Tile = RowsTile<N, BITS, NF, WR, NC, GATED, XL>;
    static_assert(!XL || NC == 1, "sixteen rows at most");
    constexpr int AHEAD = NC == 1 ? 4 : 2;
    extern __shared__ f4 part[];  // [wave][WR][NC][64]; before that, XL: x
    const int lane = threadIdx.x & 63, l16 = lane & 15, kq = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    constexpr int OUT = GATED ? 8 * WR : 16 * WR;  // outputs of a workgroup
    const int32_t j0 = blockIdx.x * OUT, r0 = blockIdx.y * 16 * NC;
    const uint8_t *wp[WR];
    const float *sp[WR];
    const typename N::T *xp[NC];
#pragma unroll
    for (int r = 0; r < WR; ++r) {
        // rows past the last one repeat it; their sums are not stored
        const int32_t j = min(j0 + (GATED ? r / 2 : r) * 16 + l16, a.m - 1);
        const int64_t row = GATED && (r & 1) ? a.m + j : j;
        wp[r] = (const uint8_t *)a.w + row * a.w_row;
        sp[r] = BITS == 16 ? nullptr : a.scale + row * a.groups;
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int32_t r = min(r0 + c * 16 + l16, a.r - 1);
        xp[c] = (const typename N::T *)a.x + r * a.x_pitch;
    }
    f4 acc[WR][NC];
#pragma unroll
    for (int r = 0; r < WR; ++r)
#pragma unroll
        for (int c = 0; c < NC; ++c)
            acc[r][c] = (f4){0, 0, 0, 0};
    // a wave's share of the steps, in one piece
    const int32_t steps = (a.k + Tile::kStep - 1) / Tile::kStep;
    const int32_t share = (steps + WAVES - 1) / WAVES;
    const int32_t first = min(wave * share, steps), last = min(first + share, steps);
    // AHEAD steps are in flight, each in registers of its own
    Tile t[AHEAD];
    auto load = [&](Tile &tile, int32_t s) { tile.load(a, wp, xp, sp, max(min(s, last - 1), 0) * Tile::kStep, kq); };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
        load(t[i], first + i);
    // x (XL): whole rows, zero up to whole steps, a row's pieces off the next one's banks
    typename N::T *xl = (typename N::T *)part;
    if constexpr (XL) {
        const int32_t kp = steps * Tile::kStep, pieces = kp / 8;
        for (int32_t e = threadIdx.x; e < a.r * pieces; e += 64 * WAVES) {
            const int32_t r = e / pieces, k = (e - r * pieces) * 8;
            u4 v = {0, 0, 0, 0};
            if (k < a.k)
                v = *(const u4 *)((const typename N::T *)a.x + r * a.x_pitch + k);
            *(u4 *)(xl + r * (kp + 8) + k) = v;
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();  // (the weights' loads stay in flight)
        asm volatile("" ::: "memory");
        xl += min(l16, a.r - 1) * (kp + 8);
    }
    int32_t s = first;
    for (; last - s > AHEAD; s += AHEAD)
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            t[i].add(acc, a, (s + i) * Tile::kStep, kq, xl);
            load(t[i], s + i + AHEAD);
        }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
        if (s + i < last)
            t[i].add(acc, a, (s + i) * Tile::kStep, kq, xl);
    if constexpr (XL)
        __syncthreads();  // x has been read
#pragma unroll
    for (int r = 0; r < WR; ++r) {
        float unscale = kUnscale<BITS>;
        if (BITS != 16 && a.groups == 1)
            unscale *= sp[r][0];
#pragma unroll
        for (int c = 0; c < NC; ++c)
            part[((wave * WR + r) * NC + c) * 64 + lane] = acc[r][c] * unscale;
    }
    __syncthreads();
    // element e of the workgroup's outputs: lane l of a tile holds column
    // l % 16 at rows 4 * (l / 16) .. + 3
    constexpr int OT = GATED ? WR / 2 : WR;
    for (int e = threadIdx.x; e < OT * NC * 64; e += 64 * WAVES) {
        const int l = e & 63, c = (e >> 6) % NC, o = (e >> 6) / NC;
        f4 t = {0, 0, 0, 0}, up = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            t += part[((w * WR + (GATED ? 2 * o : o)) * NC + c) * 64 + l];
            if constexpr (GATED)
                up += part[((w * WR + 2 * o + 1) * NC + c) * 64 + l];
        }
        const int32_t col = j0 + o * 16 + (l & 15);
        if (col >= a.m)
            continue;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int32_t row = r0 + c * 16 + 4 * (l >> 4) + i;
            if (row < a.r)
                finish<N>(a, row, col, t[i], up[i]);
        }
    }
}

template <class N, int BITS, int NF, int WR, int NC, bool GATED, bool XL, int WAVES>
hipError_t launch_rows(const MatmulArgs &a, hipStream_t s)
{
    constexpr int OUT = GATED ? 8 * WR : 16 * WR;
    const dim3 grid((a.m + OUT - 1) / OUT, (a.r + 16 * NC - 1) / (16 * NC));
    size_t lds = WAVES * WR * NC * 64 * sizeof(f4);
    if (XL && lds < rows_x_bytes<NF>(a))
        lds = rows_x_bytes<NF>(a);
    hipLaunchKernelGGL((matmul_rows_kernel<N, BITS, NF, WR, NC, GATED, XL, WAVES>), grid, dim3(64 * WAVES), lds, s, a);
    return hipGetLastError();
}

// Up to 16 rows: x is read from local memory where it fits (32 KB leave room
// for more workgroups); two blocks of rows of weights a workgroup where that
// leaves two workgroups for each compute unit, as x is then read half as often.
template <class N, int BITS, int NF, bool GATED>
hipError_t launch_rows_few(const MatmulArgs &a, hipStream_t s)
{
    const int64_t rows = GATED ? 2 * (int64_t)a.m : a.m;
    const bool local = rows_x_bytes<NF>(a) <= 32 * 1024;
    if (GATED || rows >= 32 * 512)
        return local ? launch_rows<N, BITS, NF, 2, 1, GATED, true, 8>(a, s)
                     : launch_rows<N, BITS, NF, 2, 1, GATED, false, 8>(a, s);
    if constexpr (!GATED)
        return local ? launch_rows<N, BITS, NF, 1, 1, false, true, 8>(a, s)
                     : launch_rows<N, BITS, NF, 1, 1, false, false, 8>(a, s);
    return hipErrorInvalidValue;
}

template <class N, int BITS, int NF>
hipError_t launch_rows_sized(const MatmulArgs &a, hipStream_t s)
{
    if (a.r <= 16)
        return a.gated ? launch_rows_few<N, BITS, NF, true>(a, s) : launch_rows_few<N, BITS, NF, false>(a, s);
    // (more only where the kernel of tiles cannot address the operands)
    return a.gated ? launch_rows<N, BITS, NF, 2, 4, true, false, 8>(a, s)
                   : launch_rows<N, BITS, NF, 2, 4, false, false, 8>(a, s);
}

// A lane's piece is a quarter of a group at most.
template <class N, int BITS>
hipError_t launch_rows_bits(const MatmulArgs &a, hipStream_t s)
{
    if constexpr (BITS == 16)
        return launch_rows_sized<N, 16, 1>(a, s);
    const int32_t g = a.groups > 1 ? a.group : 128;
    if (g == 32)
        return launch_rows_sized<N, BITS, 1>(a, s);
    if (g == 64 || BITS == 8)
        return launch_rows_sized<N, BITS, 2>(a, s);
    if constexpr (BITS < 8)
        return launch_rows_sized<N, BITS, 4>(a, s);
    return hipErrorInvalidValue;
}

}  // namespace qnn_lm
