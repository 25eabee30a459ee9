// The linear layer for more than 16 rows (trees of drafts, prompts).  With codes
// it is bound by the vector units, which expand them, and the matrix units, which
// hardly overlap (busy 50 and 45 % of the time in the largest tiles at 4 bits in
// groups).  With 16-bit weights no unit is full (matrix 45 %, vector 14 %, reads
// of local memory 18 %): waves wait a third of their time for the copies and the
// barriers around them, and nearly half to issue.
//
// y = x w^T on the 32x32x16 matrix instruction, A = 32 rows of x, B = 32 rows
// of weights.  A workgroup of four waves owns 32 TF rows of x and 128 WF rows of
// weights; a wave all of the former and 32 WF of the latter, so that every code
// is expanded once a workgroup, in registers, by the wave that multiplies it.
// x and the packed codes stream through local memory in steps of KS columns,
// copied there by the memory unit itself (no registers), two or three steps
// ahead, with one barrier a step.  Sixteen-byte pieces are permuted within a
// row by the row's number, so that the fragments' reads spread over the banks;
// the copy writes them in lane order, so the permutation is applied to the
// address that a lane reads from memory.
//   4096 x 4096 to 8192, bf16: 4 bits and a scale a row 250 us (1099 TFLOP/s),
//   in groups of 128 286 us, 8 bits 262 us, 16 bits 295 us, 2 bits in groups 301
//   us, 1 bit 304 us; 4096 x 11264 to 4096, 4 bits in groups: 373 us (1015
//   TFLOP/s; 368 to 398 from card to card).  A product of two 16-bit matrices of
//   the first size takes 1510 to 1600 TFLOP/s in a library.
//
// k is taken in blocks of 32: lane l holds row l % 32 at k = 16 (l / 32) .. +
// 15 of the block, two eights, the same for x and weights.
//
// Group scales: the sums are kept in units of the current group's scale and
// multiplied by the ratio of the old scale to the new one where a group ends
// (one fp32 product, where a second set of accumulators would not fit).  A
// group whose scale is zero, or 2^-40 of the row's largest before it, keeps the
// unit and has its codes cleared, as in units of its scale the sums could pass
// fp32.  Where such a group holds codes after all (a quantizer that gives empty
// groups the smallest scale there is leaves none), where a scale is 2^40 times
// those before it, or where sums have passed fp32, the wave forms its sums anew
// with an accumulator for each group (sums_by_groups).  1024 x 4096 to 4096 at 4
// bits: 56 us, 288 where every third group is 2^-70 of the others and counts, 80
// where those are empty.
#pragma once

#include "lm_matmul.h"

namespace qnn_lm {

__device__ __forceinline__ f16v mfma32(bf8 a, bf8 b, f16v c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f16v mfma32(h8 a, h8 b, f16v c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

// Copies 16 (or 4) bytes a lane from base + off to local memory at lds + 16 (4)
// * lane, without registers.  The counter of outstanding loads is waited for
// by hand (wait_copies).
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"  // (m0 is reserved; the compiler keeps nothing there)
template <int BYTES>
__device__ __forceinline__ void copy_to_lds(const void *base, uint32_t off, uint32_t lds)
{
    // (a wait state between the write of m0 and the copy that uses it)
    if constexpr (BYTES == 16)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base)
                     : "memory", "m0");
    else
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(lds), "v"(off), "s"(base)
                     : "memory", "m0");
}
#pragma clang diagnostic pop

// Until at most N of this wave's copies are outstanding and its reads of local
// memory are back.
template <int N>
__device__ __forceinline__ void wait_copies()
{
    static_assert(N < 64, "the counter has six bits");
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
}

template <int BITS, int TF, int WF, int GPB>  // GPB: groups of a step (0: one scale a row)
struct TileShape {
    static constexpr int KS = BITS == 16 ? 32 : 64;    // columns of a step
    static constexpr int BM = 32 * TF, BN = 128 * WF;  // rows of x and of weights
    static constexpr int kXRow = KS * 2, kWRow = KS * BITS / 8;  // bytes of a staged row
    static constexpr int kXChunks = kXRow / 16;
    static constexpr int kWUnit = BITS >= 4 ? 16 : 4;  // bytes of a copy of weights
    static constexpr int kWUnits = kWRow / kWUnit;     // of a row
    static constexpr int kXCopies = BM * kXRow / 1024 / 4;         // instructions of a wave a step
    static constexpr int kWCopies = BN * kWUnits / 64 / 4;
    static constexpr int kCopies = kXCopies + kWCopies;  // (now and then one of scales besides)
    static constexpr int kXBytes = BM * kXRow, kWBytes = BN * kWRow;
    static constexpr int kStage = kXBytes + kWBytes;
    // Scales come four groups at a time, 16 bytes a row (one at a time they
    // would be as many requests as x and the codes together).  A place is used
    // again when the copies ahead can no longer need it.
    static constexpr int kScaleRing = GPB == 2 ? 3 : 2, kScaleSteps = GPB == 2 ? 2 : 4;  // steps of four groups, at least
    static constexpr int kScales = GPB ? kScaleRing * BN * 16 : 0;
    // two workgroups a compute unit
    static constexpr int kStages = 4 * kStage + kScales <= 64 * 1024 ? 4 : 3 * kStage + kScales <= 80 * 1024 ? 3 : 2;
    static_assert(!GPB || kStages <= (kScaleRing - 1) * kScaleSteps, "scales are overwritten too early");
    static constexpr int kOutPitch = BN + 4;                  // floats
    static constexpr int kOut = 32 * kOutPitch * 4;
    static constexpr int kLds = kStages * kStage + kScales > kOut ? kStages * kStage + kScales : kOut;

    // Place of piece c of row r among the row's pieces: 256 bytes of local memory
    // answer at once, so the pieces that sixteen neighbouring lanes read, one a
    // row, have to lie at sixteen different places of 256 bytes.
    static __device__ __forceinline__ int x_place(int r, int c)
    {
        return c ^ (kXChunks == 8 ? (r >> 1) & 7 : (r >> 2) & 3);
    }
    static __device__ __forceinline__ int w_place(int r, int c)
    {
        if constexpr (BITS == 8 || BITS == 16)  // four pieces
            return c ^ ((r >> 2) & 3);
        else if constexpr (BITS == 4)
            return c ^ ((r >> 3) & 1);
        else
            return c;
    }
};

struct TileGrid {
    int32_t tm, tn;         // tiles of rows of x, of rows of weights
    int32_t splits, steps;  // pieces of k, of so many steps
    float *part;            // [splits][r][rows of weights] sums, where there is more than one piece
};

// Operands of one eight: every second one of a wave's is in flight while the
// other is multiplied.
template <class N, int TF, int WF>
struct Eight {
    typename N::V8 x[TF], w[WF];
};

// Codes of one block, as they lie in local memory.
template <int BITS, int WF>
struct Raw {
    uint32_t w[WF][BITS >= 2 ? BITS / 2 : 1];
};

// Reads x and expands the codes of eight F of block b.
template <class N, int BITS, int TF, int WF, int GPB, int F>
__device__ __forceinline__ void fetch(const uint8_t *xs, const Raw<BITS, WF> &raw, const uint32_t (&clear)[WF], int b,
                                      int l32, int half, Eight<N, TF, WF> &e)
{
    using S = TileShape<BITS, TF, WF, GPB>;
#pragma unroll
    for (int m = 0; m < TF; ++m) {
        const int r = m * 32 + l32;
        e.x[m] = *(const typename N::V8 *)(xs + r * S::kXRow + S::x_place(r, 4 * b + 2 * half + F) * 16);
    }
#pragma unroll
    for (int n = 0; n < WF; ++n) {
        uint32_t w[BITS >= 2 ? BITS / 2 : 1];
#pragma unroll
        for (int i = 0; i < (BITS >= 2 ? BITS / 2 : 1); ++i)
            // (a 1-bit code has no zero: its numbers are cleared instead)
            w[i] = GPB && BITS != 1 ? raw.w[n][i] & ~clear[n] : raw.w[n][i];
        e.w[n] = expand<N, BITS, F>(w);
        if constexpr (GPB && BITS == 1) {
            u4 v = __builtin_bit_cast(u4, e.w[n]);
            v &= ~clear[n];
            e.w[n] = __builtin_bit_cast(typename N::V8, v);
        }
    }
}

template <class N, int TF, int WF>
__device__ __forceinline__ void products(const Eight<N, TF, WF> &e, f16v (&acc)[TF][WF])
{
#pragma unroll
    for (int n = 0; n < WF; ++n)
#pragma unroll
        for (int m = 0; m < TF; ++m)
            acc[m][n] = mfma32(e.x[m], e.w[n], acc[m][n]);
}

// Asks for what multiplies and what prepares the next eight to alternate.
template <int PRODUCTS>
__device__ __forceinline__ void interleave()
{
#pragma unroll
    for (int i = 0; i < PRODUCTS; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // a product
        __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);  // reads of local memory
        __builtin_amdgcn_sched_group_barrier(0x002, 8, 0);  // vector instructions
    }
}

// Scales that are this many times apart are not brought to one another's unit.
constexpr float kApart = 0x1p40f;

// Whether clearing groups, or bringing the sums before one to its unit, has lost
// something of a row: a group of codes that are not all zero, a scale 1 / kApart
// of an earlier one, or codes before a scale kApart times theirs.
template <int BITS>
__device__ __forceinline__ bool groups_lost(const uint8_t *w, const float *scale, int32_t first, int32_t last, int32_t group)
{
    auto empty = [&](int32_t g) {
        if (BITS == 1)
            return false;  // (there is no code of zero)
        const uint8_t *p = w + (int64_t)g * group * BITS / 8;
        uint32_t any = 0;
        for (int i = 0; i < group * BITS / 8; i += 8) {
            const u2 v = *(const u2 *)(p + i);
            any |= v.x | v.y;
        }
        return any == 0;
    };
    float top = 0.f;
#pragma unroll 1
    for (int32_t g = first; g < last; ++g) {
        const float s = __builtin_fabsf(scale[g]);
        if (s == 0.f)
            continue;
        if (s * kApart < top && !empty(g))
            return true;
        if (top != 0.f && top * kApart < s)
            for (int32_t e = first; e < g; ++e)
                if (scale[e] != 0.f && !empty(e))
                    return true;
        top = fmaxf(top, s);
    }
    return false;
}

// The sums of a block of 32 rows of x by 32 of weights (x, w: this lane's rows)
// over groups first to last, each group's products in an accumulator of its own:
// straight from memory, for weights whose scales lie far apart.
template <class N, int BITS>
__device__ __forceinline__ f16v sums_by_groups(const typename N::T *x, const uint8_t *w, const float *scale, int32_t first,
                                               int32_t last, int32_t group, int half)
{
    f16v sum = {};
#pragma unroll 1
    for (int32_t g = first; g < last; ++g) {
        f16v part = {};
#pragma unroll 1
        for (int32_t k = g * group + 16 * half; k < (g + 1) * group; k += 32)
#pragma unroll
            for (int f = 0; f < 2; ++f) {
                uint32_t raw[2] = {0, 0};
                load_raw<BITS>(w + (int64_t)(k + 8 * f) * BITS / 8, raw);
                part = mfma32(*(const typename N::V8 *)(x + k + 8 * f), expand<N, BITS, 0>(raw), part);
            }
        sum += part * scale[g];
    }
    return sum;
}

template <class N, int BITS, int TF, int WF, int GPB, bool GATED>
__global__ void __launch_bounds__(256, 2) matmul_tile_kernel(MatmulArgs a, TileGrid g)
{
    using S = TileShape<BITS, TF, WF, GPB>;
    // A gated layer's wave holds a gate's rows and their partners: two blocks of
    // 32 (WF = 2), or the halves of one (WF = 1).
    constexpr int GR = GATED ? 16 * WF : 0, HR = GATED ? GR : 1;  // rows of a wave's half
    extern __shared__ __align__(16) uint8_t lds[];
    const int lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    constexpr int OUT = GATED ? S::BN / 2 : S::BN;  // outputs of a row

    // Tiles in an order that keeps an XCD (workgroups go round the eight of
    // them) on neighbouring tiles, eight tiles of x to a column of weights.
    const int32_t tiles = g.tm * g.tn;
    const int32_t split = blockIdx.x / tiles;
    int32_t t = blockIdx.x - split * tiles;
    {
        const int32_t q = tiles >> 3, rem = tiles & 7, x = t & 7;
        t = x * q + min(x, rem) + (t >> 3);
    }
    const int32_t band = t / (8 * g.tn), first = band * 8, high = min(8, g.tm - first);
    const int32_t in = t - band * 8 * g.tn;
    const int32_t r0 = (first + in % high) * S::BM, j0 = in / high * OUT;

    // What this lane copies: offsets from the tile's first row of x, and from
    // the first row of weights of each copy (all of a copy's rows lie in one of
    // the two halves of a gated layer).
    const uint8_t *xb = (const uint8_t *)a.x + (int64_t)r0 * a.x_pitch * 2;
    uint32_t xo[S::kXCopies], wo[S::kWCopies];
    int xc[S::kXCopies], wc[S::kWCopies];  // the piece, for the last step
#pragma unroll
    for (int i = 0; i < S::kXCopies; ++i) {
        const int e = (wave * S::kXCopies + i) * 64 + lane, r = e / S::kXChunks;
        xc[i] = S::x_place(r, e % S::kXChunks);
        xo[i] = (uint32_t)min(r, a.r - 1 - r0) * (uint32_t)(a.x_pitch * 2) + xc[i] * 16;
    }
    const uint8_t *wb[S::kWCopies];
#pragma unroll
    for (int i = 0; i < S::kWCopies; ++i) {
        const int e0 = (wave * S::kWCopies + i) * 64, e = e0 + lane, r = e / S::kWUnits;
        wc[i] = S::w_place(r, e % S::kWUnits);
        wb[i] = (const uint8_t *)a.w + (int64_t)j0 * a.w_row;
        if constexpr (GATED) {
            // staged row 2 GR w + GR f + r is row GR w + r of half f
            const int j = min(j0 + r / (2 * HR) * HR + r % HR, a.m - 1) - j0;
            if constexpr (WF == 2) {
                const int up = (e0 / S::kWUnits >> 5) & 1;
                wb[i] += (int64_t)up * a.m * a.w_row;
                wo[i] = (uint32_t)j * (uint32_t)a.w_row + wc[i] * S::kWUnit;
            } else {
                // (a copy's rows lie in both halves: the launcher sees to 32 bits)
                wo[i] = (uint32_t)((r / HR & 1) * a.m + j) * (uint32_t)a.w_row + wc[i] * S::kWUnit;
            }
        } else {
            wo[i] = (uint32_t)(min(j0 + r, a.m - 1) - j0) * (uint32_t)a.w_row + wc[i] * S::kWUnit;
        }
    }
    // Scales: four of a row a lane (gated: a half's rows, then the other's).  A
    // row's last four may lie before its place, so that nothing is read past
    // the end of all.
    const int32_t begin = split * g.steps;  // first step
    const int gshift = GPB ? __builtin_ctz(a.group) : 0;
    const int64_t most = (GATED ? 2 * (int64_t)a.m : a.m) * a.groups - 4;  // last place of four
    const float *sb = nullptr;
    int64_t sfirst = 0, srow = 0;  // elements: of sb, of this lane's row
    if constexpr (GPB) {
        const int e = (WF == 2 ? wave : wave & 1) * 64 + lane;
        const int up = GATED ? e / (S::BN / 2) : 0, j = GATED ? e % (S::BN / 2) : e;
        srow = ((int64_t)up * a.m + min(j0 + j, a.m - 1)) * a.groups;
        sfirst = ((int64_t)(GATED && WF == 2 ? wave >> 1 : 0) * a.m + j0) * a.groups - 4;
        sfirst = sfirst < 0 ? 0 : sfirst;
        sb = a.scale + sfirst;
    }
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)lds;

    auto issue = [&](int32_t step, int buf) {
        const int32_t k0 = step * S::KS, left = a.k - k0;  // a multiple of 32
        const uint32_t at = lds0 + buf * S::kStage;
        if constexpr (GPB) {
            // before the step's other copies: those are counted, this one is not
            const int32_t quad = k0 >> gshift >> 2;
            if (step == begin || (k0 & ((4 << gshift) - 1)) == 0) {
                const int64_t e = srow + 4 * quad < most ? srow + 4 * quad : most;
                copy_to_lds<16>(sb, (uint32_t)(e - sfirst) * 4,
                                lds0 + S::kStages * S::kStage + quad % S::kScaleRing * (S::BN * 16) +
                                    (WF == 2 ? wave : wave & 1) * 1024);
            }
        }
        const uint8_t *x = xb + (int64_t)k0 * 2;
        const int64_t w = (int64_t)k0 * BITS / 8;
        const uint32_t xat = at + wave * S::kXCopies * 1024,
                       wat = at + S::kXBytes + wave * S::kWCopies * 64 * S::kWUnit;
        if (left >= S::KS) {
#pragma unroll
            for (int i = 0; i < S::kXCopies; ++i)
                copy_to_lds<16>(x, xo[i], xat + i * 1024);
#pragma unroll
            for (int i = 0; i < S::kWCopies; ++i)
                copy_to_lds<S::kWUnit>(wb[i] + w, wo[i], wat + i * 64 * S::kWUnit);
        } else {
            // pieces past the row's end, never read, copy its first again
#pragma unroll
            for (int i = 0; i < S::kXCopies; ++i)
                copy_to_lds<16>(x, xc[i] * 8 < left ? xo[i] : xo[i] - xc[i] * 16, xat + i * 1024);
#pragma unroll
            for (int i = 0; i < S::kWCopies; ++i)
                copy_to_lds<S::kWUnit>(wb[i] + w, wc[i] * (S::kWUnit * 8 / BITS) < left ? wo[i] : wo[i] - wc[i] * S::kWUnit,
                                       wat + i * 64 * S::kWUnit);
        }
    };

    f16v acc[TF][WF];
#pragma unroll
    for (int m = 0; m < TF; ++m)
#pragma unroll
        for (int n = 0; n < WF; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                acc[m][n][i] = 0.f;
    float unit[WF], top[WF];  // the sums' unit, the largest scale so far
    uint32_t clear[WF];       // 0 where the group's codes count
    uint32_t low[WF];         // the smallest but zero, by bits: twice them without the sign, less one
#pragma unroll
    for (int n = 0; n < WF; ++n)
        unit[n] = 1.f, top[n] = 0.f, clear[n] = 0, low[n] = 0xFFFFFFFFu;

    const int32_t steps = min(begin + g.steps, (a.k + S::KS - 1) / S::KS);
    constexpr int BLOCKS = S::KS / 32;
    float f[BLOCKS][WF];  // old unit over new, of the group that begins with a block
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
        for (int n = 0; n < WF; ++n)
            f[b][n] = 1.f;
    Raw<BITS, WF> raw[BLOCKS];
    auto read_raw = [&](const uint8_t *ws) {
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
            for (int n = 0; n < WF; ++n) {
                const int r = (wave * WF + n) * 32 + l32;
                const uint8_t *p = ws + r * S::kWRow;
                uint32_t *to = raw[b].w[n];
                if constexpr (BITS == 16) {
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        load_words<4>(p + S::w_place(r, 2 * half + h) * 16, to + 4 * h);
                } else if constexpr (BITS == 8) {
                    load_words<4>(p + S::w_place(r, 2 * b + half) * 16, to);
                } else if constexpr (BITS == 4) {
                    load_words<2>(p + S::w_place(r, b) * 16 + half * 8, to);
                } else {
                    load_raw<2 * BITS>(p + b * 4 * BITS + half * 2 * BITS, to);
                }
            }
    };
    // Scales from a row's first to the last place of four.
    int32_t sleft[WF];
#pragma unroll
    for (int n = 0; n < WF; ++n) {
        const int q = n * 32 + l32;  // row of this wave
        const int32_t j = min(j0 + (GATED ? wave * GR + q % HR : wave * WF * 32 + q), a.m - 1);
        const int64_t left = most - ((GATED && q >= GR ? (int64_t)a.m : 0) + j) * a.groups;
        sleft[n] = (int32_t)(left < 1 << 30 ? left : 1 << 30);
    }
    // Whether block b of step s begins a group; if so its scale is the new unit.
    auto begins = [&](int32_t s, int b) {
        if constexpr (!GPB) {
            return false;
        } else {
            const int32_t k = s * S::KS + b * 32;
            if (k & (a.group - 1))
                return false;
            const int32_t group = k >> gshift, quad = group >> 2;
            const float *ss = (const float *)(lds + S::kStages * S::kStage + quad % S::kScaleRing * (S::BN * 16));
#pragma unroll
            for (int n = 0; n < WF; ++n) {
                const int at = !GATED ? (wave * WF + n) * 32 + l32
                               : WF == 2 ? n * 128 + wave * 32 + l32 : (l32 >> 4) * 64 + wave * 16 + (l32 & 15);
                const float sc = ss[at * 4 + (group & 3) + max(0, 4 * quad - sleft[n])];
                const bool small = __builtin_fabsf(sc) * kApart < top[n] || sc == 0.f;
                low[n] = min(low[n], 2 * __float_as_uint(sc) - 1);
                clear[n] = small ? 0xFFFFFFFFu : 0;
                f[b][n] = small || top[n] == 0.f ? 1.f : unit[n] / sc;  // (no sums yet)
                unit[n] = small ? unit[n] : sc;
                top[n] = fmaxf(top[n], __builtin_fabsf(sc));
            }
            return true;
        }
    };
    auto rescale = [&](int b) {
#pragma unroll
        for (int m = 0; m < TF; ++m)
#pragma unroll
            for (int n = 0; n < WF; ++n)
                acc[m][n] *= f[b][n];
    };
    // (no branch between an eight's products and the next one's preparation:
    // they are to alternate)
    auto multiply = [&](const Eight<N, TF, WF> &e) {
        products<N, TF, WF>(e, acc);
        interleave<TF * WF>();
    };

#pragma unroll
    for (int s = 0; s < S::kStages - 1; ++s)
        issue(min(begin + s, steps - 1), s);
    wait_copies<(S::kStages - 2) * S::kCopies>();
    __builtin_amdgcn_s_barrier();
    issue(min(begin + S::kStages - 1, steps - 1), S::kStages - 1);
    int buf = 0;
    // (k is a multiple of 32: the last step of all may be one block)
    const bool half_step = BLOCKS == 2 && steps * S::KS > a.k;
    const int32_t whole = half_step ? steps - 1 : steps;
    if constexpr (TF == 4) {
        // an eight ahead
        Eight<N, TF, WF> pair[2];
        read_raw(lds + S::kXBytes);
        bool scale = begins(begin, 0);
        fetch<N, BITS, TF, WF, GPB, 0>(lds, raw[0], clear, 0, l32, half, pair[0]);
        for (int32_t s = begin; s < whole; ++s) {
            const uint8_t *xs = lds + buf * S::kStage;
            if (GPB && scale)
                rescale(0);
            fetch<N, BITS, TF, WF, GPB, 1>(xs, raw[0], clear, 0, l32, half, pair[1]);
            multiply(pair[0]);
            if constexpr (BLOCKS == 2) {
                if constexpr (GPB == 2)
                    begins(s, 1);
                fetch<N, BITS, TF, WF, GPB, 0>(xs, raw[1], clear, 1, l32, half, pair[0]);
                multiply(pair[1]);
                if constexpr (GPB == 2)
                    rescale(1);
                fetch<N, BITS, TF, WF, GPB, 1>(xs, raw[1], clear, 1, l32, half, pair[1]);
                multiply(pair[0]);
            }
            // Everything of this step has been read: the next one's copies are
            // waited for, and this one's place is filled again (past the last step
            // with the last one, so that the counts stay).
            wait_copies<(S::kStages - 2) * S::kCopies>();
            __builtin_amdgcn_s_barrier();
            issue(min(s + S::kStages, steps - 1), buf);
            buf = buf == S::kStages - 1 ? 0 : buf + 1;
            const uint8_t *xn = lds + buf * S::kStage;
            read_raw(xn + S::kXBytes);
            scale = s + 1 < steps && begins(s + 1, 0);
            fetch<N, BITS, TF, WF, GPB, 0>(xn, raw[0], clear, 0, l32, half, pair[0]);
            multiply(pair[1]);
        }
        if (half_step) {
            const uint8_t *xs = lds + buf * S::kStage;
            if (GPB && scale)
                rescale(0);
            fetch<N, BITS, TF, WF, GPB, 1>(xs, raw[0], clear, 0, l32, half, pair[1]);
            multiply(pair[0]);
            multiply(pair[1]);
        }
    } else {
        // Smaller tiles have too few products in an eight to cover local
        // memory's answers, and the registers for whole steps: a step ahead.
        Eight<N, TF, WF> ahead[2][2 * BLOCKS];
        bool scale[2] = {false, false};  // a group begins with the step
        auto prepare = [&](int32_t s, Eight<N, TF, WF> (&to)[2 * BLOCKS], bool &first) {
            const uint8_t *xs = lds + buf * S::kStage;
            read_raw(xs + S::kXBytes);
            first = s < steps && begins(s, 0);
            fetch<N, BITS, TF, WF, GPB, 0>(xs, raw[0], clear, 0, l32, half, to[0]);
            fetch<N, BITS, TF, WF, GPB, 1>(xs, raw[0], clear, 0, l32, half, to[1]);
            if constexpr (BLOCKS == 2) {
                if constexpr (GPB == 2)
                    if (s < whole)
                        begins(s, 1);
                fetch<N, BITS, TF, WF, GPB, 0>(xs, raw[1], clear, 1, l32, half, to[2]);
                fetch<N, BITS, TF, WF, GPB, 1>(xs, raw[1], clear, 1, l32, half, to[3]);
            }
        };
        // The scales of step s + 1 are read while step s is multiplied: what
        // step s is brought to has been put aside.
        float g[BLOCKS][WF];
        auto set_aside = [&] {
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                for (int n = 0; n < WF; ++n)
                    g[b][n] = f[b][n];
        };
        auto bring = [&](int b) {
#pragma unroll
            for (int m = 0; m < TF; ++m)
#pragma unroll
                for (int n = 0; n < WF; ++n)
                    acc[m][n] *= g[b][n];
        };
        auto step = [&](int32_t s, const Eight<N, TF, WF> (&cur)[2 * BLOCKS], bool first, Eight<N, TF, WF> (&next)[2 * BLOCKS],
                        bool &next_first) {
            if constexpr (GPB)
                set_aside();
            // Step s has been read: its place is filled again (past the last
            // step with the last one, so that the counts stay).
            wait_copies<(S::kStages - 2) * S::kCopies>();
            __builtin_amdgcn_s_barrier();
            issue(min(s + S::kStages, steps - 1), buf);
            buf = buf == S::kStages - 1 ? 0 : buf + 1;
            prepare(s + 1, next, next_first);
            if (GPB && first)
                bring(0);
            products<N, TF, WF>(cur[0], acc);
            products<N, TF, WF>(cur[1], acc);
            if constexpr (BLOCKS == 2) {
                if constexpr (GPB == 2)
                    bring(1);
                products<N, TF, WF>(cur[2], acc);
                products<N, TF, WF>(cur[3], acc);
            }
        };
        prepare(begin, ahead[0], scale[0]);
        int32_t s = begin;
        for (; s + 1 < whole; s += 2) {
            step(s, ahead[0], scale[0], ahead[1], scale[1]);
            step(s + 1, ahead[1], scale[1], ahead[0], scale[0]);
        }
        const bool odd = s < whole;
        if (odd)
            step(s, ahead[0], scale[0], ahead[1], scale[1]);
        if (half_step) {
            if (GPB && (odd ? scale[1] : scale[0]))
                rescale(0);
            if (odd) {
                products<N, TF, WF>(ahead[1][0], acc);
                products<N, TF, WF>(ahead[1][1], acc);
            } else {
                products<N, TF, WF>(ahead[0][0], acc);
                products<N, TF, WF>(ahead[0][1], acc);
            }
        }
    }
    if constexpr (GPB != 0) {
        bool apart = false, passed = false;  // scales far apart; sums that are not finite
#pragma unroll
        for (int n = 0; n < WF; ++n)
            apart |= __uint_as_float((low[n] >> 1) + 1) * kApart < top[n];
#pragma unroll
        for (int m = 0; m < TF; ++m)
#pragma unroll
            for (int n = 0; n < WF; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    passed |= !(__builtin_fabsf(acc[m][n][i]) < INFINITY);
        if (__any(apart || passed)) {
            const uint8_t *w[WF];
            const float *scale[WF];
            const int32_t g0 = (begin * S::KS) >> gshift, g1 = (min(steps * S::KS, a.k) + a.group - 1) >> gshift;
#pragma unroll
            for (int n = 0; n < WF; ++n) {
                const int q = n * 32 + l32;  // row of this wave
                const int32_t j = min(j0 + (GATED ? wave * GR + q % HR : wave * WF * 32 + q), a.m - 1);
                const int64_t row = GATED && q >= GR ? (int64_t)a.m + j : j;
                w[n] = (const uint8_t *)a.w + row * a.w_row;
                scale[n] = a.scale + row * a.groups;
                passed |= apart && groups_lost<BITS>(w[n], scale[n], g0, g1, a.group);
            }
            if (__any(passed)) {
#pragma unroll
                for (int m = 0; m < TF; ++m) {
                    const typename N::T *x = (const typename N::T *)a.x + min(r0 + m * 32 + l32, a.r - 1) * a.x_pitch;
#pragma unroll
                    for (int n = 0; n < WF; ++n)
                        acc[m][n] = sums_by_groups<N, BITS>(x, w[n], scale[n], g0, g1, a.group, half);
                }
#pragma unroll
                for (int n = 0; n < WF; ++n)
                    unit[n] = 1.f;
            }
        }
    }
    // the copies of the last steps, made again, are there before local memory
    // is used anew
    wait_copies<0>();
    __syncthreads();

    // Epilogue: sums to results in registers, 32 rows at a time through local
    // memory, from where rows are written (and the residual read) 16 bytes a lane.
    float *out = (float *)lds;
    float bias[WF];
    // (the largest tiles are taken where there are enough of them: never in pieces)
    const bool pieces = TF < 4 && g.splits > 1;
    const int64_t rows = GATED ? 2 * (int64_t)a.m : a.m;
#pragma unroll
    for (int n = 0; n < WF; ++n) {
        const int q = n * 32 + l32;  // row of this wave
        const int32_t j = min(j0 + (GATED ? wave * GR + q % HR : wave * WF * 32 + q), a.m - 1);
        const int64_t row = GATED && q >= GR ? (int64_t)a.m + j : j;
        unit[n] *= kUnscale<BITS>;
        if (BITS != 16 && !GPB)
            unit[n] *= a.scale[row];
        bias[n] = a.bias && !pieces ? a.bias[row] : 0.f;
    }
    const bool wide = !pieces || (a.m & 7) == 0;  // (sums of pieces are written whole quads or one by one)
#pragma unroll
    for (int m = 0; m < TF; ++m) {
        if (r0 + m * 32 >= a.r)
            break;
        if (m)
            __syncthreads();
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float *p = out + (8 * (i / 4) + 4 * half + i % 4) * S::kOutPitch;
            if (GATED && WF == 2 && !pieces) {
                p[wave * 32 + l32] =
                    activate(acc[m][0][i] * unit[0] + bias[0], a.act) * (acc[m][WF - 1][i] * unit[WF - 1] + bias[WF - 1]);
            } else if (GATED && !pieces) {
                // the partner's sum is 16 lanes on
                const float v = acc[m][0][i] * unit[0] + bias[0], up = __shfl_down(v, 16, 32);
                if (l32 < 16)
                    p[wave * 16 + l32] = activate(v, a.act) * up;
            } else {
#pragma unroll
                for (int n = 0; n < WF; ++n) {
                    const float v = acc[m][n][i] * unit[n] + bias[n];
                    p[(wave * WF + n) * 32 + l32] = pieces ? v : activate(v, a.act);
                }
            }
        }
        __syncthreads();
        if (wide) {
            const int lanes = (pieces ? S::BN : OUT) / 8;  // of a row
#pragma unroll 1
            for (int r = threadIdx.x / lanes; r < 32; r += 256 / lanes) {
                const int64_t row = r0 + m * 32 + r;
                const int c = threadIdx.x % lanes * 8;
                // (pieces: staged rows 2 GR w + GR f + r of a gated layer)
                const int32_t col = j0 + (GATED && pieces ? c / (2 * HR) * HR + c % HR : c);
                if (row >= a.r || col >= a.m)
                    continue;
                float v[8];
                load8<F32>(out, r * S::kOutPitch + c, v);
                if (pieces) {
                    store8<F32>(g.part, (split * a.r + row) * rows + (GATED && (c / HR & 1) ? a.m : 0) + col, v);
                    continue;
                }
                if (col + 8 > a.m) {
                    for (int e = 0; col + e < a.m; ++e) {
                        if (a.residual)
                            v[e] += load1<N>(a.residual, row * a.residual_pitch + col + e);
                        store1<N>(a.y, row * a.y_pitch + col + e, v[e]);
                    }
                    continue;
                }
                if (a.residual) {
                    float res[8];
                    load8_any<N>(a.residual, row * a.residual_pitch + col, res);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        v[e] += res[e];
                }
                store8_any<N>(a.y, row * a.y_pitch + col, v);
            }
        } else {
            // sums of rows of any length: a lane a column
#pragma unroll 1
            for (int e = threadIdx.x; e < 32 * S::BN; e += 256) {
                const int c = e % S::BN, r = e / S::BN;
                const int64_t row = r0 + m * 32 + r;
                const int32_t col = j0 + (GATED ? c / (2 * HR) * HR + c % HR : c);
                if (row < a.r && col < a.m)
                    g.part[(split * a.r + row) * rows + (GATED && (c / HR & 1) ? a.m : 0) + col] =
                        out[r * S::kOutPitch + c];
            }
        }
    }
}

// Sums the pieces of k in their order and finishes; a thread four outputs.
template <class N>
__global__ void __launch_bounds__(256) matmul_join_kernel(MatmulArgs a, int32_t splits, const float *part)
{
    const int32_t quads = (a.m + 3) >> 2;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t row = i / quads;
    const int32_t col = (int32_t)(i - row * quads) * 4;
    if (row >= a.r)
        return;
    const int64_t rows = a.gated ? 2 * (int64_t)a.m : a.m, all = a.r * rows;
    const float *p = part + row * rows + col;
    f4 t = {0, 0, 0, 0}, up = {0, 0, 0, 0};
    if (a.m % 4 == 0) {
        // (four pieces' loads at a time; past the last piece it is read again)
        for (int s = 0; s < splits; s += 4) {
            f4 v[4], w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float *q = p + min(s + i, splits - 1) * all;
                v[i] = *(const f4 *)q;
                if (a.gated)
                    w[i] = *(const f4 *)(q + a.m);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (s + i < splits) {
                    t += v[i];
                    if (a.gated)
                        up += w[i];
                }
        }
    } else {
        for (int s = 0; s < splits; ++s)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (col + e < a.m) {
                    t[e] += p[s * all + e];
                    if (a.gated)
                        up[e] += p[s * all + a.m + e];
                }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (col + e < a.m)
            finish<N>(a, row, col + e, t[e], up[e]);
}

template <class N, int BITS, int TF, int WF, int GPB, bool GATED>
hipError_t launch_tile(const MatmulArgs &a, const TilePlan &p, void *ws, hipStream_t s)
{
    using S = TileShape<BITS, TF, WF, GPB>;
    constexpr int OUT = GATED ? S::BN / 2 : S::BN;
    TileGrid g;
    g.tm = (a.r + S::BM - 1) / S::BM;
    g.tn = (a.m + OUT - 1) / OUT;
    g.splits = p.splits;
    g.steps = p.columns / S::KS;
    g.part = (float *)ws;
    const void *kernel = (const void *)matmul_tile_kernel<N, BITS, TF, WF, GPB, GATED>;
    if constexpr (S::kLds > 64 * 1024) {
        static std::atomic<uint64_t> devices{0};
        qnn::allow_large_lds(kernel, devices);
    }
    hipLaunchKernelGGL((matmul_tile_kernel<N, BITS, TF, WF, GPB, GATED>), dim3((unsigned)(g.tm * g.tn * g.splits)), dim3(256),
                       S::kLds, s, a, g);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || g.splits == 1)
        return e;
    const int64_t threads = (int64_t)a.r * ((a.m + 3) / 4);
    hipLaunchKernelGGL(matmul_join_kernel<N>, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, s, a, g.splits, g.part);
    return hipGetLastError();
}

template <class N, int BITS, int TF, int WF>
hipError_t launch_tile_sized(const MatmulArgs &a, const TilePlan &p, void *ws, hipStream_t s)
{
    if constexpr (BITS != 16) {
        if (a.groups > 1 && a.group == 32)
            return a.gated ? launch_tile<N, BITS, TF, WF, 2, true>(a, p, ws, s) : launch_tile<N, BITS, TF, WF, 2, false>(a, p, ws, s);
        if (a.groups > 1)
            return a.gated ? launch_tile<N, BITS, TF, WF, 1, true>(a, p, ws, s) : launch_tile<N, BITS, TF, WF, 1, false>(a, p, ws, s);
    }
    return a.gated ? launch_tile<N, BITS, TF, WF, 0, true>(a, p, ws, s) : launch_tile<N, BITS, TF, WF, 0, false>(a, p, ws, s);
}

template <class N, int BITS>
hipError_t launch_tile_bits(const MatmulArgs &a, const TilePlan &p, void *ws, hipStream_t s)
{
    if constexpr (BITS != 16)
        if (p.tf == 1)
            return launch_tile_sized<N, BITS, 1, 1>(a, p, ws, s);
    if (p.tf == 2)
        return p.wf == 1 ? launch_tile_sized<N, BITS, 2, 1>(a, p, ws, s) : launch_tile_sized<N, BITS, 2, 2>(a, p, ws, s);
    return launch_tile_sized<N, BITS, 4, 2>(a, p, ws, s);
}

}  // namespace qnn_lm
