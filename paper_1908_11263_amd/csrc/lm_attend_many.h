// The attention kernel for many rows (large trees, chunks of a prompt): the
// waves of a workgroup share out the rows.
//
// Bound by the vector units (softmax, and expanding codes), so each code is
// expanded once a workgroup: 64 positions at a time go from memory through
// registers, where codes become 16-bit numbers, into local memory (two buffers,
// one barrier a tile), from where the four waves read them for 16 NR rows each.
// Loads run a tile ahead, page numbers two.
//
// The maximum that probabilities are taken against is raised only where a score
// is 2^8 above it: they stay below 2^8, their sum in fp32 loses nothing, and
// most tiles neither exchange maxima between lanes nor rescale.
//
// Values of a packed cache are multiplied as f16 whatever the queries' type
// (codes are exact, and probabilities keep 11 bits): value scales are taken
// relative to the largest so far, a power of two, so that they stay in range.
#pragma once

#include <type_traits>

#include "lm_attend.h"

namespace qnn_lm {

template <int BITS, int DIM>
struct ManyShape {
    static constexpr int KT = DIM == 256 ? 32 : 64;          // positions of a tile
    static constexpr int kChunks = DIM / 8;                  // 16-byte pieces of a staged row
    static constexpr int kRow = DIM * 2;                     // bytes of a staged row
    static constexpr int kBytes = DIM * BITS / 8;            // bytes of a slot
    static constexpr int kLanes = kBytes / 16;               // threads of a slot, 16 bytes each
    static constexpr int kLoads = KT * kLanes / 256;         // of a thread; 0: not every thread loads
    static constexpr int kMine = kLoads ? kLoads : 1;
    static constexpr int kPer = 128 / BITS;                  // numbers of a load
    static constexpr int kBuffer = 2 * KT * kRow + 2 * KT * 4;
    // workgroups a compute unit that the registers are shared out for: two,
    // but where the loads ahead (16-bit caches) or the outputs are too many
    static constexpr int groups(int nr) { return BITS == 16 && (nr == 2 || DIM == 256) ? 1 : 2; }
    // place of piece c of row r: eight rows that read one piece, and four that
    // read two neighbouring ones, find different banks
    static __device__ __forceinline__ int place(int r, int c) { return c ^ (((r & 3) << 1) | ((r >> 2) & 1)); }
};

// A load's numbers, from eight F on, to their row of local memory.
template <class N, class P, int BITS, int DIM, int F>
__device__ __forceinline__ void stage_pieces(uint8_t *kp, uint8_t *vp, const uint32_t *kr, const uint32_t *vr, int r,
                                             int load)
{
    using S = ManyShape<BITS, DIM>;
    if constexpr (F < S::kPer / 8) {
        const int at = S::place(r, load * (S::kPer / 8) + F) * 16;
        *(typename N::V8 *)(kp + at) = expand<N, BITS, F>(kr);
        *(typename P::V8 *)(vp + at) = expand<P, BITS, F>(vr);
        stage_pieces<N, P, BITS, DIM, F + 1>(kp, vp, kr, vr, r, load);
    }
}

template <class N, int BITS, int DIM, int NR>
__global__ void __launch_bounds__(256, (ManyShape<BITS, DIM>::groups(NR))) attend_many_kernel(AttendArgs a, CacheArgs c, AttendPlan pl)
{
    using S = ManyShape<BITS, DIM>;
    using P = std::conditional_t<BITS == 16, N, F16>;  // type of the second product
    constexpr int KT = S::KT, ND = DIM / 16, NK = DIM / 32, NU = KT / 16;
    extern __shared__ __align__(16) uint8_t lds[];
    const int lane = threadIdx.x & 63, l16 = lane & 15, kq = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // row tiles of one head's piece lie eight workgroups apart: on one XCD,
    // which reads the piece from memory once
    const int32_t unit = (int32_t)(blockIdx.x >> 3) / pl.row_tiles * 8 + (blockIdx.x & 7);
    const int32_t tile = (int32_t)(blockIdx.x >> 3) % pl.row_tiles;
    if (unit >= pl.splits * c.heads * c.b)
        return;
    const int32_t split = unit % pl.splits, head = unit / pl.splits % c.heads, seq = unit / pl.splits / c.heads;
    const AttendSeq sq(a, seq);
    const int32_t wg0 = tile * 64 * NR, row0 = wg0 + wave * 16 * NR;
    const int32_t end = sq.end(a, c, pl, wg0, 64 * NR);

    typename N::V8 q[NR][NK];
    int32_t draft[NR];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
        const int32_t row = row0 + n * 16 + l16;
        const int32_t dr = row / pl.g;
        const bool live = row < pl.rows && dr < sq.count;
        draft[n] = live ? dr : -1;
        const typename N::T *p =
            (const typename N::T *)a.q + seq * a.q_b + (live ? dr * a.q_t + (head * pl.g + row - dr * pl.g) * a.q_h : 0);
#pragma unroll
        for (int i = 0; i < NK; ++i) {
            u4 v = {0, 0, 0, 0};
            if (live)
                v = *(const u4 *)(p + i * 32 + kq * 8);
            q[n][i] = __builtin_bit_cast(typename N::V8, v);
        }
    }
    f4 o[NR][ND];
    float m[NR], l[NR];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
        m[n] = -INFINITY;
        l[n] = 0.f;
#pragma unroll
        for (int d = 0; d < ND; ++d)
            o[n][d] = (f4){0, 0, 0, 0};
    }
    const float qs = a.scale * 1.44269504088896f * (BITS == 4 ? 1.f / 16 : 1.f);
    int vexp = -1000;

    const int32_t tiles = (end + KT - 1) / KT;
    const int32_t share = (tiles + pl.splits - 1) / pl.splits;
    const int32_t first = split * share, last = min(first + share, tiles);

    // lane l looks position l of a tile up; page < 0: not there
    auto look = [&](int32_t t) {
        const int32_t pos = t * KT + lane;
        int32_t page = -1;
        if (t < last && lane < KT && pos < end) {
            const int32_t pg = pl.shift >= 0 ? pos >> pl.shift : (int32_t)((uint32_t)pos / (uint32_t)c.page);
            page = c.table[(int64_t)seq * c.width + pg];
            if ((uint32_t)page >= (uint32_t)c.pages)
                page = -1;
        }
        return page;
    };
    uint32_t kr[S::kMine][4], vr[S::kMine][4];
    float ks = 0.f, vs = 0.f;
    uint64_t valid = 0;
    auto load = [&](int32_t t, int32_t page) {
        const int32_t pos = t * KT + lane;
        const int32_t slot =
            pl.shift >= 0 ? pos & ((1 << pl.shift) - 1) : (int32_t)((uint32_t)pos % (uint32_t)c.page);
        valid = __ballot(page >= 0);
        if constexpr (BITS != 16) {
            ks = vs = 0.f;
            if (page >= 0) {
                const int64_t at = ((int64_t)page * c.heads + head) * c.page + slot;
                ks = c.k_scale[at];
                vs = c.v_scale[at];
            }
        }
#pragma unroll
        for (int i = 0; i < S::kMine; ++i) {
            const int e = i * 256 + threadIdx.x, r = e / S::kLanes, piece = e % S::kLanes;
            const int32_t pg = __shfl(page, r & 63, 64), sl = __shfl(slot, r & 63, 64);
#pragma unroll
            for (int w = 0; w < 4; ++w)
                kr[i][w] = vr[i][w] = 0;
            if (pg >= 0 && r < KT) {
                load_words<4>(c.k + pg * c.k_page + head * c.k_head + sl * c.k_slot + piece * 16, kr[i]);
                load_words<4>(c.v + pg * c.v_page + head * c.v_head + sl * c.v_slot + piece * 16, vr[i]);
            }
        }
    };
    // registers to local memory, codes as numbers
    auto stage = [&](uint8_t *buf) {
#pragma unroll
        for (int i = 0; i < S::kMine; ++i) {
            const int e = i * 256 + threadIdx.x, r = e / S::kLanes, piece = e % S::kLanes;
            if (S::kLoads == 0 && r >= KT)
                continue;
            uint8_t *kp = buf + r * S::kRow, *vp = kp + KT * S::kRow;
            stage_pieces<N, P, BITS, DIM, 0>(kp, vp, kr[i], vr[i], r, piece);
        }
        if constexpr (BITS != 16) {
            float *sc = (float *)(buf + 2 * KT * S::kRow);
            if (wave == 0 && lane < KT) {
                sc[lane] = ks * qs;
                sc[KT + lane] = ldexpf(vs * (BITS == 4 ? 1.f / 16 : 1.f), -vexp);
            }
        }
    };

    load(first, look(first));
    int32_t page = look(first + 1);
    for (int32_t t = first; t < last; ++t) {
        uint8_t *buf = lds + ((t - first) & 1) * S::kBuffer;
        const uint64_t there = valid;
        if constexpr (BITS != 16) {
            const int e = scale_exponent<64>(vs);
            if (e > vexp) {
                const float f = ldexpf(1.f, max(vexp - e, -300));
#pragma unroll
                for (int n = 0; n < NR; ++n)
#pragma unroll
                    for (int d = 0; d < ND; ++d)
                        o[n][d] *= f;
                vexp = e;
            }
        }
        stage(buf);
        load(t + 1, page);
        page = look(t + 2);
        // local memory is written; the loads ahead stay in flight
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");

        const uint8_t *vb = buf + KT * S::kRow;
        const float *sc = (const float *)(buf + 2 * KT * S::kRow);
        f4 s[NR][NU];
#pragma unroll
        for (int u = 0; u < NU; ++u) {
            const int r = 16 * u + l16;
#pragma unroll
            for (int n = 0; n < NR; ++n)
                s[n][u] = (f4){0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < NK; ++i) {
                const typename N::V8 kf = *(const typename N::V8 *)(buf + r * S::kRow + S::place(r, 4 * i + kq) * 16);
#pragma unroll
                for (int n = 0; n < NR; ++n)
                    s[n][u] = mfma16(kf, q[n][i], s[n][u]);
            }
            f4 ku = {qs, qs, qs, qs};
            if constexpr (BITS != 16)
                ku = *(const f4 *)(sc + 16 * u + 4 * kq);
#pragma unroll
            for (int n = 0; n < NR; ++n)
                s[n][u] *= ku;
        }
        const int32_t p0 = t * KT;
        const bool whole = there == (KT == 64 ? ~0ull : (1ull << KT) - 1) && p0 + KT <= sq.len;
        if (!whole) {
#pragma unroll
            for (int n = 0; n < NR; ++n) {
                uint64_t see = draft[n] < 0 ? 0 : seen_bits(a, seq, draft[n], p0, sq.len) & there;
                see >>= 4 * kq;
#pragma unroll
                for (int u = 0; u < NU; ++u)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        s[n][u][i] = (see >> (16 * u + i)) & 1 ? s[n][u][i] : -INFINITY;
            }
        }
        typename P::V8 p[NR][NU / 2];
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            float top = -INFINITY;
#pragma unroll
            for (int u = 0; u < NU; ++u)
#pragma unroll
                for (int i = 0; i < 4; i += 2)
                    top = fmaxf(fmaxf(s[n][u][i], s[n][u][i + 1]), top);
            if (__any(top > m[n] + 8.f)) {
                top = fmaxf(top, __shfl_xor(top, 16, 64));
                top = fmaxf(top, __shfl_xor(top, 32, 64));
                const float mn = fmaxf(m[n], top);
                // (rows that have seen nothing keep their zeros)
                const float f = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[n] - mn);
                m[n] = mn;
                l[n] *= f;
#pragma unroll
                for (int d = 0; d < ND; ++d)
                    o[n][d] *= f;
            }
            const float mm = m[n] == -INFINITY ? 0.f : m[n];
#pragma unroll
            for (int h = 0; h < NU / 2; ++h) {
                float e[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int u = 2 * h + i / 4;
                    e[i] = __builtin_amdgcn_exp2f(s[n][u][i % 4] - mm);
                    l[n] += e[i];
                }
                if constexpr (BITS != 16) {
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const f4 vu = *(const f4 *)(sc + KT + 32 * h + 16 * u + 4 * kq);
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            // (a select: what an unseen position's scale holds has no influence)
                            e[4 * u + i] = whole || s[n][2 * h + u][i] != -INFINITY ? e[4 * u + i] * vu[i] : 0.f;
                    }
                }
                const u4 r = {pack2<P>(e[0], e[1]), pack2<P>(e[2], e[3]), pack2<P>(e[4], e[5]), pack2<P>(e[6], e[7])};
                p[n][h] = __builtin_bit_cast(typename P::V8, r);
            }
        }
        bool odd = false;
        if constexpr (BITS == 16) {
            if (!whole) {
                constexpr uint32_t ex = __is_same(N, Bf16) ? 0x7F80u : 0x7C00u;
                for (int i = lane; i < KT * S::kChunks; i += 64) {
                    const u4 v = *(const u4 *)(vb + i * 16);
#pragma unroll
                    for (int w = 0; w < 4; ++w)
                        odd |= (v[w] & ex) == ex || ((v[w] >> 16) & ex) == ex;
                }
                odd = __any(odd);
            }
        }
        if (!odd) {
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int h = 0; h < NU / 2; ++h) {
                    const int r = 32 * h + 4 * kq + (l16 >> 2);
                    // (rows r and r + 16 have their pieces in the same places)
                    const uint8_t *vp = vb + r * S::kRow + S::place(r, 2 * d + ((l16 >> 1) & 1)) * 16 + (l16 & 1) * 8;
                    const s4_ x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4 *)vp);
                    const s4_ y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4 *)(vp + 16 * S::kRow));
                    const s8_ z = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
#pragma unroll
                    for (int n = 0; n < NR; ++n)
                        o[n][d] = mfma16(__builtin_bit_cast(typename P::V8, z), p[n][h], o[n][d]);
                }
        } else if constexpr (BITS == 16) {
            // an infinite or NaN value that some row does not see: one position
            // at a time, only where it is seen
#pragma unroll
            for (int n = 0; n < NR; ++n)
#pragma unroll
                for (int e = 0; e < 4 * NU; ++e)
                    for (int from = 0; from < 4; ++from) {
                        const float pe = __shfl((float)p[n][e / 8][e % 8], from * 16 + l16, 64);
                        const float se = __shfl(s[n][e / 4][e % 4], from * 16 + l16, 64);
                        if (se == -INFINITY)
                            continue;
                        const int r = 16 * (e / 4) + 4 * from + e % 4;
#pragma unroll
                        for (int d = 0; d < ND; ++d) {
                            const uint8_t *vp = vb + r * S::kRow + S::place(r, 2 * d + (kq >> 1)) * 16 + (kq & 1) * 8;
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                o[n][d][i] += pe * load1<N>(vp, i);
                        }
                    }
        }
    }
    const int64_t all = (int64_t)c.b * a.t * a.heads;
    const float f = BITS == 16 || vexp == -1000 ? 1.f : ldexpf(1.f, vexp);
#pragma unroll
    for (int n = 0; n < NR; ++n) {
        l[n] += __shfl_xor(l[n], 16, 64);
        l[n] += __shfl_xor(l[n], 32, 64);
        const int32_t row = row0 + n * 16 + l16;
        if (row >= pl.rows)
            continue;
        if (draft[n] < 0)
            m[n] = -INFINITY;  // no draft of this sequence: has seen nothing
        const bool none = m[n] == -INFINITY;
        const int32_t dr = row / pl.g;
        const int64_t index = ((int64_t)seq * a.t + dr) * a.heads + head * pl.g + row - dr * pl.g;
        const float inv = none ? 0.f : 1.f / l[n];
#pragma unroll
        for (int d = 0; d < ND; ++d) {
            const f4 v = none ? (f4){0, 0, 0, 0} : o[n][d] * f;
            store_row<N, DIM>(a, pl, all, split, index, d * 16 + 4 * kq, v, inv);
        }
        if (kq == 0)
            store_stats<DIM>(a, pl, all, split, index, m[n], none ? 0.f : l[n]);
    }
}

}  // namespace qnn_lm
