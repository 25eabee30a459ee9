// The attention kernel for few rows (a token, a small tree): the waves of a
// workgroup share out the positions, 32 of them a tile, each wave with its own
// running maximum and sums, joined at the end through local memory.
//
// Bound by memory: K goes from memory to the products' registers, V through a
// wave's local memory (it has to be transposed); no wave waits for another, and
// two tiles are in flight a wave.  Probabilities enter the second product as
// the sum of two 16-bit numbers (the matrix instructions have time to spare
// here), so that rounding them costs nothing.
//   8 heads of 128, 32 queries, bf16, 64 sequences of 8192, one token each: 16
//   bits 361 us (5.95 TB/s), 8 bits 203 us (5.46 TB/s), 4 bits 171 us (3.3 TB/s:
//   expanding the codes).  One sequence of 32768 at 8 bits: 25 us; of 1000 at 16
//   bits: 11.1 us, two launches whose chains of loads (lengths, pages, keys) set
//   the time.
#pragma once

#include <type_traits>

#include "lm_attend_far.h"

namespace qnn_lm {

constexpr int kAttendTile = 32;  // positions of a tile

template <int BITS, int DIM>
struct KvShape {
    static constexpr int kPiece = (128 / BITS < DIM / 4) ? 128 / BITS : DIM / 4;  // codes of a lane's load of K
    static constexpr int kLoads = DIM / (4 * kPiece);
    static constexpr int kWords = kPiece * BITS / 32;
    static constexpr int kSub = kPiece / 8;          // eights of a load
    static constexpr int kRow = DIM * BITS / 8;      // bytes of a slot
    static constexpr int kStaged = BITS == 16 ? 2 * DIM : DIM;  // bytes of a staged row of V
    static constexpr int kVLane = BITS == 4 ? 8 : 16;  // bytes of a lane's load of V
    static constexpr int kVLanes = kRow / kVLane;      // lanes of a row
    static constexpr int kVLoads = kAttendTile * kVLanes / 64;
    static constexpr int kVWords = kVLane / 4;
    // rows are set off so that the transposing reads, 16 or 32 rows at a time,
    // spread over the banks
    static constexpr int kPitch = kStaged + (BITS == 16 ? 32 : 16);
    static constexpr int kWaveLds = kAttendTile * kPitch + 3 * kAttendTile * 4;
};

// One tile's K and V in flight.
template <int BITS, int DIM>
struct KvTile {
    using S = KvShape<BITS, DIM>;
    uint32_t k[2][S::kLoads][S::kWords];
    uint32_t v[S::kVLoads][S::kVWords];
    float ks, vs;     // of position lane % 32
    uint32_t valid;   // positions that are in the cache and before the end

    // Page of position lane % 32 as the table says; looked at in load(), a tile
    // later (loads come back in order: a comparison here would wait for all).
    static __device__ __forceinline__ int32_t look(const CacheArgs &c, int32_t seq, int32_t p0, int32_t end,
                                                   int lane)
    {
        const int32_t pos = max(min(p0 + (lane & 31), end - 1), 0);
        const int32_t pg = qnn::fdiv((uint32_t)pos, c.page_div);
        return c.table[(int64_t)seq * c.width + pg];
    }

    // Loads are never skipped (behind a branch that may skip one, a wait for an
    // older load has to be a wait for all): what is not there is read from slot
    // 0 of page 0, and masked or cleared later.
    __device__ __forceinline__ void load(const CacheArgs &c, int32_t page, int32_t head, int32_t p0,
                                         int32_t end, int lane)
    {
        const int32_t pos = p0 + (lane & 31);
        const bool there = pos < end && (uint32_t)page < (uint32_t)c.pages;
        valid = (uint32_t)__ballot(there);
        int32_t slot = pos - (int32_t)qnn::fdiv((uint32_t)pos, c.page_div) * c.page;
        page = there ? page : 0;
        slot = there ? slot : 0;
        if constexpr (BITS != 16) {
            const int64_t at = ((int64_t)page * c.heads + head) * c.page + slot;
            ks = c.k_scale[at];
            vs = c.v_scale[at];
        }
        // lane l % 32 has looked its position up; the others take it from there
        const int l16 = lane & 15, kq = lane >> 4;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int32_t pg = __shfl(page, 16 * u + l16, 64), sl = __shfl(slot, 16 * u + l16, 64);
            const uint8_t *p = c.k + pg * c.k_page + head * c.k_head + sl * c.k_slot;
#pragma unroll
            for (int i = 0; i < S::kLoads; ++i)
                load_words<S::kWords>(p + (i * 4 + kq) * (S::kWords * 4), k[u][i]);
        }
#pragma unroll
        for (int i = 0; i < S::kVLoads; ++i) {
            const int row = i * (64 / S::kVLanes) + lane / S::kVLanes;
            const int32_t pg = __shfl(page, row, 64), sl = __shfl(slot, row, 64);
            load_words<S::kVWords>(c.v + pg * c.v_page + head * c.v_head + sl * c.v_slot + (lane % S::kVLanes) * S::kVLane,
                                   v[i]);
        }
    }

    // Clears the values and scales of positions that are not there (keys are masked).
    __device__ __forceinline__ void clear(int lane)
    {
        if (valid == 0xFFFFFFFFu)
            return;
        if (BITS != 16 && !((valid >> (lane & 31)) & 1))
            ks = vs = 0.f;
#pragma unroll
        for (int i = 0; i < S::kVLoads; ++i)
            if (!((valid >> (i * (64 / S::kVLanes) + lane / S::kVLanes)) & 1))
#pragma unroll
                for (uint32_t &w : v[i])
                    w = 0;
    }

    // s[n][u] += the I-th and later products of half u's keys with the queries
    template <class N, int I, int NR>
    __device__ __forceinline__ void scores(int u, const typename N::V8 (&q)[NR][DIM / 32], f4 (&s)[NR][2]) const
    {
        if constexpr (I < DIM / 32) {
            const typename N::V8 kf = expand<N, BITS, I % S::kSub>(k[u][I / S::kSub]);
#pragma unroll
            for (int n = 0; n < NR; ++n)
                s[n][u] = mfma16(kf, q[n][I], s[n][u]);
            scores<N, I + 1, NR>(u, q, s);
        }
    }

    // V's rows into this wave's local memory, 4-bit codes as bytes (16 times the code).
    __device__ __forceinline__ void stage(uint8_t *lds, int lane) const
    {
#pragma unroll
        for (int i = 0; i < S::kVLoads; ++i) {
            const int row = i * (64 / S::kVLanes) + lane / S::kVLanes;
            uint8_t *p = lds + row * S::kPitch + (lane % S::kVLanes) * 16;
            u4 r;
            if constexpr (BITS == 4) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t lo = (v[i][h] << 4) & 0xF0F0F0F0u, hi = v[i][h] & 0xF0F0F0F0u;
                    r[2 * h] = __builtin_amdgcn_perm(hi, lo, 0x05010400u);
                    r[2 * h + 1] = __builtin_amdgcn_perm(hi, lo, 0x07030602u);
                }
            } else {
                r = (u4){v[i][0], v[i][1], v[i][2], v[i][3]};
            }
            *(u4 *)p = r;
        }
    }

    // Whether a 16-bit value of the tile is infinite or NaN.
    template <class N>
    __device__ __forceinline__ bool odd_values() const
    {
        constexpr uint32_t e = __is_same(N, Bf16) ? 0x7F80u : 0x7C00u;
        bool odd = false;
#pragma unroll
        for (int i = 0; i < S::kVLoads; ++i)
#pragma unroll
            for (uint32_t w : v[i])
                odd |= (w & e) == e || ((w >> 16) & e) == e;
        return __any(odd);
    }
};

// The eight values of V^T at channel 16 * block + l % 16: positions 4 * (l /
// 16) .. + 3 of the tile's first half, then of its second.
template <class N, int BITS, int DIM>
__device__ __forceinline__ typename N::V8 value_frag(const uint8_t *lds, int block, int lane)
{
    using S = KvShape<BITS, DIM>;
    const int l16 = lane & 15, kq = lane >> 4;
    if constexpr (BITS == 16) {
        const uint8_t *p = lds + (4 * kq + (l16 >> 2)) * S::kPitch + block * 32 + (l16 & 3) * 8;
        const s4_ a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4 *)p);
        const s4_ b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4 *)(p + 16 * S::kPitch));
        const s8_ r = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
        return __builtin_bit_cast(typename N::V8, r);
    } else {
        const int row = 4 * kq + ((l16 >> 1) & 3) + 16 * (l16 >> 3);
        const uint8_t *p = lds + row * S::kPitch + block * 16 + (l16 & 1) * 8;
        const i2_ a = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i2 *)p);
        return expand_bytes<N>((uint32_t)a.x, (uint32_t)a.y);
    }
}

template <class N, int BITS, int DIM, int NR>
__global__ void __launch_bounds__(256) attend_kernel(AttendArgs a, CacheArgs c, AttendPlan pl)
{
    using S = KvShape<BITS, DIM>;
    using P = std::conditional_t<BITS == 16, N, F16>;  // type of the second product
    constexpr int ND = DIM / 16, NK = DIM / 32;
    extern __shared__ __align__(16) uint8_t lds[];
    const int lane = threadIdx.x & 63, l16 = lane & 15, kq = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int32_t split = blockIdx.x % pl.splits, tile = blockIdx.x / pl.splits;
    const int32_t head = blockIdx.y, seq = blockIdx.z;
    const AttendSeq sq(a, seq);
    const int32_t row0 = tile * 16 * NR;
    const int32_t end = sq.end(a, c, pl, row0, 16 * NR);

    // the channels that K's lane loads put into product i
    auto channel = [&](int i) { return (i / S::kSub) * 4 * S::kPiece + kq * S::kPiece + (i % S::kSub) * 8; };
    // this lane's rows: queries and draft numbers
    typename N::V8 q[NR][NK];
    int32_t draft[NR];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
        const int32_t row = row0 + n * 16 + l16;
        draft[n] = row < pl.rows ? row / pl.g : -1;
        const bool live = draft[n] >= 0 && draft[n] < sq.count;
        const typename N::T *p = (const typename N::T *)a.q + seq * a.q_b + max(draft[n], 0) * a.q_t +
                                 (head * pl.g + (live ? row - draft[n] * pl.g : 0)) * a.q_h;
        if (!live)
            draft[n] = -1;
#pragma unroll
        for (int i = 0; i < NK; ++i) {
            const int d = channel(i);
            u4 v = {0, 0, 0, 0};
            if (live)
                v = *(const u4 *)(p + d);
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
    const float qs = a.scale * 1.44269504088896f * (BITS == 4 ? 1.f / 16 : 1.f);  // scores in powers of two
    Unit unit;              // of the values' scales
    bool put_off = false;   // tiles with scales far from it
    uint8_t *vl = lds + wave * S::kWaveLds;
    float *scales = (float *)(vl + kAttendTile * S::kPitch);

    const int32_t tiles = (end + kAttendTile - 1) / kAttendTile;
    const int32_t share = (tiles + pl.splits - 1) / pl.splits;
    const int32_t first = split * share + wave, last = min((split + 1) * share, tiles);
    using Tile = KvTile<BITS, DIM>;
    auto look = [&](int32_t t) { return Tile::look(c, seq, t * kAttendTile, end, lane); };
    // (tiles past the last are loaded too, from slot 0 of page 0, and not used)
    auto load = [&](Tile &h, int32_t t, int32_t page) {
        h.load(c, page, head, t * kAttendTile, t < last ? end : 0, lane);
    };
    Tile ahead[2];
    const int32_t early[2] = {look(first), look(first + 4)};
    int32_t page = look(first + 8);
    load(ahead[0], first, early[0]);
    load(ahead[1], first + 4, early[1]);
    auto step = [&](Tile &cur, int32_t at) {
        const int32_t p0 = at * kAttendTile;
        cur.clear(lane);
        cur.stage(vl, lane);
        const uint32_t there = cur.valid;
        bool far = false;
        if constexpr (BITS != 16) {
            far = unit.far(cur.vs, there | (uint64_t)there << 32, o);
            if (lane < 32) {
                scales[lane] = cur.ks * qs;
                scales[32 + lane] = cur.vs * unit.inv;
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        f4 ks[2], vs[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            if constexpr (BITS != 16) {
                ks[u] = *(const f4 *)(scales + 16 * u + 4 * kq);
                vs[u] = *(const f4 *)(scales + 32 + 16 * u + 4 * kq);
            } else {
                ks[u] = (f4){qs, qs, qs, qs};
                vs[u] = (f4){1, 1, 1, 1};
            }
        }
        f4 s[NR][2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
            for (int n = 0; n < NR; ++n)
                s[n][u] = (f4){0, 0, 0, 0};
            cur.template scores<N, 0>(u, q, s);
#pragma unroll
            for (int n = 0; n < NR; ++n)
                s[n][u] *= ks[u];
        }
        const bool whole = there == 0xFFFFFFFFu && p0 + kAttendTile <= sq.len;
        bool odd = false;
        if constexpr (BITS == 16)
            odd = !whole && cur.template odd_values<N>();
        // the tile's registers are free: two tiles on, into the same ones
        const int32_t later = look(at + 12);
        load(cur, at + 8, page);
        page = later;
        if (BITS != 16 && far) {
            put_off = true;
            return;
        }
        if (!whole) {
#pragma unroll
            for (int n = 0; n < NR; ++n) {
                uint32_t see = draft[n] < 0 ? 0 : (uint32_t)seen_bits(a, seq, draft[n], p0, sq.len) & there;
                see >>= 4 * kq;
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        s[n][u][i] = (see >> (16 * u + i)) & 1 ? s[n][u][i] : -INFINITY;
            }
        }
        // (two 16-bit numbers a probability, as few rows leave room for: their
        // rounding does not show in the result)
        typename P::V8 p[NR], rest[NR];
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            float top = fmaxf(fmaxf(fmaxf(s[n][0][0], s[n][0][1]), fmaxf(s[n][0][2], s[n][0][3])),
                              fmaxf(fmaxf(s[n][1][0], s[n][1][1]), fmaxf(s[n][1][2], s[n][1][3])));
            if (__any(top > m[n] + kAbove + kSlack)) {
                top = fmaxf(top, __shfl_xor(top, 16, 64));
                top = fmaxf(top, __shfl_xor(top, 32, 64));
                const float mn = fmaxf(m[n], top - kAbove);
                // (rows that have seen nothing: 2^(-inf) = 0, of zeros)
                const float f = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[n] - mn);
                m[n] = mn;
                l[n] *= f;
#pragma unroll
                for (int d = 0; d < ND; ++d)
                    o[n][d] *= f;
            }
            const float mm = m[n] == -INFINITY ? 0.f : m[n];
            float e[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                e[i] = __builtin_amdgcn_exp2f(s[n][i / 4][i % 4] - mm);
                l[n] += e[i];
                if constexpr (BITS != 16)
                    e[i] *= vs[i / 4][i % 4];
            }
            const u4 r = {pack2<P>(e[0], e[1]), pack2<P>(e[2], e[3]), pack2<P>(e[4], e[5]), pack2<P>(e[6], e[7])};
            p[n] = __builtin_bit_cast(typename P::V8, r);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                e[i] -= (float)p[n][i];
            const u4 r2 = {pack2<P>(e[0], e[1]), pack2<P>(e[2], e[3]), pack2<P>(e[4], e[5]), pack2<P>(e[6], e[7])};
            rest[n] = __builtin_bit_cast(typename P::V8, r2);
        }
        if (!odd) {
#pragma unroll
            for (int d = 0; d < ND; ++d) {
                const typename P::V8 vf = value_frag<P, BITS, DIM>(vl, d, lane);
#pragma unroll
                for (int n = 0; n < NR; ++n)
                    o[n][d] = mfma16(vf, rest[n], mfma16(vf, p[n], o[n][d]));
            }
        } else if constexpr (BITS == 16) {
#pragma unroll
            for (int n = 0; n < NR; ++n) {
                typename N::V8 see;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    see[i] = (typename N::T)(s[n][i / 4][i % 4] != -INFINITY ? 1.f : 0.f);
#pragma unroll
                for (int d = 0; d < ND; ++d)
                    o[n][d] = add_odd_values<N>(__builtin_bit_cast(s8_, value_frag<N, BITS, DIM>(vl, d, lane)), p[n], see,
                                                o[n][d]);
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };
    for (int32_t at = first; at < last; at += 8) {
        step(ahead[0], at);
        if (at + 4 < last)
            step(ahead[1], at + 4);
    }
    if constexpr (BITS != 16)
        if (put_off)
            add_far_tiles<N, BITS, DIM, NR>(a, c, seq, head, q, draft, sq.len, first, last, 4, kAttendTile, end, qs, unit, o,
                                            m, l, channel);
#pragma unroll
    for (int n = 0; n < NR; ++n) {
        l[n] += __shfl_xor(l[n], 16, 64);
        l[n] += __shfl_xor(l[n], 32, 64);
    }
    if constexpr (BITS == 16)
        if (any_nan<NR, ND>(o, l))
            settle_infinities<N, DIM, NR>(a, c, seq, head, draft, sq.len, first, last, 4, kAttendTile, end, o);
    // join the four waves, sixteen rows at a time
    constexpr int OP = DIM + 4;  // pitch in floats
    float *jo = (float *)lds, *jm = jo + 4 * 16 * OP, *jl = jm + 64;
#pragma unroll
    for (int n = 0; n < NR; ++n) {
        const bool none = seen_nothing(draft[n], m[n], l[n]);
        __syncthreads();
        if (kq == 0) {
            jm[wave * 16 + l16] = m[n];
            jl[wave * 16 + l16] = l[n];
        }
        __syncthreads();
        float top = jm[l16];
#pragma unroll
        for (int w = 1; w < 4; ++w)
            top = fmaxf(top, jm[w * 16 + l16]);
        float f = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[n] - top);
        if constexpr (BITS != 16)
            f = ldexpf(f, BITS == 4 ? unit.e - 4 : unit.e);
#pragma unroll
        for (int d = 0; d < ND; ++d) {
            // (a row that has seen nothing may hold anything; an infinity stays
            // one when the factor is zero)
            f4 v = o[n][d] * f;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                v[i] = none ? 0.f : fabsf(o[n][d][i]) == INFINITY ? o[n][d][i] : v[i];
            *(f4 *)(jo + (wave * 16 + l16) * OP + d * 16 + 4 * kq) = v;
        }
        __syncthreads();
        // 16 threads a row
        const int r = threadIdx.x >> 4, e0 = threadIdx.x & 15;
        const int32_t row = row0 + n * 16 + r;
        if (row < pl.rows) {
            float mt = jm[r];
#pragma unroll
            for (int w = 1; w < 4; ++w)
                mt = fmaxf(mt, jm[w * 16 + r]);
            float lt = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w)
                lt += jm[w * 16 + r] == -INFINITY ? 0.f : jl[w * 16 + r] * __builtin_amdgcn_exp2f(jm[w * 16 + r] - mt);
            const int32_t dr = row / pl.g, hq = head * pl.g + row - dr * pl.g;
            const int64_t index = ((int64_t)seq * a.t + dr) * a.heads + hq;
            const int64_t all = (int64_t)c.b * a.t * a.heads;
            const float inv = pl.splits > 1 ? 1.f : (mt == -INFINITY ? 0.f : 1.f / lt);
            for (int e = e0 * 8; e < DIM; e += 128) {
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    float t = 0.f;
#pragma unroll
                    for (int w = 0; w < 4; ++w)
                        t += jo[(w * 16 + r) * OP + e + i];
                    v[i] = mt == -INFINITY ? 0.f : t * inv;
                }
                if (pl.splits > 1)
                    store8<F32>(pl.part, (split * all + index) * DIM + e, v);
                else
                    store8<N>(a.out, index * DIM + e, v);
            }
            if (e0 == 0) {
                if (pl.splits > 1) {
                    float *ml = pl.part + pl.splits * all * DIM + (split * all + index) * 2;
                    ml[0] = mt;
                    ml[1] = lt;
                } else if (a.lse) {
                    a.lse[index] = mt == -INFINITY ? -INFINITY : 0.693147180559945f * (mt + log2f(lt));
                }
            }
        }
    }
}

}  // namespace qnn_lm
