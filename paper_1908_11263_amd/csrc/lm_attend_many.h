// The attention kernel for many rows (large trees, chunks of a prompt): the
// waves of a workgroup share out the rows.
//
// Bound by the vector units (softmax, and expanding codes), so each code is
// expanded once a workgroup: 64 positions at a time go from memory through
// registers, where codes become 16-bit numbers, into local memory (two buffers,
// one barrier a tile), from where the four waves read them for 16 NR rows each.
// Loads run a tile ahead, or two where registers allow, page numbers one more.
// Probabilities are rounded to 11 bits (f16) against packed caches and to the
// queries' type against 16-bit ones: the second product takes no more, and with
// the many rows here its time counts.  The sums of the softmax take them as
// they were before that.
//   4 sequences of up to 32768 positions at 4 bits, 4 heads of 128 with 8 queries
//   each (f16), trees of 61: 211 us, 12 of them to join, 606 TFLOP/s; 8 of up to
//   8192 at 8 bits, 8 heads with 4 queries (bf16), trees of 16: 54 us and 7.  Of
//   the first the vector units are busy 43 % of the time, the matrix units 20 %,
//   local memory 38 %.  A prompt's chunk of 512 behind 8192, 8 heads with 4
//   queries, 8 bits: 151 us (470 TFLOP/s), 16 bits 226 us; 2048 from an empty
//   cache 124 and 230 us.  Measured on the first two when they took 206 and 56:
//   tiles of 32 positions 255 and 58 us, with one load ahead 265 and 65; one load
//   ahead 198 and 57 (no clear difference).
//   The error of the results, of their norm: 1.7e-3 over caches of 8 bits and up to
//   2.3e-3 over 16 bits (bf16, where one rounding of the result is 1.65e-3), 2.6 to
//   3.4e-4 (f16: 2.1e-4).
#pragma once

#include <type_traits>

#include "lm_attend_far.h"

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
    static constexpr uint64_t kWhole = KT == 64 ? ~0ull : (1ull << KT) - 1;
    static constexpr int kPer = 128 / BITS;                  // numbers of a load
    static constexpr int kBuffer = 2 * KT * kRow + 2 * KT * 4;
    // workgroups a compute unit that the registers are shared out for: two,
    // but where the loads ahead (16-bit caches) or the outputs are too many
    static constexpr int groups(int nr) { return BITS == 16 && (nr == 2 || DIM == 256) ? 1 : 2; }
    // Tiles that are loaded ahead, one set of registers each.
    static constexpr int kAhead = BITS == 16 ? 1 : 2;
    // Place of piece c of row r.  256 bytes of local memory answer at once: the
    // sixteen rows of which one piece is read (K), and the eight of which two
    // neighbouring ones are (V), have them at different places of 256 bytes.
    static __device__ __forceinline__ int place(int r, int c)
    {
        return c ^ (DIM == 64 ? ((r >> 1) & 3) << 1 | ((r >> 3) & 1) : (r & 7) << 1 | ((r >> 3) & 1));
    }
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
    const int32_t group = workgroup();
    const int32_t work = (group >> 3) / pl.row_tiles * 8 + (group & 7);
    const int32_t tile = (group >> 3) % pl.row_tiles;
    if (work >= pl.splits * c.heads * c.b)
        return;
    const int32_t split = work % pl.splits, head = work / pl.splits % c.heads, seq = work / pl.splits / c.heads;
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
    Unit unit;             // of the values' scales
    bool put_off = false;  // tiles with scales far from it

    const int32_t tiles = (end + KT - 1) / KT;
    const int32_t share = (tiles + pl.splits - 1) / pl.splits;
    const int32_t first = split * share, last = min(first + share, tiles);

    // Loads are never skipped: behind a branch that may skip one, a wait for an
    // older load has to be a wait for all.  What is not there is read from a
    // place that is (the last position's table entry, slot 0 of page 0), and
    // cleared when it is staged.
    //
    // Page of a position as the table says.  Nothing is done with the number
    // before load(): a comparison would wait for it here.
    auto find = [&](int32_t t, int32_t r) {
        const int32_t pos = max(min(t * KT + r, end - 1), 0);
        const int32_t pg = qnn::fdiv((uint32_t)pos, c.page_div);
        return c.table[(int64_t)seq * c.width + pg];
    };
    auto in_cache = [&](int32_t t, int32_t r, int32_t page) {
        return t < last && r < KT && t * KT + r < end && (uint32_t)page < (uint32_t)c.pages;
    };
    auto slot_of = [&](int32_t pos) {
        return pos - (int32_t)qnn::fdiv((uint32_t)pos, c.page_div) * c.page;
    };
    // A tile's pages: of position `lane`, and of the positions that this thread loads
    struct Pages {
        int32_t mine, of[S::kMine];
    };
    auto look = [&](int32_t t) {
        Pages p;
        p.mine = find(t, lane);
#pragma unroll
        for (int i = 0; i < S::kMine; ++i)
            p.of[i] = find(t, (i * 256 + threadIdx.x) / S::kLanes % KT);
        return p;
    };
    struct Ahead {
        uint32_t k[S::kMine][4], v[S::kMine][4];
        float ks, vs;    // scales of position `lane`
        uint64_t valid;  // positions that are in the cache
    };
    const uint8_t *kb = c.k + head * c.k_head, *vb0 = c.v + head * c.v_head;
    auto load = [&](Ahead &h, int32_t t, const Pages &p) {
        const bool there = in_cache(t, lane, p.mine);
        h.valid = __ballot(there);
        if constexpr (BITS != 16) {
            const int64_t at =
                there ? ((int64_t)p.mine * c.heads + head) * c.page + slot_of(t * KT + lane) : 0;
            h.ks = c.k_scale[at];
            h.vs = c.v_scale[at];
        }
#pragma unroll
        for (int i = 0; i < S::kMine; ++i) {
            const int e = i * 256 + threadIdx.x, r = e / S::kLanes % KT, piece = e % S::kLanes;
            const bool here = in_cache(t, r, p.of[i]);
            const int32_t pg = here ? p.of[i] : 0, sl = here ? slot_of(t * KT + r) : 0;
            load_words<4>(kb + pg * c.k_page + sl * c.k_slot + piece * 16, h.k[i]);
            load_words<4>(vb0 + pg * c.v_page + sl * c.v_slot + piece * 16, h.v[i]);
        }
    };
    // registers to local memory, codes as numbers
    auto stage = [&](Ahead &h, uint8_t *buf) {
        if (h.valid != S::kWhole) {
            // (keys that are not there are masked, values have to be zero)
#pragma unroll
            for (int i = 0; i < S::kMine; ++i)
                if (!((h.valid >> ((i * 256 + threadIdx.x) / S::kLanes % KT)) & 1))
                    h.v[i][0] = h.v[i][1] = h.v[i][2] = h.v[i][3] = 0;
        }
#pragma unroll
        for (int i = 0; i < S::kMine; ++i) {
            const int e = i * 256 + threadIdx.x, r = e / S::kLanes, piece = e % S::kLanes;
            if (S::kLoads == 0 && r >= KT)
                continue;
            uint8_t *kp = buf + r * S::kRow, *vp = kp + KT * S::kRow;
            stage_pieces<N, P, BITS, DIM, 0>(kp, vp, h.k[i], h.v[i], r, piece);
        }
        if constexpr (BITS != 16) {
            float *sc = (float *)(buf + 2 * KT * S::kRow);
            if (wave == 0 && lane < KT) {
                sc[lane] = h.ks * qs;
                sc[KT + lane] = h.vs * unit.inv;
            }
        }
    };

    Ahead ahead[S::kAhead];
    Pages early[S::kAhead];
#pragma unroll
    for (int i = 0; i < S::kAhead; ++i)
        early[i] = look(first + i);
    Pages page = look(first + S::kAhead);
#pragma unroll
    for (int i = 0; i < S::kAhead; ++i)
        load(ahead[i], first + i, early[i]);
    auto step = [&](Ahead &h, int32_t t) {
        uint8_t *buf = lds + ((t - first) & 1) * S::kBuffer;
        const uint64_t there = h.valid;
        // (a lane past a tile of 32 has no position: what it has read is another's)
        if (BITS != 16 && (KT < 64 || there != S::kWhole) && !((there >> lane) & 1))
            h.ks = h.vs = 0.f;
        bool far = false;
        if constexpr (BITS != 16)
            far = unit.far(h.vs, there, o);
        stage(h, buf);
        // (the page numbers first: loads come back in order, and these are wanted before the tile's)
        const Pages later = look(t + S::kAhead + 1);
        load(h, t + S::kAhead, page);
        page = later;
        // local memory is written; the loads ahead stay in flight
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (BITS != 16 && far) {
            put_off = true;  // (in all four waves)
            return;
        }

        const uint8_t *vb = buf + KT * S::kRow;
        const float *sc = (const float *)(buf + 2 * KT * S::kRow);
        f4 s[NR][NU];
        // (the products of a row's sixteens do not wait for each other)
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
            for (int n = 0; n < NR; ++n)
                s[n][u] = (f4){0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < NK; ++i)
#pragma unroll
            for (int u = 0; u < NU; ++u) {
                const int r = 16 * u + l16;
                const typename N::V8 kf = *(const typename N::V8 *)(buf + r * S::kRow + S::place(r, 4 * i + kq) * 16);
#pragma unroll
                for (int n = 0; n < NR; ++n)
                    s[n][u] = mfma16(kf, q[n][i], s[n][u]);
            }
#pragma unroll
        for (int u = 0; u < NU; ++u) {
            f4 ku = {qs, qs, qs, qs};
            if constexpr (BITS != 16)
                ku = *(const f4 *)(sc + 16 * u + 4 * kq);
#pragma unroll
            for (int n = 0; n < NR; ++n)
                s[n][u] *= ku;
        }
        const int32_t p0 = t * KT;
        const bool whole = there == S::kWhole && p0 + KT <= sq.len;
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
            if (__any(top > m[n] + kAbove + kSlack)) {
                top = fmaxf(top, __shfl_xor(top, 16, 64));
                top = fmaxf(top, __shfl_xor(top, 32, 64));
                const float mn = fmaxf(m[n], top - kAbove);
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
                            e[4 * u + i] *= vu[i];
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
        auto values = [&](int h, int d) {
            const int r = 32 * h + 4 * kq + (l16 >> 2);
            // (rows r and r + 16 have their pieces in the same places)
            const uint8_t *vp = vb + r * S::kRow + S::place(r, 2 * d + ((l16 >> 1) & 1)) * 16 + (l16 & 1) * 8;
            const s4_ x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4 *)vp);
            const s4_ y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4 *)(vp + 16 * S::kRow));
            return (s8_){x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
        };
        if (!odd) {
#pragma unroll
            for (int h = 0; h < NU / 2; ++h)
#pragma unroll
                for (int d = 0; d < ND; ++d) {
                    const s8_ z = values(h, d);
#pragma unroll
                    for (int n = 0; n < NR; ++n)
                        o[n][d] = mfma16(__builtin_bit_cast(typename P::V8, z), p[n][h], o[n][d]);
                }
        } else if constexpr (BITS == 16) {
#pragma unroll
            for (int h = 0; h < NU / 2; ++h)
#pragma unroll
                for (int n = 0; n < NR; ++n) {
                    typename P::V8 see;
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        see[i] = (typename P::T)(s[n][2 * h + i / 4][i % 4] != -INFINITY ? 1.f : 0.f);
#pragma unroll
                    for (int d = 0; d < ND; ++d)
                        o[n][d] = add_odd_values<P>(values(h, d), p[n][h], see, o[n][d]);
                }
        }
    };
    for (int32_t t = first; t < last; t += S::kAhead) {
        step(ahead[0], t);
        if constexpr (S::kAhead == 2)
            if (t + 1 < last)
                step(ahead[1], t + 1);
    }
    if constexpr (BITS != 16)
        if (put_off)
            add_far_tiles<N, BITS, DIM, NR>(a, c, seq, head, q, draft, sq.len, first, last, 1, KT, end, qs, unit, o, m, l,
                                            [&](int i) { return i * 32 + kq * 8; });
#pragma unroll
    for (int n = 0; n < NR; ++n) {
        l[n] += __shfl_xor(l[n], 16, 64);
        l[n] += __shfl_xor(l[n], 32, 64);
    }
    if constexpr (BITS == 16)
        if (any_nan<NR, ND>(o, l))
            settle_infinities<N, DIM, NR>(a, c, seq, head, draft, sq.len, first, last, 1, KT, end, o);
    const int64_t all = (int64_t)c.b * a.t * a.heads;
    const float f = BITS == 16 ? 1.f : ldexpf(1.f, BITS == 4 ? unit.e - 4 : unit.e);
#pragma unroll
    for (int n = 0; n < NR; ++n) {
        const int32_t row = row0 + n * 16 + l16;
        if (row >= pl.rows)
            continue;
        const bool none = seen_nothing(draft[n], m[n], l[n]);
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
