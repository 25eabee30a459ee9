// Tiles of a packed cache whose value scales are far from the unit of the
// others' (Unit, lm_attend.h): added behind the loops of both attention kernels,
// straight from memory.  Few caches have any; the code is short rather than fast,
// and takes no registers from the loops.
//   64 sequences of 8192, a token each, 8 bits: 203 us, 766 with scales from 1e-6
//   to 1e6 in every tile; 8 trees of 16 at 8 bits 56 and 246 us, at 4 bits 64 and
//   364.
#pragma once

#include "lm_attend.h"

namespace qnn_lm {

// Eight products of probabilities with their values' scales as sums of three
// bf16 numbers, for a far tile (scale: in the unit's multiples; score: the
// masked ones).  Nothing where the position is not seen, whatever it holds there;
// an infinite scale counts however small the probability.
struct FarProducts {
    bf8 part[3];

    __device__ __forceinline__ FarProducts(const float (&score)[8], const float (&scale)[8], const float (&p)[8])
    {
        float e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            e[i] = score[i] == -INFINITY ? 0.f : fabsf(scale[i]) == INFINITY ? scale[i] : p[i] * scale[i];
#pragma unroll
        for (int j = 0; j < 3; ++j) {
            const u4 r = {pack2<Bf16>(e[0], e[1]), pack2<Bf16>(e[2], e[3]), pack2<Bf16>(e[4], e[5]), pack2<Bf16>(e[6], e[7])};
            part[j] = __builtin_bit_cast(bf8, r);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                e[i] = fabsf((float)part[j][i]) == INFINITY ? 0.f : e[i] - (float)part[j][i];  // (an infinity has no rest)
        }
    }
    // o += V^T P^T
    __device__ __forceinline__ f4 add(bf8 v, f4 o) const
    {
        return mfma16(v, part[2], mfma16(v, part[1], mfma16(v, part[0], o)));
    }
};

// Adds the far tiles among first, first + stride .. (below last, of `tile`
// positions) to a wave's rows.  The unit's course over the tiles is gone through
// again, so that the same ones are found that the loop has put off; `unit` is its
// last state, which the outputs are multiples of.  q[n][i] holds eight channels
// from channel(i) on.
template <class N, int BITS, int DIM, int NR, class Channel>
__device__ __forceinline__ void add_far_tiles(const AttendArgs &a, const CacheArgs &c, int32_t seq, int32_t head,
                                              const typename N::V8 (&q)[NR][DIM / 32], const int32_t (&draft)[NR],
                                              int32_t len, int32_t first, int32_t last, int32_t stride, int32_t tile,
                                              int32_t end, float qs, const Unit &unit, f4 (&o)[NR][DIM / 16],
                                              float (&m)[NR], float (&l)[NR], Channel channel)
{
    constexpr int ND = DIM / 16, NK = DIM / 32;
    const int lane = threadIdx.x & 63, l16 = lane & 15, kq = lane >> 4;
    auto slot_of = [&](int32_t pos) { return find_slot(c, seq, pos < end ? pos : -1); };
    Unit now;
#pragma unroll 1
    for (int32_t t = first; t < last; t += stride) {
        const Slot mine = slot_of(lane < tile ? t * tile + lane : end);
        float f;
        if (!now.far(mine.page < 0 ? 0.f : c.v_scale[scale_at(c, mine, head)], __ballot(mine.page >= 0), f))
            continue;
#pragma unroll 1
        for (int32_t p0 = t * tile; p0 < min((t + 1) * tile, end); p0 += 32) {
            f4 s[NR][2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                // (keys that are not there: of slot 0 of page 0, and masked)
                Slot x = slot_of(p0 + 16 * u + l16);
                x.page = max(x.page, 0);
                const uint8_t *k = c.k + x.page * c.k_page + head * c.k_head + x.slot * c.k_slot;
#pragma unroll
                for (int n = 0; n < NR; ++n)
                    s[n][u] = (f4){0, 0, 0, 0};
#pragma unroll
                for (int i = 0; i < NK; ++i) {
                    uint32_t raw[2];
                    const uint8_t *p = k + channel(i) * BITS / 8;
                    if constexpr (BITS == 8)
                        load_words<2>(p, raw);
                    else
                        raw[0] = *(const uint32_t *)p;
                    const typename N::V8 kf = expand<N, BITS, 0>(raw);
#pragma unroll
                    for (int n = 0; n < NR; ++n)
                        s[n][u] = mfma16(kf, q[n][i], s[n][u]);
                }
            }
            // this lane's eight positions: 4 kq .. + 3 of each sixteen
            float ks[8], vs[8];
            const uint8_t *v[8];
            uint32_t there = 0;  // bit 16 u + i
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                Slot x = slot_of(p0 + 16 * (j / 4) + 4 * kq + j % 4);
                const bool is = x.page >= 0;
                there |= (uint32_t)is << (16 * (j / 4) + j % 4);
                x.page = max(x.page, 0);
                const int64_t at = scale_at(c, x, head);
                ks[j] = c.k_scale[at] * qs;
                vs[j] = c.v_scale[at] * unit.inv;
                v[j] = c.v + x.page * c.v_page + head * c.v_head + x.slot * c.v_slot;
            }
#pragma unroll
            for (int n = 0; n < NR; ++n) {
                const uint32_t see =
                    draft[n] < 0 ? 0 : (uint32_t)(seen_bits(a, seq, draft[n], p0, len) >> (4 * kq)) & there;
                float score[8], e[8], top = -INFINITY;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    score[j] = (see >> (16 * (j / 4) + j % 4)) & 1 ? s[n][j / 4][j % 4] * ks[j] : -INFINITY;
                    top = fmaxf(top, score[j]);
                }
                if (__any(top > m[n] + kAbove + kSlack)) {
                    top = fmaxf(top, __shfl_xor(top, 16, 64));
                    top = fmaxf(top, __shfl_xor(top, 32, 64));
                    const float mn = fmaxf(m[n], top - kAbove);
                    const float g = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[n] - mn);
                    m[n] = mn;
                    l[n] *= g;
#pragma unroll
                    for (int d = 0; d < ND; ++d)
                        o[n][d] *= g;
                }
                const float mm = m[n] == -INFINITY ? 0.f : m[n];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    e[j] = __builtin_amdgcn_exp2f(score[j] - mm);
                    l[n] += e[j];
                }
                const FarProducts products(score, vs, e);
#pragma unroll
                for (int d = 0; d < ND; ++d) {
                    bf8 code;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int ch = 16 * d + l16;
                        const uint32_t b = v[j][ch * BITS / 8];
                        // (a code of 4 bits 16 times, as in the loops)
                        code[j] = (__bf16)(float)(int8_t)(BITS == 8 ? b : ch & 1 ? b & 0xF0u : b << 4);
                    }
                    o[n][d] = products.add(code, o[n][d]);
                }
            }
        }
    }
}

}  // namespace qnn_lm
