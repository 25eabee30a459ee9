// Attention of a tree of drafted tokens over a paged cache
// (qnn_lm_tree_attention): one pass over the cache with the running maximum
// and sum of the softmax.
//
// The rows of a cache head are its query heads times the drafts: row = draft *
// g + query head of the group.  A workgroup owns some rows of one head of one
// sequence and one piece of its positions.  With few rows its waves share out
// the positions (lm_attend_few.h), with many the rows (lm_attend_many.h).
// Pieces are joined by a second kernel.
//
// Both products are taken transposed on the 16x16x32 matrix instruction, so
// that a lane keeps one row's statistics and never passes a probability on:
//   S^T = K Q^T  (A = 16 positions of K; B = Q): lane l
//         gets row l % 16 at positions 4 * (l / 16) .. + 3;
//   O^T = V^T P^T (B = P): lane l's eight k's are the positions that it holds
//         of the tile's two halves, in the order that A uses as well;
//         A = V^T comes from local memory by the transposing reads.
// Codes enter the products as they are (exact); a key's scale multiplies its
// scores, a value's scale its probabilities.
//
// The reference m that probabilities 2^(score - m) are taken against is not the
// maximum but kAbove below it, and is raised only where a score is kSlack above
// what it was set for: most tiles neither exchange maxima between lanes nor
// rescale.  Probabilities stay below 2^(kAbove + kSlack) = 2^14, so that f16
// holds them, and keep all its bits down to 2^-24 of the largest; sums are fp32.
// Values of a packed cache are multiplied as f16 whatever the queries' type
// (codes are exact there, and probabilities keep 11 bits): their scales multiply
// the probabilities as multiples of a unit, a power of two.  Scales within
// 2^-12 .. 2 of the unit leave a row's largest products 2^-2 and more, far above
// f16's smallest numbers.  A tile that holds any other scale but zero (one ballot
// a tile to see) is put off: it is added behind the loop, multiplied as bf16,
// which has the range of fp32, each product of a probability and its scale as the
// sum of three numbers (lm_attend_far.h).  So a scale takes no digits from a
// position with another one, nor from a row that does not see it.
#pragma once

#include "lm_cache.h"

namespace qnn_lm {

typedef short s4_ __attribute__((ext_vector_type(4)));
typedef short s8_ __attribute__((ext_vector_type(8)));
typedef int i2_ __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) s4_ lds_s4;
typedef __attribute__((address_space(3))) i2_ lds_i2;

constexpr float kAbove = 10.f, kSlack = 4.f;
// Factor that a piece of the positions joins the others with, at least: finite
// outputs do not change by it, an infinite one stays so.
constexpr float kLeast = 0x1p-126f;

struct AttendPlan {
    int32_t g;          // query heads of a cache head
    int32_t rows;       // t * g
    int32_t many;       // the waves share out the rows
    int32_t nr;         // sixteens of rows of a wave
    int32_t row_tiles;  // of 16 nr rows, or of 64 nr
    int32_t splits;     // pieces of the positions
    float *part;        // [splits][b][t][heads][dim] outputs, then their maxima and sums
};

// Sequence's lengths, bounded.
struct AttendSeq {
    int32_t len, count;
    __device__ __forceinline__ AttendSeq(const AttendArgs &a, int32_t seq)
    {
        len = max(a.lens[seq], 0);
        count = a.counts ? min(max(a.counts[seq], 0), a.t) : a.t;
    }
    // Positions that rows row0 .. row0 + rows - 1 can see end here.
    __device__ __forceinline__ int32_t end(const AttendArgs &a, const CacheArgs &c, const AttendPlan &p, int32_t row0,
                                           int32_t rows) const
    {
        const int32_t last = min(count, (min(row0 + rows, p.rows) - 1) / p.g + 1);
        const int32_t seen = row0 / p.g >= count ? 0 : a.mask ? count : last;
        return seen ? (int32_t)min((int64_t)len + seen, (int64_t)c.width * c.page) : 0;
    }
};

// Which of the 64 positions from p0 on draft i sees, as bits (cached tokens:
// all; whether a position is in the cache at all is not asked).
__device__ __forceinline__ uint64_t seen_bits(const AttendArgs &a, int32_t seq, int32_t i, int64_t p0, int32_t len)
{
    const int64_t j0 = p0 - len;  // draft of the first bit
    if (j0 <= -64)
        return ~0ull;
    if (!a.mask) {
        const int64_t n = i - j0 + 1;
        return n >= 64 ? ~0ull : n <= 0 ? 0 : (1ull << n) - 1;
    }
    const int32_t words = (a.t + 63) >> 6, w = (int32_t)(j0 >> 6), s = (int32_t)j0 & 63;
    const uint64_t *row = a.mask + ((int64_t)seq * a.t + i) * words;
    const uint64_t lo = w < 0 ? ~0ull : w < words ? row[w] : 0, hi = w + 1 < words ? row[w + 1] : 0;
    return s ? lo >> s | hi << (64 - s) : lo;
}

// Whether a row (draft < 0: one of no draft) has seen nothing; m is then
// -infinity.  NaN scores raise no maximum: a row that has seen nothing else gets
// the maximum 0, so that its sum, NaN, is not taken for nothing.
__device__ __forceinline__ bool seen_nothing(int32_t draft, float &m, float l)
{
    const bool none = draft < 0 || (m == -INFINITY && l == 0.f);
    m = none ? -INFINITY : m == -INFINITY ? 0.f : m;
    return none;
}

// A row's result from its sum l, maximum m (in powers of two) and outputs
// v = 4 channels at d: into the pieces, or finished.
template <class N, int DIM>
__device__ __forceinline__ void store_row(const AttendArgs &a, const AttendPlan &p, int64_t all, int32_t split,
                                          int64_t index, int d, f4 v, float inv)
{
    if (p.splits > 1) {
        *(f4 *)(p.part + (split * all + index) * DIM + d) = v;
    } else {
        const u2 r = {pack2<N>(v[0] * inv, v[1] * inv), pack2<N>(v[2] * inv, v[3] * inv)};
        *(u2 *)((typename N::T *)a.out + index * DIM + d) = r;
    }
}

template <int DIM>
__device__ __forceinline__ void store_stats(const AttendArgs &a, const AttendPlan &p, int64_t all, int32_t split,
                                            int64_t index, float m, float l)
{
    if (p.splits > 1) {
        float *ml = p.part + p.splits * all * DIM + (split * all + index) * 2;
        ml[0] = m;
        ml[1] = l;
    } else if (a.lse) {
        a.lse[index] = m == -INFINITY ? -INFINITY : 0.693147180559945f * (m + log2f(l));
    }
}

// o += V^T P^T for values v of which some are infinite or NaN, in a tile that
// not every row sees whole: a position counts for the rows that see it (`see`:
// 1 or 0) alone.  The finite values go through the product as ever; of the
// others three products of ones count how many +infinity, -infinity and NaN a
// row sees in a channel.
template <class P>
__device__ __forceinline__ f4 add_odd_values(s8_ v, typename P::V8 p, typename P::V8 see, f4 o)
{
    constexpr short inf = __is_same(P, Bf16) ? 0x7F80 : 0x7C00, one = __is_same(P, Bf16) ? 0x3F80 : 0x3C00;
    s8_ fin, up, down, nan;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const short mag = v[e] & 0x7FFF;
        fin[e] = mag < inf ? v[e] : 0;
        up[e] = v[e] == inf ? one : 0;
        down[e] = mag == inf && v[e] < 0 ? one : 0;
        nan[e] = mag > inf ? one : 0;
    }
    const f4 zero = {0, 0, 0, 0};
    using V = typename P::V8;
    o = mfma16(__builtin_bit_cast(V, fin), p, o);
    const f4 a = mfma16(__builtin_bit_cast(V, up), see, zero), b = mfma16(__builtin_bit_cast(V, down), see, zero),
             c = mfma16(__builtin_bit_cast(V, nan), see, zero);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        o[i] += a[i] > 0.f ? INFINITY : 0.f;
        o[i] += b[i] > 0.f ? -INFINITY : 0.f;
        o[i] += c[i] > 0.f ? NAN : 0.f;
    }
    return o;
}

// Whether a row that has seen numbers only has an output that is NaN.
template <int NR, int ND>
__device__ __forceinline__ bool any_nan(const f4 (&o)[NR][ND], const float (&l)[NR])
{
    bool nan = false;
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                nan |= o[n][d][i] != o[n][d][i] && l[n] == l[n];
    return __any(nan);
}

// Outputs that are NaN though the values that their row has seen in the channel
// are infinite of one sign at most: an infinity times a probability below the
// smallest 16-bit number, or times a probability's negative second number.  They
// become that infinity.  Whoever calls this has found a NaN; it reads the
// values of the wave's tiles (first, first + stride .. of `tile` positions)
// again, which looking for infinities in every tile would cost all calls.
template <class N, int DIM, int NR>
__device__ __forceinline__ void settle_infinities(const AttendArgs &a, const CacheArgs &c, int32_t seq, int32_t head,
                                                  const int32_t (&draft)[NR], int32_t len, int32_t first, int32_t last,
                                                  int32_t stride, int32_t tile, int32_t end, f4 (&o)[NR][DIM / 16])
{
    constexpr int ND = DIM / 16;
    constexpr uint32_t inf = __is_same(N, Bf16) ? 0x7F80 : 0x7C00;
    const int kq = (threadIdx.x & 63) >> 4;
    uint64_t up[NR], down[NR], nan[NR];  // bit 4 d + i: of this lane's channel i of sixteen d
#pragma unroll
    for (int n = 0; n < NR; ++n)
        up[n] = down[n] = nan[n] = 0;
#pragma unroll 1
    for (int32_t t = first; t < last; t += stride)
#pragma unroll 1
        for (int32_t pos = t * tile; pos < min((t + 1) * tile, end); ++pos) {
            const Slot s = find_slot(c, seq, pos);
            if (s.page < 0)
                continue;
            const uint8_t *p = c.v + s.page * c.v_page + head * c.v_head + s.slot * c.v_slot + kq * 8;
            uint64_t u = 0, w = 0, x = 0;
#pragma unroll
            for (int d = 0; d < ND; ++d) {
                const u2 r = *(const u2 *)(p + d * 32);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t v = r[i / 2] >> (16 * (i % 2)) & 0xFFFFu;
                    const uint64_t bit = 1ull << (4 * d + i);
                    u |= v == inf ? bit : 0;
                    w |= v == (inf | 0x8000u) ? bit : 0;
                    x |= (v & 0x7FFFu) > inf ? bit : 0;
                }
            }
#pragma unroll
            for (int n = 0; n < NR; ++n)
                if (draft[n] >= 0 && (seen_bits(a, seq, draft[n], pos, len) & 1)) {
                    up[n] |= u;
                    down[n] |= w;
                    nan[n] |= x;
                }
        }
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint64_t bit = 1ull << (4 * d + i);
                if (o[n][d][i] != o[n][d][i] && ((up[n] ^ down[n]) & ~nan[n] & bit))
                    o[n][d][i] = up[n] & bit ? INFINITY : -INFINITY;
            }
}

// Largest exponent of the scales that lanes hold, of either sign, at least -120
// (zeros and what is not finite do not count).
__device__ __forceinline__ int scale_exponent(float v)
{
    v = fabsf(v);
    int e = v > 0.f && v < INFINITY ? max(ilogbf(v), -120) : -120;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1)
        e = max(e, __shfl_xor(e, s, 64));
    return __builtin_amdgcn_readfirstlane(e);
}

// The unit of a packed cache's value scales.  Its exponent stays within 20 of 0,
// so that products with any scale, and outputs brought from one unit to another,
// stay within fp32.
struct Unit {
    static constexpr int kMost = 20;
    int e = -kMost;
    float inv = (float)(1 << kMost);

    __device__ __forceinline__ bool out(float vs, uint64_t there) const
    {
        const float x = fabsf(vs) * inv;
        return (__ballot(!(x < 2.f) || (x < 0x1p-12f && x > 0.f)) & there) != 0;
    }
    // Whether the tile's scales (vs: this lane's; there: lanes that hold one)
    // are far from the unit, which rises first where they are above: the outputs
    // so far are to be multiplied by f (1 if it does not rise).
    __device__ __forceinline__ bool far(float vs, uint64_t there, float &f)
    {
        if (!out(vs, there))
            return false;
        asm volatile("");  // (a branch)
        const int lane = threadIdx.x & 63;
        const int top = min(scale_exponent((there >> lane) & 1 ? vs : 0.f), kMost);
        if (top > e) {
            f = ldexpf(1.f, e - top);
            e = top;
            inv = ldexpf(1.f, -top);
        }
        return out(vs, there);
    }
    template <int NR, int ND>
    __device__ __forceinline__ bool far(float vs, uint64_t there, f4 (&o)[NR][ND])
    {
        float f = 1.f;
        const bool is = far(vs, there, f);
        if (f != 1.f)
#pragma unroll
            for (int n = 0; n < NR; ++n)
#pragma unroll
                for (int d = 0; d < ND; ++d)
                    o[n][d] *= f;
        return is;
    }
};

hipError_t launch_attend_bf16(const AttendArgs &a, const CacheArgs &c, const AttendPlan &p, int bits, int dim,
                              hipStream_t s);
hipError_t launch_attend_f16(const AttendArgs &a, const CacheArgs &c, const AttendPlan &p, int bits, int dim,
                             hipStream_t s);

}  // namespace qnn_lm
