// Writes to and reads from the paged cache: cache_append, cache_keep,
// cache_read.  All are bound by memory (and, for a few tokens, by the launch):
// DIM / 8 lanes own a token of a head, eight channels each, so that every
// access is 16 bytes of numbers or the 4 to 16 bytes of their codes.
// A thread does a token's key and its value, as working their place out takes
// as many instructions as a row's codes do (one of the two a thread: 30 us where
// it takes 20 now).
//   Append of 4 x 4001 tokens of 8 heads of 128 at 4 bits: 20 us (4.2 TB/s);
//   reading them back 17.5 us (4.7 TB/s).  8 x 16 tokens at 8 bits: 4.2 us, and 3
//   for the read; keep of 64 sequences' trees of 33: 3.9 us.
#include "lm_cache.h"

namespace qnn_lm {

struct TokenArgs {
    const void *k, *v;
    int64_t ks[3], vs[3];  // elements: sequence, token, head
    int32_t t;
    uint32_t tokens;       // b * t * heads
    qnn::FastDiv heads_div, t_div;
    const int32_t *lens, *counts;
};

// Index of this thread's token: (sequence, token, head), the head fastest.  A
// thread does its key and its value: they have the place in common.
struct Token {
    int32_t seq, i, head;
};
__device__ __forceinline__ Token token_of(uint32_t n, const qnn::FastDiv &heads, const qnn::FastDiv &t)
{
    Token o;
    const uint32_t a = qnn::fdiv(n, heads);
    o.head = n - a * heads.d;
    o.seq = qnn::fdiv(a, t);
    o.i = a - o.seq * t.d;
    return o;
}

// Codes of a token's eight numbers w (its LANES lanes hold them all), and its
// scale: the largest magnitude over the largest code.
template <class N, int BITS, int LANES>
__device__ __forceinline__ u2 codes_of(u4 w, float &scale)
{
    typedef unsigned short us2 __attribute__((ext_vector_type(2)));
    constexpr bool BF = __is_same(N, Bf16);
    constexpr float most = BITS == 8 ? 127.f : 7.f;
    // the largest magnitude, by bits: infinity and NaN are above every finite number
    us2 m = __builtin_bit_cast(us2, w[0] & 0x7FFF7FFFu);
#pragma unroll
    for (int i = 1; i < 4; ++i)
        m = __builtin_elementwise_max(m, __builtin_bit_cast(us2, w[i] & 0x7FFF7FFFu));
    uint32_t top = max(m[0], m[1]);
#pragma unroll
    for (int i = 1; i < LANES; i <<= 1)
        top = max(top, (uint32_t)__shfl_xor((int)top, i, 64));
    auto number = [](uint32_t bits) {
        return BF ? __uint_as_float(bits << 16) : (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
    };
    float v[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = number(w[i] & 0xFFFFu);
        v[2 * i + 1] = BF ? __uint_as_float(w[i] & 0xFFFF0000u) : number(w[i] >> 16);
    }
    const bool finite = top < (BF ? 0x7F80u : 0x7C00u);
    scale = finite ? number(top) / most : __uint_as_float(0x7FC00000u);
    // v / scale, correctly rounded: with the correctly rounded reciprocal y, q =
    // v y is within a unit, and q + (v - q scale) y rounds as the quotient does
    // (Markstein).  It is above the largest code by its own rounding at most;
    // adding 1.5 2^23 rounds it to a whole number, whose low bits are the code.
    uint32_t code[8];
    if (__any(!finite || (scale > 0.f && scale < 0x1p-100f))) {
        // scales whose reciprocal is not a normal number divide
#pragma unroll
        for (int e = 0; e < 8; ++e)
            code[e] = (uint32_t)(int32_t)fminf(fmaxf(rintf(finite && scale > 0.f ? v[e] / scale : 0.f), -most), most);
    } else {
        const float y = scale > 0.f ? 1.f / scale : 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float q = v[e] * y;
            code[e] = __float_as_uint(__builtin_fmaf(__builtin_fmaf(-q, scale, v[e]), y, q) + 0x1.8p23f);
        }
    }
    u2 r = {0, 0};
    if constexpr (BITS == 8) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            r[i] = __builtin_amdgcn_perm(code[4 * i + 1], code[4 * i], 0x0C0C0400u) |
                   __builtin_amdgcn_perm(code[4 * i + 3], code[4 * i + 2], 0x04000C0Cu);
    } else {
        uint32_t pair[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            pair[i] = (code[2 * i] & 15u) | code[2 * i + 1] << 4;
        r[0] = __builtin_amdgcn_perm(pair[1], pair[0], 0x0C0C0400u) | __builtin_amdgcn_perm(pair[3], pair[2], 0x04000C0Cu);
    }
    return r;
}

template <class N, int BITS, int DIM>
__global__ void __launch_bounds__(256) append_kernel(CacheArgs c, TokenArgs a)
{
    constexpr int LANES = DIM / 8;
    const uint32_t n = workgroup() * (256 / LANES) + threadIdx.x / LANES;
    const int lane = threadIdx.x % LANES;
    if (n >= a.tokens)
        return;
    const Token o = token_of(n, a.heads_div, a.t_div);
    if (a.counts && o.i >= a.counts[o.seq])
        return;
    const Slot s = find_slot(c, o.seq, (int64_t)a.lens[o.seq] + o.i);
    if (s.page < 0)
        return;
    const u4 kw = *(const u4 *)((const typename N::T *)a.k + o.seq * a.ks[0] + o.i * a.ks[1] + o.head * a.ks[2] + lane * 8);
    const u4 vw = *(const u4 *)((const typename N::T *)a.v + o.seq * a.vs[0] + o.i * a.vs[1] + o.head * a.vs[2] + lane * 8);
    uint8_t *kd = c.k + s.page * c.k_page + o.head * c.k_head + s.slot * c.k_slot + lane * BITS;
    uint8_t *vd = c.v + s.page * c.v_page + o.head * c.v_head + s.slot * c.v_slot + lane * BITS;
    if constexpr (BITS == 16) {
        *(u4 *)kd = kw;
        *(u4 *)vd = vw;
    } else {
        float ks, vs;
        const u2 kc = codes_of<N, BITS, LANES>(kw, ks), vc = codes_of<N, BITS, LANES>(vw, vs);
        if constexpr (BITS == 8) {
            *(u2 *)kd = kc;
            *(u2 *)vd = vc;
        } else {
            *(uint32_t *)kd = kc[0];
            *(uint32_t *)vd = vc[0];
        }
        if (lane == 0) {
            const int64_t at = scale_at(c, s, o.head);
            c.k_scale[at] = ks;
            c.v_scale[at] = vs;
        }
    }
}

struct ReadArgs {
    void *k, *v;
    int32_t t;
    uint32_t tokens;          // b * t * heads
    qnn::FastDiv heads_div, t_div;
    const int32_t *start;
};

// C: the number type of a 16-bit cache; N: of the result.
template <class N, class C, int BITS, int DIM>
__global__ void __launch_bounds__(256) read_kernel(CacheArgs c, ReadArgs a)
{
    constexpr int LANES = DIM / 8;
    const uint32_t n = workgroup() * (256 / LANES) + threadIdx.x / LANES;
    const int lane = threadIdx.x % LANES;
    if (n >= a.tokens)
        return;
    const Token o = token_of(n, a.heads_div, a.t_div);
    const int64_t at = (((int64_t)o.seq * a.t + o.i) * c.heads + o.head) * DIM + lane * 8;
    const Slot s = find_slot(c, o.seq, (int64_t)a.start[o.seq] + o.i);
    auto one = [&](void *dst, const uint8_t *src, const float *scales) {
        float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        if (s.page >= 0) {
            if constexpr (BITS == 16) {
                load8<C>(src, 0, v);
            } else {
                const float scale = scales[scale_at(c, s, o.head)];
                if constexpr (BITS == 8) {
                    const u2 r = *(const u2 *)src;
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        v[e] = (float)(int8_t)(r[e / 4] >> 8 * (e % 4)) * scale;
                } else {
                    const uint32_t r = *(const uint32_t *)src;
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        v[e] = (float)((int32_t)(r << (28 - 4 * e)) >> 28) * scale;
                }
            }
        }
        store8<N>(dst, at, v);
    };
    if (a.k)
        one(a.k, c.k + s.page * c.k_page + o.head * c.k_head + s.slot * c.k_slot + lane * BITS, c.k_scale);
    if (a.v)
        one(a.v, c.v + s.page * c.v_page + o.head * c.v_head + s.slot * c.v_slot + lane * BITS, c.v_scale);
}

// A workgroup owns the keys or the values of one head of one sequence, and
// moves as many tokens at a time as it has lanes for: all of them are read
// before the first is written.  Entries ascend, so a later read never finds
// what an earlier batch wrote.
template <int ROW>  // bytes of a token
__global__ void __launch_bounds__(256) keep_kernel(CacheArgs c, int32_t t, const int32_t *lens, const int32_t *path,
                                                   const int32_t *kept)
{
    constexpr int LANES = ROW / 16, BATCH = 256 / LANES;
    const int32_t seq = blockIdx.y, head = blockIdx.x >> 1, which = blockIdx.x & 1;
    const int lane = threadIdx.x % LANES;
    const int32_t count = min(kept[seq], t);
    const int64_t len = lens[seq];
    uint8_t *base = which ? c.v + head * c.v_head : c.k + head * c.k_head;
    const int64_t sp = which ? c.v_page : c.k_page, ss = which ? c.v_slot : c.k_slot;
    float *scale = which ? c.v_scale : c.k_scale;
    for (int32_t j0 = 0; j0 < count; j0 += BATCH) {
        const int32_t j = j0 + threadIdx.x / LANES;
        Slot to = {-1, 0}, from = {-1, 0};
        if (j < count) {
            const int32_t p = path[(int64_t)seq * t + j];
            if (p > j && p < t) {
                from = find_slot(c, seq, len + p);
                to = find_slot(c, seq, len + j);
            }
        }
        const bool move = from.page >= 0 && to.page >= 0;
        u4 r = {0, 0, 0, 0};
        float sc = 0;
        if (move) {
            r = *(const u4 *)(base + from.page * sp + from.slot * ss + lane * 16);
            if (scale && lane == 0)
                sc = scale[scale_at(c, from, head)];
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // every read of the batch is back
        __syncthreads();
        if (move) {
            *(u4 *)(base + to.page * sp + to.slot * ss + lane * 16) = r;
            if (scale && lane == 0)
                scale[scale_at(c, to, head)] = sc;
        }
    }
}

#define QNN_LM_DIMS(CALL) \
    switch (dim) {        \
    case 64: CALL(64)     \
    case 128: CALL(128)   \
    case 256: CALL(256)   \
    default: return hipErrorInvalidValue; \
    }                     \
    return hipGetLastError();

template <class N, int BITS>
static hipError_t append_bits(const CacheArgs &c, int dim, const TokenArgs &a, hipStream_t s)
{
#define CALL(D)                                                                                              \
    hipLaunchKernelGGL((append_kernel<N, BITS, D>), grid_of((a.tokens + 2048 / D - 1) / (2048 / D)), dim3(256), 0, s, c, a); \
    break;
    QNN_LM_DIMS(CALL)
#undef CALL
}

hipError_t launch_append(const CacheArgs &c, int bits, int dim, int type, const void *k, const void *v,
                         const int64_t *k_stride, const int64_t *v_stride, int t, const int32_t *lens,
                         const int32_t *counts, hipStream_t s)
{
    TokenArgs a;
    a.k = k;
    a.v = v;
    for (int i = 0; i < 3; ++i) {
        a.ks[i] = k_stride[i];
        a.vs[i] = v_stride[i];
    }
    a.t = t;
    a.tokens = (uint32_t)((int64_t)c.b * t * c.heads);
    a.heads_div = qnn::make_fastdiv((uint32_t)c.heads);
    a.t_div = qnn::make_fastdiv((uint32_t)t);
    a.lens = lens;
    a.counts = counts;
    if (bits == 16)
        return append_bits<Bf16, 16>(c, dim, a, s);  // 16-bit numbers are copied
    if (type == QNN_LM_BF16)
        return bits == 8 ? append_bits<Bf16, 8>(c, dim, a, s) : append_bits<Bf16, 4>(c, dim, a, s);
    return bits == 8 ? append_bits<F16, 8>(c, dim, a, s) : append_bits<F16, 4>(c, dim, a, s);
}

template <class N, class C, int BITS>
static hipError_t read_bits(const CacheArgs &c, int dim, const ReadArgs &a, hipStream_t s)
{
#define CALL(D)                                                                                              \
    hipLaunchKernelGGL((read_kernel<N, C, BITS, D>), grid_of((a.tokens + 2048 / D - 1) / (2048 / D)), dim3(256), 0, s, c, a); \
    break;
    QNN_LM_DIMS(CALL)
#undef CALL
}

template <class N>
static hipError_t read_typed(const CacheArgs &c, int bits, int dim, int cache_type, const ReadArgs &a, hipStream_t s)
{
    if (bits == 8)
        return read_bits<N, Bf16, 8>(c, dim, a, s);
    if (bits == 4)
        return read_bits<N, Bf16, 4>(c, dim, a, s);
    return cache_type == QNN_LM_BF16 ? read_bits<N, Bf16, 16>(c, dim, a, s) : read_bits<N, F16, 16>(c, dim, a, s);
}

hipError_t launch_read(const CacheArgs &c, int bits, int dim, int type, int cache_type, int t, const int32_t *start,
                       void *k, void *v, hipStream_t s)
{
    ReadArgs a;
    a.k = k;
    a.v = v;
    a.t = t;
    a.tokens = (uint32_t)((int64_t)c.b * t * c.heads);
    a.heads_div = qnn::make_fastdiv((uint32_t)c.heads);
    a.t_div = qnn::make_fastdiv((uint32_t)t);
    a.start = start;
    if (type == QNN_LM_F32)
        return read_typed<F32>(c, bits, dim, cache_type, a, s);
    return type == QNN_LM_BF16 ? read_typed<Bf16>(c, bits, dim, cache_type, a, s)
                               : read_typed<F16>(c, bits, dim, cache_type, a, s);
}

hipError_t launch_keep(const CacheArgs &c, int bits, int dim, int t, const int32_t *lens, const int32_t *path,
                       const int32_t *kept, hipStream_t s)
{
    const dim3 grid(2 * c.heads, c.b);
    switch (dim * bits / 8) {
#define CASE(ROW)                                                                                   \
    case ROW:                                                                                       \
        hipLaunchKernelGGL(keep_kernel<ROW>, grid, dim3(256), 0, s, c, t, lens, path, kept);        \
        break;
        CASE(32) CASE(64) CASE(128) CASE(256) CASE(512)
#undef CASE
    default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

}  // namespace qnn_lm
