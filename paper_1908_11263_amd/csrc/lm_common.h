// Shared by the kernels of include/qnn_lm.h: 16-bit number types, matrix
// instructions, and packed codes expanded to 16-bit numbers.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "qnn_lm.h"

namespace qnn_lm {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f16v __attribute__((ext_vector_type(16)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));

// Number types: T the element, V8 eight of them (an MFMA operand of one lane).
struct Bf16 {
    using T = __bf16;
    using V8 = bf8;
    using V2 = bf2;
};
struct F16 {
    using T = _Float16;
    using V8 = h8;
    using V2 = h2;
};
struct F32 {
    using T = float;
};

// D (16x16, fp32) += A (16 rows x 32) * B (32 x 16 columns).  Lane l holds
// row / column l % 16 of A / B at k = 8 * (l / 16) .. + 7, and of D column
// l % 16 at rows 4 * (l / 16) .. + 3.
__device__ __forceinline__ f4 mfma16(bf8 a, bf8 b, f4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f4 mfma16(h8 a, h8 b, f4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// Two floats rounded to nearest even, the first in the low half.
template <class N>
__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    const typename N::V2 v = {(typename N::T)a, (typename N::T)b};
    return __builtin_bit_cast(uint32_t, v);
}

// --- signed bytes to 16-bit numbers ------------------------------------------
// Four signed bytes (lowest first) of `a` interleaved with four of `b`:
// a0 b0 a1 b1 a2 b2 a3 b3.  bf16: a byte is converted to fp32 (one instruction
// with a byte selector) and the upper halves of two are joined: exact, for
// magnitudes up to 256.  f16: a byte plus 128 becomes the low mantissa byte of
// 1024 + .., and 1152 is subtracted, two at a time: exact.
template <class N>
__device__ __forceinline__ typename N::V8 expand_pairs(uint32_t a, uint32_t b);

__device__ __forceinline__ uint32_t join_bf16(int32_t lo, int32_t hi)
{
    return __builtin_amdgcn_perm(__float_as_uint((float)hi), __float_as_uint((float)lo), 0x07060302u);
}

template <>
__device__ __forceinline__ bf8 expand_pairs<Bf16>(uint32_t a, uint32_t b)
{
    u4 r;
    r.x = join_bf16((int8_t)a, (int8_t)b);
    r.y = join_bf16((int8_t)(a >> 8), (int8_t)(b >> 8));
    r.z = join_bf16((int8_t)(a >> 16), (int8_t)(b >> 16));
    r.w = join_bf16((int8_t)(a >> 24), (int8_t)(b >> 24));
    return __builtin_bit_cast(bf8, r);
}

// f16 of the bytes 0 and 1 (SEL 0x04010400) or 2 and 3 (0x04030402) of v ^ 0x80808080
template <uint32_t SEL>
__device__ __forceinline__ uint32_t half_pair(uint32_t v)
{
    const h2 x = __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, v, SEL));
    const h2 k = {(_Float16)-1152.f, (_Float16)-1152.f};
    return __builtin_bit_cast(uint32_t, x + k);
}

__device__ __forceinline__ h8 expand_h8(uint32_t lo, uint32_t hi)
{
    lo ^= 0x80808080u;
    hi ^= 0x80808080u;
    u4 r;
    r.x = half_pair<0x04010400u>(lo);
    r.y = half_pair<0x04030402u>(lo);
    r.z = half_pair<0x04010400u>(hi);
    r.w = half_pair<0x04030402u>(hi);
    return __builtin_bit_cast(h8, r);
}

template <>
__device__ __forceinline__ h8 expand_pairs<F16>(uint32_t a, uint32_t b)
{
    return expand_h8(__builtin_amdgcn_perm(b, a, 0x05010400u), __builtin_amdgcn_perm(b, a, 0x07030602u));
}

// Eight signed bytes in order.
template <class N>
__device__ __forceinline__ typename N::V8 expand_bytes(uint32_t lo, uint32_t hi);

template <>
__device__ __forceinline__ bf8 expand_bytes<Bf16>(uint32_t lo, uint32_t hi)
{
    u4 r;
    r.x = join_bf16((int8_t)lo, (int8_t)(lo >> 8));
    r.y = join_bf16((int8_t)(lo >> 16), (int8_t)(lo >> 24));
    r.z = join_bf16((int8_t)hi, (int8_t)(hi >> 8));
    r.w = join_bf16((int8_t)(hi >> 16), (int8_t)(hi >> 24));
    return __builtin_bit_cast(bf8, r);
}

template <>
__device__ __forceinline__ h8 expand_bytes<F16>(uint32_t lo, uint32_t hi)
{
    return expand_h8(lo, hi);
}

// --- packed codes to 16-bit numbers ------------------------------------------
// A sub-byte code is moved to the top of a byte (no sign extension), so the
// numbers are 1 / kUnscale times the codes; the caller folds kUnscale, a power
// of two, into its scale.  A 1-bit code becomes +64 or -64.
template <int BITS>
constexpr float kUnscale = BITS == 4 ? 1.f / 16 : BITS <= 2 ? 1.f / 64 : 1.f;

// Bytes B of f0, f1, f2, f3.
template <int B>
__device__ __forceinline__ uint32_t gather_bytes(uint32_t f0, uint32_t f1, uint32_t f2, uint32_t f3)
{
    constexpr uint32_t sel = 0x0C0C0000u | ((4 + B) << 8) | B;
    const uint32_t lo = __builtin_amdgcn_perm(f1, f0, sel), hi = __builtin_amdgcn_perm(f3, f2, sel);
    return lo | (hi << 16);
}

// Eight numbers whose codes are byte B of the eight words f0 .. f7.
template <class N, int B>
__device__ __forceinline__ typename N::V8 expand_fields(uint32_t f0, uint32_t f1, uint32_t f2, uint32_t f3,
                                                        uint32_t f4_, uint32_t f5, uint32_t f6, uint32_t f7)
{
    if constexpr (__is_same(N, Bf16)) {
        u4 r;
        r.x = join_bf16((int8_t)(f0 >> 8 * B), (int8_t)(f1 >> 8 * B));
        r.y = join_bf16((int8_t)(f2 >> 8 * B), (int8_t)(f3 >> 8 * B));
        r.z = join_bf16((int8_t)(f4_ >> 8 * B), (int8_t)(f5 >> 8 * B));
        r.w = join_bf16((int8_t)(f6 >> 8 * B), (int8_t)(f7 >> 8 * B));
        return __builtin_bit_cast(bf8, r);
    } else {
        return expand_h8(gather_bytes<B>(f0, f1, f2, f3), gather_bytes<B>(f4_, f5, f6, f7));
    }
}

// The F-th eight numbers of a lane's packed bytes `raw` (the first in the
// lowest bits of raw[0]).
template <class N, int BITS, int F>
__device__ __forceinline__ typename N::V8 expand(const uint32_t *raw)
{
    if constexpr (BITS == 16) {
        const u4 r = {raw[4 * F], raw[4 * F + 1], raw[4 * F + 2], raw[4 * F + 3]};
        return __builtin_bit_cast(typename N::V8, r);
    } else if constexpr (BITS == 8) {
        return expand_bytes<N>(raw[2 * F], raw[2 * F + 1]);
    } else if constexpr (BITS == 4) {
        const uint32_t v = raw[F];
        return expand_pairs<N>((v << 4) & 0xF0F0F0F0u, v & 0xF0F0F0F0u);
    } else if constexpr (BITS == 2) {
        const uint32_t v = raw[F / 2];
        const uint32_t f0 = (v << 6) & 0xC0C0C0C0u, f1 = (v << 4) & 0xC0C0C0C0u, f2 = (v << 2) & 0xC0C0C0C0u,
                       f3 = v & 0xC0C0C0C0u;
        constexpr int S = 16 * (F % 2);
        return expand_fields<N, 0>(f0 >> S, f1 >> S, f2 >> S, f3 >> S, f0 >> (S + 8), f1 >> (S + 8), f2 >> (S + 8),
                                   f3 >> (S + 8));
    } else {
        const uint32_t v = ~raw[0];
        auto field = [&](int i) { return ((v << (7 - i)) & 0x80808080u) | 0x40404040u; };
        return expand_fields<N, F>(field(0), field(1), field(2), field(3), field(4), field(5), field(6), field(7));
    }
}

// --- memory --------------------------------------------------------------------
// Two or four words from a place aligned to their size.
template <int WORDS>
__device__ __forceinline__ void load_words(const uint8_t *p, uint32_t *r)
{
    if constexpr (WORDS == 4) {
        const u4 v = *(const u4 *)p;
        r[0] = v.x, r[1] = v.y, r[2] = v.z, r[3] = v.w;
    } else {
        const u2 v = *(const u2 *)p;
        r[0] = v.x, r[1] = v.y;
    }
}

template <class N>
__device__ __forceinline__ float load1(const void *p, int64_t i)
{
    return (float)((const typename N::T *)p)[i];
}

template <class N>
__device__ __forceinline__ void store1(void *p, int64_t i, float v)
{
    ((typename N::T *)p)[i] = (typename N::T)v;
}

// Eight numbers from a 16-byte aligned place (32 bytes of F32).
template <class N>
__device__ __forceinline__ void load8(const void *p, int64_t i, float (&v)[8])
{
    if constexpr (__is_same(N, F32)) {
        const f4 a = *(const f4 *)((const float *)p + i), b = *(const f4 *)((const float *)p + i + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[e] = a[e];
            v[4 + e] = b[e];
        }
    } else {
        const typename N::V8 a = *(const typename N::V8 *)((const typename N::T *)p + i);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[e] = (float)a[e];
    }
}

// ... from and to any place of 16-bit numbers (the memory unit takes 16 bytes
// at any address).
typedef u4 u4_any __attribute__((aligned(2)));

template <class N>
__device__ __forceinline__ void load8_any(const void *p, int64_t i, float (&v)[8])
{
    const u4 r = *(const u4_any *)((const typename N::T *)p + i);
    const typename N::V8 a = __builtin_bit_cast(typename N::V8, r);
#pragma unroll
    for (int e = 0; e < 8; ++e)
        v[e] = (float)a[e];
}

template <class N>
__device__ __forceinline__ void store8_any(void *p, int64_t i, const float (&v)[8])
{
    const u4 r = {pack2<N>(v[0], v[1]), pack2<N>(v[2], v[3]), pack2<N>(v[4], v[5]), pack2<N>(v[6], v[7])};
    *(u4_any *)((typename N::T *)p + i) = r;
}

template <class N>
__device__ __forceinline__ void store8(void *p, int64_t i, const float (&v)[8])
{
    if constexpr (__is_same(N, F32)) {
        *(f4 *)((float *)p + i) = (f4){v[0], v[1], v[2], v[3]};
        *(f4 *)((float *)p + i + 4) = (f4){v[4], v[5], v[6], v[7]};
    } else {
        const u4 r = {pack2<N>(v[0], v[1]), pack2<N>(v[2], v[3]), pack2<N>(v[4], v[5]), pack2<N>(v[6], v[7])};
        *(u4 *)((typename N::T *)p + i) = r;
    }
}

}  // namespace qnn_lm
