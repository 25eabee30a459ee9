/*
 * qnn_lm.h - one step of a language model's block over packed weights and a
 * packed cache, on MI355X (gfx950).
 *
 * The entry points serve the block of a transformer whose weights and whose
 * cache of keys and values are held as the packed codes of qnn.h, with scales
 * in 32 bits, and whose activations are 16-bit numbers: the linear layer with
 * its epilogue, the norms between two blocks, the attention of a tree of
 * drafted tokens (or of one token, or of a chunk of a prompt) over a paged
 * cache, and the cache's own writes.
 *
 * Conventions as in qnn.h: caller-owned device memory, 16-byte aligned device
 * pointers (QNN_ERR_ALIGN), asynchronous on `stream` (a hipStream_t; NULL =
 * the null stream), every argument check on the host before any device call, a
 * qnn_status for every error, no device memory of the library's own.  Empty
 * inputs (no rows, no sequences) are valid and launch nothing.
 *
 * Packing.  b-bit codes (b = 8, 4, 2: two's complement; b = 1: +1 for bit 1,
 * -1 for bit 0) along the reduced axis, 8/b codes a byte, the lower index in
 * the less significant bits.
 * Arithmetic.  Products are exact (a code is an exact 16-bit number), sums,
 * softmax statistics, norms and epilogues are kept in 32-bit floating point;
 * results are rounded once, to nearest even, when they are stored.  The
 * attention's probabilities multiply the values as 16-bit numbers, each off by
 * 2^-12 of itself or 2^-35 of the row's largest at most (2^-9 of itself over a
 * cache of bf16 numbers); with up to 32 rows a cache head (16 of 256 channels) as
 * the sum of two such numbers, and next to value scales more than 2^12 apart as
 * the sum of three bf16 numbers.  Their own sum is not rounded.  The order of
 * every sum is fixed: the same call gives the same bits.
 * NaN and infinities that enter a sum come out of it as of the formula; scales
 * may have either sign.
 * Values that live on the device (lengths, page numbers, paths) cannot be
 * checked on the host.  The kernels bound every index that they make of them:
 * a position whose page number is outside of the cache, or that the table does
 * not reach, is not visible, reads as zero and is not written.
 */
#ifndef QNN_LM_H
#define QNN_LM_H

#include <stddef.h>
#include <stdint.h>

#include "qnn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Types of activations. */
typedef enum { QNN_LM_BF16 = 0, QNN_LM_F16 = 1, QNN_LM_F32 = 2 } qnn_lm_type;

typedef enum {
    QNN_LM_ACT_NONE = 0,
    QNN_LM_ACT_RELU = 1,
    QNN_LM_ACT_SILU = 2,      /* t / (1 + exp(-t)) */
    QNN_LM_ACT_GELU = 3,      /* t/2 * (1 + erf(t / sqrt(2))) */
    QNN_LM_ACT_GELU_TANH = 4  /* t/2 * (1 + tanh(sqrt(2/pi) * (t + 0.044715 t^3))) */
} qnn_lm_act;

typedef enum { QNN_LM_RMS = 0, QNN_LM_LAYER = 1 } qnn_lm_norm;

/* A linear layer: r rows of k numbers, m outputs a row. */
typedef struct {
    int32_t type;     /* of x, residual and y: QNN_LM_BF16 or QNN_LM_F16 */
    int32_t bits;     /* of the weights: 8, 4, 2, 1 (codes), or 16 (numbers of `type`) */
    int32_t r, k, m;
    int32_t group;    /* weights along k that share a scale: 32, 64 or 128, or 0 for all of a row */
    int32_t act;      /* a qnn_lm_act */
    int32_t gated;    /* 1: the weights have 2m rows, the gate's first */
    int64_t x_pitch;  /* elements from one row to the next; a multiple of 8, at least k */
    int64_t residual_pitch, y_pitch; /* at least m */
} qnn_lm_linear;

/*
 * Linear layer with its epilogue.
 *   t[i, j] = sum_k x[i, k] * w[j, k] * scale[j, k / group] + bias[j]
 *   y[i, j] = act(t[i, j]) + residual[i, j], or with gated = 1
 *   y[i, j] = act(t[i, j]) * t[i, m + j] + residual[i, j]
 * w: [m or 2m] rows of k*bits/8 bytes; k a multiple of 32 and of `group`
 * (pad with zero codes, and zeros in x).  scale: [rows][k / group] or [rows]
 * floats, NULL (and only then) at 16 bits.  bias: [rows] floats or NULL.
 * residual may be NULL and may be y itself.  ws: at least
 * qnn_lm_matmul_workspace(s) bytes, or NULL where that is 0; its contents need
 * not be set and are not kept.  Limits: k <= 2^20, rows of weights <= 2^24 (of
 * both halves together), rows of x <= 2^21, each tensor < 2^40 bytes.
 */
qnn_status qnn_lm_matmul(const qnn_lm_linear *s, const void *x, const void *w, const float *scale,
                         const float *bias, const void *residual, void *y, void *ws, size_t ws_bytes,
                         void *stream);

/* Bytes of workspace that qnn_lm_matmul takes for `s` (0 for one it refuses). */
size_t qnn_lm_matmul_workspace(const qnn_lm_linear *s);

/* The norms around a block's end. */
typedef struct {
    int32_t type;    /* of y, gate and x */
    int32_t h_type;  /* of h and h_out: `type` or QNN_LM_F32 */
    int32_t r, d;    /* rows, channels (at most 32768) */
    int32_t norm;    /* a qnn_lm_norm */
    int32_t post;    /* 1: y is normed before it is added */
    int32_t gates;   /* rows of gate: 0 (none), or a divisor of r: row i takes gate row i / (r / gates) */
    float eps, alpha, beta;
    int64_t h_pitch, y_pitch; /* elements from one row to the next */
} qnn_lm_norms;

/*
 * Norm after a block, gate, residual scale and norm before the next block:
 *   h_out = alpha * h + beta * gate * N_post(y),   x = N_pre(h_out)
 *   N(v)  = v / sqrt(mean(v^2) + eps) * weight + bias, about the row's mean
 *           first with QNN_LM_LAYER
 * Weights and biases are [d] floats or NULL (one, zero).  x is computed from
 * h_out before its rounding.  y may be NULL: x = N_pre(h), h_out is not
 * written (alpha, beta, post, gates unused).  h_out [r][d] may be h itself if
 * h_pitch = d; x [r][d] may be y if y_pitch = d.
 */
qnn_status qnn_lm_norm_residual(const qnn_lm_norms *s, const void *h, const void *y, const float *post_weight,
                                const float *post_bias, const float *pre_weight, const float *pre_bias,
                                const void *gate, void *h_out, void *x, void *stream);

/*
 * A paged cache of keys and values.  Position p of sequence i lies in slot
 * p % page of page table[i * width + p / page].  Strides are in bytes,
 * multiples of 16 (a 4-bit slot of 64 channels: 32 bytes); the channels of a
 * slot are contiguous.  Codes are symmetric (-(2^(bits-1) - 1) to its
 * opposite as written by qnn_lm_cache_append; any code is read), a value is
 * code * scale[page][head][slot].  Limits: width * page <= 2^31 - 256, b <=
 * 65535, heads <= 32767; of a call's tokens, 2 * b * t * heads <= 2^31 - 256.
 */
typedef struct {
    int32_t type;    /* of the numbers at 16 bits: QNN_LM_BF16 or QNN_LM_F16 */
    int32_t bits;    /* 16, 8 or 4 */
    int32_t pages, heads, page; /* page: slots of a page, at least 1 */
    int32_t dim;     /* channels of a head: 64, 128 or 256 */
    int64_t k_page, k_head, k_slot, v_page, v_head, v_slot;
    void *k, *v;
    float *k_scale, *v_scale; /* [pages][heads][page], NULL (and only then) at 16 bits */
    const int32_t *table;     /* [b][width] page numbers */
    int32_t b, width;
} qnn_lm_cache;

/*
 * Attention of t drafted tokens a sequence over the cache.
 *   q:      [b][t][heads][dim] with strides (in elements, multiples of 8) of
 *           q_stride; `type` numbers.  heads a multiple of the cache's heads:
 *           query head i reads cache head i / (heads / cache heads).
 *   lens:   [b] cached tokens before the drafts, seen by every draft.
 *   counts: [b] drafts of each sequence, or NULL: t.  Draft j lies at position
 *           lens + j.
 *   mask:   [b][t][words] 64-bit words, words = ceil(t / 64): bit j % 64 of
 *           word j / 64 says whether a draft sees draft j; NULL: draft i sees
 *           drafts 0 .. i.
 *   out:    [b][t][heads][dim] `type` numbers; lse: [b][t][heads] floats, the
 *           natural logarithm of the sum of exponentials, or NULL.
 * A draft that sees nothing (or nothing but scores of -infinity), and one at or
 * past its count, gets zeros and -infinity.  What an unseen position holds has no
 * influence.  Limits: t * heads <= 2^24, b * t * heads <= 2^31 - 256.
 */
typedef struct {
    int32_t type;   /* of q and out (at 16 bits the cache's type) */
    int32_t t, heads;
    float scale;    /* of the scores; usually 1 / sqrt(dim) */
    int64_t q_stride[3]; /* sequence, draft, head */
} qnn_lm_queries;

qnn_status qnn_lm_tree_attention(const qnn_lm_queries *s, const void *q, const qnn_lm_cache *c,
                                 const int32_t *lens, const int32_t *counts, const uint64_t *mask, void *out,
                                 float *lse, void *ws, size_t ws_bytes, void *stream);

/* Bytes of workspace that qnn_lm_tree_attention takes (0 for a call it refuses). */
size_t qnn_lm_tree_attention_workspace(const qnn_lm_queries *s, const qnn_lm_cache *c);

/* New tokens: [b][t][heads][dim] numbers of `type`, strides in elements
 * (multiples of 8) of the sequence, the token and the head. */
typedef struct {
    int32_t type, t;
    int64_t k_stride[3], v_stride[3];
} qnn_lm_tokens;

/*
 * Writes token j < counts[i] (NULL: t) of each sequence to position lens[i] +
 * j.  At 8 and 4 bits a token's scale is, for each head, its largest magnitude
 * / (2^(bits-1) - 1) in 32 bits, a code the whole number nearest to value /
 * scale (ties to even; all zero where the scale is zero; a token that holds
 * infinity or NaN gets scale NaN).
 */
qnn_status qnn_lm_cache_append(const qnn_lm_tokens *s, const void *k, const void *v, const qnn_lm_cache *c,
                               const int32_t *lens, const int32_t *counts, void *stream);

/*
 * Moves the accepted drafts to the front: position lens[i] + j takes what
 * position lens[i] + path[i * t + j] holds, for j < kept[i].  path ascends
 * strictly within 0 .. t - 1 (a token whose entry is smaller than its index or
 * not below t is not moved).
 */
qnn_status qnn_lm_cache_keep(const qnn_lm_cache *c, int32_t t, const int32_t *lens, const int32_t *path,
                             const int32_t *kept, void *stream);

/*
 * Positions start[i] .. start[i] + t - 1 of each sequence as numbers of
 * `type`: k and v are [b][t][heads][dim], contiguous; either may be NULL.
 */
qnn_status qnn_lm_cache_read(const qnn_lm_cache *c, int32_t type, int32_t t, const int32_t *start, void *k,
                             void *v, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* QNN_LM_H */
