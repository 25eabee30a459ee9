// C ABI of include/qnn_lm.h: argument checks (all on the host, before any
// device call) and dispatch.
#include "lm_internal.h"

using namespace qnn_lm;

namespace {

constexpr int64_t kMostBytes = (int64_t)1 << 40;

bool aligned16(const void *p) { return ((uintptr_t)p & 15u) == 0; }

qnn_status launched(hipError_t e) { return e == hipSuccess ? QNN_OK : QNN_ERR_LAUNCH; }

bool type16(int32_t t) { return t == QNN_LM_BF16 || t == QNN_LM_F16; }

int64_t type_bytes(int32_t t) { return t == QNN_LM_F32 ? 4 : 2; }

// n >= 0 rows `pitch` elements apart stay below kMostBytes
bool fits(int64_t n, int64_t pitch, int64_t bytes) { return pitch <= kMostBytes / bytes / (n > 1 ? n : 1); }

qnn_status check_linear(const qnn_lm_linear *s)
{
    if (!s)
        return QNN_ERR_NULL;
    if (s->bits != 16 && s->bits != 8 && s->bits != 4 && s->bits != 2 && s->bits != 1)
        return QNN_ERR_BITS;
    if (!type16(s->type) || s->act < QNN_LM_ACT_NONE || s->act > QNN_LM_ACT_GELU_TANH || (s->gated != 0 && s->gated != 1))
        return QNN_ERR_PARAM;
    if (s->group != 0 && s->group != 32 && s->group != 64 && s->group != 128)
        return QNN_ERR_PARAM;
    if (s->bits == 16 && s->group != 0)
        return QNN_ERR_PARAM;
    if (s->r < 0 || s->k < 1 || s->m < 1 || s->r > 1 << 21 || s->m > (s->gated ? 1 << 23 : 1 << 24))
        return QNN_ERR_SHAPE;
    if (s->k % 32 != 0 || (s->group && s->k % s->group != 0))
        return QNN_ERR_SHAPE;
    if (s->k > 1 << 20)
        return QNN_ERR_UNSUPPORTED;
    if (s->x_pitch < s->k || s->y_pitch < s->m || s->residual_pitch < 0)
        return QNN_ERR_SHAPE;
    if (s->x_pitch % 8 != 0)
        return QNN_ERR_ALIGN;
    const int64_t rows = s->gated ? 2 * (int64_t)s->m : s->m;
    if (!fits(s->r, s->x_pitch, 2) || !fits(s->r, s->y_pitch, 2) || !fits(s->r, s->residual_pitch, 2) ||
        !fits(rows, s->k, 2))
        return QNN_ERR_SHAPE;
    return QNN_OK;
}

MatmulArgs matmul_args(const qnn_lm_linear *s)
{
    MatmulArgs a = {};
    a.r = s->r;
    a.k = s->k;
    a.m = s->m;
    a.group = s->group ? s->group : s->k;
    a.groups = s->group ? s->k / s->group : 1;
    a.act = s->act;
    a.gated = s->gated;
    a.x_pitch = s->x_pitch;
    a.residual_pitch = s->residual_pitch;
    a.y_pitch = s->y_pitch;
    a.w_row = (int64_t)s->k * s->bits / 8;
    return a;
}

qnn_status check_stride(int64_t n, int64_t stride, int64_t least)
{
    if (stride < (n > 1 ? least : 0) || !fits(n, stride, 1))
        return QNN_ERR_SHAPE;
    return stride % 16 != 0 ? QNN_ERR_ALIGN : QNN_OK;
}

qnn_status check_cache(const qnn_lm_cache *c)
{
    if (!c)
        return QNN_ERR_NULL;
    if (c->bits != 16 && c->bits != 8 && c->bits != 4)
        return QNN_ERR_BITS;
    if (!type16(c->type))
        return QNN_ERR_PARAM;
    if (c->pages < 1 || c->heads < 1 || c->page < 1 || c->b < 0 || c->width < 1)
        return QNN_ERR_SHAPE;
    if (c->dim != 64 && c->dim != 128 && c->dim != 256)
        return QNN_ERR_UNSUPPORTED;
    // a table reaches positions of 31 bits; sequences and heads are grid sizes
    if ((int64_t)c->width * c->page > 0x7FFFFF00 || c->b > 65535 || c->heads > 32767)
        return QNN_ERR_SHAPE;
    const int64_t row = (int64_t)c->dim * c->bits / 8;
    const int64_t n[6] = {c->pages, c->heads, c->page, c->pages, c->heads, c->page};
    const int64_t st[6] = {c->k_page, c->k_head, c->k_slot, c->v_page, c->v_head, c->v_slot};
    for (int i = 0; i < 6; ++i) {
        const qnn_status e = check_stride(n[i], st[i], row);
        if (e != QNN_OK)
            return e;
    }
    return QNN_OK;
}

qnn_status check_cache_pointers(const qnn_lm_cache *c, bool k, bool v)
{
    if ((k && !c->k) || (v && !c->v) || !c->table)
        return QNN_ERR_NULL;
    if (c->bits == 16 ? (c->k_scale || c->v_scale) : ((k && !c->k_scale) || (v && !c->v_scale)))
        return c->bits == 16 ? QNN_ERR_PARAM : QNN_ERR_NULL;
    if (!aligned16(c->k) || !aligned16(c->v) || !aligned16(c->k_scale) || !aligned16(c->v_scale) || !aligned16(c->table))
        return QNN_ERR_ALIGN;
    return QNN_OK;
}

CacheArgs cache_args(const qnn_lm_cache *c)
{
    CacheArgs a;
    a.k = (uint8_t *)c->k;
    a.v = (uint8_t *)c->v;
    a.k_scale = c->k_scale;
    a.v_scale = c->v_scale;
    a.table = c->table;
    a.pages = c->pages;
    a.heads = c->heads;
    a.page = c->page;
    a.b = c->b;
    a.width = c->width;
    a.k_page = c->k_page;
    a.k_head = c->k_head;
    a.k_slot = c->k_slot;
    a.v_page = c->v_page;
    a.v_head = c->v_head;
    a.v_slot = c->v_slot;
    a.page_div = qnn::make_fastdiv((uint32_t)c->page);
    return a;
}

qnn_status check_element_strides(const int64_t *st, int64_t b, int64_t t, int64_t heads)
{
    const int64_t n[3] = {b, t, heads};
    for (int i = 0; i < 3; ++i) {
        if (st[i] < 0 || !fits(n[i], st[i], 2))
            return QNN_ERR_SHAPE;
        if (st[i] % 8 != 0)
            return QNN_ERR_ALIGN;
    }
    return QNN_OK;
}

qnn_status check_queries(const qnn_lm_queries *s, const qnn_lm_cache *c)
{
    if (!s)
        return QNN_ERR_NULL;
    const qnn_status e = check_cache(c);
    if (e != QNN_OK)
        return e;
    if (!type16(s->type))
        return QNN_ERR_PARAM;
    if (c->bits == 16 && c->type != s->type)
        return QNN_ERR_PARAM;
    if (s->t < 0 || s->heads < 1 || s->heads % c->heads != 0)
        return QNN_ERR_SHAPE;
    if ((int64_t)s->t * s->heads > 1 << 24 || (int64_t)c->b * s->t * s->heads > 0x7FFFFF00)
        return QNN_ERR_SHAPE;
    if (!(s->scale == s->scale) || s->scale - s->scale != 0.f)  // NaN, infinity
        return QNN_ERR_PARAM;
    return check_element_strides(s->q_stride, c->b, s->t, s->heads);
}

AttendArgs attend_args(const qnn_lm_queries *s)
{
    AttendArgs a = {};
    a.t = s->t;
    a.heads = s->heads;
    a.scale = s->scale;
    a.q_b = s->q_stride[0];
    a.q_t = s->q_stride[1];
    a.q_h = s->q_stride[2];
    return a;
}

// Tokens are numbered in 32 bits.
bool token_count(const qnn_lm_cache *c, int32_t t) { return (int64_t)c->b * t <= 0x7FFFFF00 / (2 * (int64_t)c->heads); }

}  // namespace

extern "C" {

size_t qnn_lm_matmul_workspace(const qnn_lm_linear *s)
{
    if (check_linear(s) != QNN_OK || s->r == 0)
        return 0;
    return matmul_workspace(matmul_args(s), s->type, s->bits);
}

qnn_status qnn_lm_matmul(const qnn_lm_linear *s, const void *x, const void *w, const float *scale, const float *bias,
                         const void *residual, void *y, void *ws, size_t ws_bytes, void *stream)
{
    qnn_status e = check_linear(s);
    if (e != QNN_OK)
        return e;
    if (!w || (s->r && (!x || !y)) || (s->bits != 16 && !scale))
        return QNN_ERR_NULL;
    if (s->bits == 16 && scale)
        return QNN_ERR_PARAM;
    if (residual && s->residual_pitch < s->m)
        return QNN_ERR_SHAPE;
    if (!aligned16(x) || !aligned16(w) || !aligned16(scale) || !aligned16(bias) || !aligned16(residual) || !aligned16(y) ||
        !aligned16(ws))
        return QNN_ERR_ALIGN;
    if (s->r == 0)
        return QNN_OK;
    MatmulArgs a = matmul_args(s);
    const size_t need = matmul_workspace(a, s->type, s->bits);
    if (need && !ws)
        return QNN_ERR_NULL;
    if (ws_bytes < need)
        return QNN_ERR_SHAPE;
    if ((e = qnn_device_check()) != QNN_OK)
        return e;
    a.x = x;
    a.w = w;
    a.scale = scale;
    a.bias = bias;
    a.residual = residual;
    a.y = y;
    return launched(launch_matmul(a, s->type, s->bits, ws, (hipStream_t)stream));
}

qnn_status qnn_lm_norm_residual(const qnn_lm_norms *s, const void *h, const void *y, const float *post_weight,
                                const float *post_bias, const float *pre_weight, const float *pre_bias,
                                const void *gate, void *h_out, void *x, void *stream)
{
    if (!s)
        return QNN_ERR_NULL;
    if (s->type < QNN_LM_BF16 || s->type > QNN_LM_F32 || (s->h_type != s->type && s->h_type != QNN_LM_F32) ||
        (s->norm != QNN_LM_RMS && s->norm != QNN_LM_LAYER) || (s->post != 0 && s->post != 1) || !(s->eps >= 0.f))
        return QNN_ERR_PARAM;
    if (s->r < 0 || s->d < 1 || s->gates < 0 || s->h_pitch < s->d || (y && s->y_pitch < s->d))
        return QNN_ERR_SHAPE;
    if (s->d > 32768)
        return QNN_ERR_UNSUPPORTED;
    if (y && s->gates && s->r % s->gates != 0)
        return QNN_ERR_SHAPE;
    if (!fits(s->r, s->h_pitch, type_bytes(s->h_type)) || (y && !fits(s->r, s->y_pitch, type_bytes(s->type))))
        return QNN_ERR_SHAPE;
    if (s->r && (!h || !x || (y && !h_out) || (y && s->gates && !gate)))
        return QNN_ERR_NULL;
    if (!aligned16(h) || !aligned16(y) || !aligned16(post_weight) || !aligned16(post_bias) || !aligned16(pre_weight) ||
        !aligned16(pre_bias) || !aligned16(gate) || !aligned16(h_out) || !aligned16(x))
        return QNN_ERR_ALIGN;
    if (s->r == 0)
        return QNN_OK;
    const qnn_status e = qnn_device_check();
    if (e != QNN_OK)
        return e;
    NormArgs a;
    a.h = h;
    a.y = y;
    a.gate = gate;
    a.post_weight = post_weight;
    a.post_bias = post_bias;
    a.pre_weight = pre_weight;
    a.pre_bias = pre_bias;
    a.h_out = h_out;
    a.x = x;
    a.r = s->r;
    a.d = s->d;
    a.layer = s->norm == QNN_LM_LAYER;
    a.post = s->post;
    a.gates = y ? s->gates : 0;
    a.gate_rows = a.gates ? s->r / a.gates : 1;
    a.eps = s->eps;
    a.alpha = s->alpha;
    a.beta = s->beta;
    a.h_pitch = s->h_pitch;
    a.y_pitch = s->y_pitch;
    return launched(launch_norm(a, s->type, s->h_type, (hipStream_t)stream));
}

size_t qnn_lm_tree_attention_workspace(const qnn_lm_queries *s, const qnn_lm_cache *c)
{
    if (check_queries(s, c) != QNN_OK || c->b == 0 || s->t == 0)
        return 0;
    return attend_workspace(attend_args(s), cache_args(c), c->dim);
}

qnn_status qnn_lm_tree_attention(const qnn_lm_queries *s, const void *q, const qnn_lm_cache *c, const int32_t *lens,
                                 const int32_t *counts, const uint64_t *mask, void *out, float *lse, void *ws,
                                 size_t ws_bytes, void *stream)
{
    qnn_status e = check_queries(s, c);
    if (e != QNN_OK)
        return e;
    if (c->b == 0 || s->t == 0)
        return QNN_OK;
    if (!q || !lens || !out)
        return QNN_ERR_NULL;
    if ((e = check_cache_pointers(c, true, true)) != QNN_OK)
        return e;
    if (!aligned16(q) || !aligned16(lens) || !aligned16(counts) || !aligned16(mask) || !aligned16(out) ||
        !aligned16(lse) || !aligned16(ws))
        return QNN_ERR_ALIGN;
    AttendArgs a = attend_args(s);
    const CacheArgs ca = cache_args(c);
    const size_t need = attend_workspace(a, ca, c->dim);
    if (need && !ws)
        return QNN_ERR_NULL;
    if (ws_bytes < need)
        return QNN_ERR_SHAPE;
    if ((e = qnn_device_check()) != QNN_OK)
        return e;
    a.q = q;
    a.lens = lens;
    a.counts = counts;
    a.mask = mask;
    a.out = out;
    a.lse = lse;
    return launched(launch_attend(a, ca, c->bits, c->dim, s->type, ws, (hipStream_t)stream));
}

qnn_status qnn_lm_cache_append(const qnn_lm_tokens *s, const void *k, const void *v, const qnn_lm_cache *c,
                               const int32_t *lens, const int32_t *counts, void *stream)
{
    if (!s)
        return QNN_ERR_NULL;
    qnn_status e = check_cache(c);
    if (e != QNN_OK)
        return e;
    if (!type16(s->type) || (c->bits == 16 && c->type != s->type))
        return QNN_ERR_PARAM;
    if (s->t < 0 || !token_count(c, s->t))
        return QNN_ERR_SHAPE;
    if ((e = check_element_strides(s->k_stride, c->b, s->t, c->heads)) != QNN_OK ||
        (e = check_element_strides(s->v_stride, c->b, s->t, c->heads)) != QNN_OK)
        return e;
    if (c->b == 0 || s->t == 0)
        return QNN_OK;
    if (!k || !v || !lens)
        return QNN_ERR_NULL;
    if ((e = check_cache_pointers(c, true, true)) != QNN_OK)
        return e;
    if (!aligned16(k) || !aligned16(v) || !aligned16(lens) || !aligned16(counts))
        return QNN_ERR_ALIGN;
    if ((e = qnn_device_check()) != QNN_OK)
        return e;
    return launched(launch_append(cache_args(c), c->bits, c->dim, s->type, k, v, s->k_stride, s->v_stride, s->t, lens,
                                  counts, (hipStream_t)stream));
}

qnn_status qnn_lm_cache_keep(const qnn_lm_cache *c, int32_t t, const int32_t *lens, const int32_t *path,
                             const int32_t *kept, void *stream)
{
    qnn_status e = check_cache(c);
    if (e != QNN_OK)
        return e;
    if (t < 0 || !token_count(c, t))
        return QNN_ERR_SHAPE;
    if (c->b == 0 || t == 0)
        return QNN_OK;
    if (!lens || !path || !kept)
        return QNN_ERR_NULL;
    if ((e = check_cache_pointers(c, true, true)) != QNN_OK)
        return e;
    if (!aligned16(lens) || !aligned16(path) || !aligned16(kept))
        return QNN_ERR_ALIGN;
    if ((e = qnn_device_check()) != QNN_OK)
        return e;
    return launched(launch_keep(cache_args(c), c->bits, c->dim, t, lens, path, kept, (hipStream_t)stream));
}

qnn_status qnn_lm_cache_read(const qnn_lm_cache *c, int32_t type, int32_t t, const int32_t *start, void *k, void *v,
                             void *stream)
{
    qnn_status e = check_cache(c);
    if (e != QNN_OK)
        return e;
    if (type < QNN_LM_BF16 || type > QNN_LM_F32)
        return QNN_ERR_PARAM;
    if (t < 0 || !token_count(c, t))
        return QNN_ERR_SHAPE;
    if (c->b == 0 || t == 0)
        return QNN_OK;
    if ((!k && !v) || !start)
        return QNN_ERR_NULL;
    if ((e = check_cache_pointers(c, k != nullptr, v != nullptr)) != QNN_OK)
        return e;
    if (!aligned16(start) || !aligned16(k) || !aligned16(v))
        return QNN_ERR_ALIGN;
    if ((e = qnn_device_check()) != QNN_OK)
        return e;
    return launched(launch_read(cache_args(c), c->bits, c->dim, type, c->type, t, start, k, v, (hipStream_t)stream));
}

}  // extern "C"
