// The host's path of lm.py's calls: torch tensors to the C structures of
// include/qnn_lm.h and back.
//
// Argument marshalling only, like the rest of the binding, but compiled: a call
// of a small layer takes a few microseconds on the device, and looking at ten
// tensors from Python takes longer.  What only a binding can see (a tensor's
// type, shape, strides, device) is checked here and raises ValueError; what the
// library refuses raises QnnError.  The library's entry points are handed in by
// lm.py (init), so that there is one loaded library in a process.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/core/grad_mode.h>
#include <ATen/ops/clone.h>
#include <ATen/ops/empty.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <stdexcept>
#include <string>
#include <vector>

#include "qnn_lm.h"

namespace {

struct Entry {
    decltype(&qnn_lm_matmul) matmul;
    decltype(&qnn_lm_matmul_workspace) matmul_workspace;
    decltype(&qnn_lm_norm_residual) norm_residual;
    decltype(&qnn_lm_tree_attention) tree_attention;
    decltype(&qnn_lm_tree_attention_workspace) tree_attention_workspace;
    decltype(&qnn_lm_cache_append) cache_append;
    decltype(&qnn_lm_cache_keep) cache_keep;
    decltype(&qnn_lm_cache_read) cache_read;
} g_lib;
PyObject *g_error = nullptr;  // qnn.QnnError(status, where)
bool g_gpu = false;           // a device is there

using at::Tensor;

struct Refused {
    qnn_status status;
    const char *where;
};

[[noreturn]] void bad(const std::string &what) { throw std::invalid_argument(what); }

const Tensor &tensor(PyObject *o, const char *what)
{
    if (!THPVariable_Check(o))
        bad(std::string(what) + " must be a tensor");
    const Tensor &t = THPVariable_Unpack(o);
    // (a result without a gradient would look like one that has none)
    if (t.requires_grad() && at::GradMode::is_enabled())
        bad(std::string(what) + " requires a gradient, which these operators do not have: call them under torch.no_grad()");
    return t;
}

const Tensor *maybe(PyObject *o, const char *what) { return o == Py_None ? nullptr : &tensor(o, what); }

int type_of(at::ScalarType t)
{
    return t == at::kBFloat16 ? QNN_LM_BF16 : t == at::kHalf ? QNN_LM_F16 : t == at::kFloat ? QNN_LM_F32 : -1;
}

int type16_of(at::ScalarType t)
{
    const int k = type_of(t);
    return k == QNN_LM_F32 ? -1 : k;
}

// All tensors of a call live on the device of its first one, which is the
// current one (or, with no device at all, on the host: the library refuses).
struct Place {
    at::Device device;
    std::vector<Tensor> copies;
    explicit Place(const Tensor &t) : device(t.device()) {}
    void same(const Tensor &t) const
    {
        if (t.device() != device)
            bad("all tensors must be on one device: got one on " + t.device().str());
    }
    void *stream() const
    {
        if (!device.is_cuda()) {
            if (g_gpu)
                bad("tensors must be on the current device: got some on " + device.str());
            return nullptr;
        }
        const auto now = c10::hip::current_device();
        if (device.index() != now)
            bad("tensors must be on the current device (cuda:" + std::to_string((int)now) + "): got some on " + device.str());
        return (void *)c10::hip::getCurrentHIPStream(now).stream();
    }
    const float *vector(const Tensor *t, int64_t n, const char *what) const
    {
        if (!t)
            return nullptr;
        if (t->scalar_type() != at::kFloat || t->numel() != n || !t->is_contiguous())
            bad(std::string(what) + " must be contiguous float32 of " + std::to_string(n) + " elements");
        same(*t);
        return (const float *)t->data_ptr();
    }
    // Lengths, page numbers, paths and masks may be slices of larger tensors (a
    // part of a batch): what the library's alignment refuses is copied.
    const void *whole(const Tensor &t)
    {
        if (((uintptr_t)t.data_ptr() & 15u) == 0)
            return t.data_ptr();
        copies.push_back(t.clone());
        return copies.back().data_ptr();
    }
    const int32_t *ints(const Tensor *t, int64_t n, const char *what)
    {
        if (!t)
            return nullptr;
        if (t->scalar_type() != at::kInt || t->dim() != 1 || t->numel() != n || !t->is_contiguous())
            bad(std::string(what) + " must be contiguous int32 of " + std::to_string(n));
        same(*t);
        return (const int32_t *)whole(*t);
    }
};

int32_t int32_of(int64_t v, const char *what)
{
    if (v != (int32_t)v)
        bad(std::string(what) + " is too large");
    return (int32_t)v;
}

// Elements from one row of n to the next of a matrix, or of a stack of them that is one.
int64_t pitch_of(const Tensor &t, int64_t n, const char *what)
{
    if (t.is_contiguous())
        return n;
    if (t.dim() != 2 || (t.stride(1) != 1 && n > 1))
        bad(std::string(what) + " must be contiguous along its last axis, and altogether with more than two axes");
    return t.size(0) > 1 ? t.stride(0) : n;
}

int64_t rows_of(const Tensor &t)
{
    int64_t r = 1;
    for (int64_t i = 0; i + 1 < t.dim(); ++i)
        r *= t.size(i);
    return r;
}

bool like(const Tensor &t, at::IntArrayRef shape, at::ScalarType type) { return t.scalar_type() == type && t.sizes() == shape; }

Tensor make(at::IntArrayRef shape, const Tensor &on, at::ScalarType type)
{
    return at::empty(shape, on.options().dtype(type).requires_grad(false));
}

void *data(const Tensor &t) { return t.data_ptr(); }

long number(PyObject *o)
{
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        bad("a whole number was expected");
    }
    return v;
}

float real(PyObject *o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) {
        PyErr_Clear();
        bad("a number was expected");
    }
    return (float)v;
}

bool truth(PyObject *o)
{
    const int v = PyObject_IsTrue(o);
    if (v < 0) {
        PyErr_Clear();
        bad("True or False was expected");
    }
    return v != 0;
}

template <class F>
PyObject *guarded(F f)
{
    try {
        return f();
    } catch (const Refused &r) {
        PyObject *e = PyObject_CallFunction(g_error, "is", (int)r.status, r.where);
        if (e) {
            PyErr_SetObject(g_error, e);
            Py_DECREF(e);
        }
    } catch (const std::invalid_argument &e) {
        PyErr_SetString(PyExc_ValueError, e.what());
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

void check(qnn_status s, const char *where)
{
    if (s != QNN_OK)
        throw Refused{s, where};
}

void arguments(Py_ssize_t n, Py_ssize_t want)
{
    if (n != want)
        bad("wrong number of arguments");
}

// x, w, bits, scale, bias, act, gated, residual, out
PyObject *matmul(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&] {
        arguments(n, 9);
        const Tensor &x = tensor(a[0], "x"), &w = tensor(a[1], "w");
        const long bits = number(a[2]);
        const Tensor *scale = maybe(a[3], "scale"), *bias = maybe(a[4], "bias"), *residual = maybe(a[7], "residual");
        const at::ScalarType type = x.scalar_type();
        qnn_lm_linear s;
        s.type = type16_of(type);
        if (s.type < 0 || x.dim() < 1)
            bad("x must be [..., k] bfloat16 or float16");
        const int64_t k = x.size(-1);
        s.bits = (int32_t)bits;
        s.k = int32_of(k, "k");
        s.r = int32_of(rows_of(x), "the number of rows");
        s.x_pitch = pitch_of(x, k, "x");
        const Place at(x);
        if (w.scalar_type() != (bits == 16 ? type : at::kByte))
            bad("w must be uint8 packed codes, or at 16 bits of x's type");
        if (w.dim() != 2 || !w.is_contiguous() || w.size(1) * (bits == 16 ? 16 : 8) != k * bits)
            bad("w must be contiguous rows of " + std::to_string(k) + " channels of " + std::to_string(bits) + " bits");
        at.same(w);
        const int64_t rows = w.size(0);
        s.gated = truth(a[6]) ? 1 : 0;
        if (s.gated && rows % 2)
            bad("a gated layer has an even number of rows");
        const int64_t m = s.gated ? rows / 2 : rows;
        s.m = int32_of(m, "the number of outputs");
        s.act = (int32_t)number(a[5]);
        s.group = 0;
        if (scale) {
            if (scale->scalar_type() != at::kFloat || scale->dim() < 1 || scale->dim() > 2 || scale->size(0) != rows ||
                !scale->is_contiguous())
                bad("scale must be contiguous float32 [rows] or [rows, groups]");
            if (scale->dim() == 2 && scale->size(1) != 1) {
                if (scale->size(1) == 0 || k % scale->size(1))
                    bad("scale has " + std::to_string(scale->size(1)) + " groups for " + std::to_string(k) + " channels");
                s.group = (int32_t)(k / scale->size(1));
            }
            at.same(*scale);
        }
        const float *bp = at.vector(bias, rows, "bias");
        at::DimVector shape(x.sizes());
        shape.back() = m;
        s.residual_pitch = s.y_pitch = m;
        if (residual) {
            if (!like(*residual, shape, type))
                bad("residual must be of x's type and the result's shape");
            at.same(*residual);
            s.residual_pitch = pitch_of(*residual, m, "residual");
        }
        void *stream = at.stream();
        const Tensor *given = maybe(a[8], "out");
        Tensor made;
        if (given) {
            if (!like(*given, shape, type))
                bad("out must be of x's type and the result's shape");
            at.same(*given);
            s.y_pitch = pitch_of(*given, m, "out");
        } else {
            made = make(shape, x, type);
        }
        const Tensor &out = given ? *given : made;
        const size_t size = g_lib.matmul_workspace(&s);
        Tensor ws;
        if (size)
            ws = make({(int64_t)size}, x, at::kByte);
        check(g_lib.matmul(&s, data(x), data(w), scale ? (const float *)data(*scale) : nullptr, bp,
                           residual ? data(*residual) : nullptr, data(out), size ? data(ws) : nullptr, size, stream),
              "qnn_lm_matmul");
        if (given) {
            Py_INCREF(a[8]);
            return a[8];
        }
        return THPVariable_Wrap(made);
    });
}

PyObject *pair(PyObject *a, PyObject *b)  // takes both references
{
    PyObject *t = a && b ? PyTuple_New(2) : nullptr;
    if (!t) {
        Py_XDECREF(a);
        Py_XDECREF(b);
        return nullptr;
    }
    PyTuple_SET_ITEM(t, 0, a);
    PyTuple_SET_ITEM(t, 1, b);
    return t;
}

PyObject *own(PyObject *o)
{
    Py_INCREF(o);
    return o;
}

// h, y, norm, post, post_weight, post_bias, pre_weight, pre_bias, gate, alpha, beta, eps, like, h_out, out
PyObject *norm_residual(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&] {
        arguments(n, 15);
        const Tensor &h = tensor(a[0], "h");
        const Tensor *y = maybe(a[1], "y"), *gate = maybe(a[8], "gate"), *as = maybe(a[12], "like");
        const at::ScalarType htype = h.scalar_type(), type = y ? y->scalar_type() : as ? as->scalar_type() : htype;
        qnn_lm_norms s;
        s.type = type_of(type);
        s.h_type = type_of(htype);
        if (s.type < 0 || s.h_type < 0 || h.dim() < 1)
            bad("h and y must be [..., d] bfloat16, float16 or float32");
        const int64_t d = h.size(-1);
        s.d = int32_of(d, "the number of channels");
        s.r = int32_of(rows_of(h), "the number of rows");
        s.norm = (int32_t)number(a[2]);
        s.post = truth(a[3]) ? 1 : 0;
        s.gates = 0;
        s.alpha = real(a[9]);
        s.beta = real(a[10]);
        s.eps = real(a[11]);
        s.h_pitch = pitch_of(h, d, "h");
        s.y_pitch = d;
        const Place at(h);
        void *stream = at.stream();
        const Tensor *hg = maybe(a[13], "h_out"), *og = maybe(a[14], "out");
        Tensor hm, om;
        if (y) {
            if (y->sizes() != h.sizes())
                bad("h and y must have one shape");
            at.same(*y);
            s.y_pitch = pitch_of(*y, d, "y");
            if (gate) {
                if (gate->scalar_type() != type || gate->dim() < 1 || gate->dim() > 2 || gate->size(-1) != d ||
                    !gate->is_contiguous())
                    bad("gate must be contiguous [d] or [gates, d] of y's type");
                at.same(*gate);
                s.gates = d ? int32_of(gate->numel() / d, "the number of gates") : 0;
            }
            if (hg) {
                if (!like(*hg, h.sizes(), htype) || !hg->is_contiguous())
                    bad("h_out must be contiguous and like h");
                at.same(*hg);
            } else {
                hm = make(h.sizes(), h, htype);
            }
        }
        if (og) {
            if (!like(*og, h.sizes(), type) || !og->is_contiguous())
                bad("out must be contiguous, of h's shape and y's type");
            at.same(*og);
        } else {
            om = make(h.sizes(), h, type);
        }
        const float *v[4];
        static const char *const names[4] = {"post_weight", "post_bias", "pre_weight", "pre_bias"};
        for (int i = 0; i < 4; ++i)
            v[i] = at.vector(maybe(a[4 + i], names[i]), d, names[i]);
        check(g_lib.norm_residual(&s, data(h), y ? data(*y) : nullptr, v[0], v[1], v[2], v[3],
                                  s.gates ? data(*gate) : nullptr, y ? data(hg ? *hg : hm) : nullptr, data(og ? *og : om),
                                  stream),
              "qnn_lm_norm_residual");
        return pair(!y ? own(a[0]) : hg ? own(a[13]) : THPVariable_Wrap(hm), og ? own(a[14]) : THPVariable_Wrap(om));
    });
}

// A lm.Cache (k, v, k_scale, v_scale, bits) and its table.
struct Cache {
    qnn_lm_cache c;
    at::ScalarType type;  // of the numbers at 16 bits

    Cache(PyObject *o, PyObject *t, int64_t b, Place &at)
    {
        if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 5)
            bad("a cache is a lm.Cache");
        const Tensor &k = tensor(PyTuple_GET_ITEM(o, 0), "a cache's k"), &v = tensor(PyTuple_GET_ITEM(o, 1), "a cache's v");
        const Tensor *scale[2] = {maybe(PyTuple_GET_ITEM(o, 2), "k_scale"), maybe(PyTuple_GET_ITEM(o, 3), "v_scale")};
        const long bits = number(PyTuple_GET_ITEM(o, 4));
        if (k.dim() != 4 || v.sizes() != k.sizes() || v.scalar_type() != k.scalar_type())
            bad("k and v of a cache must be [pages, heads, page, dim], alike");
        if (k.stride(3) != 1 || v.stride(3) != 1)
            bad("the channels of a cache must be contiguous");
        type = k.scalar_type();
        int64_t unit = 1, dim = k.size(3);
        c.type = QNN_LM_BF16;
        c.k_scale = c.v_scale = nullptr;
        if (bits == 16) {
            c.type = type16_of(type);
            unit = 2;
            if (c.type < 0 || scale[0] || scale[1])
                bad("a cache of 16 bits holds bfloat16 or float16 and no scales");
        } else {
            if (type != at::kByte || (bits != 8 && bits != 4))
                bad("a cache holds uint8 codes of 8 or 4 bits, or numbers of 16 bits");
            if (bits == 4)
                dim *= 2;
            for (const Tensor *s : scale) {
                if (!s || s->scalar_type() != at::kFloat || s->sizes() != k.sizes().slice(0, 3) || !s->is_contiguous())
                    bad("the scales of a cache must be contiguous float32 [pages, heads, page]");
                at.same(*s);
            }
            c.k_scale = (float *)data(*scale[0]);
            c.v_scale = (float *)data(*scale[1]);
        }
        const Tensor &table = tensor(t, "table");
        if (table.scalar_type() != at::kInt || table.dim() != 2 || table.size(0) != b || !table.is_contiguous())
            bad("table must be contiguous int32 [" + std::to_string(b) + ", pages of a sequence]");
        at.same(k);
        at.same(v);
        at.same(table);
        c.bits = (int32_t)bits;
        c.pages = int32_of(k.size(0), "the number of pages");
        c.heads = int32_of(k.size(1), "the number of heads");
        c.page = int32_of(k.size(2), "a page");
        c.dim = int32_of(dim, "a head");
        c.k_page = k.stride(0) * unit;
        c.k_head = k.stride(1) * unit;
        c.k_slot = k.stride(2) * unit;
        c.v_page = v.stride(0) * unit;
        c.v_head = v.stride(1) * unit;
        c.v_slot = v.stride(2) * unit;
        c.k = data(k);
        c.v = data(v);
        c.table = (const int32_t *)at.whole(table);
        c.b = int32_of(b, "the number of sequences");
        c.width = int32_of(table.size(1), "the table");
    }
    bool holds(at::ScalarType t) const { return c.bits != 16 || t == type; }
};

// q, cache, table, lens, mask, counts, scale, out, want_lse
PyObject *tree_attention(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&] {
        arguments(n, 9);
        const Tensor &q = tensor(a[0], "q");
        if (q.dim() != 4 || q.stride(3) != 1)
            bad("q must be [b, t, heads, dim], contiguous along dim");
        const int64_t b = q.size(0), t = q.size(1), dim = q.size(3);
        Place at(q);
        const Cache cache(a[1], a[2], b, at);
        qnn_lm_queries s;
        s.type = type16_of(q.scalar_type());
        if (s.type < 0 || !cache.holds(q.scalar_type()))
            bad("q must be bfloat16 or float16, and of the type of a cache of 16 bits");
        if (cache.c.dim != dim)
            bad("q has heads of " + std::to_string(dim) + " channels, the cache of " + std::to_string(cache.c.dim));
        s.t = int32_of(t, "the number of drafts");
        s.heads = int32_of(q.size(2), "the number of heads");
        s.scale = real(a[6]);
        for (int i = 0; i < 3; ++i)
            s.q_stride[i] = q.stride(i);
        const int32_t *lens = at.ints(&tensor(a[3], "lens"), b, "lens");
        const int32_t *counts = at.ints(maybe(a[5], "counts"), b, "counts");
        const Tensor *mask = maybe(a[4], "mask"), *given = maybe(a[7], "out");
        if (mask) {
            if (mask->scalar_type() != at::kLong || mask->dim() != 3 || mask->size(0) != b || mask->size(1) != t ||
                mask->size(2) != (t + 63) / 64 || !mask->is_contiguous())
                bad("mask must be contiguous int64 [b, t, ceil(t / 64)]");
            at.same(*mask);
        }
        void *stream = at.stream();
        Tensor made, lse, ws;
        if (given) {
            if (!like(*given, q.sizes(), q.scalar_type()) || !given->is_contiguous())
                bad("out must be contiguous and like q");
            at.same(*given);
        } else {
            made = make(q.sizes(), q, q.scalar_type());
        }
        const bool want = truth(a[8]);
        if (want)
            lse = make(q.sizes().slice(0, 3), q, at::kFloat);
        const size_t size = g_lib.tree_attention_workspace(&s, &cache.c);
        if (size)
            ws = make({(int64_t)size}, q, at::kByte);
        check(g_lib.tree_attention(&s, data(q), &cache.c, lens, counts,
                                   mask ? (const uint64_t *)at.whole(*mask) : nullptr, data(given ? *given : made),
                                   want ? (float *)data(lse) : nullptr, size ? data(ws) : nullptr, size, stream),
              "qnn_lm_tree_attention");
        PyObject *out = given ? own(a[7]) : THPVariable_Wrap(made);
        return want ? pair(out, THPVariable_Wrap(lse)) : out;
    });
}

// k, v, cache, table, lens, counts
PyObject *cache_append(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&] {
        arguments(n, 6);
        const Tensor &k = tensor(a[0], "k"), &v = tensor(a[1], "v");
        if (k.dim() != 4 || v.sizes() != k.sizes() || v.scalar_type() != k.scalar_type())
            bad("k and v must be [b, t, heads, dim], alike");
        if (k.stride(3) != 1 || v.stride(3) != 1)
            bad("k and v must be contiguous along dim");
        const int64_t b = k.size(0);
        Place at(k);
        const Cache cache(a[2], a[3], b, at);
        qnn_lm_tokens s;
        s.type = type16_of(k.scalar_type());
        if (s.type < 0 || !cache.holds(k.scalar_type()))
            bad("k and v must be bfloat16 or float16, and of the type of a cache of 16 bits");
        if (k.size(2) != cache.c.heads || k.size(3) != cache.c.dim)
            bad("k and v have other heads than the cache");
        at.same(v);
        s.t = int32_of(k.size(1), "the number of tokens");
        for (int i = 0; i < 3; ++i) {
            s.k_stride[i] = k.stride(i);
            s.v_stride[i] = v.stride(i);
        }
        const int32_t *lens = at.ints(&tensor(a[4], "lens"), b, "lens");
        const int32_t *counts = at.ints(maybe(a[5], "counts"), b, "counts");
        check(g_lib.cache_append(&s, data(k), data(v), &cache.c, lens, counts, at.stream()), "qnn_lm_cache_append");
        return own(Py_None);
    });
}

// cache, table, lens, path, kept
PyObject *cache_keep(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&] {
        arguments(n, 5);
        const Tensor &path = tensor(a[3], "path");
        if (path.scalar_type() != at::kInt || path.dim() != 2 || !path.is_contiguous())
            bad("path must be contiguous int32 [b, t]");
        const int64_t b = path.size(0);
        Place at(path);
        const Cache cache(a[0], a[1], b, at);
        const int32_t *lens = at.ints(&tensor(a[2], "lens"), b, "lens"), *kept = at.ints(&tensor(a[4], "kept"), b, "kept");
        check(g_lib.cache_keep(&cache.c, int32_of(path.size(1), "the number of drafts"), lens,
                               (const int32_t *)at.whole(path), kept, at.stream()),
              "qnn_lm_cache_keep");
        return own(Py_None);
    });
}

// cache, table, start, n, type (an empty tensor's)
PyObject *cache_read(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&] {
        arguments(n, 5);
        const Tensor &start = tensor(a[2], "start");
        const int64_t b = start.numel(), t = number(a[3]);
        static const at::ScalarType types[3] = {at::kBFloat16, at::kHalf, at::kFloat};
        const long type = number(a[4]);
        if (type < 0 || type > 2 || t < 0)
            bad("n must not be negative, dtype bfloat16, float16 or float32");
        Place at(start);
        const Cache cache(a[0], a[1], b, at);
        const int32_t *from = at.ints(&start, b, "start");
        void *stream = at.stream();
        const Tensor k = make({b, t, cache.c.heads, cache.c.dim}, start, types[type]);
        const Tensor v = make({b, t, cache.c.heads, cache.c.dim}, start, types[type]);
        check(g_lib.cache_read(&cache.c, (int32_t)type, int32_of(t, "n"), from, data(k), data(v), stream),
              "qnn_lm_cache_read");
        return pair(THPVariable_Wrap(k), THPVariable_Wrap(v));
    });
}

// QnnError, whether a device is there, then the addresses of the entry points in Entry's order
PyObject *init(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&] {
        arguments(n, 10);
        Py_XDECREF(g_error);
        g_error = own(a[0]);
        g_gpu = truth(a[1]);
        void *p[8];
        for (int i = 0; i < 8; ++i)
            p[i] = PyLong_AsVoidPtr(a[2 + i]);
        static_assert(sizeof(Entry) == sizeof(p), "one address each");
        memcpy(&g_lib, p, sizeof(p));
        return own(Py_None);
    });
}

#define FAST(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(init),         FAST(matmul),     FAST(norm_residual), FAST(tree_attention),
                         FAST(cache_append), FAST(cache_keep), FAST(cache_read),    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_lm_bind", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__lm_bind(void) { return PyModule_Create(&module); }
