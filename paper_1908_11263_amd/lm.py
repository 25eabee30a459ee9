"""ctypes binding of include/qnn_lm.h: one step of a language model's block
over packed weights and a packed cache.

Argument marshalling only, as in qnn.py: every computation runs in the
library's HIP kernels, there is no fallback.  Tensors live on the current HIP
device; work is enqueued on torch's current stream or on `stream`, and what a
call allocates (its result, its workspace) belongs to that stream.  What the
library can check it refuses with QnnError; what only the binding can see (a
tensor's type, shape, strides, device) raises ValueError.

A cache is a `Cache`: k and v are [pages, heads, page, dim] tensors of 16-bit
numbers (bits = 16), or uint8 tensors whose last axis holds dim codes of 8 or 4
bits, with k_scale and v_scale [pages, heads, page] in 32 bits.  Any strides
will do whose last is 1 and whose others are multiples of 16 bytes: a view of
[pages, page, heads, dim] is as good.
"""
import collections
import ctypes
import math
import os
import struct

import torch

from . import qnn
from .qnn import QnnError

HEADER = os.path.join(os.path.dirname(qnn.HEADER), "qnn_lm.h")

BF16, F16, F32 = 0, 1, 2
_TYPES = {torch.bfloat16: BF16, torch.float16: F16, torch.float32: F32}
_ACTS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3, "gelu_tanh": 4}
_NORMS = {"rms": 0, "layer": 1}

# bits: 16, 8 or 4; the scales are None at 16 bits
Cache = collections.namedtuple("Cache", "k v k_scale v_scale bits")

# the C structures as packed bytes (what ctypes structures cost a call is what
# a small layer takes)
_pack_linear = struct.Struct("@8i3q").pack
_pack_norms = struct.Struct("@7i3f2q").pack
_pack_cache = struct.Struct("@6i6q5P2i").pack
_pack_queries = struct.Struct("@3if3q").pack
_pack_tokens = struct.Struct("@2i6q").pack

_f = {}


def _load():
    L = qnn.lib()
    P, I, S, Z = ctypes.c_void_p, ctypes.c_int32, ctypes.c_char_p, ctypes.c_size_t
    for name, restype, args in (
            ("qnn_lm_matmul", ctypes.c_int, [S, P, P, P, P, P, P, P, Z, P]),
            ("qnn_lm_matmul_workspace", Z, [S]),
            ("qnn_lm_norm_residual", ctypes.c_int, [S, P, P, P, P, P, P, P, P, P, P]),
            ("qnn_lm_tree_attention", ctypes.c_int, [S, P, S, P, P, P, P, P, P, Z, P]),
            ("qnn_lm_tree_attention_workspace", Z, [S, S]),
            ("qnn_lm_cache_append", ctypes.c_int, [S, P, P, S, P, P, P]),
            ("qnn_lm_cache_keep", ctypes.c_int, [S, I, P, P, P, P]),
            ("qnn_lm_cache_read", ctypes.c_int, [S, I, I, P, P, P, P])):
        f = L[name]
        f.restype, f.argtypes = restype, args
        _f[name] = f
    return _f


def _fn(name):
    return _f.get(name) or _load()[name]


def _check(status, name):
    if status != 0:
        raise QnnError(status, name)


def _bad(what):
    raise ValueError(what)


def _on_device(*tensors):
    """All given tensors live on the current device."""
    device = torch.cuda.current_device() if torch.cuda.is_initialized() or torch.cuda.is_available() else -1
    for t in tensors:
        if t is not None and t.get_device() != device:
            _bad("tensors must be on the current device (cuda:%d): got one on %s" % (device, t.device))


def _ptr(t):
    return None if t is None else t.data_ptr()


def _alloc(shape, dtype, like, stream):
    """Uninitialised memory of the stream that will use it."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=like.device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=like.device)


def _vector(t, n, what):
    """A contiguous float32 vector of n, or None."""
    if t is not None and (t.dtype is not torch.float32 or t.numel() != n or not t.is_contiguous()):
        _bad("%s must be contiguous float32 of %d elements" % (what, n))
    return t


def _ints(t, shape, what):
    if t is not None and (t.dtype is not torch.int32 or tuple(t.shape) != shape or not t.is_contiguous()):
        _bad("%s must be contiguous int32 of shape %s" % (what, shape))
    return t


def _rows(t, what):
    """(rows, channels, pitch) of a matrix, or of a stack of them that is one."""
    if t.dim() < 1 or (t.shape[-1] > 1 and t.stride(-1) != 1):
        _bad("%s must be contiguous along its last axis" % what)
    n = t.shape[-1]
    if t.dim() == 1:
        return 1, n, n
    if t.dim() == 2:
        return t.shape[0], n, t.stride(0) if t.shape[0] > 1 else n
    if not t.is_contiguous():
        _bad("%s: more than two axes must be contiguous" % what)
    return t.numel() // n if n else 0, n, n


def matmul(x, w, bits, scale=None, bias=None, act="none", gated=False, residual=None, out=None, stream=None):
    """Linear layer with its epilogue (qnn_lm_matmul):
    act(x w^T * scale + bias) + residual, or with gated=True
    act(gate) * up + residual, the first half of w's rows being the gate's.

    x: [..., k] bfloat16 or float16.  w: [rows, k * bits / 8] uint8 packed codes
    (bits 8, 4, 2, 1), or [rows, k] numbers of x's type (bits = 16).  scale:
    float32 [rows] or [rows, groups], k / groups being 32, 64 or 128.  bias:
    float32 [rows].  Returns [..., m] of x's type; out may be residual."""
    dtype = x.dtype
    kind = _TYPES.get(dtype, F32)
    if kind == F32:
        _bad("x must be bfloat16 or float16")
    r, k, pitch = _rows(x, "x")
    if r == 1 or pitch < k:
        pitch = k if k % 8 == 0 else k + -k % 8
    if w.dim() != 2 or not w.is_contiguous() or w.dtype is not (dtype if bits == 16 else torch.uint8):
        _bad("w must be a contiguous matrix of uint8 (or, at 16 bits, of x's type)")
    rows = w.shape[0]
    if w.shape[1] * (1 if bits == 16 else 8) != k * (1 if bits == 16 else bits):
        _bad("w has rows of %d for %d channels of %s bits" % (w.shape[1], k, bits))
    if gated and rows % 2:
        _bad("a gated layer has an even number of rows")
    m = rows // 2 if gated else rows
    group = 0
    if scale is not None:
        if scale.dtype is not torch.float32 or not scale.is_contiguous() or scale.shape[0] != rows or scale.dim() > 2:
            _bad("scale must be contiguous float32 [rows] or [rows, groups]")
        if scale.dim() == 2 and scale.shape[1] != 1:
            groups = scale.shape[1]
            if groups == 0 or k % groups:
                _bad("scale has %d groups for %d channels" % (groups, k))
            group = k // groups
    _vector(bias, rows, "bias")
    shape = x.shape[:-1] + (m,)
    rpitch = m
    if residual is not None:
        if residual.dtype is not dtype or residual.shape != shape:
            _bad("residual must be of x's type and the result's shape")
        rr, _, rpitch = _rows(residual, "residual")
    if out is None:
        out = _alloc(shape, dtype, x, stream)
        ypitch = m
    else:
        if out.dtype is not dtype or out.shape != shape:
            _bad("out must be of x's type and shape %s" % (tuple(shape),))
        _, _, ypitch = _rows(out, "out")
    _on_device(x, w, scale, bias, residual, out)
    s = _pack_linear(kind, bits, r, k, m, group, _ACTS[act], 1 if gated else 0, pitch, rpitch, ypitch)
    size = _fn("qnn_lm_matmul_workspace")(s)
    ws = _alloc((size,), torch.uint8, x, stream) if size else None
    _check(_f["qnn_lm_matmul"](s, x.data_ptr(), w.data_ptr(), _ptr(scale), _ptr(bias), _ptr(residual), out.data_ptr(),
                               _ptr(ws), size, qnn._stream_int(stream)), "qnn_lm_matmul")
    return out


def norm_residual(h, y=None, norm="rms", post=True, post_weight=None, post_bias=None, pre_weight=None, pre_bias=None,
                  gate=None, alpha=1.0, beta=1.0, eps=1e-6, dtype=None, h_out=None, out=None, stream=None):
    """Norm after a block, gate, residual scale and norm before the next block
    (qnn_lm_norm_residual): h' = alpha * h + beta * gate * N_post(y),
    x = N_pre(h').  Returns (h', x).

    h: [..., d], of y's type or float32; y: [..., d] bfloat16, float16 or
    float32, or None: x = N_pre(h) of type `dtype` (h's if not given), and h
    itself is returned beside it.  norm: "rms" or "layer"; post=False adds y
    without a norm.  Weights and biases: float32 [d] or None.  gate: [d] or
    [gates, d] of y's type, each row for as many consecutive rows of y.  h_out
    may be h, out may be y."""
    r, d, hpitch = _rows(h, "h")
    ytype = (dtype or h.dtype) if y is None else y.dtype
    kind, hkind = _TYPES.get(ytype), _TYPES.get(h.dtype)
    if kind is None or hkind is None:
        _bad("h and y must be bfloat16, float16 or float32")
    if r == 1:
        hpitch = d
    ypitch, gates = d, 0
    if y is not None:
        if y.shape != h.shape:
            _bad("h and y must have one shape")
        _, _, ypitch = _rows(y, "y")
        if r == 1:
            ypitch = d
        if gate is not None:
            if gate.dtype is not ytype or gate.shape[-1] != d or gate.dim() > 2 or not gate.is_contiguous():
                _bad("gate must be contiguous [d] or [gates, d] of y's type")
            gates = gate.numel() // d if d else 0
        if h_out is None:
            h_out = _alloc(h.shape, h.dtype, h, stream)
        elif h_out.shape != h.shape or h_out.dtype is not h.dtype or not h_out.is_contiguous():
            _bad("h_out must be contiguous and like h")
    if out is None:
        out = _alloc(h.shape, ytype, h, stream)
    elif out.shape != h.shape or out.dtype is not ytype or not out.is_contiguous():
        _bad("out must be contiguous, of h's shape and y's type")
    for v, what in ((post_weight, "post_weight"), (post_bias, "post_bias"), (pre_weight, "pre_weight"),
                    (pre_bias, "pre_bias")):
        if v is not None:
            _vector(v, d, what)
    _on_device(h, y, post_weight, post_bias, pre_weight, pre_bias, gate, h_out, out)
    s = _pack_norms(kind, hkind, r, d, _NORMS[norm], 1 if post else 0, gates, eps, alpha, beta, hpitch, ypitch)
    _check(_fn("qnn_lm_norm_residual")(s, h.data_ptr(), _ptr(y), _ptr(post_weight), _ptr(post_bias), _ptr(pre_weight),
                                       _ptr(pre_bias), _ptr(gate), _ptr(h_out) if y is not None else None,
                                       out.data_ptr(), qnn._stream_int(stream)), "qnn_lm_norm_residual")
    return (h if y is None else h_out), out


def make_cache(pages, heads, page, dim, bits, dtype=torch.bfloat16, device="cuda"):
    """An empty Cache of `bits` bits (16: numbers of `dtype`)."""
    if bits == 16:
        k, v = (torch.zeros((pages, heads, page, dim), dtype=dtype, device=device) for _ in range(2))
        return Cache(k, v, None, None, 16)
    k, v = (torch.zeros((pages, heads, page, dim * bits // 8), dtype=torch.uint8, device=device) for _ in range(2))
    ks, vs = (torch.zeros((pages, heads, page), dtype=torch.float32, device=device) for _ in range(2))
    return Cache(k, v, ks, vs, bits)


def _cache(cache, table, b):
    """(the C structure, heads, dim, number type or None at fewer bits)"""
    k, v, ks, vs, bits = cache
    if k.dim() != 4 or k.shape != v.shape or k.dtype is not v.dtype:
        _bad("k and v of a cache must be [pages, heads, page, dim], alike")
    pages, heads, page, width = k.shape
    if bits == 16:
        kind = _TYPES.get(k.dtype, F32)
        if kind == F32:
            _bad("a cache of 16 bits holds bfloat16 or float16")
        unit, dim = 2, width
    else:
        if k.dtype is not torch.uint8 or bits not in (8, 4):
            _bad("a cache holds uint8 codes of 8 or 4 bits, or numbers of 16 bits")
        kind, unit, dim = BF16, 1, width * 8 // bits
        for s in (ks, vs):
            if s is None or s.dtype is not torch.float32 or s.shape != k.shape[:3] or not s.is_contiguous():
                _bad("the scales of a cache must be contiguous float32 [pages, heads, page]")
    a, c = k.stride(), v.stride()
    if a[3] != 1 or c[3] != 1:
        _bad("the channels of a cache must be contiguous")
    if table.dtype is not torch.int32 or table.dim() != 2 or table.shape[0] != b or not table.is_contiguous():
        _bad("table must be contiguous int32 [%d, pages of a sequence]" % b)
    _on_device(k, v, ks, vs, table)
    return (_pack_cache(kind, bits, pages, heads, page, dim, a[0] * unit, a[1] * unit, a[2] * unit, c[0] * unit,
                        c[1] * unit, c[2] * unit, k.data_ptr(), v.data_ptr(), ks.data_ptr() if ks is not None else 0,
                        vs.data_ptr() if vs is not None else 0, table.data_ptr(), b, table.shape[1]),
            heads, dim, k.dtype if bits == 16 else None)


def tree_attention(q, cache, table, lens, mask=None, counts=None, scale=None, out=None, want_lse=False, stream=None):
    """Attention of drafted tokens over a paged cache (qnn_lm_tree_attention).

    q: [b, t, heads, dim] bfloat16 or float16, any strides that are multiples of
    8 elements.  table: int32 [b, pages of a sequence].  lens: int32 [b], tokens
    before the drafts; draft j lies at position lens + j.  counts: int32 [b] or
    None (t each).  mask: int64 [b, t, ceil(t / 64)], bit j % 64 of word j // 64
    set where a draft sees draft j; None: draft i sees drafts 0 .. i (a chunk of
    a prompt; t = 1: plain decoding).  scale: of the scores, 1 / sqrt(dim) if
    not given.  Returns [b, t, heads, dim], with want_lse also float32
    [b, t, heads]."""
    if q.dim() != 4 or q.stride(3) != 1:
        _bad("q must be [b, t, heads, dim], contiguous along dim")
    b, t, heads, dim = q.shape
    kind = _TYPES.get(q.dtype, F32)
    c, _, cdim, ctype = _cache(cache, table, b)
    if kind == F32 or (ctype is not None and ctype is not q.dtype):
        _bad("q must be bfloat16 or float16, and of the type of a cache of 16 bits")
    if cdim != dim:
        _bad("q has heads of %d channels, the cache of %d" % (dim, cdim))
    _ints(lens, (b,), "lens")
    _ints(counts, (b,), "counts")
    if mask is not None and (mask.dtype is not torch.int64 or tuple(mask.shape) != (b, t, (t + 63) // 64)
                             or not mask.is_contiguous()):
        _bad("mask must be contiguous int64 [b, t, ceil(t / 64)]")
    if out is None:
        out = _alloc((b, t, heads, dim), q.dtype, q, stream)
    elif out.shape != q.shape or out.dtype is not q.dtype or not out.is_contiguous():
        _bad("out must be contiguous and like q")
    lse = _alloc((b, t, heads), torch.float32, q, stream) if want_lse else None
    _on_device(q, lens, counts, mask, out)
    st = q.stride()
    s = _pack_queries(kind, t, heads, 1 / math.sqrt(dim) if scale is None else scale, st[0], st[1], st[2])
    size = _fn("qnn_lm_tree_attention_workspace")(s, c)
    ws = _alloc((size,), torch.uint8, q, stream) if size else None
    _check(_f["qnn_lm_tree_attention"](s, q.data_ptr(), c, lens.data_ptr(), _ptr(counts), _ptr(mask), out.data_ptr(),
                                       _ptr(lse), _ptr(ws), size, qnn._stream_int(stream)), "qnn_lm_tree_attention")
    return (out, lse) if want_lse else out


def cache_append(k, v, cache, table, lens, counts=None, stream=None):
    """Writes new tokens into the cache (qnn_lm_cache_append): k and v
    [b, t, heads, dim] bfloat16 or float16, token j of a sequence to position
    lens + j where j < counts (None: t)."""
    if k.dim() != 4 or k.shape != v.shape or k.dtype is not v.dtype or k.stride(3) != 1 or v.stride(3) != 1:
        _bad("k and v must be [b, t, heads, dim], alike, contiguous along dim")
    b, t, heads, dim = k.shape
    kind = _TYPES.get(k.dtype, F32)
    c, cheads, cdim, ctype = _cache(cache, table, b)
    if kind == F32 or (ctype is not None and ctype is not k.dtype):
        _bad("k and v must be bfloat16 or float16, and of the type of a cache of 16 bits")
    if (heads, dim) != (cheads, cdim):
        _bad("k and v have %d heads of %d channels, the cache %d of %d" % (heads, dim, cheads, cdim))
    _ints(lens, (b,), "lens")
    _ints(counts, (b,), "counts")
    _on_device(k, v, lens, counts)
    a, d = k.stride(), v.stride()
    s = _pack_tokens(kind, t, a[0], a[1], a[2], d[0], d[1], d[2])
    _check(_fn("qnn_lm_cache_append")(s, k.data_ptr(), v.data_ptr(), c, lens.data_ptr(), _ptr(counts),
                                      qnn._stream_int(stream)), "qnn_lm_cache_append")


def cache_keep(cache, table, lens, path, kept, stream=None):
    """Moves the accepted drafts to the front (qnn_lm_cache_keep): position
    lens + j takes position lens + path[:, j] for j < kept.  path: int32 [b, t],
    strictly ascending; kept: int32 [b]."""
    if path.dim() != 2:
        _bad("path must be [b, t]")
    b, t = path.shape
    c = _cache(cache, table, b)[0]
    _ints(path, (b, t), "path")
    _ints(lens, (b,), "lens")
    _ints(kept, (b,), "kept")
    _on_device(lens, path, kept)
    _check(_fn("qnn_lm_cache_keep")(c, t, lens.data_ptr(), path.data_ptr(), kept.data_ptr(), qnn._stream_int(stream)),
           "qnn_lm_cache_keep")


def cache_read(cache, table, start, n, dtype=torch.bfloat16, stream=None):
    """The values at positions start .. start + n - 1 of each sequence
    (qnn_lm_cache_read): (k, v), each [b, n, heads, dim] of `dtype`; zeros where
    the table does not reach."""
    kind = _TYPES.get(dtype)
    if kind is None:
        _bad("dtype must be bfloat16, float16 or float32")
    b = start.shape[0]
    c, heads, dim, _ = _cache(cache, table, b)
    _ints(start, (b,), "start")
    _on_device(start)
    k = _alloc((b, n, heads, dim), dtype, start, stream)
    v = _alloc((b, n, heads, dim), dtype, start, stream)
    _check(_fn("qnn_lm_cache_read")(c, kind, n, start.data_ptr(), k.data_ptr(), v.data_ptr(), qnn._stream_int(stream)),
           "qnn_lm_cache_read")
    return k, v
