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
import os
import struct

import torch

from . import qnn
from .qnn import QnnError

HEADER = os.path.join(os.path.dirname(qnn.HEADER), "qnn_lm.h")

BF16, F16, F32 = 0, 1, 2
_TYPES = {torch.bfloat16: BF16, torch.float16: F16, torch.float32: F32}
_TYPES16 = {torch.bfloat16: BF16, torch.float16: F16}
_U8, _I32, _F32 = torch.uint8, torch.int32, torch.float32
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


def _bad(what):
    raise ValueError(what)


# A call of a small layer takes a few microseconds on the device: what follows
# is written for the host's time (no helper call per tensor where one line
# does, one read of an attribute that costs 0.1 us).
_current = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda d: torch.cuda.current_stream(d).cuda_stream)


def _stream(d, stream):
    """The stream's handle; d: the device of the call's tensors, which must be the current one."""
    if d < 0:
        if torch.cuda.is_available():
            _bad("tensors must be on the current device")
        return None  # (no device at all: the library says so)
    if d != _current():
        _bad("tensors must be on the current device (cuda:%d): got some on cuda:%d" % (_current(), d))
    return _raw_stream(d) if stream is None else stream.cuda_stream


def _elsewhere(t):
    _bad("all tensors must be on one device: got one on %s" % t.device)


def _alloc(shape, dtype, like, stream):
    """Uninitialised memory of the stream that will use it."""
    if stream is None:
        return like.new_empty(shape, dtype=dtype)
    with torch.cuda.stream(stream):
        return like.new_empty(shape, dtype=dtype)


def _alloc_like(t, stream):
    """The same for a tensor like the contiguous t."""
    if stream is None:
        return torch.empty_like(t)
    with torch.cuda.stream(stream):
        return torch.empty_like(t)


def _vector(t, n, d, what):
    """The address of a contiguous float32 vector of n."""
    if t.dtype is not _F32 or t.numel() != n or not t.is_contiguous():
        _bad("%s must be contiguous float32 of %d elements" % (what, n))
    if t.get_device() != d:
        _elsewhere(t)
    return t.data_ptr()


def _ints(t, n, d, what):
    """The address of a contiguous int32 vector of n."""
    if t.dtype is not _I32 or t.dim() != 1 or t.numel() != n or not t.is_contiguous():
        _bad("%s must be contiguous int32 of %d" % (what, n))
    if t.get_device() != d:
        _elsewhere(t)
    return t.data_ptr()


def _pitch(t, n, what):
    """Elements from one row of n to the next of a matrix, or of a stack of them that is one."""
    if t.is_contiguous():
        return n
    st = t.stride()
    if len(st) != 2 or (st[1] != 1 and n > 1):
        _bad("%s must be contiguous along its last axis, and altogether with more than two axes" % what)
    return st[0] if t.shape[0] > 1 else n


def matmul(x, w, bits, scale=None, bias=None, act="none", gated=False, residual=None, out=None, stream=None):
    """Linear layer with its epilogue (qnn_lm_matmul):
    act(x w^T * scale + bias) + residual, or with gated=True
    act(gate) * up + residual, the first half of w's rows being the gate's.

    x: [..., k] bfloat16 or float16.  w: [rows, k * bits / 8] uint8 packed codes
    (bits 8, 4, 2, 1), or [rows, k] numbers of x's type (bits = 16).  scale:
    float32 [rows] or [rows, groups], k / groups being 32, 64 or 128.  bias:
    float32 [rows].  Returns [..., m] of x's type; out may be residual."""
    dtype = x.dtype
    kind = _TYPES16.get(dtype)
    if kind is None or not x.dim():
        _bad("x must be [..., k] bfloat16 or float16")
    shape = x.shape
    k = shape[-1]
    lead = shape[:-1]
    r = lead.numel()
    pitch = k if x.is_contiguous() else _pitch(x, k, "x")
    d = x.get_device()
    if bits == 16:
        if w.dtype is not dtype:
            _bad("w must be of x's type at 16 bits")
    elif w.dtype is not _U8:
        _bad("w must be uint8 packed codes")
    wshape = w.shape
    if len(wshape) != 2 or not w.is_contiguous() or wshape[1] * (16 if bits == 16 else 8) != k * bits:
        _bad("w must be contiguous rows of %d channels of %s bits: got %s" % (k, bits, tuple(wshape)))
    if w.get_device() != d:
        _elsewhere(w)
    rows = wshape[0]
    m = rows
    if gated:
        if rows % 2:
            _bad("a gated layer has an even number of rows")
        m = rows // 2
    group = 0
    sp = bp = rp = None
    if scale is not None:
        st = scale.shape
        if scale.dtype is not _F32 or not 1 <= len(st) <= 2 or st[0] != rows or not scale.is_contiguous():
            _bad("scale must be contiguous float32 [rows] or [rows, groups]")
        if len(st) == 2 and st[1] != 1:
            if st[1] == 0 or k % st[1]:
                _bad("scale has %d groups for %d channels" % (st[1], k))
            group = k // st[1]
        if scale.get_device() != d:
            _elsewhere(scale)
        sp = scale.data_ptr()
    if bias is not None:
        bp = _vector(bias, rows, d, "bias")
    shape = lead + (m,)
    rpitch = ypitch = m
    if residual is not None:
        if residual.dtype is not dtype or residual.shape != shape:
            _bad("residual must be of x's type and the result's shape")
        if residual.get_device() != d:
            _elsewhere(residual)
        rpitch = _pitch(residual, m, "residual")
        rp = residual.data_ptr()
    handle = _stream(d, stream)
    if out is None:
        if stream is not None:
            out = _alloc(shape, dtype, x, stream)
        else:
            out = x.new_empty(shape)
    else:
        if out.dtype is not dtype or out.shape != shape:
            _bad("out must be of x's type and shape %s" % (tuple(shape),))
        if out.get_device() != d:
            _elsewhere(out)
        ypitch = _pitch(out, m, "out")
    s = _pack_linear(kind, bits, r, k, m, group, _ACTS[act], 1 if gated else 0, pitch, rpitch, ypitch)
    f = _f or _load()
    size = f["qnn_lm_matmul_workspace"](s)
    ws = _alloc((size,), _U8, x, stream) if size else None
    status = f["qnn_lm_matmul"](s, x.data_ptr(), w.data_ptr(), sp, bp, rp, out.data_ptr(),
                                None if ws is None else ws.data_ptr(), size, handle)
    if status:
        raise QnnError(status, "qnn_lm_matmul")
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
    hdtype = h.dtype
    ytype = (dtype or hdtype) if y is None else y.dtype
    kind, hkind = _TYPES.get(ytype), _TYPES.get(hdtype)
    if kind is None or hkind is None or not h.dim():
        _bad("h and y must be [..., d] bfloat16, float16 or float32")
    shape = h.shape
    d = shape[-1]
    r = shape[:-1].numel()
    hpitch = d if h.is_contiguous() else _pitch(h, d, "h")
    dev = h.get_device()
    handle = _stream(dev, stream)
    ypitch, gates = d, 0
    yp = gp = hop = a = b = c = e = None
    if y is not None:
        if y.shape != shape:
            _bad("h and y must have one shape")
        if y.get_device() != dev:
            _elsewhere(y)
        ypitch = d if y.is_contiguous() else _pitch(y, d, "y")
        yp = y.data_ptr()
        if gate is not None:
            if gate.dtype is not ytype or gate.dim() > 2 or gate.shape[-1:] != shape[-1:] or not gate.is_contiguous():
                _bad("gate must be contiguous [d] or [gates, d] of y's type")
            if gate.get_device() != dev:
                _elsewhere(gate)
            gates = gate.numel() // d if d else 0
            gp = gate.data_ptr()
        if h_out is None:
            h_out = _alloc_like(h, stream) if hpitch == d else _alloc(shape, hdtype, h, stream)
        elif h_out.shape != shape or h_out.dtype is not hdtype or not h_out.is_contiguous():
            _bad("h_out must be contiguous and like h")
        elif h_out.get_device() != dev:
            _elsewhere(h_out)
        hop = h_out.data_ptr()
    else:
        h_out = h
    if out is None:
        out = _alloc_like(y, stream) if yp and ypitch == d else _alloc(shape, ytype, h, stream)
    elif out.shape != shape or out.dtype is not ytype or not out.is_contiguous():
        _bad("out must be contiguous, of h's shape and y's type")
    elif out.get_device() != dev:
        _elsewhere(out)
    if post_weight is not None:
        a = _vector(post_weight, d, dev, "post_weight")
    if post_bias is not None:
        b = _vector(post_bias, d, dev, "post_bias")
    if pre_weight is not None:
        c = _vector(pre_weight, d, dev, "pre_weight")
    if pre_bias is not None:
        e = _vector(pre_bias, d, dev, "pre_bias")
    s = _pack_norms(kind, hkind, r, d, _NORMS[norm], 1 if post else 0, gates, eps, alpha, beta, hpitch, ypitch)
    status = (_f or _load())["qnn_lm_norm_residual"](s, h.data_ptr(), yp, a, b, c, e, gp, hop, out.data_ptr(), handle)
    if status:
        raise QnnError(status, "qnn_lm_norm_residual")
    return h_out, out


def make_cache(pages, heads, page, dim, bits, dtype=torch.bfloat16, device="cuda"):
    """An empty Cache of `bits` bits (16: numbers of `dtype`)."""
    if bits == 16:
        k, v = (torch.zeros((pages, heads, page, dim), dtype=dtype, device=device) for _ in range(2))
        return Cache(k, v, None, None, 16)
    k, v = (torch.zeros((pages, heads, page, dim * bits // 8), dtype=torch.uint8, device=device) for _ in range(2))
    ks, vs = (torch.zeros((pages, heads, page), dtype=torch.float32, device=device) for _ in range(2))
    return Cache(k, v, ks, vs, bits)


def _cache(cache, table, b, d):
    """(the C structure, heads, dim, the numbers' type at 16 bits or None); d: the device."""
    k, v, ks, vs, bits = cache
    shape, dtype = k.shape, k.dtype
    if len(shape) != 4 or v.shape != shape or v.dtype is not dtype:
        _bad("k and v of a cache must be [pages, heads, page, dim], alike")
    pages, heads, page, dim = shape
    a0, a1, a2, a3 = k.stride()
    c0, c1, c2, c3 = v.stride()
    if a3 != 1 or c3 != 1:
        _bad("the channels of a cache must be contiguous")
    ksp = vsp = 0
    if bits == 16:
        kind = _TYPES16.get(dtype)
        if kind is None or ks is not None or vs is not None:
            _bad("a cache of 16 bits holds bfloat16 or float16 and no scales")
        a0, a1, a2, c0, c1, c2 = 2 * a0, 2 * a1, 2 * a2, 2 * c0, 2 * c1, 2 * c2
    else:
        if dtype is not _U8 or (bits != 8 and bits != 4):
            _bad("a cache holds uint8 codes of 8 or 4 bits, or numbers of 16 bits")
        kind, dtype = 0, None
        if bits == 4:
            dim *= 2
        for s in (ks, vs):
            if s is None or s.dtype is not _F32 or s.shape != shape[:3] or not s.is_contiguous():
                _bad("the scales of a cache must be contiguous float32 [pages, heads, page]")
            if s.get_device() != d:
                _elsewhere(s)
        ksp, vsp = ks.data_ptr(), vs.data_ptr()
    t = table.shape
    if len(t) != 2 or t[0] != b or table.dtype is not _I32 or not table.is_contiguous():
        _bad("table must be contiguous int32 [%d, pages of a sequence]" % b)
    if k.get_device() != d or v.get_device() != d or table.get_device() != d:
        _bad("the cache and its table must be on the other tensors' device")
    return (_pack_cache(kind, bits, pages, heads, page, dim, a0, a1, a2, c0, c1, c2, k.data_ptr(), v.data_ptr(), ksp, vsp,
                        table.data_ptr(), b, t[1]), heads, dim, dtype)


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
    st = q.stride()
    if len(st) != 4 or st[3] != 1:
        _bad("q must be [b, t, heads, dim], contiguous along dim")
    shape = q.shape
    b, t, heads, dim = shape
    dtype = q.dtype
    kind = _TYPES16.get(dtype)
    d = q.get_device()
    c, _, cdim, ctype = _cache(cache, table, b, d)
    if kind is None or (ctype is not None and ctype is not dtype):
        _bad("q must be bfloat16 or float16, and of the type of a cache of 16 bits")
    if cdim != dim:
        _bad("q has heads of %d channels, the cache of %d" % (dim, cdim))
    handle = _stream(d, stream)
    lp = _ints(lens, b, d, "lens")
    cp = mp = sp = None
    if counts is not None:
        cp = _ints(counts, b, d, "counts")
    if mask is not None:
        if mask.dtype is not torch.int64 or mask.shape != (b, t, (t + 63) // 64) or not mask.is_contiguous():
            _bad("mask must be contiguous int64 [b, t, ceil(t / 64)]")
        if mask.get_device() != d:
            _elsewhere(mask)
        mp = mask.data_ptr()
    if out is None:
        out = _alloc_like(q, stream) if q.is_contiguous() else _alloc(shape, dtype, q, stream)
    elif out.shape != shape or out.dtype is not dtype or not out.is_contiguous():
        _bad("out must be contiguous and like q")
    elif out.get_device() != d:
        _elsewhere(out)
    lse = None
    if want_lse:
        lse = _alloc(shape[:3], _F32, q, stream)
        sp = lse.data_ptr()
    s = _pack_queries(kind, t, heads, dim ** -0.5 if scale is None else scale, st[0], st[1], st[2])
    f = _f or _load()
    size = f["qnn_lm_tree_attention_workspace"](s, c)
    ws = wp = None
    if size:
        ws = _alloc(size, _U8, q, stream)
        wp = ws.data_ptr()
    status = f["qnn_lm_tree_attention"](s, q.data_ptr(), c, lp, cp, mp, out.data_ptr(), sp, wp, size, handle)
    if status:
        raise QnnError(status, "qnn_lm_tree_attention")
    return (out, lse) if want_lse else out


def cache_append(k, v, cache, table, lens, counts=None, stream=None):
    """Writes new tokens into the cache (qnn_lm_cache_append): k and v
    [b, t, heads, dim] bfloat16 or float16, token j of a sequence to position
    lens + j where j < counts (None: t)."""
    shape, dtype = k.shape, k.dtype
    if len(shape) != 4 or v.shape != shape or v.dtype is not dtype:
        _bad("k and v must be [b, t, heads, dim], alike")
    a0, a1, a2, a3 = k.stride()
    c0, c1, c2, c3 = v.stride()
    if a3 != 1 or c3 != 1:
        _bad("k and v must be contiguous along dim")
    b, t, heads, dim = shape
    kind = _TYPES16.get(dtype)
    d = k.get_device()
    c, cheads, cdim, ctype = _cache(cache, table, b, d)
    if kind is None or (ctype is not None and ctype is not dtype):
        _bad("k and v must be bfloat16 or float16, and of the type of a cache of 16 bits")
    if heads != cheads or dim != cdim:
        _bad("k and v have %d heads of %d channels, the cache %d of %d" % (heads, dim, cheads, cdim))
    if v.get_device() != d:
        _elsewhere(v)
    s = _pack_tokens(kind, t, a0, a1, a2, c0, c1, c2)
    status = (_f or _load())["qnn_lm_cache_append"](
        s, k.data_ptr(), v.data_ptr(), c, _ints(lens, b, d, "lens"),
        None if counts is None else _ints(counts, b, d, "counts"), _stream(d, stream))
    if status:
        raise QnnError(status, "qnn_lm_cache_append")


def cache_keep(cache, table, lens, path, kept, stream=None):
    """Moves the accepted drafts to the front (qnn_lm_cache_keep): position
    lens + j takes position lens + path[:, j] for j < kept.  path: int32 [b, t],
    strictly ascending; kept: int32 [b]."""
    if path.dim() != 2 or path.dtype is not _I32 or not path.is_contiguous():
        _bad("path must be contiguous int32 [b, t]")
    b, t = path.shape
    d = path.get_device()
    status = (_f or _load())["qnn_lm_cache_keep"](
        _cache(cache, table, b, d)[0], t, _ints(lens, b, d, "lens"), path.data_ptr(), _ints(kept, b, d, "kept"),
        _stream(d, stream))
    if status:
        raise QnnError(status, "qnn_lm_cache_keep")


def cache_read(cache, table, start, n, dtype=torch.bfloat16, stream=None):
    """The values at positions start .. start + n - 1 of each sequence
    (qnn_lm_cache_read): (k, v), each [b, n, heads, dim] of `dtype`; zeros where
    the table does not reach."""
    kind = _TYPES.get(dtype)
    if kind is None:
        _bad("dtype must be bfloat16, float16 or float32")
    b, d = start.numel(), start.get_device()
    c, heads, dim, _ = _cache(cache, table, b, d)
    sp, handle = _ints(start, b, d, "start"), _stream(d, stream)
    k = _alloc((b, n, heads, dim), dtype, start, stream)
    v = _alloc_like(k, stream)
    status = (_f or _load())["qnn_lm_cache_read"](c, kind, n, sp, k.data_ptr(), v.data_ptr(), handle)
    if status:
        raise QnnError(status, "qnn_lm_cache_read")
    return k, v
