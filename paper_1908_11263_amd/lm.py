"""Binding of include/qnn_lm.h: one step of a language model's block over packed
weights and a packed cache.

Argument marshalling only, as in qnn.py: every computation runs in the
library's HIP kernels, there is no fallback.  The marshalling itself is compiled
(csrc/lm_bind.cpp): a call of a small layer takes a few microseconds on the
device, and looking at its tensors from Python takes longer.  Tensors live on
the current HIP device; work is enqueued on torch's current stream or on
`stream`, and what a call allocates (its result, its workspace) belongs to that
stream.  Tensors start on 16 bytes; lengths, counts, tables, masks and paths that
do not (lens[1:], a part of a batch) are copied.  What the library can check it
refuses with QnnError; what only the binding can see (a tensor's type, shape,
strides, device) raises ValueError.  The operators are forward only: a tensor
that requires a gradient is refused while torch records them (torch.no_grad()
says that none is meant).

A cache is a `Cache`: k and v are [pages, heads, page, dim] tensors of 16-bit
numbers (bits = 16), or uint8 tensors whose last axis holds dim codes of 8 or 4
bits, with k_scale and v_scale [pages, heads, page] in 32 bits.  Any strides
will do whose last is 1 and whose others are multiples of 16 bytes: a view of
[pages, page, heads, dim] is as good.
"""
import collections
import ctypes
import importlib.util
import os

import torch

from . import qnn
from .qnn import QnnError  # noqa: F401

HEADER = os.path.join(os.path.dirname(qnn.HEADER), "qnn_lm.h")
BINDING = os.path.join(qnn.HERE, "_lm_bind.so")

_TYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
_ACTS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3, "gelu_tanh": 4}
_NORMS = {"rms": 0, "layer": 1}

# bits: 16, 8 or 4; the scales are None at 16 bits
Cache = collections.namedtuple("Cache", "k v k_scale v_scale bits")

# in the order that the compiled part takes their addresses
ENTRIES = ("qnn_lm_matmul", "qnn_lm_matmul_workspace", "qnn_lm_norm_residual", "qnn_lm_tree_attention",
           "qnn_lm_tree_attention_workspace", "qnn_lm_cache_append", "qnn_lm_cache_keep", "qnn_lm_cache_read")


class _Unloaded:
    """Loads the compiled part (and libqnn.so) at the first call."""

    def __getattr__(self, name):
        global _bind
        if not os.path.exists(BINDING):
            raise RuntimeError("_lm_bind.so is not built (run __graft_entry__.build()); there is no fallback")
        L = qnn.lib()
        spec = importlib.util.spec_from_file_location("_lm_bind", BINDING)
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
        module.init(qnn.QnnError, torch.cuda.is_available(),
                    *(ctypes.cast(L[entry], ctypes.c_void_p).value for entry in ENTRIES))
        _bind = module
        return getattr(module, name)


_bind = _Unloaded()


def _on(stream, *tensors):
    """Makes `stream` the current one for a call, so that what it allocates is the
    stream's, and tells the allocator that the stream uses the call's tensors: a
    caller may drop them when the call returns."""
    for t in tensors:
        if isinstance(t, torch.Tensor):
            if t.is_cuda:
                t.record_stream(stream)
        elif isinstance(t, Cache):
            _on(stream, *t)
    return torch.cuda.stream(stream)


def matmul(x, w, bits, scale=None, bias=None, act="none", gated=False, residual=None, out=None, stream=None):
    """Linear layer with its epilogue (qnn_lm_matmul):
    act(x w^T * scale + bias) + residual, or with gated=True
    act(gate) * up + residual, the first half of w's rows being the gate's.

    x: [..., k] bfloat16 or float16.  w: [rows, k * bits / 8] uint8 packed codes
    (bits 8, 4, 2, 1), or [rows, k] numbers of x's type (bits = 16).  scale:
    float32 [rows] or [rows, groups], k / groups being 32, 64 or 128.  bias:
    float32 [rows].  Returns [..., m] of x's type; out may be residual."""
    if stream is not None:
        with _on(stream, x, w, scale, bias, residual, out):
            return matmul(x, w, bits, scale, bias, act, gated, residual, out)
    return _bind.matmul(x, w, bits, scale, bias, _ACTS[act], gated, residual, out)


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
    if stream is not None:
        with _on(stream, h, y, post_weight, post_bias, pre_weight, pre_bias, gate, h_out, out):
            return norm_residual(h, y, norm, post, post_weight, post_bias, pre_weight, pre_bias, gate, alpha, beta, eps,
                                 dtype, h_out, out)
    like = torch.empty(0, dtype=dtype) if dtype is not None and y is None else None
    return _bind.norm_residual(h, y, _NORMS[norm], post, post_weight, post_bias, pre_weight, pre_bias, gate, alpha, beta,
                               eps, like, h_out, out)


def make_cache(pages, heads, page, dim, bits, dtype=torch.bfloat16, device="cuda"):
    """An empty Cache of `bits` bits (16: numbers of `dtype`)."""
    if bits == 16:
        k, v = (torch.zeros((pages, heads, page, dim), dtype=dtype, device=device) for _ in range(2))
        return Cache(k, v, None, None, 16)
    k, v = (torch.zeros((pages, heads, page, dim * bits // 8), dtype=torch.uint8, device=device) for _ in range(2))
    ks, vs = (torch.zeros((pages, heads, page), dtype=torch.float32, device=device) for _ in range(2))
    return Cache(k, v, ks, vs, bits)


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
    if stream is not None:
        with _on(stream, q, cache, table, lens, mask, counts, out):
            return tree_attention(q, cache, table, lens, mask, counts, scale, out, want_lse)
    return _bind.tree_attention(q, cache, table, lens, mask, counts, q.shape[-1] ** -0.5 if scale is None else scale, out,
                                want_lse)


def cache_append(k, v, cache, table, lens, counts=None, stream=None):
    """Writes new tokens into the cache (qnn_lm_cache_append): k and v
    [b, t, heads, dim] bfloat16 or float16, token j of a sequence to position
    lens + j where j < counts (None: t)."""
    if stream is not None:
        with _on(stream, k, v, cache, table, lens, counts):
            return cache_append(k, v, cache, table, lens, counts)
    return _bind.cache_append(k, v, cache, table, lens, counts)


def cache_keep(cache, table, lens, path, kept, stream=None):
    """Moves the accepted drafts to the front (qnn_lm_cache_keep): position
    lens + j takes position lens + path[:, j] for j < kept.  path: int32 [b, t],
    strictly ascending; kept: int32 [b]."""
    if stream is not None:
        with _on(stream, cache, table, lens, path, kept):
            return cache_keep(cache, table, lens, path, kept)
    return _bind.cache_keep(cache, table, lens, path, kept)


def cache_read(cache, table, start, n, dtype=torch.bfloat16, stream=None):
    """The values at positions start .. start + n - 1 of each sequence
    (qnn_lm_cache_read): (k, v), each [b, n, heads, dim] of `dtype`; zeros where
    the table does not reach."""
    if stream is not None:
        with _on(stream, cache, table, start):
            return cache_read(cache, table, start, n, dtype)
    return _bind.cache_read(cache, table, start, n, _TYPES.get(dtype, -1))
