"""include/qnn_lm.h without a GPU: the library exports what the header
declares, its arguments are checked on the host before any device call, and
the binding refuses tensors that are not what a call takes."""
import ctypes
import re
import struct

import pytest
import torch

OK, NULL, BITS, SHAPE, PARAM, ALIGN, UNSUPPORTED, DEVICE = 0, 1, 2, 3, 4, 5, 7, 8
P = 1 << 20  # a 16-byte aligned address that is never read
BF, HF, F, I = torch.bfloat16, torch.float16, torch.float32, torch.int32


class Raw:
    """The library's entry points with plain arguments, and the C structures as packed bytes."""
    _pack_linear = staticmethod(struct.Struct("@8i3q").pack)
    _pack_norms = staticmethod(struct.Struct("@7i3f2q").pack)
    _pack_cache = staticmethod(struct.Struct("@6i6q5P2i").pack)
    _pack_queries = staticmethod(struct.Struct("@3if3q").pack)
    _pack_tokens = staticmethod(struct.Struct("@2i6q").pack)

    def __init__(self):
        from paper_1908_11263_amd import lm, qnn
        self.HEADER = lm.HEADER
        P, I, S, Z = ctypes.c_void_p, ctypes.c_int32, ctypes.c_char_p, ctypes.c_size_t
        arguments = {"qnn_lm_matmul": [S, P, P, P, P, P, P, P, Z, P], "qnn_lm_matmul_workspace": [S],
                     "qnn_lm_norm_residual": [S] + 10 * [P], "qnn_lm_tree_attention": [S, P, S, P, P, P, P, P, P, Z, P],
                     "qnn_lm_tree_attention_workspace": [S, S], "qnn_lm_cache_append": [S, P, P, S, P, P, P],
                     "qnn_lm_cache_keep": [S, I, P, P, P, P], "qnn_lm_cache_read": [S, I, I, P, P, P, P]}
        assert sorted(arguments) == sorted(lm.ENTRIES)
        self.f = {}
        for name, types in arguments.items():
            f = qnn.lib()[name]
            f.restype, f.argtypes = Z if name.endswith("workspace") else ctypes.c_int, types
            self.f[name] = f

    def _fn(self, name):
        return self.f[name]


@pytest.fixture(scope="module")
def lm():
    return Raw()


@pytest.fixture(scope="module")
def binding():
    from paper_1908_11263_amd import lm
    return lm


def reached():
    """What a call that passes every check gives where there is no GPU."""
    return (DEVICE,)


def test_exports_every_header_function(lm):
    with open(lm.HEADER) as f:
        text = re.sub(r"/\*.*?\*/", "", f.read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(qnn_lm_[a-z0-9_]+)\s*\(", text)))
    assert len(names) == 8
    for name in names:
        assert lm._fn(name)


needs_no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="calls that pass every check are not made on a GPU")


def linear(lm, type=0, bits=4, r=3, k=256, m=64, group=0, act=0, gated=0, xp=256, rp=64, yp=64, x=P, w=P, scale=P,
           bias=None, res=None, y=P, ws=None, size=0):
    s = lm._pack_linear(type, bits, r, k, m, group, act, gated, xp, rp, yp)
    return lm._fn("qnn_lm_matmul")(s, x, w, scale, bias, res, y, ws, size, None)


@needs_no_gpu
def test_matmul_refusals(lm):
    f = lambda **a: linear(lm, **a)  # noqa: E731
    assert f() in reached()
    assert f(bits=16, scale=None) in reached()
    assert f(r=0, x=None, y=None) == OK
    for bits in (0, 3, 5, 32, -8):
        assert f(bits=bits) == BITS
    for bad in (dict(type=2), dict(type=-1), dict(act=5), dict(act=-1), dict(gated=2), dict(group=16), dict(group=96),
                dict(bits=16, group=32, scale=None), dict(bits=16)):
        assert f(**bad) == PARAM, bad
    for bad in (dict(r=-1), dict(k=0), dict(m=0), dict(k=40, xp=40), dict(k=96, xp=96, group=64), dict(xp=248),
                dict(yp=63), dict(res=P, rp=63), dict(r=1 << 22), dict(m=1 << 25, yp=1 << 25), dict(rp=-8),
                dict(xp=1 << 62), dict(yp=1 << 62), dict(rp=1 << 62, res=P)):
        assert f(**bad) == SHAPE, bad
    assert f(k=1 << 21, xp=1 << 21) == UNSUPPORTED
    for bad in (dict(x=None), dict(w=None), dict(scale=None), dict(y=None)):
        assert f(**bad) == NULL, bad
    for bad in (dict(xp=257), dict(x=P + 8), dict(w=P + 4), dict(scale=P + 4), dict(bias=P + 4), dict(res=P + 2),
                dict(y=P + 2), dict(ws=P + 1, size=1 << 30)):
        assert f(**bad) == ALIGN, bad
    assert lm._fn("qnn_lm_matmul")(None, P, P, P, None, None, P, None, 0, None) == NULL
    assert lm._fn("qnn_lm_matmul_workspace")(None) == 0


def norms(lm, type=0, ht=0, r=4, d=64, norm=0, post=1, gates=0, eps=1e-6, hp=64, yp=64, h=P, y=P, pw=None, gate=None,
          ho=P, x=P):
    s = lm._pack_norms(type, ht, r, d, norm, post, gates, eps, 1.0, 1.0, hp, yp)
    return lm._fn("qnn_lm_norm_residual")(s, h, y, pw, None, None, None, gate, ho, x, None)


@needs_no_gpu
def test_norm_refusals(lm):
    f = lambda **a: norms(lm, **a)  # noqa: E731
    assert f() in reached()
    assert f(y=None, ho=None) in reached()
    assert f(ht=2) in reached()
    assert f(r=0, h=None, y=None, x=None) == OK
    for bad in (dict(type=3), dict(ht=1), dict(type=2, ht=0), dict(norm=2), dict(post=2), dict(eps=-1.0),
                dict(eps=float("nan"))):
        assert f(**bad) == PARAM, bad
    for bad in (dict(r=-1), dict(d=0), dict(gates=3, gate=P), dict(gates=-1), dict(hp=63), dict(yp=63), dict(hp=1 << 61)):
        assert f(**bad) == SHAPE, bad
    assert f(d=32769, hp=32769, yp=32769) == UNSUPPORTED
    for bad in (dict(h=None), dict(x=None), dict(ho=None), dict(gates=2)):
        assert f(**bad) == NULL, bad
    for bad in (dict(h=P + 4), dict(y=P + 2), dict(pw=P + 4), dict(x=P + 8), dict(ho=P + 8)):
        assert f(**bad) == ALIGN, bad


def cache(lm, type=0, bits=8, pages=10, heads=2, page=16, dim=64, st=(2048, 1024, 64) * 2, k=P, v=P, ks=P, vs=P, table=P,
          b=2, width=4):
    ptr = lambda p: p or 0  # noqa: E731
    return lm._pack_cache(type, bits, pages, heads, page, dim, *st, ptr(k), ptr(v), ptr(ks), ptr(vs), ptr(table), b, width)


CACHES = [
    (dict(), None), (dict(bits=4), None), (dict(bits=16, ks=None, vs=None, st=(4096, 2048, 128) * 2), None),
    (dict(st=(2048, 64, 128) * 2), None), (dict(bits=2), BITS), (dict(bits=1), BITS), (dict(type=2), PARAM),
    (dict(bits=16, st=(4096, 2048, 128) * 2), PARAM), (dict(pages=0), SHAPE), (dict(heads=0), SHAPE), (dict(page=0), SHAPE),
    (dict(b=-1), SHAPE), (dict(width=0), SHAPE), (dict(dim=96), UNSUPPORTED), (dict(dim=32), UNSUPPORTED),
    (dict(width=1 << 28), SHAPE), (dict(b=65536), SHAPE), (dict(st=(2048, 1024, 48) * 2), SHAPE),
    (dict(st=(2048, 1024, 72) * 2), ALIGN), (dict(st=(-2048, 1024, 64) * 2), SHAPE),
    (dict(st=(1 << 61, 1024, 64) * 2), SHAPE), (dict(k=None), NULL), (dict(v=None), NULL), (dict(table=None), NULL),
    (dict(ks=None), NULL), (dict(vs=None), NULL), (dict(k=P + 8), ALIGN), (dict(vs=P + 4), ALIGN), (dict(table=P + 4), ALIGN),
]


def attend(lm, c, type=0, t=3, heads=4, scale=0.125, st=(768, 256, 64), q=P, lens=P, counts=None, mask=None, out=P,
           lse=None, ws=P, size=1 << 40):
    s = lm._pack_queries(type, t, heads, scale, *st)
    return lm._fn("qnn_lm_tree_attention")(s, q, c, lens, counts, mask, out, lse, ws, size, None)


def append(lm, c, type=0, t=3, st=(384, 128, 64) * 2, k=P, v=P, lens=P, counts=None):
    return lm._fn("qnn_lm_cache_append")(lm._pack_tokens(type, t, *st), k, v, c, lens, counts, None)


def keep(lm, c, t=3, lens=P, path=P, kept=P):
    return lm._fn("qnn_lm_cache_keep")(c, t, lens, path, kept, None)


def read(lm, c, type=0, t=3, start=P, k=P, v=P):
    return lm._fn("qnn_lm_cache_read")(c, type, t, start, k, v, None)


@needs_no_gpu
@pytest.mark.parametrize("args,status", CACHES)
def test_cache_refusals(lm, args, status):
    c = cache(lm, **args)
    for call in (attend, append, keep, read):
        got = call(lm, c)
        assert got in reached() if status is None else got == status, call.__name__


@needs_no_gpu
def test_attention_refusals(lm):
    c = cache(lm)
    f = lambda **a: attend(lm, c, **a)  # noqa: E731
    assert f() in reached()
    assert f(t=0, q=None, out=None) == OK and attend(lm, cache(lm, b=0)) == OK
    for bad in (dict(type=2), dict(scale=float("nan")), dict(scale=float("inf"))):
        assert f(**bad) == PARAM, bad
    assert attend(lm, cache(lm, bits=16, type=1, ks=None, vs=None, st=(4096, 2048, 128) * 2)) == PARAM
    for bad in (dict(t=-1), dict(heads=3), dict(heads=0), dict(t=1 << 23), dict(st=(-8, 256, 64)), dict(st=(1 << 62, 256, 64))):
        assert f(**bad) == SHAPE, bad
    for bad in (dict(q=None), dict(lens=None), dict(out=None)):
        assert f(**bad) == NULL, bad
    # few rows over a cache of many tiles: pieces, joined through the workspace
    wide = cache(lm, width=1000)
    need = lm._fn("qnn_lm_tree_attention_workspace")(lm._pack_queries(0, 3, 4, 0.125, 768, 256, 64), wide)
    assert need > 0
    assert attend(lm, wide, size=need) in reached()
    assert attend(lm, wide, size=need - 1) == SHAPE and attend(lm, wide, ws=None) == NULL
    for bad in (dict(st=(768, 256, 60)), dict(q=P + 8), dict(lens=P + 4), dict(counts=P + 4), dict(mask=P + 8),
                dict(out=P + 2), dict(lse=P + 4), dict(ws=P + 8)):
        assert f(**bad) == ALIGN, bad
    assert lm._fn("qnn_lm_tree_attention")(None, P, c, P, None, None, P, None, None, 0, None) == NULL
    assert lm._fn("qnn_lm_tree_attention")(lm._pack_queries(0, 1, 2, 1.0, 0, 0, 0), P, None, P, None, None, P, None, None,
                                           0, None) == NULL
    assert lm._fn("qnn_lm_tree_attention_workspace")(None, c) == 0


@needs_no_gpu
def test_token_refusals(lm):
    c = cache(lm)
    assert append(lm, c) in reached() and keep(lm, c) in reached() and read(lm, c, k=None) in reached()
    assert append(lm, c, t=0, k=None) == OK and keep(lm, c, t=0, path=None) == OK and read(lm, c, t=0, k=None, v=None) == OK
    assert append(lm, c, type=2) == PARAM and read(lm, c, type=3) == PARAM
    assert append(lm, c, st=(384, 128, 60) * 2) == ALIGN and append(lm, c, st=(384, -128, 64) * 2) == SHAPE
    for call in (append, keep, read):
        assert call(lm, c, t=-1) == SHAPE
        assert call(lm, c, t=1 << 29) == SHAPE
    assert append(lm, c, v=None) == NULL and append(lm, c, lens=None) == NULL
    assert keep(lm, c, path=None) == NULL and keep(lm, c, kept=None) == NULL
    assert read(lm, c, k=None, v=None) == NULL and read(lm, c, start=None) == NULL
    assert append(lm, c, k=P + 2) == ALIGN and keep(lm, c, path=P + 4) == ALIGN and read(lm, c, v=P + 4) == ALIGN


def refused(f, *args, **kw):
    with pytest.raises(ValueError):
        f(*args, **kw)


def test_binding_refuses(binding):
    lm = binding
    z = torch.zeros
    x, w, s = z(3, 64, dtype=BF), z(8, 32, dtype=torch.uint8), z(8)
    for bad in (dict(x=z(3, 64)), dict(x=z(64, 3, dtype=BF).t()), dict(w=z(8, 31, dtype=torch.uint8)), dict(w=z(8, 32)),
                dict(w=z(32, 8, dtype=torch.uint8).t()), dict(scale=z(7)), dict(scale=z(8, dtype=BF)), dict(scale=z(8, 3)),
                dict(scale=z(8, 0)), dict(bias=z(9)), dict(bias=z(8, dtype=BF)), dict(residual=z(3, 9, dtype=BF)),
                dict(residual=z(3, 8)), dict(out=z(2, 8, dtype=BF)), dict(out=z(3, 8)), dict(out=z(8, 3, dtype=BF).t()),
                dict(w=z(7, 32, dtype=torch.uint8), scale=z(7), gated=True)):
        a = dict(x=x, w=w, bits=4, scale=s) | bad
        refused(lm.matmul, **a)
    with pytest.raises(KeyError):
        lm.matmul(x, w, 4, scale=s, act="tanh")
    h = z(3, 64, dtype=BF)
    for bad in (dict(y=z(3, 63, dtype=BF)), dict(y=z(3, 64, dtype=torch.int32)), dict(gate=z(2, 63, dtype=BF)),
                dict(gate=z(3, 64)), dict(pre_weight=z(63)), dict(post_bias=z(64, dtype=BF)), dict(h_out=z(3, 64)),
                dict(out=z(3, 64)), dict(out=z(64, 3, dtype=BF).t())):
        refused(lm.norm_residual, **(dict(h=h, y=h) | bad))
    c = lm.make_cache(4, 2, 16, 64, 8, device="cpu")
    assert c.k.shape == (4, 2, 16, 64) and lm.make_cache(4, 2, 16, 64, 4, device="cpu").k.shape == (4, 2, 16, 32)
    table, lens = z(1, 4, dtype=I), z(1, dtype=I)
    q = z(1, 3, 4, 64, dtype=BF)
    mask = z(1, 3, 1, dtype=torch.int64)
    for bad in (dict(q=z(1, 3, 4, 64)), dict(q=z(3, 4, 64, dtype=BF)), dict(q=z(1, 3, 4, 128, dtype=BF)),
                dict(table=z(2, 4, dtype=I)), dict(table=z(1, 4)), dict(lens=z(2, dtype=I)), dict(lens=z(1)),
                dict(counts=z(2, dtype=I)), dict(mask=z(1, 3, 2, dtype=torch.int64)), dict(mask=z(1, 3, 1, dtype=I)),
                dict(out=z(1, 3, 4, 64)), dict(cache=c._replace(bits=16)), dict(cache=c._replace(k_scale=None)),
                dict(cache=c._replace(v=c.v[:3])), dict(cache=c._replace(v_scale=z(4, 2, 15))), dict(cache=c._replace(bits=2)),
                dict(cache=lm.make_cache(4, 2, 16, 64, 16, HF, "cpu"))):
        refused(lm.tree_attention, **(dict(q=q, cache=c, table=table, lens=lens, mask=mask) | bad))
    kv = z(1, 3, 2, 64, dtype=BF)
    for bad in (dict(k=z(1, 3, 2, 64)), dict(k=z(1, 2, 2, 64, dtype=BF)), dict(k=z(1, 3, 1, 64, dtype=BF), v=z(1, 3, 1, 64, dtype=BF)),
                dict(lens=z(3, dtype=I)), dict(counts=z(1))):
        refused(lm.cache_append, **(dict(k=kv, v=kv, cache=c, table=table, lens=lens) | bad))
    path = z(1, 3, dtype=I)
    for bad in (dict(path=z(1, 3)), dict(path=z(3, dtype=I)), dict(kept=z(2, dtype=I)), dict(lens=z(1, 1, dtype=I))):
        refused(lm.cache_keep, **(dict(cache=c, table=table, lens=lens, path=path, kept=lens) | bad))
    refused(lm.cache_read, c, table, lens, 3, dtype=torch.int32)
    refused(lm.cache_read, c, table, z(1), 3)

