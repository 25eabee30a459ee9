"""The operators of include/qnn_lm.h on the GPU against their formulas in 64
bits (lm_reference.py): sizes that fill no tile, every bit-width, masks that
leave rows empty, strides, streams and graphs."""
import math

import pytest
import torch

import lm_reference as ref

pytestmark = pytest.mark.gpu

BF, HF, F = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def lm():
    from paper_1908_11263_amd import lm
    return lm


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(g, *shape, dtype=F):
    return torch.randn(shape, generator=g, device="cuda", dtype=F).to(dtype)


def layer(g, r, k, m, bits, group, dtype, gated=False, bias=False, residual=False):
    rows = 2 * m if gated else m
    x = randn(g, r, k, dtype=dtype)
    if bits == 16:
        w, scale = randn(g, rows, k, dtype=dtype) * k ** -0.5, None
    else:
        w = torch.randint(0, 256, (rows, k * bits // 8), generator=g, device="cuda", dtype=torch.uint8)
        shape = (rows, k // group) if group else (rows,)
        scale = (0.2 + torch.rand(shape, generator=g, device="cuda")) / (2 ** (bits - 1) * k ** 0.5)
    return dict(x=x, w=w, scale=scale, bias=randn(g, rows) if bias else None,
                residual=randn(g, r, m, dtype=dtype) if residual else None)


def check_matmul(lm, L, bits, act="none", gated=False):
    y = lm.matmul(L["x"], L["w"], bits, scale=L["scale"], bias=L["bias"], act=act, gated=gated, residual=L["residual"])
    want, bound = ref.matmul(L["x"], L["w"], bits, L["scale"], L["bias"], act, gated, L["residual"])
    ref.close(y, want, bound, "matmul")
    return y


SIZES = [(1, 32, 1), (1, 4096, 64), (2, 128, 17), (3, 96, 100), (5, 1056, 33), (15, 256, 16), (16, 384, 48),
         (17, 160, 31), (31, 512, 129), (64, 2080, 65), (65, 224, 130), (127, 640, 257), (128, 128, 128),
         (129, 1184, 96), (257, 320, 300), (300, 2048, 511), (513, 96, 770)]


@pytest.mark.parametrize("bits", [16, 8, 4, 2, 1])
@pytest.mark.parametrize("r,k,m", SIZES)
def test_matmul_sizes(lm, bits, r, k, m):
    g = gen(r * 7 + k + m + bits)
    for dtype in (BF, HF):
        check_matmul(lm, layer(g, r, k, m, bits, 0, dtype), bits)


@pytest.mark.parametrize("bits", [8, 4, 2, 1])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("r,k,m", [(1, 128, 16), (7, 1152, 50), (33, 640, 200), (200, 1408, 272), (400, 256, 129)])
def test_matmul_groups(lm, bits, group, r, k, m):
    g = gen(r + k + m + bits + group)
    dtype = BF if (r + bits) % 2 else HF
    check_matmul(lm, layer(g, r, k, m, bits, group, dtype, bias=True, residual=True), bits)


@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("r,bits,group", [(1, 4, 128), (20, 8, 0), (70, 16, 0), (210, 4, 64), (333, 2, 32)])
def test_matmul_epilogues(lm, act, gated, r, bits, group):
    g = gen(r + bits)
    for bias, residual in ((False, False), (True, False), (True, True)):
        check_matmul(lm, layer(g, r, 384, 75, bits, group, BF, gated, bias, residual), bits, act, gated)


@pytest.mark.parametrize("r", [1, 4, 40, 300])
def test_matmul_extremes_of_codes(lm, r):
    """Rows of the lowest and the highest code, and of one code alone: every code expands exactly."""
    for bits in (8, 4, 2, 1):
        n = 1 << bits
        codes = torch.arange(n, device="cuda", dtype=torch.uint8).repeat_interleave(256).reshape(n, 256)
        w = ref.pack(codes, bits)
        x = torch.zeros(r, 256, device="cuda", dtype=BF)
        x[:, 37] = 1.0
        for dtype in (BF, HF):
            y = lm.matmul(x.to(dtype), w, bits, scale=torch.ones(n, device="cuda"))
            want = ref.values(w, bits)[:, 37].expand(r, n)
            assert torch.equal(y.double(), want), bits


@pytest.mark.parametrize("r", [2, 24, 150])
@pytest.mark.parametrize("bits", [16, 4])
def test_matmul_infinities_stay_in_their_rows(lm, r, bits):
    g = gen(3)
    L = layer(g, r, 256, 90, bits, 0, BF)
    L["x"][1, 5] = math.inf
    L["x"][0, 7] = math.nan
    y = lm.matmul(L["x"], L["w"], bits, scale=L["scale"])
    assert torch.isnan(y[0]).all()
    w5 = L["w"][:, 5].double() if bits == 16 else ref.values(L["w"], bits)[:, 5]
    assert torch.equal(y[1].isposinf(), w5 > 0) and torch.equal(y[1].isneginf(), w5 < 0)
    want, bound = ref.matmul(L["x"][2:], L["w"], bits, L["scale"])
    ref.close(y[2:], want, bound, "rows beside")


@pytest.mark.parametrize("r", [1, 9, 70, 260])
def test_matmul_strides_and_places(lm, r):
    """Padded rows in x, residual and out; the result in the residual's place; a stack of matrices."""
    g = gen(r)
    L = layer(g, r, 192, 52, 4, 64, BF, bias=True, residual=True)
    want, bound = ref.matmul(L["x"], L["w"], 4, L["scale"], L["bias"], "silu", False, L["residual"])
    wide = torch.full((r, 200), math.nan, device="cuda", dtype=BF)
    wide[:, :192] = L["x"]
    res = torch.zeros(r, 61, device="cuda", dtype=BF)
    res[:, :52] = L["residual"]
    out = torch.zeros(r, 55, device="cuda", dtype=BF)
    y = lm.matmul(wide[:, :192], L["w"], 4, scale=L["scale"], bias=L["bias"], act="silu", residual=res[:, :52],
                  out=out[:, :52])
    assert y.data_ptr() == out.data_ptr()
    ref.close(y, want, bound, "strided")
    assert not bool(out[:, 52:].any()) and not bool(res[:, 52:].any())
    h = L["residual"].clone()
    lm.matmul(L["x"], L["w"], 4, scale=L["scale"], bias=L["bias"], act="silu", residual=h, out=h)
    ref.close(h, want, bound, "in place")
    if r % 2 == 0:
        y = lm.matmul(L["x"].reshape(2, r // 2, 192), L["w"], 4, scale=L["scale"], bias=L["bias"], act="silu",
                      residual=L["residual"].reshape(2, r // 2, 52))
        assert y.shape == (2, r // 2, 52)
        ref.close(y, want, bound, "stacked")
    assert lm.matmul(L["x"][:0], L["w"], 4, scale=L["scale"]).shape == (0, 52)


@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("r,d", [(1, 1), (1, 64), (3, 7), (5, 1000), (4, 1024), (2, 1025), (1, 2056), (7, 4096),
                                 (3, 4097), (130, 520), (2, 8192), (2, 9001), (1, 16384), (2, 32768), (1, 32767)])
def test_norm_sizes(lm, norm, r, d):
    g = gen(r + d)
    for dtype, hdtype in ((BF, BF), (BF, F), (HF, F), (F, F)):
        h, y = randn(g, r, d, dtype=hdtype) * 3, randn(g, r, d, dtype=dtype) + 0.5
        w = [1 + 0.2 * randn(g, d) for _ in range(2)]
        b = [0.1 * randn(g, d) for _ in range(2)]
        gate = randn(g, d, dtype=dtype)
        args = dict(norm=norm, post_weight=w[0], post_bias=b[0], pre_weight=w[1], pre_bias=b[1], gate=gate, alpha=0.8,
                    beta=0.6, eps=1e-5)
        ho, x = lm.norm_residual(h, y, **args)
        wh, wx, eh, ex = ref.norm_residual(h, y, norm, True, w[0], b[0], w[1], b[1], gate, 0.8, 0.6, 1e-5)
        ref.close(ho, wh, eh, "h")
        ref.close(x, wx, ex, "x")
        assert ho.dtype is hdtype and x.dtype is dtype


@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("gates", [0, 1, 3, 12])
def test_norm_gates_and_parts(lm, post, gates):
    g = gen(gates)
    h, y = randn(g, 12, 264, dtype=BF), randn(g, 12, 264, dtype=BF)
    gate = randn(g, gates, 264, dtype=BF) if gates else None
    ho, x = lm.norm_residual(h, y, post=post, gate=gate)
    wh, wx, eh, ex = ref.norm_residual(h, y, "rms", post, None, None, None, None, gate, 1.0, 1.0, 1e-6)
    ref.close(ho, wh, eh, "h")
    ref.close(x, wx, ex, "x")
    same, x = lm.norm_residual(h, None, pre_weight=randn(gen(9), 264), norm="layer")
    assert same is h
    _, wx, _, ex = ref.norm_residual(h, None, "layer", False, None, None, randn(gen(9), 264), None, None, 1, 1, 1e-6)
    ref.close(x, wx, ex, "first norm")


def test_norm_in_place_strides_and_means(lm):
    g = gen(4)
    y = randn(g, 6, 500, dtype=BF)
    h = randn(g, 6, 500)
    wh, wx, eh, ex = ref.norm_residual(h, y, "layer", True, None, None, None, None, None, 1.0, 1.0, 1e-6)
    h2, y2 = h.clone(), y.clone()
    lm.norm_residual(h2, y2, norm="layer", h_out=h2, out=y2)
    ref.close(h2, wh, eh, "h in place")
    ref.close(y2, wx, ex, "x in place")
    wide = randn(g, 6, 512, dtype=BF)
    wide[:, :500] = y
    ho, x = lm.norm_residual(h, wide[:, :500], norm="layer")
    ref.close(x, wx, ex, "strided")
    # a mean that is far larger than the deviation
    h = 1000 + randn(g, 3, 2048)
    _, x = lm.norm_residual(h, None, norm="layer")
    _, wx, _, ex = ref.norm_residual(h, None, "layer", False, None, None, None, None, None, 1, 1, 1e-6)
    ref.close(x, wx, ex, "large mean")
    # rows of zeros, and of infinities beside sound ones
    h = randn(g, 3, 256)
    h[0] = 0
    h[1, 3] = math.inf
    _, x = lm.norm_residual(h, None)
    assert not bool(x[0].any()) and not bool(torch.isfinite(x[1, 3]))
    _, wx, _, ex = ref.norm_residual(h[2:], None, "rms", False, None, None, None, None, None, 1, 1, 1e-6)
    ref.close(x[2:], wx, ex, "row beside")
    a, b = lm.norm_residual(h[:0], h[:0])
    assert a.shape == b.shape == (0, 256)


def make_cache(lm, g, pages, heads, page, dim, bits, dtype, permuted=False):
    """Random codes and scales; `permuted`: a view of [pages, page, heads, dim]."""
    width = dim if bits == 16 else dim * bits // 8
    shape = (pages, page, heads, width) if permuted else (pages, heads, page, width)
    if bits == 16:
        k, v = randn(g, *shape, dtype=dtype), randn(g, *shape, dtype=dtype)
        s = (None, None)
    else:
        k, v = (torch.randint(0, 256, shape, generator=g, device="cuda", dtype=torch.uint8) for _ in range(2))
        s = [(0.5 + torch.rand((pages, heads, page), generator=g, device="cuda")) / (70 if bits == 8 else 4.5)
             for _ in range(2)]
    if permuted:
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    return lm.Cache(k, v, s[0], s[1], bits)


def words(mask, t):
    """Lists of seen drafts -> int64 words [b, t, ceil(t / 64)]."""
    n = (t + 63) // 64
    out = []
    for rows in mask:
        for row in rows:
            w = [0] * n
            for j in row:
                w[j // 64] |= 1 << (j % 64)
            out.append([x - (1 << 64) if x >> 63 else x for x in w])
    return torch.tensor(out, dtype=torch.int64, device="cuda").reshape(len(mask), t, n)


def random_mask(rng, b, t):
    """Trees, with a few rows that see nothing and a few that do not see themselves."""
    out = []
    for _ in range(b):
        rows = []
        for i in range(t):
            kind = rng.random()
            if kind < 0.1:
                rows.append([])
            else:
                up = rows[rng.randrange(i)] if i and kind < 0.8 else []
                rows.append(up + ([i] if kind < 0.9 else []))
        out.append(rows)
    return out


def check_attention(lm, g, b, t, heads, hk, dim, page, bits, dtype, lens, counts, mask, permuted=False, scale=None,
                    extra=0):
    width = max(1, -(-(max(max(lens), 0) + t) // page) + extra)
    pages = b * width + 1
    cache = make_cache(lm, g, pages, hk, page, dim, bits, dtype, permuted)
    table = torch.randperm(pages, generator=g, device="cuda")[:b * width].int().reshape(b, width)
    q = 1.5 * randn(g, b, t, heads, dim, dtype=dtype)
    il = torch.tensor(lens, dtype=torch.int32, device="cuda")
    ic = None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda")
    out, lse = lm.tree_attention(q, cache, table, il, mask=None if mask is None else words(mask, t), counts=ic,
                                 scale=scale, want_lse=True)
    wo, wl, eo, el = ref.attention(q, cache, table, lens, mask, counts, dim ** -0.5 if scale is None else scale)
    ref.close(lse, wl, el, "lse")
    ref.close(out, wo, eo, "out")
    return q, cache, table, il, ic, out


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_attention_types(lm, bits, dim, dtype):
    import random
    rng = random.Random(bits + dim)
    check_attention(lm, gen(1), 2, 5, 4, 2, dim, 16, bits, dtype, [70, 3], [5, 4], random_mask(rng, 2, 5))
    check_attention(lm, gen(2), 1, 1, 3, 1, dim, 64, bits, dtype, [300], None, None)
    check_attention(lm, gen(3), 1, 20, 4, 1, dim, 32, bits, dtype, [45], None, random_mask(rng, 1, 20), permuted=True)


@pytest.mark.parametrize("t,heads,hk", [(1, 1, 1), (1, 8, 8), (1, 32, 4), (3, 5, 1), (16, 2, 2), (17, 3, 3), (33, 4, 2),
                                        (63, 2, 1), (64, 1, 1), (65, 2, 1), (130, 1, 1), (9, 16, 1)])
@pytest.mark.parametrize("masked", [False, True])
def test_attention_rows(lm, t, heads, hk, masked):
    import random
    rng = random.Random(t)
    mask = random_mask(rng, 2, t) if masked else None
    check_attention(lm, gen(t), 2, t, heads, hk, 64, 16, 8, BF, [40, 0], [t, max(1, t - 2)], mask)


@pytest.mark.parametrize("page", [1, 3, 7, 16, 31, 33, 64, 100, 128])
def test_attention_pages(lm, page):
    """Pages that end inside a tile, of any size."""
    check_attention(lm, gen(page), 2, 4, 4, 2, 64, page, 8, BF, [95, 130], None, None)
    check_attention(lm, gen(page), 1, 2, 2, 1, 128, page, 16, HF, [129], None, [[[0], []]])


@pytest.mark.parametrize("lens", [[0], [1], [31], [32], [33], [127], [128], [129], [1000], [5000]])
@pytest.mark.parametrize("bits", [16, 8])
def test_attention_lengths(lm, lens, bits):
    check_attention(lm, gen(lens[0]), 1, 1, 4, 2, 128, 32, bits, BF, lens, None, None)
    check_attention(lm, gen(lens[0]), 1, 6, 4, 2, 64, 32, bits, HF, lens, [4], [[[]] * 6])


def test_attention_many_splits_and_sequences(lm):
    """Long caches in pieces, tables that reach further than the lengths, sequences of every length."""
    check_attention(lm, gen(1), 1, 2, 2, 1, 64, 64, 4, BF, [20000], None, None, extra=5)
    check_attention(lm, gen(2), 6, 3, 2, 1, 64, 16, 8, HF, [0, 1, 17, 600, 1500, 64], [3, 0, 1, 2, 3, 3], None, extra=40)


def test_attention_large_scores_and_tiny_values(lm):
    """Scores far apart, and scales of values from 1e-7 to 1e4 side by side: f16 keeps their digits."""
    g = gen(5)
    for bits in (8, 4):
        for dtype in (BF, HF):
            cache = make_cache(lm, g, 9, 1, 16, 64, bits, dtype)
            for factor in (1e-7, 1e-4, 1.0):
                c = cache._replace(v_scale=cache.v_scale * factor, k_scale=cache.k_scale * 4)
                q = 2 * randn(g, 1, 2, 2, 64, dtype=dtype)
                table = torch.arange(9, device="cuda", dtype=torch.int32).reshape(1, 9)
                out, lse = lm.tree_attention(q, c, table, torch.tensor([140], dtype=torch.int32, device="cuda"),
                                             want_lse=True)
                wo, wl, eo, el = ref.attention(q, c, table, [140], None, None, 64 ** -0.5)
                ref.close(lse, wl, el, "lse")
                # (results below f16's normal range are rounded to 2^-25)
                ref.close(out, wo, eo + (2.0 ** -25 if dtype is HF else 0), "out")


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_attention_ignores_what_is_not_seen(lm, bits, dtype):
    """Slots past the end, drafts that a row does not see and pages that do not exist: NaN and infinities there
    change nothing."""
    g = gen(6)
    t, n = 6, 37
    mask = [[[0], [0, 1], [2], [], [0, 4], [5]]]
    cache = make_cache(lm, g, 5, 2, 16, 64, bits, dtype)
    table = torch.tensor([[3, 0, 4, 1]], dtype=torch.int32, device="cuda")
    q = randn(g, 1, t, 4, 64, dtype=dtype)
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    counts = torch.tensor([5], dtype=torch.int32, device="cuda")
    base, lse0 = lm.tree_attention(q, cache, table, lens, mask=words(mask, t), counts=counts, want_lse=True)
    assert not bool(base[0, 5].any()) and bool(torch.isneginf(lse0[0, 5]).all())

    def spoil(pos, what):
        page, slot = int(table[0, pos // 16]), pos % 16
        if bits == 16:
            k[page, :, slot], v[page, :, slot] = what, what
        else:
            ks[page, :, slot], vs[page, :, slot] = what, what

    k, v = cache.k.clone(), cache.v.clone()
    ks, vs = (None, None) if bits == 16 else (cache.k_scale.clone(), cache.v_scale.clone())
    for what, pos in ((math.nan, n + 5), (math.inf, n + 6), (math.nan, 60)):  # at and past the count
        spoil(pos, what)
    k[2], v[2] = 0, 0
    spoiled = lm.Cache(k, v, ks, vs, bits)
    out, lse = lm.tree_attention(q, spoiled, table, lens, mask=words(mask, t), counts=counts, want_lse=True)
    assert torch.equal(out, base) and torch.equal(lse, lse0)
    # draft 2 is seen by itself alone: the other rows stay as they are
    spoil(n + 2, math.inf)
    out, lse = lm.tree_attention(q, spoiled, table, lens, mask=words(mask, t), counts=counts, want_lse=True)
    rows = [0, 1, 3, 4, 5]
    assert torch.equal(lse[:, rows], lse0[:, rows])
    # (rows beside an infinite value may be summed in another order)
    d = (out[:, rows].double() - base[:, rows].double()).abs().max()
    assert float(d) <= 8 * ref.U[dtype] * float(base[:, rows].abs().max())
    assert not bool(torch.isfinite(out[0, 2]).all())


def test_attention_bad_tables_and_lengths(lm):
    """Page numbers outside of the cache, lengths past the table, negative lengths: those positions are not there."""
    g = gen(7)
    cache = make_cache(lm, g, 4, 1, 16, 64, 8, BF)
    q = randn(g, 4, 2, 2, 64, dtype=BF)
    table = torch.tensor([[0, 99, 1], [0, 1, 2], [0, -1, 2], [3, 2, 1]], dtype=torch.int32, device="cuda")
    lens = [40, 1000, 20, -5]
    out, lse = lm.tree_attention(q, cache, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), want_lse=True)
    wo, wl, eo, el = ref.attention(q, cache, table, lens, None, None, 64 ** -0.5)
    ref.close(lse, wl, el, "lse")
    ref.close(out, wo, eo, "out")


def test_attention_strided_queries(lm):
    """Queries that are a slice of a projection's output."""
    g = gen(8)
    qkv = randn(g, 3, 4, (4 + 2 + 2) * 64, dtype=BF)
    q = qkv[..., :256].unflatten(-1, (4, 64))
    cache = make_cache(lm, g, 12, 2, 16, 64, 8, BF)
    table = torch.arange(12, device="cuda", dtype=torch.int32).reshape(3, 4)
    lens = torch.tensor([9, 33, 50], dtype=torch.int32, device="cuda")
    out = lm.tree_attention(q, cache, table, lens)
    assert torch.equal(out, lm.tree_attention(q.contiguous(), cache, table, lens))
    wo, _, eo, _ = ref.attention(q, cache, table, [9, 33, 50], None, None, 0.125)
    ref.close(out, wo, eo, "strided")


def codes_of(cache, which):
    p = getattr(cache, which)
    return p if cache.bits == 16 else ref.values(p, cache.bits).long()


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("permuted", [False, True])
def test_cache_append_and_read(lm, bits, dim, dtype, permuted):
    g = gen(bits + dim)
    b, t, heads, page, width = 3, 9, 2, 7, 5
    cache = make_cache(lm, g, 20, heads, page, dim, bits, dtype, permuted)
    table = torch.randperm(20, generator=g, device="cuda")[:15].int().reshape(b, width)
    kv = randn(g, b, t, 2, heads, dim, dtype=dtype)
    kv[0, 0] = 0
    kv[1, 2, 0, 1, 5] = math.nan
    kv[1, 3, 1, 0, 6] = -math.inf
    kv[2, 1] *= 1e-3
    k, v = kv[:, :, 0], kv[:, :, 1]
    lens, counts = [0, 13, 29], [9, 7, 9]  # the last sequence runs past its table
    il, ic = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (lens, counts))
    want = {}
    for which, new in (("k", k), ("v", v)):
        pages = getattr(cache, which).clone()
        scales = None if bits == 16 else getattr(cache, which + "_scale").clone()
        for i in range(b):
            for j in range(counts[i]):
                pos = lens[i] + j
                if pos >= width * page:
                    continue
                at = (int(table[i, pos // page]), slice(None), pos % page)
                if bits == 16:
                    pages[at] = new[i, j]
                else:
                    code, scale = ref.quantize(new[i, j], bits)
                    pages[at] = ref.pack((code & ((1 << bits) - 1)).to(torch.uint8), bits).cuda()
                    scales[at] = scale.cuda()
        want[which] = (pages, scales)
    lm.cache_append(k, v, cache, table, il, counts=ic)
    for which in "kv":
        pages, scales = want[which]
        assert torch.equal(torch.nan_to_num(getattr(cache, which).float(), 7.0, 8.0, 9.0), torch.nan_to_num(pages.float(), 7.0, 8.0, 9.0)), which
        if bits != 16:
            assert torch.equal(torch.nan_to_num(getattr(cache, which + "_scale"), -1.0), torch.nan_to_num(scales, -1.0))
    # back as numbers: code times scale in 32 bits, rounded once; zeros past the table
    for out_type in (BF, HF, F):
        got = lm.cache_read(cache, table, il, t + 1, out_type)
        for which, x in zip("kv", got):
            full = getattr(cache, which).float() if bits == 16 else (
                codes_of(cache, which).float() * getattr(cache, which + "_scale").unsqueeze(-1))
            for i in range(b):
                for j in range(t + 1):
                    pos = lens[i] + j
                    w = torch.zeros(heads, dim, device="cuda") if pos >= width * page else (
                        full[int(table[i, pos // page]), :, pos % page])
                    assert torch.equal(torch.nan_to_num(x[i, j].float(), 7.0, 8.0, 9.0),
                                       torch.nan_to_num(w.to(out_type).float(), 7.0, 8.0, 9.0))


@pytest.mark.parametrize("bits,dim", [(16, 64), (16, 256), (8, 64), (8, 128), (4, 64), (4, 256)])
@pytest.mark.parametrize("t", [1, 5, 64, 200])
def test_cache_keep(lm, bits, dim, t):
    import random
    rng = random.Random(t)
    g = gen(t + bits)
    b, heads, page = 4, 2, 16
    width = -(-(40 + t) // page)
    cache = make_cache(lm, g, b * width, heads, page, dim, bits, BF, permuted=t % 2 == 0)
    table = torch.randperm(b * width, generator=g, device="cuda").int().reshape(b, width)
    lens = [0, 17, 40, 33]
    kept = [0, t, max(1, t // 2), max(1, t // 3)]
    path = [sorted(rng.sample(range(t), n)) + [0] * (t - n) for n in kept]
    names = ["k", "v"] + ([] if bits == 16 else ["k_scale", "v_scale"])
    want = {}
    for which in names:
        new, old = getattr(cache, which).clone(), getattr(cache, which).clone()
        for i in range(b):
            for j in range(kept[i]):
                to, fr = lens[i] + j, lens[i] + path[i][j]
                new[int(table[i, to // page]), :, to % page] = old[int(table[i, fr // page]), :, fr % page]
        want[which] = new
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    lm.cache_keep(cache, table, i32(lens), i32(path), i32(kept))
    for which in names:
        assert torch.equal(getattr(cache, which), want[which]), which
    # entries that do not ascend or lie outside move nothing
    lm.cache_keep(cache, table, i32(lens), i32([[0] * t, [-7] * t, [t] * t, [1 << 30] * t]), i32([t, t, t, 1 << 30]))
    for which in names:
        assert torch.equal(getattr(cache, which), want[which]), which


def test_offsets_past_32_bits(lm):
    """A cache of more than 4 GiB, and rows of x more than 2^32 bytes apart."""
    pages, page = 70000, 64  # 70000 * 64 * 2 * 256 * ... bytes
    k = torch.zeros((pages, 1, page, 1024), dtype=torch.uint8, device="cuda")[..., :128]
    v = torch.zeros((pages, 1, page, 1024), dtype=torch.uint8, device="cuda")[..., :128]
    ks, vs = torch.zeros((pages, 1, page), device="cuda"), torch.zeros((pages, 1, page), device="cuda")
    cache = lm.Cache(k, v, ks, vs, 8)
    assert k.stride(0) * (pages - 1) > 1 << 32
    g = gen(1)
    table = torch.tensor([[pages - 1, 3, pages - 2]], dtype=torch.int32, device="cuda")
    new = randn(g, 1, 150, 1, 128, dtype=BF)
    zero, n = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.tensor([149], dtype=torch.int32, device="cuda")
    lm.cache_append(new, new, cache, table, zero)
    got, _ = lm.cache_read(cache, table, zero, 150, F)
    code, scale = ref.quantize(new[0], 8)
    assert torch.equal(got[0].cpu(), code.float() * scale.unsqueeze(-1))
    q = randn(g, 1, 1, 2, 128, dtype=BF)
    out, lse = lm.tree_attention(q, cache, table, n, want_lse=True)
    small = lm.Cache(k[[pages - 1, 3, pages - 2]].contiguous(), v[[pages - 1, 3, pages - 2]].contiguous(),
                     ks[[pages - 1, 3, pages - 2]].contiguous(), vs[[pages - 1, 3, pages - 2]].contiguous(), 8)
    order = torch.arange(3, device="cuda", dtype=torch.int32).reshape(1, 3)
    wo, wl, eo, el = ref.attention(q, small, order, [149], None, None, 128 ** -0.5)
    ref.close(out, wo, eo, "out")
    ref.close(lse, wl, el, "lse")


def pass_through(lm, s, stream=None):
    """One call of each operator on the state s."""
    y = lm.matmul(s["x"], s["w"], 4, scale=s["scale"], stream=stream)
    h, x = lm.norm_residual(s["x"], s["x"], stream=stream)
    lm.cache_append(s["k"], s["k"], s["cache"], s["table"], s["lens"], stream=stream)
    o = lm.tree_attention(s["q"], s["cache"], s["table"], s["lens"], stream=stream)
    lm.cache_keep(s["cache"], s["table"], s["lens"], s["path"], s["kept"], stream=stream)
    k, v = lm.cache_read(s["cache"], s["table"], s["lens"], 4, stream=stream)
    return [y, h, x, o, k, v]


def state(lm, seed):
    g = gen(seed)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    L = layer(g, 40, 512, 256, 4, 128, BF)
    return dict(L, k=randn(g, 2, 4, 2, 64, dtype=BF), q=randn(g, 2, 4, 8, 64, dtype=BF),
                cache=make_cache(lm, g, 64, 2, 64, 64, 8, BF),
                table=torch.randperm(64, generator=g, device="cuda").int().reshape(2, 32), lens=i32([1900, 77]),
                path=i32([[0, 2, 3, 0], [1, 3, 0, 0]]), kept=i32([3, 2]))


def test_same_call_same_bits(lm):
    for seed in range(3):
        a, b = pass_through(lm, state(lm, seed)), pass_through(lm, state(lm, seed))
        for x, y in zip(a, b):
            assert torch.equal(x, y)


def test_other_streams(lm):
    want = pass_through(lm, state(lm, 1))
    s = state(lm, 1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = pass_through(lm, s, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for x, y in zip(got, want):
        assert torch.equal(x, y)
    s = state(lm, 1)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = pass_through(lm, s)
    torch.cuda.current_stream().wait_stream(side)
    for x, y in zip(got, want):
        assert torch.equal(x, y)


def test_graph_replays(lm):
    """Captured once, replayed with new inputs, with eager work between the replays."""
    s = state(lm, 0)
    warm = torch.cuda.Stream()
    warm.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(warm):
        pass_through(lm, state(lm, 0))
    torch.cuda.current_stream().wait_stream(warm)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = pass_through(lm, s)
    for seed in (3, 4, 5):
        new = state(lm, seed)
        for name in ("x", "w", "scale", "k", "q", "table", "lens", "path", "kept"):
            s[name].copy_(new[name])
        for a, b in zip(s["cache"][:4], new["cache"][:4]):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        want = pass_through(lm, new)
        for x, y in zip(out, want):
            assert torch.equal(x, y)


@pytest.mark.parametrize("bits", [8, 4, 2, 1])
@pytest.mark.parametrize("r", [2, 50, 140])
def test_matmul_zero_and_uneven_scales(lm, bits, r):
    """Groups whose scale is zero, first, last and in a row, and groups of very different scales."""
    g = gen(bits)
    for group in (32, 64, 128):
        L = layer(g, r, 1280, 150, bits, group, BF)
        s = L["scale"]
        s *= 10.0 ** torch.randint(-6, 7, s.shape, generator=g, device="cuda")
        s[torch.rand(s.shape, generator=g, device="cuda") < 0.3] = 0
        s[3], s[4, :-1], s[5, 1:] = 0, 0, 0
        s[6, 1] = -s[6, 1]
        s[7, 0] = 1e-42  # no normal number
        check_matmul(lm, L, bits)


@pytest.mark.parametrize("bits", [8, 4, 2, 1])
@pytest.mark.parametrize("r", [3, 20, 70, 300])
def test_matmul_scales_of_empty_groups(lm, bits, r):
    """Groups that a quantizer gave the smallest scale there is, beside ordinary ones: nothing passes fp32."""
    g = gen(bits + r)
    for group in (32, 64, 128):
        for tiny in (torch.finfo(torch.float32).tiny, 1e-45, 1e-30):
            L = layer(g, r, 1280, 150, bits, group, BF)
            L["x"] *= 1000
            s = L["scale"]
            empty = torch.rand(s.shape, generator=g, device="cuda") < 0.4
            empty[:, 2], empty[3, -1], empty[4, 0] = False, False, False  # (the results are normal numbers)
            s[empty] = tiny
            s[3, :-1], s[4, 1:] = tiny, tiny
            s[6, 0], s[6, 1] = 0, tiny
            s[7] = 10.0 ** -torch.arange(s.shape[1], device="cuda")  # down by tens
            check_matmul(lm, L, bits)
