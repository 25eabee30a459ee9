"""The operators of include/qnn_lm.h where numbers are not ordinary: NaN and
infinities, scales far apart or negative, places that a call must not look at.
Against the formulas in 64 bits (lm_reference.py), with its bounds."""
import math

import pytest
import torch

import lm_reference as ref
from test_lm_gpu import lm, gen, randn, make_cache, words, layer  # noqa: F401

pytestmark = pytest.mark.gpu

BF, HF, F = torch.bfloat16, torch.float16, torch.float32
ROWS = [(1, 4), (5, 4), (20, 2), (40, 2)]  # drafts and query heads of a cache head: few rows to many


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def check(lm, q, cache, table, lens, mask=None, extra=0.0):
    t = q.shape[1]
    out, lse = lm.tree_attention(q, cache, table, i32(lens), mask=None if mask is None else words(mask, t), want_lse=True)
    wo, wl, eo, el = ref.attention(q, cache, table, lens, mask, None, q.shape[-1] ** -0.5)
    ref.close(lse, wl, el, "lse")
    ref.close(out, wo, eo + extra, "out")
    return out, lse


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("t,g", [(5, 4), (20, 1), (9, 8)])
def test_scales_of_other_sequences(lm, bits, t, g):
    """A scale that belongs to no position of the sequence (the cache's very first place, on a page that the table does
    not name) changes no bit, whatever it holds."""
    for dim in (256, 128, 64):
        r = gen(dim + t)
        cache = make_cache(lm, r, 8, 1, 32, dim, bits, BF)
        table = i32([[3, 5, 1, 7]])
        q = randn(r, 1, t, g, dim, dtype=BF)
        base = lm.tree_attention(q, cache, table, i32([96 - t]), want_lse=True)
        for huge in (1e6, 1e12, 1e30, math.inf, math.nan):
            vs, ks = cache.v_scale.clone(), cache.k_scale.clone()
            vs[0, 0, 0] = ks[0, 0, 0] = huge
            got = lm.tree_attention(q, cache._replace(v_scale=vs, k_scale=ks), table, i32([96 - t]), want_lse=True)
            assert torch.equal(got[0], base[0]) and torch.equal(got[1], base[1]), (dim, huge)


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("t,g", ROWS)
@pytest.mark.parametrize("n", [20, 3000])
def test_nan_queries(lm, bits, t, g, n):
    """A query that holds NaN gives NaN, the rows beside it what they always give."""
    r = gen(t + g + n)
    page = 64
    width = -(-(n + t) // page)
    for dim, dtype in ((64, BF), (128, HF), (256, BF)):
        cache = make_cache(lm, r, width, 1, page, dim, bits, dtype)
        q = randn(r, 1, t, g, dim, dtype=dtype)
        q[0, 0, 0, 5] = math.nan
        q[0, t - 1, g - 1, dim - 1] = math.nan
        out, lse = check(lm, q, cache, torch.arange(width, device="cuda", dtype=torch.int32).reshape(1, width), [n])
        assert bool(out[0, 0, 0].isnan().all()) and bool(lse[0, 0, 0].isnan())


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("t,g", ROWS)
def test_nan_keys(lm, bits, t, g):
    """Keys that are NaN: all that a draft sees, or a stretch of a long cache that one wave or one piece has to itself."""
    for dim, dtype in ((128, BF), (64, HF)):
        r = gen(t + g + dim)
        page = 32
        width = -(-(3000 + t) // page)
        table = torch.randperm(width, generator=r, device="cuda").int().reshape(1, width)
        q = randn(r, 1, t, g, dim, dtype=dtype)

        def spoiled(cache, positions):
            k, ks = cache.k.clone(), None if bits == 16 else cache.k_scale.clone()
            for pos in positions:
                pg, slot = int(table[0, pos // page]), pos % page
                if bits == 16:
                    k[pg, :, slot] = math.nan
                else:
                    ks[pg, :, slot] = math.nan
            return cache._replace(k=k, k_scale=ks)

        cache = make_cache(lm, r, width, 1, page, dim, bits, dtype)
        # an empty cache: draft 0 sees its own key alone
        out, _ = check(lm, q, spoiled(cache, [0]), table, [0])
        assert bool(out.isnan().all())
        mask = [[[0] if i == 0 else [i] for i in range(t)]]
        out, _ = check(lm, q, spoiled(cache, [0]), table, [0], mask)
        assert bool(out[0, 0].isnan().all()) and not bool(out[0, 1:].isnan().any())
        for first, last in ((0, 32), (96, 128), (128, 256), (2944, 3000)):
            out, _ = check(lm, q, spoiled(cache, range(first, last)), table, [3000])
            assert bool(out.isnan().all()), first


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("t,g", ROWS)
@pytest.mark.parametrize("low", [False, True])
def test_infinite_values(lm, dtype, t, g, low):
    """Infinite values of cached tokens, in tiles that every row sees whole: infinities of their sign, NaN where both
    signs meet, the other channels as ever; also where such a token's probability is below the smallest 16-bit number."""
    for dim in (64, 128, 256):
        for n in (200, 2000):
            r = gen(t + dim)
            page = 16
            width = -(-(n + t) // page)
            table = torch.randperm(width, generator=r, device="cuda").int().reshape(1, width)
            cache = make_cache(lm, r, width, 1, page, dim, 16, dtype)
            base = randn(r, dim)
            q = (base + 0.1 * randn(r, 1, t, g, dim)).to(dtype)
            for pos, channel, what in ((70, 3, math.inf), (90, 5, -math.inf), (71, 7, math.inf), (140, 7, -math.inf),
                                       (n - 1, 9, math.inf)):
                pg, slot = int(table[0, pos // page]), pos % page
                cache.v[pg, 0, slot, channel] = what
                if low:
                    # scores about 50 below the others'
                    cache.k[pg, 0, slot] = (base * (-50 * dim ** 0.5 / float(base @ base))).to(dtype)
            out, _ = check(lm, q, cache, table, [n])
            assert bool(out[..., 3].isposinf().all()) and bool(out[..., 5].isneginf().all())
            assert bool(out[..., 7].isnan().all()) and bool(out[..., 9].isposinf().all())


@pytest.mark.parametrize("t,g", ROWS)
def test_infinite_values_far_below(lm, t, g):
    """An infinite value in a stretch of positions whose scores all lie 100 below the others': no factor between parts
    of the positions makes zero of it."""
    for dim in (64, 128, 256):
        for n in (200, 2000):
            r = gen(t + dim)
            page = 32
            width = -(-(n + t) // page)
            cache = make_cache(lm, r, width, 1, page, dim, 16, BF)
            base = randn(r, dim)
            q = (base + 0.1 * randn(r, 1, t, g, dim)).to(BF)
            cache.k[1:5, 0] = (base * (-100 * dim ** 0.5 / float(base @ base))).to(BF)
            cache.v[2, 0, 9, 3] = math.inf
            out, _ = check(lm, q, cache, torch.arange(width, device="cuda", dtype=torch.int32).reshape(1, width), [n])
            assert bool(out[..., 3].isposinf().all())


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("t,g", ROWS)
def test_infinite_scales(lm, bits, t, g):
    """A value's scale that is infinite: infinities of the codes' signs, NaN for code zero."""
    for dim, dtype in ((64, HF), (128, BF), (256, BF)):
        for n in (150, 2000):
            r = gen(t + dim)
            page = 16
            width = -(-(n + t) // page)
            table = torch.randperm(width, generator=r, device="cuda").int().reshape(1, width)
            cache = make_cache(lm, r, width, 1, page, dim, bits, dtype)
            cache.v_scale[int(table[0, 5]), 0, 3] = math.inf
            q = randn(r, 1, t, g, dim, dtype=dtype)
            out, _ = check(lm, q, cache, table, [n])
            assert bool((~torch.isfinite(out)).all())


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("t,g", ROWS)
@pytest.mark.parametrize("n", [20, 1000])
def test_negative_scales(lm, bits, t, g, n):
    for dim, dtype in ((64, BF), (128, HF), (256, HF)):
        r = gen(t + dim)
        page = 16
        width = -(-(n + t) // page)
        table = torch.randperm(width, generator=r, device="cuda").int().reshape(1, width)
        cache = make_cache(lm, r, width, 1, page, dim, bits, dtype)
        q = randn(r, 1, t, g, dim, dtype=dtype)
        for sign in (-1.0, None):
            for s in (cache.k_scale, cache.v_scale):
                s *= sign or torch.where(randn(r, *s.shape) < 0, -1.0, 1.0)
            check(lm, q, cache, table, [n])


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("t,g", ROWS)
@pytest.mark.parametrize("n", [20, 1000])
def test_scales_far_apart(lm, bits, t, g, n):
    """Values' scales from 1e-9 to 1e9 side by side, seen by every row, with scores that favour small and large ones."""
    for dim in (64, 128, 256):
        r = gen(t + dim)
        page = 16
        width = -(-(n + t) // page)
        table = torch.randperm(width, generator=r, device="cuda").int().reshape(1, width)
        cache = make_cache(lm, r, width, 1, page, dim, bits, BF)
        base = randn(r, dim)
        q = (base + 0.1 * randn(r, 1, t, g, dim)).to(BF)
        check(lm, q, cache._replace(v_scale=cache.v_scale * 10.0 ** (18 * torch.rand(cache.v_scale.shape, generator=r, device="cuda") - 9)),
              table, [n])
        # one token far larger than the others, whose probability makes it smaller than they are: early, then late
        for pos in (3, n - 2):
            pg, slot = int(table[0, pos // page]), pos % page
            for gap, scale in ((30, 1e6), (45, 1e10), (60, 1e18)):
                most = 127 if bits == 8 else 7
                want = base * (-gap * dim ** 0.5 / float(base @ base))
                code, ks = ref.quantize(want, bits)
                k, s, v = cache.k.clone(), cache.k_scale.clone(), cache.v_scale.clone()
                k[pg, 0, slot] = ref.pack((code & (2 * most + 1)).to(torch.uint8), bits).cuda()
                s[pg, 0, slot] = float(ks)
                v[pg, 0, slot] = scale
                check(lm, q, cache._replace(k=k, k_scale=s, v_scale=v), table, [n])


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("t,g", ROWS)
@pytest.mark.parametrize("n", [0, 20, 1000])
def test_large_scales_of_unseen_drafts(lm, bits, t, g, n):
    """A draft whose values are far larger than all others, and that few rows or none see: the others do not change by
    more than sums in another order do."""
    if t < 2:
        return
    for dim in (64, 128, 256):
        r = gen(t + dim)
        page = 16
        width = -(-(n + t) // page)
        table = torch.randperm(width, generator=r, device="cuda").int().reshape(1, width)
        cache = make_cache(lm, r, width, 1, page, dim, bits, BF)
        q = randn(r, 1, t, g, dim, dtype=BF)
        for seen in (True, False):
            mask = [[[j for j in range(i + 1) if j != 1 or (seen and i == 1)] for i in range(t)]]
            pos = n + 1
            for huge in (1e6, 1e12, 1e30):
                v = cache.v_scale.clone()
                v[int(table[0, pos // page]), 0, pos % page] = huge
                check(lm, q, cache._replace(v_scale=v), table, [n], mask)


@pytest.mark.parametrize("bits", [8, 4, 2, 1])
@pytest.mark.parametrize("r", [5, 24, 70, 300])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_group_scales_in_any_order(lm, bits, r, group):
    """Scales more than 2^60 apart, the large one first, last or between, where x is zero in the columns of the large
    one; and numbers of x that bring a group's sums near the end of 32 bits."""
    for gated in (False, True):
        g = gen(bits + r)
        L = layer(g, r, 1280, 150, bits, group, BF, gated)
        n = 1280 // group
        for at in (0, n // 2, n - 1):
            x, s = L["x"].clone(), torch.full_like(L["scale"], 2.0 ** -75)
            s[:, at] = 1.0
            x[:, at * group:(at + 1) * group] = 0
            if r > 1:
                x[1] = L["x"][1]  # one row that the large group counts for
            act = "relu" if gated else "none"
            y = lm.matmul(x, L["w"], bits, scale=s, act=act, gated=gated)
            want, bound = ref.matmul(x, L["w"], bits, s, None, act, gated)
            ref.close(y, want, bound, "at %d" % at)
            if gated:
                continue
            x, s = L["x"].clone(), torch.full_like(L["scale"], 2.0 ** -58)
            s[:, at] = 1.0
            x[:, at * group:(at + 1) * group] *= 1e25
            y = lm.matmul(x, L["w"], bits, scale=s)
            want, bound = ref.matmul(x, L["w"], bits, s)
            ref.close(y, want, bound, "large x at %d" % at)


@pytest.mark.parametrize("bits,group", [(8, 128), (4, 64), (4, 32), (2, 128), (1, 32)])
@pytest.mark.parametrize("r", [2033, 1003])
def test_group_scales_in_large_tiles(lm, bits, group, r):
    """The same in tiles of 128 x 256 and of 64 x 256: a few rows of weights, and a few of x, are the odd ones."""
    g = gen(bits + r)
    L = layer(g, r, 512, 8001, bits, group, BF)
    x, s = L["x"], L["scale"]
    s[1000] = 2.0 ** -75
    s[1000, -1], s[4000, 0] = 1.0, 2.0 ** 70
    x[7, 512 - group:] = 0
    x[:4, :group] = 0
    x[11, :group] *= 1e25
    want, bound = ref.matmul(x, L["w"], bits, s)
    # (row 4000's results for the large x pass the type)
    most = torch.finfo(BF).max * (1 + 2.0 ** -9)
    want = torch.where(want.abs() >= most, want.sign() * math.inf, want)
    ref.close(lm.matmul(x, L["w"], bits, scale=s), want, bound, "large tiles")
    # rows of nothing but the smallest scale and codes of zero (the lowest codes at one bit) in every second group
    if bits > 1:
        s = torch.full_like(s, 2.0 ** -4)
        s[:, ::2] = 1e-45
        w = L["w"].reshape(8001, -1, group * bits // 8).clone()
        w[:, ::2] = 0
        w = w.reshape(8001, -1)
        ref.close(lm.matmul(L["x"], w, bits, scale=s), *ref.matmul(L["x"], w, bits, s), "empty groups")
