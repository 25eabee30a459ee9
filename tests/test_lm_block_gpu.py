"""The block's operators together, as a serving program runs them
(network.tree_step, network.accept_path)."""
import math
import random

import pytest
import torch

import lm_reference as ref

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32
D, HEADS, KV, DIM, FF = 256, 8, 2, 64, 320


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def layer(g, rows, k, bits, group):
    if bits == 16:
        return dict(w=(torch.randn((rows, k), generator=g, device="cuda") / math.sqrt(k)).to(BF), bits=16)
    w = torch.randint(0, 256, (rows, k * bits // 8), generator=g, device="cuda", dtype=torch.uint8)
    shape = (rows, k // group) if group else (rows,)
    rms = {8: 73.9, 4: 4.6, 2: 1.2, 1: 1.0}[bits]
    return dict(w=w, bits=bits, scale=(0.5 + torch.rand(shape, generator=g, device="cuda")) / (rms * math.sqrt(k)))


def make_block(g, bits, post=True):
    weight = lambda: 1 + 0.1 * torch.randn(D, generator=g, device="cuda")  # noqa: E731
    return dict(heads=HEADS, kv_heads=KV, dim=DIM, act="silu", norm="rms", eps=1e-6, alpha=1.0, beta=0.5,
                qkv=layer(g, (HEADS + 2 * KV) * DIM, D, bits, 64), out=layer(g, D, HEADS * DIM, bits, 128),
                up=layer(g, 2 * FF, D, bits, 0), down=layer(g, D, FF, bits, 32),
                attn_norm=weight() if post else None, mlp_norm=weight() if post else None, mid_norm=weight(),
                next_norm=weight())


def make(seed, bits, cache_bits, blocks, b, longest, page=16, post=True):
    from paper_1908_11263_amd import lm
    g = gen(seed)
    width = -(-longest // page)
    caches = [lm.make_cache(b * width, KV, page, DIM, cache_bits) for _ in range(blocks)]
    table = torch.randperm(b * width, generator=g, device="cuda").int().reshape(b, width)
    return g, [make_block(g, bits, post) for _ in range(blocks)], caches, table


def words(mask, t):
    out = torch.zeros(len(mask), t, (t + 63) // 64, dtype=torch.int64)
    for i, rows in enumerate(mask):
        for j, row in enumerate(rows):
            for k in row:
                out[i, j, k // 64] |= torch.tensor(1 << (k % 64) if k % 64 < 63 else -(1 << 63))
    return out.cuda()


def exact_layer(x, L):
    wv = L["w"].double() if L["bits"] == 16 else ref.values(L["w"], L["bits"])
    if L["bits"] != 16:
        s = L["scale"].double().reshape(wv.shape[0], -1)
        wv = wv * s.repeat_interleave(wv.shape[1] // s.shape[1], 1)
    return x @ wv.t()


def exact_block(h, x, k, b, t):
    """A block in 64 bits without a cache: the drafts are all that there is, causal."""
    qkv = exact_layer(x, k["qkv"]).reshape(b, t, HEADS + 2 * KV, DIM)
    q, key, v = qkv[:, :, :HEADS], qkv[:, :, HEADS:HEADS + KV], qkv[:, :, HEADS + KV:]
    key, v = key.repeat_interleave(HEADS // KV, 2), v.repeat_interleave(HEADS // KV, 2)
    s = torch.stack([torch.stack([q[i, :, j] @ key[i, :, j].t().contiguous() for j in range(HEADS)]) for i in range(b)])
    s = s / math.sqrt(DIM) + torch.full((t, t), -math.inf, dtype=torch.float64, device=s.device).triu(1)
    p = torch.softmax(s, -1)
    o = torch.stack([torch.stack([p[i, j] @ v[i, :, j] for j in range(HEADS)], 1) for i in range(b)])
    for y, post, pre in ((exact_layer(o.reshape(b, t, -1), k["out"]), "attn_norm", "mid_norm"), (None, "mlp_norm", "next_norm")):
        if y is None:
            u = exact_layer(x, k["up"])
            y = exact_layer(torch.nn.functional.silu(u[..., :FF]) * u[..., FF:], k["down"])
        if k[post] is not None:
            y = ref.normed(y, "rms", k[post], None, 1e-6)
        h = h + 0.5 * y
        x = ref.normed(h, "rms", k[pre], None, 1e-6)
    return h, x


@pytest.mark.parametrize("bits", [16, 8, 4, 2])
@pytest.mark.parametrize("post", [True, False])
def test_block_against_64_bits(bits, post):
    """A prompt from an empty cache of 16 bits.  The activations between the calls are rounded to 8 significant bits
    (half a unit: 2^-9 of a number) at eight places of a block, two blocks: their norm is off by 16 * 2^-8 at most, were
    all of them to point one way and each to be carried on by a factor of two."""
    from paper_1908_11263_amd import network
    b, t = 2, 37
    g, blocks, caches, table = make(bits, bits, 16, 2, b, t, post=post)
    h = torch.randn((b, t, D), generator=g, device="cuda")
    first = 1 + 0.1 * torch.randn(D, generator=g, device="cuda")
    lens = torch.zeros(b, dtype=torch.int32, device="cuda")
    gh, gx = network.tree_step(h, first, blocks, caches, table, lens, dtype=BF)
    assert gh.dtype is F and gx.dtype is BF
    wh, wx = h.double(), ref.normed(h.double(), "rms", first, None, 1e-6)
    for k in blocks:
        wh, wx = exact_block(wh, wx, k, b, t)
    for got, want in ((gh, wh), (gx, wx)):
        assert float((got.double() - want).norm() / want.norm()) < 16 * 2.0 ** -8


@pytest.mark.parametrize("cache_bits", [16, 8, 4])
@pytest.mark.parametrize("bits", [8, 4])
def test_tree_then_path(bits, cache_bits):
    """What a draft of a tree gets is what it gets alone with its ancestors, and after the accepted path has been kept
    the caches hold what they would hold had the path alone been drafted."""
    from paper_1908_11263_amd import lm, network
    rng = random.Random(cache_bits)
    b, t, prompt = 3, 12, 50
    g, blocks, caches, table = make(7, bits, cache_bits, 2, b, prompt + t)
    first = torch.ones(D, device="cuda")
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    lens = i32([prompt, prompt - 7, 20])
    network.tree_step(torch.randn((b, prompt, D), generator=g, device="cuda"), first, blocks, caches, table, i32([0] * b),
                      counts=lens, dtype=BF)
    parents = [[-1] + [rng.randrange(-1, i) for i in range(1, t)] for _ in range(b)]
    sees = []
    for row in parents:
        s = []
        for i, up in enumerate(row):
            s.append((s[up] if up >= 0 else []) + [i])
        sees.append(s)
    h = torch.randn((b, t, D), generator=g, device="cuda")
    copies = [lm.Cache(*(x.clone() if x is not None else None for x in c[:4]), c.bits) for c in caches]
    _, tree = network.tree_step(h, first, blocks, caches, table, lens, mask=words(sees, t), dtype=BF)
    # the longest path of each tree, drafted alone
    paths = [max(s, key=len) for s in sees]
    n = max(len(p) for p in paths)
    kept = i32([len(p) for p in paths])
    path = i32([p + [t - 1] * (n - len(p)) for p in paths])
    ph = torch.gather(h, 1, path.long().unsqueeze(-1).expand(b, n, D)).contiguous()
    _, alone = network.tree_step(ph, first, blocks, copies, table, lens, counts=kept, dtype=BF)
    full = i32([p + [0] * (t - len(p)) for p in paths])
    new = network.accept_path(caches, table, lens, full, kept)
    assert torch.equal(new, lens + kept)
    for i, p in enumerate(paths):
        a, c = tree[i, p].double(), alone[i, :len(p)].double()
        # sums in another order: a unit of 2^-8 here and there, in each of two blocks' sixteen roundings
        assert float((a - c).norm() / c.norm()) < 16 * 2.0 ** -9
    for x, y in zip(caches, copies):
        for i, p in enumerate(paths):
            s = new[i:i + 1] * 0
            k1, v1 = lm.cache_read(x, table[i:i + 1].contiguous(), s, int(new[i]), F)
            k2, v2 = lm.cache_read(y, table[i:i + 1].contiguous(), s, int(new[i]), F)
            for u, w in ((k1, k2), (v1, v2)):
                step = 2.0 ** -4 if cache_bits == 16 else (0.02 if cache_bits == 8 else 0.3)
                assert torch.equal(u[:, :int(lens[i])], w[:, :int(lens[i])])
                assert float((u - w).abs().max()) <= step * float(w.abs().max())
