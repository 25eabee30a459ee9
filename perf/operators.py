"""The operators of a language model's block over packed weights and a packed
cache (paper_1908_11263_amd.lm), as cases to measure.

A case is a dict of plain values; its "kind" is one of

  matmul   a linear layer: 16-bit activations times packed 8/4/2/1-bit codes
           with a scale per channel or group (or 16-bit weights), then bias,
           activation, gate and residual
  norm     norm after a block, gate, residual scale, norm before the next one
  attend   attention of a tree of drafted tokens over a paged cache
  append   new keys and values into the cache, and the values that it then
           stands for
  keep     the accepted path of the tree moved to the front, and the values
           that the cache then holds there

Where `own` is false, `run` computes them from elementary torch operations in
32 bits, rounded once at the end; where it is true, by the library's calls.

Sizes are generic ones of a serving step: hidden sizes of 1024 to 8192, heads
of 64 and 128, caches of up to 32768 tokens, trees of 1 to 64 drafted tokens.
"""
import math

import torch

own = False

_DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _mm(name, dtype, bits, group, r, k, m, act="none", gated=False, bias=False, residual=False):
    return dict(name=name, kind="matmul", dtype=dtype, bits=bits, group=group, r=r, k=k, m=m, act=act,
                gated=gated, bias=bias, residual=residual)


def _norm(name, dtype, hdtype, r, d, norm, gates, post=True):
    return dict(name=name, kind="norm", dtype=dtype, hdtype=hdtype, r=r, d=d, norm=norm, gates=gates, post=post)


def _attend(name, dtype, bits, b, t, heads, kv_heads, d, length, page, ragged):
    return dict(name=name, kind="attend", dtype=dtype, bits=bits, b=b, t=t, heads=heads, kv_heads=kv_heads, d=d,
                length=length, page=page, ragged=ragged)


def _cache(name, kind, dtype, bits, b, t, kv_heads, d, length, page):
    return dict(name=name, kind=kind, dtype=dtype, bits=bits, b=b, t=t, kv_heads=kv_heads, d=d, length=length,
                page=page)


def listed():
    return [
        # one token through one projection: nothing but the weights' bytes and the call
        _mm("matmul4_token", "bf16", 4, 128, 1, 4096, 4096, residual=True),
        # eight sequences' trees of eight drafts through the gated half of a feed-forward layer
        _mm("matmul4_tree_gated", "bf16", 4, 128, 64, 4096, 11264, act="silu", gated=True),
        # a prompt through a wide layer: sizes that fill no tile, 8-bit weights, GELU with bias
        _mm("matmul8_prompt_odd", "f16", 8, 0, 1777, 2080, 6001, act="gelu", bias=True),
        # the largest: a batch of prompts through a feed-forward layer's second half
        _mm("matmul4_prompts", "bf16", 4, 128, 4096, 11264, 4096, residual=True),
        # one token between two blocks
        _norm("norm_token", "bf16", "bf16", 1, 4096, "rms", 0),
        # a batch of prompts with a gate per sequence and a residual stream in 32 bits, a width of no power of two
        _norm("norm_prompts", "bf16", "f32", 8192, 5120, "layer", 16),
        # plain decoding: one sequence, one token, a cache of 16-bit numbers
        _attend("attend_token", "bf16", 16, 1, 1, 32, 8, 128, 1000, 64, False),
        # trees of 16 drafts over 8-bit caches of different lengths
        _attend("attend8_trees", "bf16", 8, 8, 16, 32, 8, 128, 8192, 64, True),
        # large trees over long caches of 4-bit codes
        _attend("attend4_long", "f16", 4, 4, 61, 32, 4, 128, 32768, 32, True),
        # the drafts' keys and values into 8-bit caches
        _cache("append8_trees", "append", "bf16", 8, 8, 16, 8, 128, 8192, 64),
        # prompts into 4-bit caches
        _cache("append4_prompts", "append", "f16", 4, 4, 4001, 8, 128, 77, 32),
        # the accepted paths of a large batch's trees
        _cache("keep8_trees", "keep", "bf16", 8, 64, 33, 8, 128, 1000, 64),
    ]


def _log_int(rng, lo, hi):
    n = max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))
    return n + 1 if n == 3072 else n


def draw(rng):
    kind = rng.choice(["matmul"] * 5 + ["attend"] * 4 + ["norm"] * 2 + ["append", "keep"])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    if kind == "matmul":
        bits = rng.choice([16, 8, 4, 4, 2, 1])
        group = 0 if bits == 16 else rng.choice([0, 0, 32, 64, 128])
        unit = group or 32
        r, k, m = _log_int(rng, 1, 8192), unit * _log_int(rng, 512 // unit, 12288 // unit), _log_int(rng, 256, 16384)
        gated = rng.random() < 0.3
        k += unit if k == 3072 else 0
        # no more than the largest listed case: 1.9e11 multiply-adds
        r = max(1, min(r, int(1.8e11 / (k * m * (2 if gated else 1)))))
        return dict(kind=kind, dtype=dtype, bits=bits, group=group, r=r, k=k, m=m,
                    act=rng.choice(["silu", "gelu", "relu"]) if gated else rng.choice(["none", "none", "gelu", "gelu_tanh"]),
                    gated=gated, bias=rng.random() < 0.4, residual=rng.random() < 0.4)
    if kind == "norm":
        d = _log_int(rng, 512, 8192)
        if rng.random() < 0.7:
            d = d // 64 * 64 + (64 if d // 64 == 48 else 0)
        gates = rng.choice([0, 1, 1, 4])
        r = max(gates, _log_int(rng, 1, 16384))
        r = min(r, 40_000_000 // d)
        r = r // gates * gates if gates else r
        return dict(kind=kind, dtype=rng.choice([dtype, dtype, "f32"]), hdtype=rng.choice(["same", "f32"]), r=r, d=d,
                    norm=rng.choice(["rms", "rms", "layer"]), gates=gates, post=rng.random() < 0.7)
    bits = rng.choice([16, 8, 8, 4])
    d = rng.choice([64, 128, 128])
    kv = rng.choice([1, 2, 4, 8])
    page = rng.choice([16, 32, 64, 128])
    if kind == "attend":
        b, t, length = _log_int(rng, 1, 64), _log_int(rng, 1, 64), _log_int(rng, 1, 32768)
        heads = kv * rng.choice([1, 2, 4, 5, 8])
        # no more keys than the largest listed case has, nor more products
        length = max(1, min(length, 524288 // (b * kv), int(3.2e10 / (b * t * heads * d))))
        return dict(kind=kind, dtype=dtype, bits=bits, b=b, t=t, heads=heads, kv_heads=kv, d=d, length=length,
                    page=page, ragged=rng.random() < 0.7)
    b = _log_int(rng, 1, 64)
    t = _log_int(rng, 1, 64) if kind == "keep" else max(1, min(_log_int(rng, 1, 4096), 16384 // b))
    return dict(kind=kind, dtype=dtype, bits=bits, b=b, t=t, kv_heads=kv, d=d,
                length=min(_log_int(rng, 1, 8192), 65536 // b), page=page)


# --- sizes that follow from a case --------------------------------------------

def _lens(c):
    """Cached tokens of each sequence: all alike, or spread over a quarter below the longest."""
    if not c.get("ragged", True):
        return [c["length"]] * c["b"]
    return [c["length"] - (37 * i) % (c["length"] // 4 + 1) for i in range(c["b"])]


def _counts(c):
    """Drafted tokens of each sequence."""
    if c["kind"] == "append" or not c.get("ragged", True):
        return [c["t"]] * c["b"]
    return [max(1, c["t"] - i % 4) for i in range(c["b"])]


def _kept(c):
    """Accepted tokens of each sequence: from none to all."""
    return [(5 * i + 3) % (c["t"] + 1) for i in range(c["b"])]


def _token_bytes(c):
    """Bytes of one token of one head in the cache: its codes and their scale."""
    return c["d"] * c["bits"] // 8 + (0 if c["bits"] == 16 else 4)


def work(case):
    c = case
    if c["kind"] == "matmul":
        rows = c["m"] * (2 if c["gated"] else 1)
        scales = 0 if c["bits"] == 16 else 4 * rows * (c["k"] // c["group"] if c["group"] else 1)
        byts = 2 * c["r"] * (c["k"] + c["m"] * (2 if c["residual"] else 1)) + rows * c["k"] * c["bits"] // 8 + scales
        return {"bytes": byts + (4 * rows if c["bias"] else 0), "flops": 2 * c["r"] * rows * c["k"]}
    if c["kind"] == "norm":
        y = 4 if c["dtype"] == "f32" else 2
        h = 4 if c["hdtype"] == "f32" else y
        n = c["r"] * c["d"]
        return {"bytes": n * (2 * y + 2 * h) + c["d"] * (c["gates"] * y + 8), "flops": 12 * n}
    lens, counts = _lens(c), _counts(c)
    if c["kind"] == "attend":
        seen = sum(n + k for n, k in zip(lens, counts))
        q = sum(counts) * c["heads"]
        return {"bytes": 2 * seen * c["kv_heads"] * _token_bytes(c) + q * (4 * c["d"] + 4),
                "flops": 4 * c["heads"] * c["d"] * sum((n + k) * k for n, k in zip(lens, counts))}
    n = sum(counts) if c["kind"] == "append" else sum(_kept(c))
    # append: the numbers in, the codes out; keep: the codes in and out.  Then the codes in, the values out.
    back = n if c["kind"] == "append" else c["b"] * c["t"]
    into = 2 * c["d"] + _token_bytes(c) if c["kind"] == "append" else 2 * _token_bytes(c)
    return {"bytes": 2 * c["kv_heads"] * (n * into + back * (_token_bytes(c) + 2 * c["d"])),
            "flops": 8 * n * c["kv_heads"] * c["d"]}


# --- inputs -------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 7919 + 23)
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _bytes(g, *shape):
    return torch.randint(0, 256, shape, generator=g, device="cuda", dtype=torch.uint8)


def _pages(g, c, pages):
    """Pages of one of the two: 16-bit numbers, or codes and a scale for each token and head."""
    d, h, page, bits = c["d"], c["kv_heads"], c["page"], c["bits"]
    if bits == 16:
        return torch.randn((pages, h, page, d), generator=g, device="cuda", dtype=_DT[c["dtype"]]), None
    # a token's largest number is about 2.5 to 3.5 of its deviations, and takes the largest code
    if bits == 8:
        v = torch.randn((pages, h, page, d), generator=g, device="cuda", dtype=torch.bfloat16)
        codes = v.mul_(40.0).round_().clamp_(-127, 127).to(torch.int8).view(torch.uint8)
        return codes, (0.6 + 0.8 * torch.rand((pages, h, page), generator=g, device="cuda")) / 40.0
    lo = torch.randn((pages, h, page, d // 2), generator=g, device="cuda", dtype=torch.bfloat16)
    hi = torch.randn((pages, h, page, d // 2), generator=g, device="cuda", dtype=torch.bfloat16)
    lo, hi = (v.mul_(2.4).round_().clamp_(-7, 7).to(torch.int8).view(torch.uint8) & 15 for v in (lo, hi))
    return lo | (hi << 4), (0.6 + 0.8 * torch.rand((pages, h, page), generator=g, device="cuda")) / 2.4


def _tree(g, c):
    """Ancestor bits of random trees [b, t, words]: each draft sees itself and its ancestors."""
    b, t = c["b"], c["t"]
    parent = (torch.rand((b, t), generator=g, device="cuda").sqrt() * torch.arange(t, device="cuda")).long() - 1
    parent = parent.cpu()
    sees = torch.zeros(b, t + 1, t, dtype=torch.bool)  # (row t: the parent of a root)
    at = torch.arange(b)
    for i in range(t):
        up = parent[:, i].clamp(min=-1)
        sees[:, i] = sees[at, torch.where(up < 0, t, up)]
        sees[:, i, i] = True
    words = -(-t // 64)
    bits = torch.nn.functional.pad(sees[:, :t], (0, words * 64 - t)).reshape(b, t, words, 64).long()
    return (bits << torch.arange(64)).sum(-1).cuda()


def prepare(case, seed):
    c, g = case, _gen(seed)
    s = dict(case=c)
    if c["kind"] == "matmul":
        rows, dt = c["m"] * (2 if c["gated"] else 1), _DT[c["dtype"]]
        k, bits = c["k"], c["bits"]
        s["x"] = torch.randn((c["r"], k), generator=g, device="cuda", dtype=dt)
        s["scale"] = None
        if bits == 16:
            s["w"] = torch.randn((rows, k), generator=g, device="cuda", dtype=dt) * (1 / math.sqrt(k))
        else:
            s["w"] = _bytes(g, rows, k * bits // 8)
            rms = {8: 73.9, 4: 4.64, 2: 1.22, 1: 1.0}[bits]
            shape = (rows, k // c["group"]) if c["group"] else (rows,)
            s["scale"] = (0.5 + torch.rand(shape, generator=g, device="cuda")) / (rms * math.sqrt(k))
        s["bias"] = 0.5 * _randn(g, rows) if c["bias"] else None
        s["residual"] = torch.randn((c["r"], c["m"]), generator=g, device="cuda", dtype=dt) if c["residual"] else None
        return s
    if c["kind"] == "norm":
        dt = _DT[c["dtype"]]
        hd = torch.float32 if c["hdtype"] == "f32" else dt
        r, d = c["r"], c["d"]
        s["h"] = (3 * _randn(g, r, d)).to(hd)
        s["y"] = (_randn(g, r, d) * (0.1 + _randn(g, r, 1).abs()) + 0.3).to(dt)
        s["post_weight"] = 1 + 0.2 * _randn(g, d) if c["post"] else None
        s["pre_weight"] = 1 + 0.2 * _randn(g, d)
        layer = c["norm"] == "layer"
        s["post_bias"] = 0.1 * _randn(g, d) if layer and c["post"] else None
        s["pre_bias"] = 0.1 * _randn(g, d) if layer else None
        s["gate"] = (1 + 0.3 * _randn(g, c["gates"], d)).to(dt) if c["gates"] else None
        return s
    lens, counts = _lens(c), _counts(c)
    wide = -(-(max(lens) + c["t"]) // c["page"])
    pages = c["b"] * wide
    s["k_pages"], s["k_scale"] = _pages(g, c, pages)
    s["v_pages"], s["v_scale"] = _pages(g, c, pages)
    s["table"] = torch.randperm(pages, generator=g, device="cuda").int().reshape(c["b"], wide)
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    s["counts"] = torch.tensor(counts, dtype=torch.int32, device="cuda")
    dt = _DT[c["dtype"]]
    if c["kind"] == "attend":
        s["q"] = 1.5 * torch.randn((c["b"], c["t"], c["heads"], c["d"]), generator=g, device="cuda", dtype=dt)
        s["mask"] = _tree(g, c)
    elif c["kind"] == "append":
        # as they come from a projection: side by side, some channels larger than others
        big = 1 + 3 * (torch.rand(2 * c["kv_heads"] * c["d"], generator=g, device="cuda") > 0.95)
        kv = (torch.randn((c["b"], c["t"], 2 * c["kv_heads"] * c["d"]), generator=g, device="cuda", dtype=dt) * big).to(dt)
        s["kv"] = kv.reshape(c["b"], c["t"], 2, c["kv_heads"], c["d"])
    else:
        kept = _kept(c)
        s["kept"] = torch.tensor(kept, dtype=torch.int32, device="cuda")
        order = torch.rand((c["b"], c["t"]), generator=g, device="cuda").argsort(1)
        first = torch.arange(c["t"], device="cuda") < s["kept"].unsqueeze(1)
        # `kept` drafts of each tree, in ascending order; what is behind them is not read
        s["path"] = torch.where(first, order, c["t"]).sort(1).values.clamp(max=c["t"] - 1).int()
    return s


# --- plain forms --------------------------------------------------------------

def _codes(w, bits):
    """Two's complement codes (or +-1) of packed bytes, the lower channel in the lower bits, as 32-bit numbers."""
    if bits == 8:
        return w.view(torch.int8).float()
    sh = torch.arange(0, 8, bits, device=w.device, dtype=torch.uint8)
    v = ((w.unsqueeze(-1) >> sh) & ((1 << bits) - 1)).flatten(-2)
    if bits == 1:
        return v.float() * 2 - 1
    half = 1 << (bits - 1)
    return (v ^ half).float() - half


def _act(t, act):
    if act == "relu":
        return t.clamp(min=0)
    if act == "silu":
        return t / (1 + torch.exp(-t))
    if act == "gelu":
        return 0.5 * t * (1 + torch.erf(t * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * t * (1 + torch.tanh(math.sqrt(2 / math.pi) * (t + 0.044715 * t * t * t)))
    return t


def _plain_matmul(s):
    c = s["case"]
    if c["bits"] == 16:
        w = s["w"].float()
    else:
        w = _codes(s["w"], c["bits"])
        n = c["k"] // c["group"] if c["group"] else 1
        w = (w.reshape(w.shape[0], n, -1) * s["scale"].reshape(-1, n, 1)).reshape(w.shape[0], -1)
    t = s["x"].float() @ w.t()
    if c["bias"]:
        t = t + s["bias"]
    if c["gated"]:
        t = _act(t[:, :c["m"]], c["act"]) * t[:, c["m"]:]
    else:
        t = _act(t, c["act"])
    if c["residual"]:
        t = t + s["residual"].float()
    return t.to(s["x"].dtype)


_EPS, _ALPHA, _BETA = 1e-6, 0.9, 0.7


def _plain_norm_of(v, norm, weight, bias):
    if norm == "layer":
        v = v - v.mean(-1, keepdim=True)
    v = v / torch.sqrt((v * v).mean(-1, keepdim=True) + _EPS)
    v = v * weight
    return v if bias is None else v + bias


def _plain_norm(s):
    c = s["case"]
    z = s["y"].float()
    if c["post"]:
        z = _plain_norm_of(z, c["norm"], s["post_weight"], s["post_bias"])
    if c["gates"]:
        z = (z.reshape(c["gates"], -1, c["d"]) * s["gate"].float().unsqueeze(1)).reshape(z.shape)
    h = _ALPHA * s["h"].float() + _BETA * z
    x = _plain_norm_of(h, c["norm"], s["pre_weight"], s["pre_bias"])
    return {"h": h.to(s["h"].dtype), "x": x.to(s["y"].dtype)}


def _gather(s, which):
    """The cache of each sequence as numbers [b, heads, tokens, d]."""
    c, table = s["case"], s["table"].long()
    v = s[which + "_pages"][table]  # [b, pages, heads, page, bytes]
    v = v.float() if c["bits"] == 16 else _codes(v, c["bits"]) * s[which + "_scale"][table].unsqueeze(-1)
    return v.transpose(1, 2).reshape(c["b"], c["kv_heads"], -1, c["d"])


def _plain_attend(s):
    c = s["case"]
    b, t, hk, d = c["b"], c["t"], c["kv_heads"], c["d"]
    g = c["heads"] // hk
    k, v = _gather(s, "k"), _gather(s, "v")
    n = k.shape[2]
    q = s["q"].float().reshape(b, t, hk, g, d).permute(0, 2, 1, 3, 4).reshape(b, hk, t * g, d)
    p = torch.matmul(q, k.transpose(2, 3)) * (1 / math.sqrt(d))
    # which positions a draft sees: all cached ones, and of the drafts those that its bits name
    lens, counts = s["lens"].long().view(b, 1, 1), s["counts"].long().view(b, 1, 1)
    j = torch.arange(n, device=k.device).view(1, 1, n) - lens
    at = j.clamp(0, t - 1)
    word = torch.gather(s["mask"], 2, (at >> 6).expand(b, t, n))
    sees = (j < 0) | ((j < counts) & (((word >> (at & 63)) & 1) != 0))
    sees = sees & (torch.arange(t, device=k.device).view(1, t, 1) < counts)
    p = p.reshape(b, hk, t, g, n).masked_fill_(~sees.view(b, 1, t, 1, n), -math.inf).reshape(b, hk, t * g, n)
    top = p.amax(-1, keepdim=True).clamp(min=-3e38)
    p = torch.exp(p - top)
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, v) / total.clamp(min=1e-38)
    lse = torch.where(total > 0, top + torch.log(total), -math.inf)
    out = out.reshape(b, hk, t, g, d).permute(0, 2, 1, 3, 4).reshape(b, t, hk * g, d)
    lse = lse.reshape(b, hk, t, g).permute(0, 2, 1, 3).reshape(b, t, hk * g)
    return {"out": out.to(s["q"].dtype), "lse": lse}


def _slots(s, start, n):
    """(page, slot) of the n positions from `start` on, each [b, n]."""
    c = s["case"]
    pos = start.long().unsqueeze(1) + torch.arange(n, device=start.device)
    return torch.gather(s["table"].long(), 1, pos // c["page"]), pos % c["page"]


def _plain_read(s, which, page, slot):
    """Values [b, n, heads, d] at (page, slot)."""
    c = s["case"]
    v = s[which + "_pages"][page, :, slot]
    v = v.float() if c["bits"] == 16 else _codes(v, c["bits"]) * s[which + "_scale"][page, :, slot].unsqueeze(-1)
    return v.to(_DT[c["dtype"]])


def _plain_append(s):
    c, out = s["case"], {}
    page, slot = _slots(s, s["lens"], c["t"])
    for i, which in enumerate("kv"):
        v = s["kv"][:, :, i]
        if c["bits"] == 16:
            s[which + "_pages"][page, :, slot] = v
        else:
            v = v.float()
            most = (1 << (c["bits"] - 1)) - 1
            scale = v.abs().amax(-1) / torch.full((), most, device=v.device)
            code = torch.round(v / scale.clamp(min=1e-38).unsqueeze(-1)).clamp(-most, most).to(torch.int8).view(torch.uint8)
            if c["bits"] == 4:
                code = (code[..., 0::2] & 15) | (code[..., 1::2] << 4)
            s[which + "_pages"][page, :, slot] = code
            s[which + "_scale"][page, :, slot] = scale
        out[which] = _plain_read(s, which, page, slot)
    return out


def _plain_keep(s):
    c, out = s["case"], {}
    n = c["t"]
    page, slot = _slots(s, s["lens"], n)
    live = torch.arange(n, device=page.device) < s["kept"].unsqueeze(1)
    # positions behind the kept ones stay as they are
    at = torch.where(live, s["path"].long(), torch.arange(n, device=page.device))
    fpage, fslot = torch.gather(page, 1, at), torch.gather(slot, 1, at)
    for which in "kv":
        v = s[which + "_pages"]
        v[page, :, slot] = v[fpage, :, fslot]
        if c["bits"] != 16:
            v = s[which + "_scale"]
            v[page, :, slot] = v[fpage, :, fslot]
        out[which] = _plain_read(s, which, page, slot)
    return out


# --- one pass -----------------------------------------------------------------

def _own(s):
    from paper_1908_11263_amd import lm
    c = s["case"]
    if c["kind"] == "matmul":
        return lm.matmul(s["x"], s["w"], c["bits"], scale=s["scale"], bias=s["bias"], act=c["act"], gated=c["gated"],
                         residual=s["residual"])
    if c["kind"] == "norm":
        h, x = lm.norm_residual(s["h"], s["y"], norm=c["norm"], post=c["post"], post_weight=s["post_weight"],
                                post_bias=s["post_bias"], pre_weight=s["pre_weight"], pre_bias=s["pre_bias"],
                                gate=s["gate"], alpha=_ALPHA, beta=_BETA, eps=_EPS)
        return {"h": h, "x": x}
    cache = lm.Cache(s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"], c["bits"])
    if c["kind"] == "attend":
        out, lse = lm.tree_attention(s["q"], cache, s["table"], s["lens"], mask=s["mask"], counts=s["counts"],
                                     want_lse=True)
        return {"out": out, "lse": lse}
    if c["kind"] == "append":
        lm.cache_append(s["kv"][:, :, 0], s["kv"][:, :, 1], cache, s["table"], s["lens"])
    else:
        lm.cache_keep(cache, s["table"], s["lens"], s["path"], s["kept"])
    k, v = lm.cache_read(cache, s["table"], s["lens"], c["t"], _DT[c["dtype"]])
    return {"k": k, "v": v}


_PLAIN = {"matmul": _plain_matmul, "norm": _plain_norm, "attend": _plain_attend, "append": _plain_append,
          "keep": _plain_keep}


def run(state):
    return _own(state) if own else _PLAIN[state["case"]["kind"]](state)


# --- the definitions in 64 bits -----------------------------------------------

def _exact_values(packed, bits):
    """Values that packed bytes stand for, by a table of all 256 bytes."""
    per, table = 8 // bits, []
    for byte in range(256):
        for i in range(per):
            f = (byte >> (i * bits)) % (1 << bits)
            table.append((1 if f else -1) if bits == 1 else f - (1 << bits) if f >> (bits - 1) else f)
    table = torch.tensor(table, dtype=torch.float64, device=packed.device).reshape(256, per)
    return table[packed.long()].reshape(*packed.shape[:-1], -1)


def _exact_act(t, act):
    f = torch.nn.functional
    return {"none": lambda v: v, "relu": f.relu, "silu": f.silu, "gelu": f.gelu,
            "gelu_tanh": lambda v: f.gelu(v, approximate="tanh")}[act](t)


def _exact_matmul(s):
    c = s["case"]
    x, parts = s["x"].double(), []
    rows = s["w"].shape[0]
    for a in range(0, rows, 4096):
        e = min(rows, a + 4096)
        if c["bits"] == 16:
            w = s["w"][a:e].double()
        else:
            w = _exact_values(s["w"][a:e], c["bits"])
            sc = s["scale"][a:e].double().reshape(e - a, -1)
            w *= sc.repeat_interleave(c["k"] // sc.shape[1], 1)
        parts.append(torch.mm(w, x.t()).t())
    t = torch.cat(parts, 1)
    if s["bias"] is not None:
        t = t + s["bias"].double()
    t = _exact_act(t[:, :c["m"]], c["act"]) * t[:, c["m"]:] if c["gated"] else _exact_act(t, c["act"])
    return t if s["residual"] is None else t + s["residual"].double()


def _exact_normed(v, kind, weight, bias):
    var = v.var(-1, unbiased=False, keepdim=True) if kind == "layer" else v.pow(2).mean(-1, keepdim=True)
    mean = v.mean(-1, keepdim=True) if kind == "layer" else 0.0
    v = (v - mean) * torch.rsqrt(var + _EPS) * weight.double()
    return v if bias is None else v + bias.double()


def _exact_norm(s):
    c = s["case"]
    z = s["y"].double()
    if c["post"]:
        z = _exact_normed(z, c["norm"], s["post_weight"], s["post_bias"])
    if s["gate"] is not None:
        z = z * s["gate"].double().repeat_interleave(c["r"] // c["gates"], 0)
    h = s["h"].double() * _ALPHA + z * _BETA
    return {"h": h, "x": _exact_normed(h, c["norm"], s["pre_weight"], s["pre_bias"])}


def _exact_tokens(s, which, b, first, n):
    """Values [heads, n, d] of positions first .. first + n - 1 of sequence b."""
    c = s["case"]
    pos = torch.arange(first, first + n, device=s["table"].device)
    page = s["table"][b].long()[torch.div(pos, c["page"], rounding_mode="floor")]
    v = s[which + "_pages"].transpose(1, 2)[page, pos.remainder(c["page"])]
    if c["bits"] == 16:
        return v.double().transpose(0, 1)
    scale = s[which + "_scale"].transpose(1, 2)[page, pos.remainder(c["page"])]
    return (_exact_values(v, c["bits"]) * scale.double().unsqueeze(-1)).transpose(0, 1)


def _exact_attend(s):
    c = s["case"]
    g, t = c["heads"] // c["kv_heads"], c["t"]
    out = torch.zeros(c["b"], t, c["heads"], c["d"], dtype=torch.float64, device="cuda")
    lse = torch.full((c["b"], t, c["heads"]), -math.inf, dtype=torch.float64, device="cuda")
    for b, (n, count) in enumerate(zip(_lens(c), _counts(c))):
        k, v = _exact_tokens(s, "k", b, 0, n + count), _exact_tokens(s, "v", b, 0, n + count)
        words = s["mask"][b, :count].cpu().tolist()
        see = torch.tensor([[(w[j // 64] >> (j % 64)) & 1 for j in range(count)] for w in words], device="cuda").bool()
        bias = torch.zeros(count, n + count, dtype=torch.float64, device="cuda")
        bias[:, n:][~see] = -math.inf
        for h in range(c["heads"]):
            w = s["q"][b, :count, h].double() @ k[h // g].t().contiguous() / math.sqrt(c["d"]) + bias
            lse[b, :count, h] = torch.logsumexp(w, -1)
            out[b, :count, h] = torch.softmax(w, -1) @ v[h // g]
    return {"out": out, "lse": lse}


def _exact_append(s):
    c, out = s["case"], {}
    for i, which in enumerate("kv"):
        v = s["kv"][:, :, i].double()
        if c["bits"] != 16:
            # the scale is held in 32 bits; a code is the whole number next to v / scale
            top = float(2 ** (c["bits"] - 1) - 1)
            scale = (v.abs().amax(-1, keepdim=True) / top).float().double()
            v = torch.where(scale > 0, torch.clamp(torch.round(v / scale), -top, top) * scale, torch.zeros_like(v))
        out[which] = v
    return out


def _exact_keep(s):
    c, out = s["case"], {}
    path, kept, lens = s["path"].cpu().tolist(), _kept(c), _lens(c)
    for which in "kv":
        rows = []
        for b in range(c["b"]):
            drafts = _exact_tokens(s, which, b, lens[b], c["t"]).transpose(0, 1)
            rows.append(drafts[[path[b][j] if j < kept[b] else j for j in range(c["t"])]])
        out[which] = torch.stack(rows)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"matmul": _exact_matmul, "norm": _exact_norm, "attend": _exact_attend, "append": _exact_append,
            "keep": _exact_keep}[case["kind"]](s)
