"""The operators of include/qnn_lm.h from their formulas, in 64 bits, with the
bounds that an implementation in 32-bit sums and one rounding keeps."""
import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -23}  # twice the rounding's bound


def pack(codes, bits):
    """uint8 codes (each < 2^bits) along the last axis -> packed bytes."""
    per = 8 // bits
    sh = torch.arange(0, 8, bits, dtype=torch.uint8)
    return (codes.reshape(*codes.shape[:-1], -1, per) << sh.to(codes.device)).sum(-1).to(torch.uint8)


def values(packed, bits):
    """The whole numbers that packed bytes stand for, in 64 bits."""
    v = packed.long().unsqueeze(-1)
    f = torch.cat([(v >> s) & ((1 << bits) - 1) for s in range(0, 8, bits)], -1).flatten(-2)
    if bits == 1:
        return (2 * f - 1).double()
    return (f - ((f >> (bits - 1)) << bits)).double()


def act(t, kind):
    if kind == "relu":
        return t.clamp(min=0)
    if kind == "silu":
        return t * torch.sigmoid(t)
    if kind == "gelu":
        return 0.5 * t * torch.erfc(-t * math.sqrt(0.5))
    if kind == "gelu_tanh":
        return 0.5 * t * (1 + torch.tanh(math.sqrt(2 / math.pi) * (t + 0.044715 * t ** 3)))
    return t


def matmul(x, w, bits, scale=None, bias=None, kind="none", gated=False, residual=None):
    """(result, bound): sums of k exact products in 32 bits, in any order, lose
    at most about k units of 2^-24 of the sum of magnitudes (twice that is
    allowed: the matrix instruction may cut off where it does not round);
    activations have slopes below 1.2 and 32-bit rounding of their own."""
    wv = w.double() if bits == 16 else values(w, bits)
    rows, k = wv.shape
    if scale is not None:
        s = scale.double().reshape(rows, -1)
        wv = wv * s.repeat_interleave(k // s.shape[1], 1)
    xv = x.double().reshape(-1, k)
    t, mag = xv @ wv.t(), xv.abs() @ wv.abs().t()
    if bias is not None:
        t, mag = t + bias.double(), mag + bias.double().abs()
    e = 2 * (k + 16) * 2.0 ** -24 * mag
    if gated:
        m = rows // 2
        a, up = act(t[:, :m], kind), t[:, m:]
        e = 1.2 * e[:, :m] * (up.abs() + e[:, m:]) + a.abs() * e[:, m:] + 1e-6 * (a * up).abs() + 1e-6 * up.abs()
        y = a * up
    else:
        y = act(t, kind)
        e = (1.2 * e + 1e-6 * (1 + t.abs())) if kind != "none" else e
    if residual is not None:
        r = residual.double().reshape(y.shape)
        y, e = y + r, e + 2.0 ** -23 * (y.abs() + r.abs())
    return y, e + U[x.dtype] * y.abs()


def normed(v, norm, weight, bias, eps):
    if norm == "layer":
        v = v - v.mean(-1, keepdim=True)
    v = v / (v.pow(2).mean(-1, keepdim=True) + eps).sqrt()
    if weight is not None:
        v = v * weight.double()
    return v if bias is None else v + bias.double()


def norm_residual(h, y, norm, post, pw, pb, w, b, gate, alpha, beta, eps):
    """(h', x, bound of h', bound of x).  A sum over a row in 32 bits is a tree
    of short sums: a few 1e-6 of its magnitudes; the bounds take 1e-5 of every
    term, and of the row's largest number over its deviation for the mean."""
    hv = h.double()
    e = torch.zeros_like(hv)
    if y is not None:
        z = y.double()
        spread = torch.ones_like(z[..., :1])
        if post:
            spread = 1 + z.abs().amax(-1, keepdim=True) / (z.var(-1, unbiased=False, keepdim=True) + eps).sqrt()
            z = normed(z, norm, pw, pb, eps)
        size = z.abs() + (1 if pw is None else pw.double().abs()) * spread if post else z.abs()
        if gate is not None:
            g = gate.double().reshape(-1, gate.shape[-1])
            g = g.repeat_interleave(z.reshape(-1, z.shape[-1]).shape[0] // g.shape[0], 0).reshape(z.shape)
            z, size = z * g, size * g.abs()
        e = 1e-5 * ((alpha * hv).abs() + abs(beta) * size)
        hv = alpha * hv + beta * z
    x = normed(hv, norm, w, b, eps)
    dev = hv.var(-1, unbiased=False, keepdim=True) if norm == "layer" else hv.pow(2).mean(-1, keepdim=True)
    dev = (dev + eps).sqrt()
    wv = 1.0 if w is None else w.double().abs()
    ex = wv * (e + e.mean(-1, keepdim=True) + 1e-5 * hv.abs().amax(-1, keepdim=True)) / dev + 1e-5 * x.abs()
    ex = ex + 2 * x.abs() * (e.amax(-1, keepdim=True) / dev)
    if b is not None:
        ex = ex + 1e-6 * b.double().abs()
    return hv, x, e + U[h.dtype] * hv.abs() + 1e-30, ex + U[(h if y is None else y).dtype] * x.abs() + 1e-30


def cache_values(pages, scale, bits):
    """[pages, heads, page, dim] in 64 bits."""
    return pages.double() if bits == 16 else values(pages, bits) * scale.double().unsqueeze(-1)


def attention(q, cache, table, lens, mask, counts, scale):
    """(out, lse, bound of out, bound of lse, rows that see something), one
    sequence, head and draft at a time.  mask: [b][i] -> list of drafts that
    draft i sees, or None for 0 .. i."""
    b, t, heads, dim = q.shape
    kv, vv = cache_values(cache.k, cache.k_scale, cache.bits), cache_values(cache.v, cache.v_scale, cache.bits)
    pages, hk, page, _ = kv.shape
    g = heads // hk
    out = torch.zeros(b, t, heads, dim, dtype=torch.float64, device=q.device)
    lse = torch.full((b, t, heads), -math.inf, dtype=torch.float64, device=q.device)
    eo, el = torch.zeros_like(out), torch.zeros_like(lse)
    u = U[q.dtype]
    tab = table.cpu().tolist()
    for i in range(b):
        count = t if counts is None else min(max(counts[i], 0), t)
        for d in range(count):
            drafts = range(d + 1) if mask is None else [j for j in mask[i][d] if j < count]
            pos = list(range(max(lens[i], 0))) + [max(lens[i], 0) + j for j in drafts]
            at = [(tab[i][p // page], p % page) for p in pos if p < page * len(tab[i])]
            at = [(pg, s) for pg, s in at if 0 <= pg < pages]
            if not at:
                continue
            pg = torch.tensor([x for x, _ in at], device=q.device)
            sl = torch.tensor([x for _, x in at], device=q.device)
            k = kv[pg, :, sl].repeat_interleave(g, 1)  # [n, heads, dim]
            v = vv[pg, :, sl].repeat_interleave(g, 1)
            qd = q[i, d].double()
            s = (k * qd).sum(-1) * scale
            mag = (k * qd).abs().sum(-1) * abs(scale)
            es = (2 * (dim + 16) * 2.0 ** -24 * mag + 1e-6 * s.abs()).amax(0)  # [heads]
            p = torch.softmax(s, 0)
            lse[i, d] = torch.logsumexp(s, 0)
            el[i, d] = es + 2e-6 * (1 + lse[i, d].abs()) + len(at) * 2.0 ** -24
            out[i, d] = (p.unsqueeze(-1) * v).sum(0)
            pv = (p.unsqueeze(-1) * v.abs()).sum(0)
            # probabilities and results are rounded to 16 bits; f16 probabilities below 2^-14 to 2^-25
            eo[i, d] = (u + 3 * es.unsqueeze(-1) + len(at) * 2.0 ** -22) * pv + u * out[i, d].abs()
            if q.dtype == torch.float16:
                eo[i, d] += 2.0 ** -24 * v.abs().sum(0)
    return out, lse, eo + 1e-30, el


def quantize(v, bits):
    """(codes, scales) of 32-bit numbers along the last axis, as the cache keeps them."""
    most = (1 << (bits - 1)) - 1
    v = v.float().cpu()
    scale = v.abs().amax(-1) / torch.tensor(float(most))
    code = torch.where(scale.unsqueeze(-1) > 0, torch.round(v / scale.unsqueeze(-1)), torch.zeros_like(v))
    code = code.clamp(-most, most)
    bad = ~torch.isfinite(v).all(-1)
    scale = torch.where(bad, torch.full_like(scale, math.nan), scale)
    code = torch.where(bad.unsqueeze(-1), torch.zeros_like(code), code)
    return code.to(torch.int64), scale


def close(got, want, bound, what):
    """|got - want| <= bound, and NaN and infinities in the same places."""
    got, want, bound = got.double().reshape(want.shape), want, bound.reshape(want.shape)
    fine = torch.isfinite(want)
    assert torch.equal(torch.isfinite(got), fine), "%s: not finite at other places" % what
    assert torch.equal(torch.isnan(got), torch.isnan(want)), "%s: NaN at other places" % what
    rest = ~fine & ~torch.isnan(want)
    assert torch.equal(got[rest], want[rest]), "%s: other infinities" % what
    off = (got - want).abs()[fine]
    bad = off > bound[fine]
    if bool(bad.any()):
        i = int((off - bound[fine]).argmax())
        raise AssertionError("%s: %d of %d off, worst %g against %g at %g" % (
            what, int(bad.sum()), bad.numel(), float(off[i]), float(bound[fine][i]), float(want[fine][i])))
