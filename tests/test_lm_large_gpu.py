"""Calls of more threads than a launch has along one axis (2^32)."""
import pytest
import torch

import lm_reference as ref
from test_lm_gpu import lm, gen, randn, make_cache  # noqa: F401

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16


@pytest.mark.parametrize("r,d", [((1 << 24) + 5, 1), ((1 << 24) + 3, 7), ((1 << 26) + 1, 8)])
def test_norm_of_many_rows(lm, r, d):
    g = gen(d)
    h, y = randn(g, r, d, dtype=HF), randn(g, r, d, dtype=HF)
    ho, x = lm.norm_residual(h, y, post=False)
    for part in (slice(0, 1000), slice(r // 2 - 500, r // 2 + 500), slice(r - 1000, r)):
        wh, wx, eh, ex = ref.norm_residual(h[part], y[part], "rms", False, None, None, None, None, None, 1.0, 1.0, 1e-6)
        # (results below f16's normal range are rounded to 2^-25)
        ref.close(ho[part], wh, eh + 2.0 ** -25, "h")
        ref.close(x[part], wx, ex + 2.0 ** -25, "x")


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_append_of_many_tokens(lm, bits):
    """A token repeated 2^29 times and more, of which the table reaches the last hundred."""
    g = gen(bits)
    t = (1 << 29) + 1000
    cache = make_cache(lm, g, 5, 1, 32, 64, bits, BF)
    table = torch.tensor([[3, 1, 4, 0]], dtype=torch.int32, device="cuda")
    new = randn(g, 1, 1, 1, 64, dtype=BF)
    start = torch.tensor([100 - t], dtype=torch.int32, device="cuda")
    zero = torch.zeros(1, dtype=torch.int32, device="cuda")
    before, _ = lm.cache_read(cache, table, zero, 128, torch.float32)
    k = new.expand(1, t, 1, 64)
    lm.cache_append(k, k, cache, table, start)
    got, _ = lm.cache_read(cache, table, zero, 128, torch.float32)
    if bits == 16:
        want = new.float()
    else:
        code, scale = ref.quantize(new, bits)
        want = (code.float() * scale.unsqueeze(-1)).cuda()
    assert torch.equal(got[:, :100], want.expand(1, 100, 1, 64))
    assert torch.equal(got[:, 100:], before[:, 100:])
