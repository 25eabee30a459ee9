"""The linear layer's activations at every number of f16 in reach, through
weights of ones on the diagonal: the sums are exact, so what is left is the
activation's own error and one rounding."""
import math

import pytest
import torch

from test_lm_gpu import lm  # noqa: F401

pytestmark = pytest.mark.gpu


def every_f16(most):
    """All numbers of f16 from 2^-10 to `most` in magnitude, both signs."""
    bits = torch.arange(0x1400, 0x7C00, dtype=torch.int32)
    v = bits.to(torch.int16).view(torch.float16)
    v = v[v.double() <= most]
    v = torch.cat([v, -v])
    return torch.cat([v, torch.zeros(-v.numel() % 256, dtype=torch.float16)]).cuda()


@pytest.mark.parametrize("rows", [16, 1 << 20])
def test_gelu(lm, rows):
    """Numbers within 3e-6 of the formula's for |t| < 5 (1e-5 to 9), rounded to nearest: half a spacing of f16 besides,
    2^-11 of the power of two below the result, and 2^-25 at least.  (1 + erf in 32 bits is off by 3e-4 at -3.5.)"""
    t = every_f16(9.0)
    w = torch.eye(256, device="cuda", dtype=torch.int8).view(torch.uint8)
    x = t.reshape(-1, 256)
    y = torch.cat([lm.matmul(part, w, 8, scale=torch.ones(256, device="cuda"), act="gelu") for part in x.split(rows)])
    v = x.double()
    want = 0.5 * v * torch.erfc(-v * math.sqrt(0.5))
    half = (2.0 ** (torch.frexp(want)[1].double() - 12)).clamp(min=2.0 ** -25)
    own = torch.where(v.abs() < 5, 3e-6, 1e-5) * want.abs()
    off = (y.double() - want).abs()
    assert bool((off <= half + own).all()), float((off - half - own).max())
