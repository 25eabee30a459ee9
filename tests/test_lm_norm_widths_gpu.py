"""Norms of rows whose width is no multiple of 8: one element an access, and no worse than that."""
import pytest
import torch

from test_lm_gpu import lm, gen, randn  # noqa: F401

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32


def best(f):
    """Microseconds of a call, the best of several rounds."""
    for _ in range(3):
        f()
    times = []
    for _ in range(5):
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        for _ in range(10):
            f()
        b.record()
        torch.cuda.synchronize()
        times.append(a.elapsed_time(b) * 100)
    return min(times)


@pytest.mark.parametrize("d", [1000, 2048, 4096, 7288, 16384])
def test_odd_widths_are_not_many_times_slower(lm, d):
    """Eight times the accesses at most (a kernel that kept the row in scratch memory took 60 times as long)."""
    g = gen(d)
    h, y = randn(g, 2000, d + 1), randn(g, 2000, d + 1, dtype=BF)
    even = best(lambda: lm.norm_residual(h[:, :d].contiguous(), y[:, :d].contiguous()))
    odd = best(lambda: lm.norm_residual(h, y))
    assert odd < 8 * even, (odd, even)
