"""network.tree_step and accept_path on a stream of their own, with what they read produced there."""
import random

import pytest
import torch

from test_lm_block_gpu import D, BF, F, make, words

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def steps(stream, lens, path, kept, h, first, blocks, caches, table, mask):
    """Two steps with an accepted path between them."""
    from paper_1908_11263_amd import network
    _, x1 = network.tree_step(h, first, blocks, caches, table, lens, mask=mask, dtype=BF, stream=stream)
    new = network.accept_path(caches, table, lens, path, kept, stream=stream)
    _, x2 = network.tree_step(h, first, blocks, caches, table, new, mask=mask, dtype=BF, stream=stream)
    return x1, new, x2


def busy():
    """Some milliseconds of work on the current stream."""
    a = torch.ones(4096, 4096, device="cuda")
    for _ in range(8):
        a = a @ a * 2.0 ** -12
    return a


def test_steps_on_a_side_stream():
    """Lengths and kept counts that the side stream writes late, behind other work of its own."""
    t, b = 6, 2
    rng = random.Random(1)
    sees = [[(lambda up: up + [i])([rng.randrange(i)] if i else []) for i in range(t)] for _ in range(b)]
    got = []
    for side in (None, torch.cuda.Stream()):
        g, blocks, caches, table = make(3, 4, 8, 2, b, 40 + 2 * t)
        h, first = torch.randn((b, t, D), generator=g, device="cuda"), torch.ones(D, device="cuda", dtype=F)
        mask, path = words(sees, t), i32([[0, 2, 3, 0, 0, 0], [1, 2, 0, 0, 0, 0]])
        lens, kept = i32([40, 17]), i32([3, 2])
        if side is None:
            got.append(steps(None, lens, path, kept, h, first, blocks, caches, table, mask))
            continue
        late_lens, late_kept = torch.zeros_like(lens), torch.zeros_like(kept)
        torch.cuda.synchronize()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            busy()
            late_lens.copy_(lens)
            late_kept.copy_(kept)
        got.append(steps(side, late_lens, path, late_kept, h, first, blocks, caches, table, mask))
        torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert got[1][1].tolist() == [43, 19]
    for x, y in zip(*got):
        assert torch.equal(x, y)


def test_arguments_dropped_at_once():
    """Arguments made for a call on a side stream and dropped when it returns: their memory is not given to others
    before the side stream has read them."""
    from paper_1908_11263_amd import lm
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    x = torch.randn((512, 1024), generator=g, device="cuda").to(BF)
    w = torch.randn((256, 1024), generator=g, device="cuda").to(BF)
    want, (_, normed) = lm.matmul(x, w, 16), lm.norm_residual(x, x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        busy()
    torch.cuda.synchronize()  # (what busy() compiles or loads has been)
    got = []
    for call in (lambda v: lm.matmul(v, w, 16, stream=side), lambda v: lm.norm_residual(v, x, stream=side)[1]):
        copy = x.clone()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            busy()
        got.append(call(copy))
        del copy
        others = [torch.full_like(x, float("nan")) for _ in range(4)]
        torch.cuda.synchronize()
        del others
    assert torch.equal(got[0], want) and torch.equal(got[1], normed)
