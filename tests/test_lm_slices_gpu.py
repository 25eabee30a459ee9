"""A part of a batch: slices of lengths, counts, tables, masks and paths, which start at any word."""
import pytest
import torch

from test_lm_gpu import lm, gen, randn, make_cache, words, random_mask  # noqa: F401

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32


@pytest.mark.parametrize("first", [1, 2, 3])
def test_parts_of_a_batch(lm, first):
    import random
    b, t, width = 4, 3, 5
    g = gen(first)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    table = torch.randperm(b * width, generator=g, device="cuda").int().reshape(b, width)
    lens, counts, kept = i32([40, 7, 61, 30]), i32([3, 2, 3, 1]), i32([2, 1, 2, 0])
    path = i32([[0, 2, 0], [1, 0, 0], [1, 2, 0], [0, 0, 0]])
    mask = words(random_mask(random.Random(first), b, t), t)
    q, kv = randn(g, b, t, 4, 64, dtype=BF), randn(g, b, t, 2, 64, dtype=BF)
    one = make_cache(lm, g, b * width, 2, 16, 64, 8, BF)
    two = lm.Cache(*(x.clone() for x in one[:4]), 8)
    part = slice(first, None)
    assert lens[part].data_ptr() % 16 and table[part].data_ptr() % 16
    results = []
    for cache, s in ((one, slice(None)), (two, part)):
        lm.cache_append(kv[s], kv[s], cache, table[s], lens[s], counts=counts[s])
        o, lse = lm.tree_attention(q[s], cache, table[s], lens[s], mask=mask[s], counts=counts[s], want_lse=True)
        lm.cache_keep(cache, table[s], lens[s], path[s], kept[s])
        k, v = lm.cache_read(cache, table[s], lens[s], t, F)
        results.append([o, lse, k, v])
    for a, c in zip(*results):
        assert torch.equal(a[part], c)
