"""What the binding of include/qnn_lm.h refuses about a call's tensors besides their types and shapes."""
import pytest
import torch

BF, I = torch.bfloat16, torch.int32


@pytest.fixture(scope="module")
def lm():
    from paper_1908_11263_amd import lm
    return lm


def calls(lm):
    """Each operator with its arguments, and the names of those that can require a gradient."""
    z = torch.zeros
    c = lm.make_cache(4, 2, 16, 64, 16, BF, "cpu")
    table, lens = z(1, 4, dtype=I), z(1, dtype=I)
    x, y = z(3, 64, dtype=BF), z(3, 8, dtype=BF)
    kv = z(1, 3, 2, 64, dtype=BF)
    w = z(64)
    yield lm.matmul, dict(x=x, w=z(8, 64, dtype=BF), bits=16, bias=z(8), residual=y), ("x", "w", "bias", "residual")
    yield lm.matmul, dict(x=x, w=z(8, 32, dtype=torch.uint8), bits=4, scale=z(8)), ("x", "scale")
    yield (lm.norm_residual, dict(h=x, y=x, post_weight=w, post_bias=w, pre_weight=w, pre_bias=w, gate=x[:1]),
           ("h", "y", "post_weight", "post_bias", "pre_weight", "pre_bias", "gate"))
    yield lm.tree_attention, dict(q=z(1, 3, 4, 64, dtype=BF), cache=c, table=table, lens=lens), ("q", "cache.k", "cache.v")
    yield lm.cache_append, dict(k=kv, v=kv, cache=c, table=table, lens=lens), ("k", "v", "cache.k")
    yield lm.cache_read, dict(cache=c, table=table, start=lens, n=2), ("cache.v",)


def test_gradients_are_refused(lm):
    """While torch records gradients, a tensor that requires one is named; without recording the call goes on (and is
    refused for lying on the host)."""
    for f, args, names in calls(lm):
        for name in names:
            a = dict(args)
            if name.startswith("cache."):
                part = name[6:]
                a["cache"] = a["cache"]._replace(**{part: getattr(a["cache"], part).clone().requires_grad_()})
            else:
                a[name] = a[name].clone().requires_grad_()
            with pytest.raises(ValueError, match="gradient"):
                f(**a)
            with torch.no_grad(), pytest.raises((ValueError, RuntimeError)) as e:
                f(**a)
            assert "gradient" not in str(e.value)


def test_flags_without_a_truth_value(lm):
    """A flag that is neither true nor false is refused, not taken for true with the error left behind."""
    (matmul, a, _), (_, b, _), (norm, c, _), (attend, d, _) = list(calls(lm))[:4]
    neither = torch.zeros(2)
    for f, args in ((matmul, dict(a, residual=None, gated=neither)), (norm, dict(c, post=neither)),
                    (attend, dict(d, want_lse=neither))):
        with pytest.raises(ValueError, match="True or False"):
            f(**args)
