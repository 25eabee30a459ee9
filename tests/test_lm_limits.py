"""The limits that include/qnn_lm.h names are where the library refuses (the first call past each; the last within goes
on, to be refused for having no GPU)."""
import re

import pytest
import torch

from test_lm_host import DEVICE, SHAPE, UNSUPPORTED, Raw, append, attend, cache, keep, linear, read

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="calls that pass every check are not made on a GPU")


@pytest.fixture(scope="module")
def lm():
    return Raw()


def test_linear(lm):
    big = dict(ws=1 << 20, size=1 << 50)
    f = lambda **a: linear(lm, **{**big, **a})  # noqa: E731
    assert f(r=1 << 21) == DEVICE and f(r=(1 << 21) + 1) == SHAPE
    assert f(m=1 << 24, yp=1 << 24) == DEVICE and f(m=(1 << 24) + 1, yp=1 << 25) == SHAPE
    assert f(m=1 << 23, yp=1 << 23, gated=1) == DEVICE and f(m=(1 << 23) + 1, yp=1 << 24, gated=1) == SHAPE
    assert f(k=1 << 20, xp=1 << 20) == DEVICE and f(k=(1 << 20) + 32, xp=1 << 21) == UNSUPPORTED
    assert f(xp=1 << 37, r=4) == DEVICE and f(xp=(1 << 37) + 8, r=4) == SHAPE


def test_cache_and_attention(lm):
    most = (1 << 31) - 256
    for call in (attend, append, keep, read):
        assert call(lm, cache(lm, width=most // 16)) == DEVICE, call.__name__
        assert call(lm, cache(lm, width=most // 16 + 1)) == SHAPE
        assert call(lm, cache(lm, b=65535)) == DEVICE and call(lm, cache(lm, b=65536)) == SHAPE
    heads = dict(st=(1 << 22, 64, 64) * 2)
    assert read(lm, cache(lm, heads=32767, **heads), t=1) == DEVICE and read(lm, cache(lm, heads=32768, **heads), t=1) == SHAPE
    for call in (append, keep, read):
        assert call(lm, cache(lm), t=most // 8) == DEVICE and call(lm, cache(lm), t=most // 8 + 1) == SHAPE
    assert attend(lm, cache(lm), t=1 << 22) == DEVICE and attend(lm, cache(lm), t=(1 << 22) + 1) == SHAPE
    c = cache(lm, b=256)
    assert attend(lm, c, t=(1 << 21) - 1) == DEVICE and attend(lm, c, t=1 << 21) == SHAPE


def test_header_names_them(lm):
    with open(lm.HEADER) as f:
        text = re.sub(r"[\s*]+", " ", f.read())
    for words in ("k <= 2^20, rows of weights <= 2^24", "rows of x <= 2^21, each tensor < 2^40 bytes",
                  "width page <= 2^31 - 256, b <= 65535, heads <= 32767", "2 b t heads <= 2^31 - 256",
                  "t heads <= 2^24, b t heads <= 2^31 - 256"):
        assert words in text, words
