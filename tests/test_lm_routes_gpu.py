"""Every kernel instance that the operators of include/qnn_lm.h choose between,
by sizes that their rules send to it: the linear layer's tiles, its kernels for
few rows, the attention's, the norms' and the cache's, against the formulas in 64
bits."""
import random

import pytest
import torch

import lm_reference as ref
from test_lm_gpu import lm, gen, randn, layer, make_cache, check_attention, random_mask  # noqa: F401

pytestmark = pytest.mark.gpu

BF, HF, F = torch.bfloat16, torch.float16, torch.float32
FORMS = [(16, 0)] + [(bits, group) for bits in (8, 4, 2, 1) for group in (0, 32, 64, 128)]
TYPES = pytest.mark.parametrize("dtype", [BF, HF])


def check_matmul(lm, L, bits, act="none", gated=False):
    y = lm.matmul(L["x"], L["w"], bits, scale=L["scale"], bias=L["bias"], act=act, gated=gated, residual=L["residual"])
    want, bound = ref.matmul(L["x"], L["w"], bits, L["scale"], L["bias"], act, gated, L["residual"])
    # (results below f16's normal range are rounded to 2^-25)
    ref.close(y, want, bound + (2.0 ** -25 if y.dtype is HF else 0), "matmul")


# 16 tiles of 128 rows of x (or of 64) by 32 of 256 rows of weights: 512 and more tiles, the last of each not full;
# k ends with a step of a half where it is an odd multiple of 32
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("bits,group", FORMS)
@pytest.mark.parametrize("r,k", [(2033, 384), (2033, 160), (1003, 640), (1003, 96)])
@TYPES
def test_large_tiles(lm, dtype, r, k, bits, group, gated):
    """Tiles of 128 x 256 (r = 2033) and of 64 x 256 (r = 1003)."""
    k = -(-k // (group or 32)) * (group or 32)
    m = 4001 if gated else 8001
    L = layer(gen(r + k), r, k, m, bits, group, dtype, gated, bias=True, residual=bool(k & 64))
    check_matmul(lm, L, bits, "silu" if gated else "gelu", gated)


@pytest.mark.parametrize("bits,group", FORMS)
@pytest.mark.parametrize("r", [40, 64, 30, 130])
@pytest.mark.parametrize("m", [72, 76, 75])
@TYPES
def test_gated_tiles_in_pieces(lm, dtype, r, bits, group, m):
    """Gated layers whose k is cut in pieces, joined by a kernel of their own: outputs in eights, in fours and odd."""
    L = layer(gen(r + m), r, 2304, m, bits, group, dtype, True, bias=True, residual=r == 40)
    check_matmul(lm, L, bits, "silu", True)


@pytest.mark.parametrize("bits,group", FORMS)
@pytest.mark.parametrize("r", [17, 32, 50, 128])
@TYPES
def test_small_tiles(lm, dtype, r, bits, group):
    """Tiles of 32 x 128 and of 64 x 128, whole and in pieces."""
    for k, m in ((384, 150), (2304, 152), (4224, 131)):
        check_matmul(lm, layer(gen(r + m), r, k, m, bits, group, dtype, residual=True), bits)


@pytest.mark.parametrize("bits,group", FORMS)
@pytest.mark.parametrize("gated", [False, True])
@TYPES
def test_few_rows_past_local_memory(lm, dtype, bits, group, gated):
    """Up to 16 rows of x that local memory does not hold, narrow and wide layers (two blocks of weights a workgroup
    from 16384 rows of weights on)."""
    for r, k, m in ((16, 1280, 33), (16, 8192, 100), (5, 4224, 70), (1, 33 * 512, 20), (3, 384, 40)):
        check_matmul(lm, layer(gen(r + k), r, k, m, bits, group, dtype, gated, bias=True), bits, "none", gated)
    m = 8200 if gated else 16400
    for r, k in ((1, 384), (16, 512), (16, 1152)):
        check_matmul(lm, layer(gen(r + k), r, k, m, bits, group, dtype, gated), bits, "none", gated)


@pytest.mark.parametrize("r", [17, 64, 65, 130])
@pytest.mark.parametrize("bits", [8, 4, 2, 1])
@TYPES
def test_fewer_than_four_scales(lm, dtype, r, bits):
    """One output and two or three groups: the kernel of few rows, 64 rows a workgroup."""
    for group in (32, 64, 128):
        for n in (2, 3):
            check_matmul(lm, layer(gen(r), r, n * group, 1, bits, group, dtype, bias=True), bits)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("r", [3, 17, 70, 260])
@TYPES
def test_rows_of_x_far_apart(lm, dtype, r, gated):
    """Rows of x 2^23 elements apart and more (at r = 260 the last lies past 2^32 bytes)."""
    pitch = (1 << 23) + 8
    x = torch.empty(r * pitch, device="cuda", dtype=dtype).view(r, pitch)[:, :384]
    for bits, group in FORMS:
        L = layer(gen(r + bits), r, 384, 75, bits, group, dtype, gated, bias=True, residual=True)
        x.copy_(L["x"])
        y = lm.matmul(x, L["w"], bits, scale=L["scale"], bias=L["bias"], act="silu", gated=gated, residual=L["residual"])
        want, bound = ref.matmul(L["x"], L["w"], bits, L["scale"], L["bias"], "silu", gated, L["residual"])
        ref.close(y, want, bound + (2.0 ** -25 if dtype is HF else 0), "far apart")


# drafts and query heads of a cache head: up to 16 rows, 32, 64 and more
@pytest.mark.parametrize("t,g", [(3, 1), (4, 4), (17, 1), (8, 4), (11, 3), (16, 4), (13, 5), (33, 4)])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("bits", [16, 8, 4])
@TYPES
def test_attention_kernels(lm, dtype, t, g, dim, bits):
    """Whole in one piece and over lengths that are cut in pieces, with and without a mask."""
    rng = random.Random(t + dim)
    check_attention(lm, gen(t), 2, t, 2 * g, 2, dim, 16, bits, dtype, [100, 31], None, random_mask(rng, 2, t))
    check_attention(lm, gen(t), 2, t, 2 * g, 2, dim, 64, bits, dtype, [1500, 700], [t, max(1, t - 3)], None)


@pytest.mark.parametrize("dtype,hdtype", [(BF, BF), (BF, F), (HF, HF), (HF, F), (F, F)])
@pytest.mark.parametrize("d", [512, 1536, 4000, 5120, 8192, 9000, 333, 4099, 9001])
def test_norm_kernels(lm, d, dtype, hdtype):
    """A wave a row and a workgroup a row of every width, by eights and one by one."""
    g = gen(d)
    h, y = 3 * randn(g, 5, d, dtype=hdtype), randn(g, 5, d, dtype=dtype)
    for norm in ("rms", "layer"):
        ho, x = lm.norm_residual(h, y, norm=norm, alpha=0.9, beta=0.5)
        wh, wx, eh, ex = ref.norm_residual(h, y, norm, True, None, None, None, None, None, 0.9, 0.5, 1e-6)
        least = 2.0 ** -25 if dtype is HF else 0
        ref.close(ho, wh, eh + (2.0 ** -25 if hdtype is HF else 0), "h")
        ref.close(x, wx, ex + least, "x")


@pytest.mark.parametrize("bits,dim", [(4, 64), (8, 64), (8, 128), (16, 128), (8, 256), (16, 256)])
@TYPES
def test_keep_of_every_width(lm, dtype, bits, dim):
    """Tokens of 32 to 512 bytes: every second draft of forty kept."""
    cache = make_cache(lm, gen(dim), 6, 2, 16, dim, bits, dtype)
    table = torch.tensor([[4, 0, 5, 2]], dtype=torch.int32, device="cuda")
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    before = lm.cache_read(cache, table, i32([0]), 64, F)
    lm.cache_keep(cache, table, i32([9]), i32([[2 * j + 1 for j in range(20)] + [0] * 20]), i32([20]))
    after = lm.cache_read(cache, table, i32([0]), 64, F)
    order = list(range(9)) + [9 + 2 * j + 1 for j in range(20)] + list(range(29, 64))
    for a, b in zip(after, before):
        assert torch.equal(a, b[:, order])
