"""The ways of the dense operators' kernels that calls of many rows, and of
large products, take: against plain implementations in 64 bits, with the
tolerances of test_gpu_dense.py. (A thread of the norms' way for many rows takes
16 features of a row, and sums go up a tree of 9 levels at most: less than what
those allow for.)"""

import pytest
import torch

from test_gpu_dense import BF16, DEV, F32, SUM, apart, check_product, codes_of, gen, hidden, normal, plain_norm, rounding

from paper_2603_18599_gb300 import dense

pytestmark = pytest.mark.gpu

# rows of 2 blocks an SM and one, and a number that no number of blocks times two divides
MANY = [305, 2501]
# features: of blocks with threads that have no or one piece, of two to four stages of rows on
# their way, and (4097) rows that cannot be accessed 16 bytes at a time
WIDE = [520, 1000, 1600, 4096, 4097, 5120, 8192]


def many(t):
    assert t > 2 * torch.cuda.get_device_properties(0).multi_processor_count


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d", [513, *WIDE])
@pytest.mark.parametrize("t", MANY)
def test_quantise_of_many_rows(t, d, dtype):
    many(t)
    g = gen(t + d)
    x = hidden(g, t, d, dtype)
    x[t // 2], x[t - 1, d - 1] = 0, float("inf")
    top = x.float().abs().amax(1) / torch.full((), 127.0, device=DEV)
    want = (x.float() / torch.where(top > 0, top, 1.0)[:, None]).round().nan_to_num(0.0).to(torch.int8)
    for v in (x, apart(x, 8), apart(x, 5, 1)):
        codes, scale = dense.quantise(v)
        assert torch.equal(scale[:-1], top[:-1]) and scale[-1].isnan()
        assert torch.equal(codes[:-1], want[:-1]) and (codes[-1] == 0).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("centre,gain,bias,residual", [(False, True, False, True), (True, True, True, False), (True, False, True, True),
                                                       (False, False, False, False)])
@pytest.mark.parametrize("d", WIDE)
@pytest.mark.parametrize("t", MANY)
def test_norm_of_many_rows(t, d, centre, gain, bias, residual, dtype):
    many(t)
    g = gen(t + d)
    x, res = hidden(g, t, d, dtype) + (3.0 if centre else 0.0), hidden(g, t, d, dtype)
    w, b = (1 + 0.2 * normal(g, d) if gain else None), (normal(g, d) if bias else None)
    h = (x.float() + res.float()).to(dtype) if residual else x
    want, _, _, size = plain_norm(h, w, b, 1e-6, centre)
    tol = SUM * size * 1.01 + want.abs() * rounding(dtype)
    top, err = want.abs().amax(1), SUM * size.amax(1) * 1.01
    for spread in (lambda v: v, lambda v: apart(v, 8), lambda v: apart(v, 5, 1)):
        r = spread(res) if residual else None
        got = dense.norm(spread(x), w, b, residual=r, eps=1e-6, centre=centre)
        y = got[0] if residual else got
        assert y.dtype == dtype and ((y.double() - want).abs() <= tol).all()
        codes, scale, *rest = dense.norm_codes(spread(x), w, b, residual=r, eps=1e-6, centre=centre)
        if residual:
            assert torch.equal(got[1], h) and torch.equal(rest[0], h)
        assert ((scale.double() * 127 - top).abs() <= err + top * 2.0 ** -23).all()
        off = (codes.double() * scale.double()[:, None] - want).abs()
        assert (off <= scale.double()[:, None] * (0.5 + 2.0 ** -16) + err[:, None]).all()


def workspace(t, n, k, tokens, cut):
    """What a product asks for that goes in tiles of `tokens`, and with `cut`
    has tiles that several pairs of blocks share."""
    pairs = min(torch.cuda.get_device_properties(0).multi_processor_count // 2, 80)
    per, token_tiles = -(-k // 64), -(-t // tokens)
    slots = (2 if cut else 0) + (1 if per > 16 else 0)
    return 4096 + -(-4 * t // 256) * 256 + token_tiles * tokens * per * 128 + 2 * pairs * slots * (-(-tokens // 32) * 32) * 512


# tokens, channels, features; tokens of a tile; whether the last rounds are cut into equal runs.
# Tiles of 256 channels: 76 pairs of blocks take them.
PRODUCTS = [
    (256, 16384, 4096, 256, False),     # one accumulator; 64 tiles
    (203, 13435, 426, 208, False),
    (219, 19875, 2164, 224, True),      # one accumulator, 78 tiles in 76 runs
    (230, 20886, 2188, 240, True),      # runs longer than a tile: a part, a whole tile, a part
    (226, 39095, 2058, 240, True),      # a round of whole tiles, then runs
    (200, 65536, 4096, 208, True),      # two rounds, then longer runs
    (128, 65536, 4096, 128, True),      # the same with two accumulators
    (2048, 16384, 4096, 192, True),     # 704 tiles: eight rounds, then longer runs
    (64, 25600, 2048, 64, True),        # 100 tiles in runs
    (10, 39990, 1332, 16, True),
    (9, 20208, 924, 16, True),          # 79 tiles whose sums stay within 24 bits
    (318, 267, 1537, 16, True),         # 40 tiles in 76 runs
    (2048, 6144, 4096, 176, False),
]


@pytest.mark.parametrize("kind", ["any", "largest", "drift"])
@pytest.mark.parametrize("t,n,k,tokens,cut", PRODUCTS)
def test_ways_of_a_product(t, n, k, tokens, cut, kind):
    """Equal bit for bit. That a call still goes the way it stands here for is
    seen from the workspace that it asks for."""
    assert dense._size(0, "sjd_product_workspace_size", t, n, k) == workspace(t, n, k, tokens, cut)
    g = gen(t + k)
    x, w = codes_of(g, t, k), codes_of(g, n, k)
    if kind == "largest":               # sums of 2^24 and more, in parts of 1024 features
        x.fill_(-128)
        w.fill_(-128)
        w[:, ::7] = 1
        x[::3, ::5] = 3
    elif kind == "drift":
        x.copy_(x.abs().clamp(max=127) | 1)
        w.copy_(w.abs().clamp(max=127) | 1)
    check_product(g, x, w, kind != "largest", kind == "any", F32 if kind == "drift" else BF16, 5 if kind == "any" else 0)
