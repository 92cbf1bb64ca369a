"""The dense operators against plain implementations in 64 bits: products of
8-bit codes, norms and their gradient, the embedding and its gradient, at the
sizes, types and contents where they can go wrong.

Tolerances come from the arithmetic the operators declare (include/sjd.h):
- a product's sum is exact, and what follows is rounded step by step: equal,
  bit for bit;
- a sum over a row of up to 16384 features is taken by threads of at most 32
  of them and trees of 10 levels: off by 42 * 2^-24 of the sum of magnitudes at
  most. A mean is off by that share of the mean magnitude, 1 / sqrt(mean
  square) by half of it (21 * 2^-24), and a value takes at most 6 more
  roundings: 2^-18 (64 * 2^-24) of the magnitudes that it is made of;
- a column's sum takes the rows of a block one after another (at most
  ROWS_OF_A_BLOCK in these tests) and the blocks in 32 parts;
- codes are x / s rounded to nearest: half a step off;
- results in bf16 are half a unit off, 2^-8 of their value.
"""

import pytest
import torch

from paper_2603_18599_gb300 import dense, sjd

pytestmark = pytest.mark.gpu

DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16
SUM = 2.0 ** -18


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def normal(g, *shape):
    return torch.randn(*shape, device=DEV, generator=g)


def codes_of(g, *shape):
    return torch.randint(-128, 128, shape, device=DEV, generator=g).to(torch.int8)


def apart(x, by, offset=0):
    """The same values in wider rows, `offset` elements from their start."""
    wide = torch.full((*x.shape[:-1], x.shape[-1] + by), 77, dtype=x.dtype, device=x.device)
    wide[..., offset:offset + x.shape[-1]] = x
    return wide[..., offset:offset + x.shape[-1]]


def rounding(dtype):
    return 2.0 ** -8 if dtype == BF16 else 2.0 ** -24


# --- products -------------------------------------------------------------------

def plain_product(codes, scale, w, sw, bias, residual, dtype):
    y = (codes.double() @ w.double().T).float() * scale[:, None] * sw
    if bias is not None:
        y = y + bias
    if residual is not None:
        y = y + residual.float()
    return y.to(dtype)


def check_product(g, codes, w, bias, residual, dtype, offset=0):
    t, n = codes.shape[0], w.shape[0]
    scale, sw = normal(g, t).abs() + 0.01, normal(g, n).abs() + 0.01
    b = normal(g, n) if bias else None
    r = normal(g, t, n).to(dtype) if residual else None
    packed = dense.Weight(w, sw)
    got = dense.product(apart(codes, 9, offset) if offset else codes, scale, packed, bias=b,
                        residual=apart(r, 3, 1) if offset and residual else r, dtype=dtype)
    assert packed.sync() == sjd.SJD_OK
    assert torch.equal(got, plain_product(codes, scale, w, sw, b, r, dtype))


@pytest.mark.parametrize("dtype,bias,residual,offset", [(BF16, False, False, 0), (F32, True, True, 0), (BF16, True, True, 5), (F32, False, True, 1)])
@pytest.mark.parametrize("t,n,k", [
    (1, 1, 1), (2, 3, 5), (1, 128, 128), (2, 6144, 4096), (7, 300, 1000), (16, 256, 640), (17, 257, 129), (32, 4096, 4096), (33, 130, 16384),
    (64, 1000, 127), (65, 128, 4097), (100, 515, 2048), (128, 2048, 300), (129, 777, 1024), (200, 640, 1025), (256, 384, 8192), (257, 4096, 1600),
    (333, 10007, 1000), (513, 100, 100), (1000, 1, 3000), (2049, 1100, 384), (1, 20000, 64), (8, 1, 65536),
])
def test_product(t, n, k, dtype, bias, residual, offset):
    g = gen(t + n + k)
    check_product(g, codes_of(g, t, k), codes_of(g, n, k), bias, residual, dtype, offset)


@pytest.mark.parametrize("t,n,k", [(3, 200, 65536), (40, 130, 16384), (300, 300, 8191), (600, 4096, 4096), (5000, 300, 2200)])
@pytest.mark.parametrize("kind", ["largest", "lowest", "opposite", "drift", "one row", "one channel"])
def test_sums_beyond_24_bits_are_exact(t, n, k, kind):
    """The fp32 of a tensor core's accumulator holds integers up to 2^24; sums
    go up to 2^30, with odd addends all the way."""
    g = gen(k)
    x, w = codes_of(g, t, k), codes_of(g, n, k)
    if kind in ("largest", "lowest"):
        x.fill_(127 if kind == "largest" else -128)
        w.copy_(x[:1, :].expand(n, k))
        w[:, ::7] = 1
    elif kind == "opposite":                    # far up, and back down to almost nothing
        x.fill_(127)
        w[:, :k // 2], w[:, k // 2:] = 127, -127
        w[:, 3] = 1
    elif kind == "drift":
        x.copy_((x.abs().clamp(max=127) | 1))
        w.copy_((w.abs().clamp(max=127) | 1))
    else:                                       # the others' sums are small
        rows = x if kind == "one row" else w
        rows[:] = rows // 64
        (w if kind == "one row" else x).abs_().clamp_(min=100, max=127)
        rows[rows.shape[0] // 2] = 127
    check_product(g, x, w, False, False, F32)


@pytest.mark.parametrize("high", [2 ** 24, 2 ** 23, 2 ** 22])
def test_small_addends_beside_a_large_accumulator(high):
    """Sums that climb to just below `high` and then take addends of one, of
    either sign, in the same step of the tensor core and in later ones."""
    k = 2048
    big = (high - 1) // (127 * 127)
    x = torch.zeros(5, k, dtype=torch.int8, device=DEV)
    w = torch.zeros(130, k, dtype=torch.int8, device=DEV)
    x[:, :big], w[:, :big] = 127, 127
    g = gen(1)
    ones = torch.randint(-1, 2, (130, k - big), device=DEV, generator=g).to(torch.int8)
    w[:, big:], x[:, big:] = ones, 1
    perm = torch.randperm(k, device=DEV, generator=g)
    check_product(g, x, w, False, False, F32)
    check_product(g, x[:, perm].contiguous(), w[:, perm].contiguous(), False, False, F32)


def test_product_of_many_dimensions_no_rows_and_scales_that_are_no_numbers():
    g = gen(3)
    w, sw = codes_of(g, 40, 96), normal(g, 40).abs()
    packed = dense.Weight(w, sw)
    codes, scale = codes_of(g, 2, 3, 5, 96), normal(g, 2, 3, 5).abs()
    scale[1, 2, 4], scale[0, 0, 0] = float("nan"), 0.0
    codes[1, 2, 4] = 0
    residual = normal(g, 2, 3, 5, 40).bfloat16()
    y = dense.product(codes, scale, packed, residual=residual)
    want = plain_product(codes.view(30, 96), scale.view(30), w, sw, None, residual.view(30, 40), BF16).view(2, 3, 5, 40)
    assert y.shape == (2, 3, 5, 40) and y[1, 2, 4].isnan().all() and torch.equal(y[0], want[0]) and torch.equal(y[0, 0, 0], residual[0, 0, 0])
    assert not y[:1].isnan().any() and not y[1, :2].isnan().any()
    assert dense.product(codes[:0], scale[:0], packed).shape == (0, 3, 5, 40)
    assert torch.equal(dense.product(codes[0, 0, 0], scale[0, 0, 0], packed), torch.zeros(40, dtype=BF16, device=DEV))


def test_a_rows_product_does_not_depend_on_the_others():
    g = gen(4)
    w, sw, codes, scale = codes_of(g, 1000, 4096), normal(g, 1000).abs(), codes_of(g, 700, 4096), normal(g, 700).abs()
    packed = dense.Weight(w, sw)
    whole = dense.product(codes, scale, packed)
    for n in (1, 16, 40, 100, 300):
        assert torch.equal(dense.product(codes[:n], scale[:n], packed), whole[:n])


def test_a_weight_may_lie_in_wider_rows_and_go_at_once():
    g = gen(5)
    w, sw, codes, scale = codes_of(g, 300, 200), normal(g, 300).abs(), codes_of(g, 9, 200), normal(g, 9).abs()
    view = apart(w, 5, 3)
    packed = dense.Weight(view, sw)
    view.fill_(9)
    got = dense.product(codes, scale, packed)
    del packed
    assert torch.equal(got, plain_product(codes, scale, w, sw, None, None, BF16))


def test_offsets_past_32_bits_in_a_product():
    """The output's last rows are more than 2^32 elements from its first, the
    residual's too, and so are the codes of a large weight."""
    g = gen(6)
    t, n = 66000, 65600
    w, sw, codes, scale = codes_of(g, n, 64), normal(g, n).abs(), codes_of(g, t, 64), normal(g, t).abs()
    y = dense.product(codes, scale, dense.Weight(w, sw))
    for rows in (slice(0, 40), slice(65480, 65560), slice(t - 40, t)):
        assert torch.equal(y[rows], plain_product(codes[rows], scale[rows], w, sw, None, None, BF16))
    z = dense.product(codes, scale, dense.Weight(w, sw), residual=y)
    rows = slice(t - 40, t)
    assert torch.equal(z[rows], plain_product(codes[rows], scale[rows], w, sw, None, y[rows], BF16))
    del y, z
    n, k = 70000, 65536
    w = torch.randint(-128, 128, (n // 100, k), device=DEV, generator=g, dtype=torch.int32).to(torch.int8).repeat(100, 1)
    sw, codes, scale = normal(g, n).abs(), codes_of(g, 3, k), normal(g, 3).abs()
    y = dense.product(codes, scale, dense.Weight(w, sw), dtype=F32)
    assert torch.equal(y[:, -200:], plain_product(codes, scale, w[-200:], sw[-200:], None, None, F32))


# --- rows as codes --------------------------------------------------------------

DIMS = [1, 2, 7, 8, 31, 64, 100, 255, 256, 257, 512, 1000, 1600, 2048, 4096, 4097, 5120, 8191, 8192, 8200, 16383, 16384]


def hidden(g, t, d, dtype):
    x = normal(g, t, d) * torch.exp(normal(g, t, 1)) * (1 + 5 * (torch.rand(d, device=DEV, generator=g) < 0.02))
    return x.to(dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d", DIMS)
def test_quantise(d, dtype):
    g = gen(d)
    x = hidden(g, 37, d, dtype)
    x[3] = 0
    for v in (x, apart(x, 8), apart(x, 5, 1)):
        codes, scale = dense.quantise(v)
        top = x.float().abs().amax(1) / torch.full((), 127.0, device=DEV)
        assert torch.equal(scale, top)
        want = (x.float() / torch.where(top > 0, top, 1.0)[:, None]).round().to(torch.int8)
        assert torch.equal(codes, want)


def test_quantise_rows_that_are_not_finite_and_subnormal_ones():
    x = torch.ones(6, 300, device=DEV)
    x[0, 17], x[1, 299], x[2, 0] = float("nan"), float("inf"), -float("inf")
    x[3] = 2.0 ** -149 * 100
    x[3, 5] = 2.0 ** -149 * 190
    x[4] = 3e38
    codes, scale = dense.quantise(x)
    assert scale[:3].isnan().all() and (codes[:3] == 0).all()
    assert (codes[3] >= -127).all() and scale[3] > 0 and (codes[4] == 127).all() and (codes[5] == 127).all()
    assert ((codes[3].double() * scale[3].double() - x[3].double()).abs() <= 2.0 ** -149 * 100).all()


# --- norms ----------------------------------------------------------------------

def plain_norm(h, gain, bias, eps, centre):
    """y, the normed rows without gain, r and the error's scale, in 64 bits."""
    h = h.double()
    m = h.mean(1, keepdim=True) if centre else torch.zeros(h.shape[0], 1, dtype=torch.float64, device=DEV)
    r = ((h - m).square().mean(1, keepdim=True) + eps).rsqrt()
    u = (h - m) * r
    y = u * (gain.double() if gain is not None else 1.0)
    size = y.abs() + (h.abs().mean(1, keepdim=True) * r * (gain.double().abs() if gain is not None else 1.0) if centre else 0.0)
    if bias is not None:
        y, size = y + bias.double(), size + bias.double().abs()
    return y, u, r, size


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("centre,gain,bias,residual", [(False, True, False, True), (True, True, True, False), (True, False, True, True),
                                                       (False, False, False, False)])
@pytest.mark.parametrize("d", DIMS)
def test_norm(d, centre, gain, bias, residual, dtype):
    g = gen(d + 1)
    t = 45
    x, res = hidden(g, t, d, dtype) + (3.0 if centre else 0.0), hidden(g, t, d, dtype)
    w, b = (1 + 0.2 * normal(g, d) if gain else None), (normal(g, d) if bias else None)
    h = (x.float() + res.float()).to(dtype) if residual else x
    want, _, _, size = plain_norm(h, w, b, 1e-6, centre)
    tol = SUM * size * 1.01 + want.abs() * rounding(dtype)
    for spread in (lambda v: v, lambda v: apart(v, 8), lambda v: apart(v, 5, 1)):
        got = dense.norm(spread(x), w, b, residual=spread(res) if residual else None, eps=1e-6, centre=centre)
        y = got
        if residual:
            y = got[0]
            assert torch.equal(got[1], h)
        assert y.dtype == dtype and ((y.double() - want).abs() <= tol).all()
        codes, scale, *rest = dense.norm_codes(spread(x), w, b, residual=spread(res) if residual else None, eps=1e-6, centre=centre)
        if residual:
            assert torch.equal(rest[0], h)
        top = want.abs().amax(1)
        err = SUM * size.amax(1) * 1.01
        assert ((scale.double() * 127 - top).abs() <= err + top * 2.0 ** -23).all()
        off = (codes.double() * scale.double()[:, None] - want).abs()
        assert (off <= scale.double()[:, None] * (0.5 + 2.0 ** -16) + err[:, None]).all()


def test_norm_of_zeros_and_of_rows_that_are_not_finite():
    x = torch.ones(5, 333, device=DEV)
    x[0] = 0
    x[1, 7], x[2, 8] = float("nan"), float("inf")
    for centre in (False, True):
        y = dense.norm(x, eps=1e-6, centre=centre)
        assert (y[0] == 0).all() and y[1].isnan().all() and y[2, 8].isnan()
        assert torch.equal(y[3], y[4]) and not y[3:].isnan().any()
        codes, scale = dense.norm_codes(x, eps=1e-6, centre=centre)
        assert scale[1].isnan() and scale[2].isnan() and (codes[1:3] == 0).all() and scale[0] == 0 and (codes[0] == 0).all()
    assert dense.norm(x[:0]).shape == (0, 333)
    assert dense.norm(x.view(5, 1, 333)).shape == (5, 1, 333) and dense.norm(x[3]).shape == (333,)


@pytest.mark.parametrize("t", [1, 2, 31, 3000])
def test_long_rows_far_from_zero(t):
    """A mean that is a thousand times the spread around it."""
    g = gen(t)
    x = 1000.0 + normal(g, t, 4096)
    want, _, _, size = plain_norm(x, None, None, 1e-6, True)
    assert ((dense.norm(x, centre=True).double() - want).abs() <= SUM * size + want.abs() * 2.0 ** -24).all()


# --- the norm's gradient ----------------------------------------------------------

ROWS_OF_A_BLOCK = 20


def plain_norm_gradient(dy, x, gain, eps, centre, dh):
    _, u, r, _ = plain_norm(x, None, None, eps, centre)
    dy = dy.double()
    w = gain.double() if gain is not None else torch.ones(x.shape[1], dtype=torch.float64, device=DEV)
    g = dy * w
    along = (g * u).mean(1, keepdim=True)
    dx = r * (g - u * along - (g.mean(1, keepdim=True) if centre else 0.0))
    shift = x.double().abs().mean(1, keepdim=True) * r if centre else torch.zeros_like(r)   # the mean's part in u
    mag = (g.abs() * (u.abs() + shift)).mean(1, keepdim=True)
    size = r * (g.abs() + g.abs().mean(1, keepdim=True) + (u.abs() + shift) * mag)
    if dh is not None:
        dx, size = dx + dh.double(), size + dh.double().abs()
    return dx, (dy * u).sum(0), dy.sum(0), size, (dy.abs() * (u.abs() + shift)).sum(0), dy.abs().sum(0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("centre,gain,dh", [(False, True, True), (True, True, False), (True, False, True), (False, False, False)])
@pytest.mark.parametrize("t,d", [(1, 64), (3, 1), (45, 7), (700, 100), (333, 256), (1000, 1000), (5000, 1600), (40, 4096), (2500, 4097), (600, 8192),
                                 (350, 8200), (310, 16384), (9, 16383)])
def test_norm_gradient(t, d, centre, gain, dh, dtype):
    g = gen(t + d)
    x, dy = hidden(g, t, d, dtype) + (1.0 if centre else 0.0), normal(g, t, d).to(dtype)
    w, r = (1 + 0.2 * normal(g, d) if gain else None), (normal(g, t, d).to(dtype) if dh else None)
    dx, dg, db, size, gsize, bsize = plain_norm_gradient(dy, x, w, 1e-6, centre, r)
    columns = (ROWS_OF_A_BLOCK + 64 + 64) * 2.0 ** -24
    for spread in (lambda v: v, lambda v: apart(v, 8), lambda v: apart(v, 5, 1)):
        got = dense.norm_gradient(spread(dy), spread(x), w, 1e-6, centre, dh=spread(r) if dh else None, bias=centre)
        # (three terms, each off by the sums in it and by those in r: 2.5 times a value's)
        assert ((got[0].double() - dx).abs() <= 2.5 * SUM * size * 1.01 + dx.abs() * rounding(dtype)).all()
        assert ((got[1].double() - dg).abs() <= columns * gsize).all()
        if centre:
            assert ((got[2].double() - db).abs() <= columns * bsize).all()
        else:
            assert got[2] is None


@pytest.mark.parametrize("centre", [False, True])
def test_norm_gradient_against_differences(centre):
    """Along random directions, the definition's central differences in 64 bits
    (error of second order: 1e-4 squared times third derivatives near 1)."""
    g = gen(8)
    t, d = 7, 96
    x, dy, w = normal(g, t, d), normal(g, t, d), 1 + 0.2 * normal(g, d)
    dx, dgain, dbias = dense.norm_gradient(dy, x, w, 1e-6, centre, bias=True)
    b = torch.zeros(d, device=DEV)

    def loss(x, w, b):
        m = x.mean(1, keepdim=True) if centre else 0.0
        return (dy.double() * ((x - m) / ((x - m).square().mean(1, keepdim=True) + 1e-6).sqrt() * w + b)).sum()

    for _ in range(5):
        vx, vw, vb = normal(g, t, d).double(), normal(g, d).double(), normal(g, d).double()
        e = 1e-4
        up = loss(x.double() + e * vx, w.double() + e * vw, b.double() + e * vb)
        down = loss(x.double() - e * vx, w.double() - e * vw, b.double() - e * vb)
        along = (dx.double() * vx).sum() + (dgain.double() * vw).sum() + (dbias.double() * vb).sum()
        # (sums of 700 products, each off by 2^-16, and the differences' 1e-8 of a third derivative below 100 a row)
        terms = (dx.double() * vx).abs().sum() + (dgain.double() * vw).abs().sum() + (dbias.double() * vb).abs().sum()
        assert abs((up - down) / (2 * e) - along) <= 2.0 ** -16 * terms + 1e-6 * t * 100


# --- embedding ------------------------------------------------------------------

@pytest.mark.parametrize("table,dtype", [(BF16, BF16), (BF16, F32), (F32, BF16), (F32, F32)])
@pytest.mark.parametrize("t,v,d", [(1, 1, 1), (32, 1000, 4096), (7, 300, 100), (1000, 17, 257), (70000, 5, 8), (3, 9, 65536), (5, 100, 1030)])
def test_embed(t, v, d, table, dtype):
    g = gen(t + d)
    E = normal(g, v, d).to(table)
    tokens = torch.randint(-2, v + 2, (t,), device=DEV, generator=g).int()
    tokens[0] = v - 1
    if t > 2:
        tokens[1], tokens[2] = 2 ** 31 - 1, -2 ** 31
    inside = (tokens >= 0) & (tokens < v)
    want = (E.float()[tokens.long().clamp(0, v - 1)] * 1.7).to(dtype) * inside[:, None]
    for view in (E, apart(E, 8), apart(E, 5, 1)):
        assert torch.equal(dense.embed(view, tokens, scale=1.7, dtype=dtype), want)
    assert torch.equal(dense.embed(E, tokens.view(t, 1, 1), 1.7, dtype), want.view(t, 1, 1, d))
    assert dense.embed(E, tokens[:0]).shape == (0, d)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("t,v,d,skew", [(1, 1, 1, 1), (32, 1000, 4096, 1), (700, 300, 100, 3), (5000, 17, 257, 1), (3000, 1, 64, 1), (40000, 70000, 36, 3),
                                        (20, 513, 65536, 1), (2000, 512, 1000, 4), (1025, 256, 8, 8)])
def test_embed_gradient(t, v, d, skew, dtype):
    g = gen(t + d)
    dy = normal(g, t, d).to(dtype)
    tokens = (v * torch.rand(t, device=DEV, generator=g) ** skew).long().clamp(max=v - 1).int()
    if t > 3:
        tokens[1], tokens[2], tokens[3] = -1, v, -2 ** 31
    inside = (tokens >= 0) & (tokens < v)
    at = tokens.long()[inside]

    def sums(values):
        return torch.zeros(v, d, dtype=torch.float64, device=DEV).index_add_(0, at, values[inside])

    want = sums(dy.double()) * 0.3
    # (one addition after another, and the product with the scale, itself rounded to fp32)
    count = torch.bincount(at, minlength=v).double()[:, None]
    tol = (count + 2) * 2.0 ** -24 * sums(dy.double().abs()) * 0.3
    first = None
    for view in (dy, apart(dy, 8), apart(dy, 5, 1)):
        got = dense.embed_gradient(view, tokens, v, scale=0.3)
        assert ((got.double() - want).abs() <= tol).all()
        first = got if first is None else first
        assert torch.equal(got, first)
    # the gradient is the transpose: <dy, embed(E)> = <gradient, E>, each product and sum off by less than 2^-16 of the magnitudes
    E = normal(g, v, d)
    y = dense.embed(E, tokens, scale=0.3, dtype=F32).double()
    assert ((dy.double() * y).sum() - (first.double() * E).sum()).abs() <= 2.0 ** -16 * ((dy.double() * y).abs().sum() + (first.double() * E).abs().sum())
    assert torch.equal(dense.embed_gradient(dy[:0], tokens[:0], v), torch.zeros(v, d, device=DEV))


def test_offsets_past_32_bits_in_an_embedding():
    g = gen(9)
    v, d = 70000, 65536
    E = torch.empty(v, d, dtype=BF16, device=DEV)
    E[-3:] = normal(g, 3, d).bfloat16()
    tokens = torch.full((66000,), v - 2, dtype=torch.int32, device=DEV)
    tokens[-1] = v - 1
    y = dense.embed(E, tokens)
    assert torch.equal(y[-1], E[-1]) and torch.equal(y[-2], E[-2])
    del y
    grad = dense.embed_gradient(E[-3:], tokens[-3:], v)
    assert torch.equal(grad[-1], E[-1].float()) and torch.equal(grad[-2], E[-3].float() + E[-2].float())


# --- shapes and strides that documents allow and callers seldom use -------------------

@pytest.mark.parametrize("d", [64, 100, 1600, 4096])
def test_rows_that_repeat_single_rows_and_vectors_off_boundaries(d):
    """Rows of stride 0 (a broadcast), one row without a dimension for it, and
    gains, biases and scales that do not start on 16-byte boundaries: the same bits as
    from contiguous copies (whose sums are taken in the same order where the ways
    are the same; else within the norm's bound)."""
    g = gen(d)
    row, dy = normal(g, 1, d).bfloat16(), normal(g, 1, d).bfloat16()
    many, dys = row.expand(7, d), dy.expand(7, d)
    ids = torch.arange(7, device=DEV).int() // 3
    for a, b in ((dense.norm(many), dense.norm(many.contiguous())), (dense.quantise(many)[0], dense.quantise(many.contiguous())[0]),
                 *zip(dense.norm_gradient(dys, many, bias=True), dense.norm_gradient(dys.contiguous(), many.contiguous(), bias=True)),
                 (dense.embed_gradient(dys, ids, 4), dense.embed_gradient(dys.contiguous(), ids, 4))):
        assert torch.equal(a, b)
    assert torch.equal(dense.norm(row[0]), dense.norm(row)[0])
    E, token = normal(g, 5, d), torch.tensor(3, dtype=torch.int32, device=DEV)
    assert torch.equal(dense.embed(E, token), E[3])
    assert torch.equal(dense.embed_gradient(E[1], token, 5)[3], E[1])
    held = normal(g, 3, d + 1)
    w, b = held[0, 1:], held[1, 1:]
    x = normal(g, 40, d)
    for centre in (False, True):
        want, _, _, size = plain_norm(x, w, b, 1e-6, centre)
        assert ((dense.norm(x, w, b, centre=centre).double() - want).abs() <= SUM * size + want.abs() * 2.0 ** -24).all()
        dx, dg, db, size, gsize, bsize = plain_norm_gradient(x, x, w, 1e-6, centre, None)
        got = dense.norm_gradient(x, x, w, 1e-6, centre, bias=True)
        assert ((got[0].double() - dx).abs() <= 2.5 * SUM * size * 1.01 + dx.abs() * 2.0 ** -24).all()
        assert ((got[1].double() - dg).abs() <= (ROWS_OF_A_BLOCK + 128) * 2.0 ** -24 * gsize).all()
    codes, weight = codes_of(g, 41, d), codes_of(g, 72, d)
    scale, sw, bias = held[2, :1].abs().expand(41).contiguous(), normal(g, 73)[1:].abs(), normal(g, 73)[1:]
    for n in (1, 3, 7, 41):
        got = dense.product(codes[:n], scale[:n], dense.Weight(weight, sw), bias=bias, dtype=F32)
        assert torch.equal(got, plain_product(codes[:n], scale[:n], weight, sw, bias, None, F32))
    repeated = codes[:1].expand(30, d)
    assert torch.equal(dense.product(repeated, scale[:30], dense.Weight(weight, sw), dtype=F32),
                       plain_product(repeated, scale[:30], weight, sw, None, None, F32))


# --- streams, graphs, refusals -----------------------------------------------------

def chain(s):
    """Every operator, one after another."""
    x = dense.embed(s["table"], s["tokens"], scale=2.0)
    codes, scale, h = dense.norm_codes(x, s["gain"], residual=s["x"])
    y = dense.product(codes, scale, s["weight"], bias=s["bias"], residual=h)
    out = dense.norm(y, s["gain"], s["bias"], centre=True)
    dy, dgain, dbias = dense.norm_gradient(out, y, s["gain"], centre=True, bias=True, dh=h)
    return {"out": out, "y": y, "dy": dy, "dgain": dgain, "dbias": dbias, "grad": dense.embed_gradient(dy, s["tokens"], s["table"].shape[0], 2.0)}


def chain_inputs(seed, t=50, d=512, v=300):
    g = gen(seed)
    return {"table": normal(g, v, d).bfloat16(), "tokens": torch.randint(-1, v, (t,), device=DEV, generator=g).int(), "gain": 1 + 0.1 * normal(g, d),
            "bias": normal(g, d), "x": normal(g, t, d).bfloat16(), "weight": dense.Weight.quantise(normal(g, d, d))}


def test_a_chain_on_another_stream_and_in_graphs():
    """Two captured graphs of the same calls, replayed in turn with other
    inputs, and calls on a side stream behind a long one: the same bits as alone."""
    a, b = chain_inputs(1), chain_inputs(2)
    want = [chain(a), chain(b)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    big = normal(gen(3), 4000, 4000)
    with torch.cuda.stream(side):
        for _ in range(20):
            big = (big @ big).clamp(-1, 1)
        got = chain(a)
    side.synchronize()
    assert all(torch.equal(got[k], want[0][k]) for k in got)

    held = chain_inputs(4)
    held["weight"] = a["weight"]
    graphs, outs = [torch.cuda.CUDAGraph() for _ in range(2)], []
    chain(held)
    torch.cuda.synchronize()
    for graph in graphs:
        with torch.cuda.graph(graph):
            outs.append(chain(held))
    for turn in range(3):
        for k, v in held.items():
            if k != "weight":
                v.copy_((a, b)[turn % 2][k])
        for graph in graphs:
            graph.replay()
        expected = want[0] if turn % 2 == 0 else chain(dict(b, weight=a["weight"]))
        for out in outs:
            assert all(torch.equal(out[k], expected[k]) for k in out), turn
    assert a["weight"].sync() == sjd.SJD_OK


def test_two_streams_at_once():
    """Calls of both streams in flight together share no workspace."""
    ins = [chain_inputs(s, t=600, d=1024) for s in (5, 6)]
    want = [chain(s) for s in ins]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ins]
    got = []
    for _ in range(5):
        for s, stream in zip(ins, streams):
            with torch.cuda.stream(stream):
                got.append(chain(s))
    torch.cuda.synchronize()
    for i, out in enumerate(got):
        assert all(torch.equal(out[k], want[i % 2][k]) for k in out)


def test_a_weight_may_go_while_its_last_call_runs():
    side = torch.cuda.Stream()
    g = gen(7)
    w, sw, codes, scale = codes_of(g, 512, 512), normal(g, 512).abs(), codes_of(g, 9, 512), normal(g, 9).abs()
    packed = dense.Weight(w, sw)
    size = packed._packed.numel()
    big = normal(g, 4000, 4000)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):
            big = (big @ big).clamp(-1, 1)
        y = dense.product(codes, scale, packed)
    del packed
    other = torch.zeros(size, dtype=torch.uint8, device=DEV)
    side.synchronize()
    assert torch.equal(y, plain_product(codes, scale, w, sw, None, None, BF16)) and not other.any()


def test_refusals():
    g = gen(8)
    x, xb, v = normal(g, 4, 64), normal(g, 4, 64).bfloat16(), normal(g, 64)
    codes, scale = codes_of(g, 4, 64), v[:4].abs()
    weight = dense.Weight(codes_of(g, 32, 64), v[:32].abs())
    tokens = torch.zeros(4, dtype=torch.int32, device=DEV)
    wants = normal(g, 4, 64).requires_grad_()
    calls = [
        lambda: dense.Weight(codes.float(), scale), lambda: dense.Weight(codes, scale[:3]), lambda: dense.Weight(codes.T, v),
        lambda: dense.Weight(codes, scale.double()), lambda: dense.Weight(codes, None), lambda: dense.Weight(codes[:0], scale[:0]),
        lambda: dense.Weight(codes[None], scale), lambda: dense.Weight.quantise(x.half()),
        lambda: dense.product(codes[:, :63], scale, weight), lambda: dense.product(codes, scale[:3], weight), lambda: dense.product(x, scale, weight),
        lambda: dense.product(codes, scale.double(), weight), lambda: dense.product(codes, scale, weight, dtype=torch.float16),
        lambda: dense.product(codes, scale, weight, bias=v), lambda: dense.product(codes, scale, weight, bias=v[:32].bfloat16()),
        lambda: dense.product(codes, scale, weight, residual=xb), lambda: dense.product(codes, scale, weight, residual=x[:, :32]),
        lambda: dense.product(codes.T.contiguous().T, scale, weight), lambda: dense.product(codes.cpu(), scale, weight),
        lambda: dense.quantise(x.half()), lambda: dense.quantise(wants), lambda: dense.quantise(x.T), lambda: dense.quantise(x[:, :0]),
        lambda: dense.quantise(torch.zeros(1, 16385, device=DEV)), lambda: dense.quantise(torch.zeros((), device=DEV)),
        lambda: dense.norm(x, v[:63]), lambda: dense.norm(x, v.bfloat16()), lambda: dense.norm(x, v, v[None]), lambda: dense.norm(x, eps=-1.0),
        lambda: dense.norm(x, eps=float("nan")), lambda: dense.norm(x, residual=xb), lambda: dense.norm(x, residual=x[:3]), lambda: dense.norm(wants),
        lambda: dense.norm(x, residual=wants), lambda: dense.norm(x, v.clone().requires_grad_()), lambda: dense.norm(normal(g, 4, 6, 64).transpose(0, 1)),
        lambda: dense.norm_codes(x.double()), lambda: dense.norm_codes(wants),
        lambda: dense.norm_gradient(xb, x), lambda: dense.norm_gradient(x[:2], x), lambda: dense.norm_gradient(x, x, dh=xb),
        lambda: dense.norm_gradient(x, x, v[:5]), lambda: dense.norm_gradient(x, wants),
        lambda: dense.embed(x, tokens.long()), lambda: dense.embed(x, tokens.cpu()), lambda: dense.embed(wants, tokens), lambda: dense.embed(x[:0], tokens),
        lambda: dense.embed(x, tokens, dtype=torch.float16), lambda: dense.embed(codes, tokens), lambda: dense.embed(v, tokens),
        lambda: dense.embed(x, tokens.repeat(2)[::2]),
        lambda: dense.embed_gradient(x, tokens[:3], 5), lambda: dense.embed_gradient(x, tokens.long(), 5), lambda: dense.embed_gradient(x, tokens, 0),
        lambda: dense.embed_gradient(wants, tokens, 5), lambda: dense.embed_gradient(x.half(), tokens, 5),
    ]
    for i, call in enumerate(calls):
        with pytest.raises(ValueError):
            call()
            pytest.fail("call %d was taken" % i)
    with torch.no_grad():
        assert torch.equal(dense.norm(wants), dense.norm(wants.detach()))
    # what the binding sees to itself: a workspace, and one that is large enough
    L = dense.load()
    codes, y = codes_of(g, 20, 64), torch.empty(20, 32, dtype=BF16, device=DEV)
    size, room = L.sjd_product_workspace_size(20, 32, 64), torch.empty(1 << 20, dtype=torch.uint8, device=DEV)
    assert size > 0 and L.sjd_product_workspace_size(2, 32, 64) == 0
    args = [weight._at, 32, 64, dense._pack(codes), v.data_ptr(), 20, None, None, sjd.SJD_BF16, dense._pack(y), None, size, None]
    assert L.sjd_product(*args) == sjd.SJD_ERR_ARG
    args[10:12] = room.data_ptr(), size - 1
    assert L.sjd_product(*args) == sjd.SJD_ERR_CAPACITY
    size = L.sjd_norm_gradient_workspace_size(4, 64, sjd.SJD_F32)
    assert L.sjd_norm_gradient(dense._pack(x), dense._pack(x), None, 1e-6, 0, None, 4, 64, sjd.SJD_F32, dense._pack(x.clone()), v.data_ptr(), None,
                               room.data_ptr(), size - 1, None) == sjd.SJD_ERR_CAPACITY
