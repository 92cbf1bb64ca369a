"""Attention over an 8-bit cache whose values' scales lie far apart, against
the definition in 64 bits: keys that a row does not see, or sees with next to
no weight, whatever the size of their values; keys of most of the weight whose
values are small or zero; and values near the ends of fp32's range.

Tolerances, from the arithmetic that include/sjd.h declares for an 8-bit cache:
- a weight times its value's scale is rounded to fp16, 2^-11 of it, or loses
  at most 2^-29 of the row's largest such product where it is far below that:
  2^-11 size + 2^-29 max(p s) sum |code|, both times 1.05 for what the fp32
  steps before add;
- a result is rounded to bf16 once: half a unit, at most 2^-8 of the value;
  over many results 2^-9 / sqrt(3) of 1.4, the middle of an octave, at most in
  the 2-norm, 0.0016 (0.002 is held to);
- scores are fp32 sums of D products, 2^-17 of the sum of magnitudes at most.
"""

import math

import pytest
import torch

import test_gpu_kv as base
from paper_2603_18599_gb300 import kv, sjd

pytestmark = pytest.mark.gpu

DEV = "cuda"
EIGHT = [torch.float8_e4m3fn, torch.int8]
D = 64
# (heads, kv_heads, new tokens): the rows of a key head, 32, 64, 128 and more, take different kernels
ROWS = [(8, 2, 7), (8, 2, 12), (8, 2, 30), (4, 2, 140)]


def held(h, layer, table, b, last):
    """Codes and scales of the first `last` tokens of a sequence, f64."""
    rows = torch.arange(last, device=DEV)
    page, slot = table[b].long()[rows // h.cfg.page_size], rows % h.cfg.page_size
    out = []
    for name in ("k", "v"):
        cache = getattr(layer, name)
        codes = cache.view(torch.uint8)[page, :, slot].contiguous().view(cache.dtype).double()
        out += [codes, getattr(layer, name + "_scale")[page, :, slot].double()]
    return out


def check(h, layer, q, table, starts, mask, got, lse, scale=None):
    """mask [B or 1, n, n] of the chunk's own keys."""
    c = h.cfg
    n, G = q.shape[1], c.heads // c.kv_heads
    scale = c.head_dim ** -0.5 if scale is None else scale
    errors, sizes = [], []
    for b, s in enumerate(starts):
        kc, ks, vc, vs = held(h, layer, table, b, s + n)
        seen = torch.ones(n, s + n, dtype=torch.bool, device=DEV)
        seen[:, s:] = mask[b if mask.shape[0] > 1 else 0]
        for head in range(c.heads):
            x, g = q[b, :, head].double(), head // G
            score = (x @ (kc[:, g] * ks[:, g, None]).T * scale).masked_fill(~seen, -math.inf)
            spread = (x.abs() @ (kc[:, g].abs() * ks[:, g, None]).T * abs(scale)).masked_fill(~seen, 0).amax(-1)
            p = torch.softmax(score, -1).nan_to_num(0.0)          # (a row that sees nothing)
            ps = p * vs[:, g]
            o, size = ps @ vc[:, g], ps @ vc[:, g].abs()
            lost = 2.0 ** -29 * ps.amax(-1, keepdim=True) * (seen.double() @ vc[:, g].abs())
            wrong = 2.0 ** -17 * spread + 2e-6
            tol = 1.05 * (2.0 ** -11 * size + lost) + 2.0 ** -8 * o.abs() + 2 * wrong[:, None] * size
            mine = got[b, :, head].double()
            assert mine.isfinite().all()
            off = (mine - o).abs()
            assert (off <= tol).all(), (b, head, (off / tol.clamp(min=1e-300)).amax())
            # (results that cancel, or are next to nothing beside the row's largest, say little)
            some = o.norm(dim=-1) > 0.05 * size.norm(dim=-1)
            errors.append(((mine - o).norm(dim=-1) / o.norm(dim=-1))[some])
            sizes.append(some.sum())
            want = torch.logsumexp(score, -1)
            assert ((lse[b, :, head].double() - want).abs() <= wrong + 1e-6 * want.abs())[want.isfinite()].all()
            assert (lse[b, :, head][want == -math.inf] == -math.inf).all()
    errors = torch.cat(errors)
    if errors.numel() > 20:
        assert errors.square().mean().sqrt() <= 0.002, errors.square().mean().sqrt()


def causal(n):
    return torch.ones(1, n, n, dtype=torch.bool, device=DEV).tril()


class Scene:
    """A cache that holds keys and values of one's own making: `edit(k, v)`
    changes them, [B, tokens, kv_heads, D] in f32, before they are written.
    Element 0 of every query is 8 and of every key 0, so that a key's element
    0 moves its scores alone."""

    def __init__(self, dtype, heads, kv_heads, n, starts, edit, page=24, seed=0, spread=0.3):
        self.starts, self.n = starts, n
        B, most = len(starts), max(starts) + n
        self.h, self.layer, self.table, self.start, g = base.make(B, heads, kv_heads, D, dtype, page, starts, n, seed=seed)
        k = base.normal(g, B, most, kv_heads, D)
        k[..., 0] = 0.0
        v = base.normal(g, B, most, kv_heads, D) * torch.exp(spread * base.normal(g, B, most, kv_heads, 1))
        edit(k, v)
        whole = kv.KV(B, heads, kv_heads, D, self.h.cfg.n_pages, page, self.h.cfg.max_pages, most, dtype)
        whole.write(kv.Layer(*self.layer._t), k, v, self.table, torch.zeros_like(self.start), self.start + n)
        assert whole.sync() == sjd.SJD_OK
        self.q = base.normal(g, B, n, heads, D).bfloat16()
        self.q[..., 0] = 8.0

    def attend(self, mask=None):
        o, lse = self.h.attend(self.layer, self.q, self.table, self.start, mask="causal" if mask is None else mask, lse=True)
        assert self.h.sync() == sjd.SJD_OK
        return o, lse

    def check(self, mask=None):
        o, lse = self.attend(mask)
        check(self.h, self.layer, self.q, self.table, self.starts, causal(self.n) if mask is None else mask, o, lse)
        return o


@pytest.mark.parametrize("dtype", EIGHT)
@pytest.mark.parametrize("rows", ROWS)
def test_values_of_one_size(dtype, rows):
    """The declared precision where no value stands out, several tiles to a block."""
    Scene(dtype, *rows, [1500 - 70 * b for b in range(14)], lambda k, v: None).check()


@pytest.mark.parametrize("dtype", EIGHT)
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("power", [6, 12, 20, 24, 28, 32, 40, 90])
def test_large_values_of_unseen_keys_change_nothing(dtype, rows, power):
    """The chunk's last token, and under a mask a token in the middle, has
    values 2^power times the others': the rows that do not see it give the
    same as without it."""
    heads, kv_heads, n = rows
    starts = [130, 613]
    for given in (False, True):
        mask = torch.ones(1, n, n, dtype=torch.bool, device=DEV).tril() if given else None
        where = n // 2 if given else n - 1
        if given:
            mask[0, :, where] = False

        def edit(k, v, by=2.0 ** power):
            for b, s in enumerate(starts):
                v[b, s + where] *= by

        o = Scene(dtype, *rows, starts, edit).check(mask)
        plain = Scene(dtype, *rows, starts, lambda k, v: None).attend(mask)[0]
        rest = [t for t in range(n) if given or t != where]
        off = (o[:, rest].double() - plain[:, rest].double()).norm() / plain[:, rest].double().norm()
        assert off <= 0.003, off


@pytest.mark.parametrize("dtype", EIGHT)
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("power,score", [(12, -200), (20, -200), (28, -200), (40, -200), (40, -20), (20, -25), (20, -14), (90, -60), (90, -80)])
def test_large_values_of_keys_of_little_weight(dtype, rows, power, score):
    """A key that every row sees with a score far below the others'; in the
    first tile, in the middle and in the last one."""
    starts = [700, 650, 300]

    def edit(k, v):
        for b, (s, at) in enumerate(zip(starts, (3, 400, 298))):
            v[b, at] *= 2.0 ** power
            k[b, at, :, 0] = score / 8.0 * D ** 0.5
    Scene(dtype, *rows, starts, edit).check()


@pytest.mark.parametrize("dtype", EIGHT)
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("power", [-40, 20, 40, 80])
def test_what_came_before_the_largest_scores(dtype, rows, power):
    """The first tiles hold scores far below the later ones' and values far
    from theirs: several tiles to a block, so that the row's unit has to fall,
    or rise, with its reference."""
    starts = [1500 - 60 * b for b in range(14)]

    def edit(k, v):
        v[:, :700] *= 2.0 ** power
        k[:, :300, :, 0] = -160.0 / 8.0 * D ** 0.5
        k[:, 300:700, :, 0] = -90.0 / 8.0 * D ** 0.5
    Scene(dtype, *rows, starts, edit).check()


@pytest.mark.parametrize("dtype", EIGHT)
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("factor", [0.0, 2.0 ** -12, 2.0 ** -30, 2.0 ** -60])
def test_small_values_of_the_key_with_the_weight(dtype, rows, factor):
    """A key that has nearly all of every row's weight, and values of little
    size or zeros: the result is what the others leave."""
    starts = [1500 - 60 * b for b in range(14)]

    def edit(k, v):
        v[:, 5] *= factor
        k[:, 5, :, 0] = 25.0 / 8.0 * D ** 0.5
        v[:, 9] = 0.0
    Scene(dtype, *rows, starts, edit).check()


@pytest.mark.parametrize("dtype", EIGHT)
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("spread", [1.0, 4.0])
def test_values_of_many_sizes(dtype, rows, spread):
    """Values whose sizes are spread over 2^10 and 2^40."""
    Scene(dtype, *rows, [1300 - 60 * b for b in range(14)], lambda k, v: None, spread=spread).check()


@pytest.mark.parametrize("dtype", EIGHT)
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("size", [1e-33, 1e-20, 1e20, 1e33])
def test_values_near_the_ends_of_the_range(dtype, rows, size):
    """Scores spread over 2^30: the sum of the weights keeps the small ones."""
    def edit(k, v):
        v *= size
        k[..., 0] = torch.linspace(-10.0, 10.0, k.shape[1], device=DEV)[:, None] / 8.0 * D ** 0.5
    Scene(dtype, *rows, [900, 641], edit).check()


@pytest.mark.parametrize("dtype", EIGHT)
@pytest.mark.parametrize("rows", ROWS)
def test_caches_of_zeros(dtype, rows):
    """Values that are all zeros, of all keys and of a tile's: results of
    zeros, and finite sums."""
    def zeros(k, v):
        v.zero_()
    assert (Scene(dtype, *rows, [500, 129], zeros).check() == 0).all()

    def tile(k, v):
        v[:, 128:256] = 0.0
        v[:, 300:] = 0.0
    Scene(dtype, *rows, [500, 129], tile).check()
