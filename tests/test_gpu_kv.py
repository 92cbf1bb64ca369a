"""The window forward's operators against plain implementations in 64 bits:
rotary positions with several axes, the paged cache (write, quantise, read)
and attention of a chunk over it, at the sizes, masks and contents where
they can go wrong.

Tolerances come from the arithmetic the operators declare (include/sjd.h):
- a rotation rounds the angle to 24 bits of half a turn (1.9e-7), sincospi
  is within 2 ulp, and a result takes three fp32 roundings: 8e-7 (|u| + |w|);
  plus half a unit of bf16 (at most 2^-8 of the value: 8 bits) where the
  result is bf16;
- codes are x / s rounded to nearest in fp32 arithmetic: equal, bit for bit,
  where the input is not rotated; half a step off at most where it is;
- an attention's weights are rounded to bf16 (2^-8 each), its scores are
  fp32 sums of D products (2^-17 of the sum of magnitudes at D = 128, on
  both sides of the softmax), its result is rounded to bf16 once.
"""

import math

import pytest
import torch

from paper_2603_18599_gb300 import kv, sjd

pytestmark = pytest.mark.gpu

DEV = "cuda"
MOST = {torch.float8_e4m3fn: 448.0, torch.int8: 127.0}
TYPES = [torch.bfloat16, torch.float8_e4m3fn, torch.int8]


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def normal(g, *shape):
    return torch.randn(*shape, device=DEV, generator=g)


# --- rotary positions ---------------------------------------------------------

def rotated(x, positions, freq, axis, interleaved, inverse=False):
    """x [B, n, H, D] f64, turned by the definition."""
    m = len(freq)
    angle = positions.double()[:, :, torch.tensor(axis, device=x.device)] * torch.tensor(freq, dtype=torch.float64, device=x.device)
    cos, sin = angle.cos()[:, :, None], angle.sin()[:, :, None] * (-1 if inverse else 1)
    y = x.clone()
    a, b = (slice(0, 2 * m, 2), slice(1, 2 * m, 2)) if interleaved else (slice(0, m), slice(m, 2 * m))
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., a] * sin + x[..., b] * cos
    return y


def pair_sizes(x, m, interleaved):
    """|u| + |w| of the pair each element belongs to."""
    s = x.abs()
    a, b = (slice(0, 2 * m, 2), slice(1, 2 * m, 2)) if interleaved else (slice(0, m), slice(m, 2 * m))
    t = s.clone()
    t[..., a] = s[..., a] + s[..., b]
    t[..., b] = t[..., a]
    return t


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("B,n,H,D,sections", [
    (1, 1, 1, 8, (4,)), (2, 16, 32, 128, (16, 24, 24)), (3, 5, 7, 80, (20, 20)), (1, 33, 2, 96, (12,)),
    (2, 3, 5, 256, (64, 32, 32)), (1, 129, 3, 64, (8, 8, 8, 8)), (1, 2, 40, 120, (60,)),
])
def test_rotate(B, n, H, D, sections, inverse, interleaved, dtype):
    g = gen(n + D)
    rope = kv.Rope.sections(sections, interleaved=interleaved)
    axis = [a for a, m in enumerate(sections) for _ in range(m)]
    freq = [10000.0 ** (-i / m) for m in sections for i in range(m)]
    x = normal(g, B, n, H, D).to(dtype)
    positions = torch.randint(-50, 40000, (B, n, len(sections)), device=DEV, generator=g).int()
    positions[0, 0, 0] = 0
    y = rope.rotate(x, positions, inverse=inverse)
    want = rotated(x.double(), positions, freq, axis, interleaved, inverse)
    tol = 8e-7 * pair_sizes(x.double(), len(freq), interleaved)
    if dtype == torch.bfloat16:
        tol = tol * 1.01 + want.abs() * 2.0 ** -8
    assert ((y.double() - want).abs() <= tol).all()
    kept = 2 * len(freq)
    assert torch.equal(y[..., kept:], x[..., kept:])


def test_rotate_at_the_largest_positions():
    rope = kv.Rope([1.0, 0.3, 1e-3, 1e-9], [0, 0, 0, 0])
    pos = [0, 1, -1, 2 ** 31 - 1, -2 ** 31, 2 ** 30 + 12345]
    positions = torch.tensor(pos, dtype=torch.int32, device=DEV).view(1, -1, 1)
    x = torch.zeros(1, len(pos), 1, 8, device=DEV)
    x[..., :4] = 1.0
    y = rope.rotate(x, positions)[0, :, 0].cpu()
    for p, row in zip(pos, y):
        for i, f in enumerate((1.0, 0.3, 1e-3, 1e-9)):
            # the frequency itself is held to 53 bits: 2^31 * 2^-53 turns
            tol = 8e-7 + abs(p) * f * 2.0 ** -52
            assert abs(row[i].item() - math.cos(p * f)) < tol and abs(row[4 + i].item() - math.sin(p * f)) < tol, (p, f)


def test_rotate_in_place_on_strided_and_unaligned_views():
    g = gen(5)
    rope = kv.Rope.sections((8, 8))
    positions = torch.randint(0, 4000, (2, 9, 2), device=DEV, generator=g).int()
    for dtype in (torch.float32, torch.bfloat16):
        packed = normal(g, 2, 9, 1 + 5 * 48).to(dtype)
        for offset in (0, 1):   # 1: no vector starts on a boundary of more than its type
            view = packed[:, :, offset:offset + 240].unflatten(2, (5, 48))
            dense = view.clone()
            want = rope.rotate(dense, positions)
            before = packed.clone()
            assert rope.rotate(view, positions, out=view) is view
            assert torch.equal(view, want)
            rest = [0] if offset else [240]
            assert torch.equal(packed[:, :, rest], before[:, :, rest])
        transposed = normal(g, 2, 5, 9, 48).to(dtype).transpose(1, 2)   # heads before tokens
        assert torch.equal(rope.rotate(transposed, positions), rope.rotate(transposed.contiguous(), positions))


def test_rotate_gradient_is_the_transpose():
    """Against the formula's and against differences (the map is linear, so
    a difference is exact but for rounding)."""
    g = gen(6)
    for interleaved in (False, True):
        rope = kv.Rope.sections((6, 10, 8), interleaved=interleaved)
        positions = torch.randint(0, 900, (2, 7, 3), device=DEV, generator=g).int()
        x, gy, e = (normal(g, 2, 7, 3, 56) for _ in range(3))
        gx = rope.rotate(gy, positions, inverse=True)
        lhs = ((rope.rotate(x + e, positions).double() - rope.rotate(x - e, positions).double()) * gy.double()).sum() / 2
        rhs = (gx.double() * e.double()).sum()
        size = (gx.double() * e.double()).abs().sum()
        assert abs(lhs - rhs) <= 1e-5 * size
        back = rope.rotate(rope.rotate(x, positions), positions, inverse=True)
        assert (back - x).abs().max() <= 4e-6 * x.abs().max()


# --- the paged cache ----------------------------------------------------------

def make(B, heads, kv_heads, D, dtype, page, starts, n, seed=0, extra=2, stale=True):
    """A handle, a layer whose every slot holds stale values, and a table of
    scattered pages with -1 behind them."""
    g = gen(seed)
    pages = [max(1, -(-(s + n) // page)) for s in starts]
    total = sum(pages) + extra
    order = torch.randperm(total, device=DEV, generator=g).int().tolist()
    table, at = [], 0
    for m in pages:
        table.append(order[at:at + m] + [-1] * (max(pages) - m))
        at += m
    h = kv.KV(B, heads, kv_heads, D, total, page, max(pages), n, dtype)
    layer = h.new_layer()
    if stale:
        for name in ("k", "v"):
            c = getattr(layer, name)
            if dtype == torch.bfloat16:
                c.fill_(math.nan)
            else:
                c.view(torch.uint8).fill_(0x55)
                getattr(layer, name + "_scale").fill_(math.nan)
    return h, layer, torch.tensor(table, dtype=torch.int32, device=DEV), torch.tensor(starts, dtype=torch.int32, device=DEV), g


def quantised(x, dtype):
    """(codes, scale) of f32 vectors by the declared arithmetic."""
    top = torch.full((), MOST[dtype], device=x.device)
    scale = x.abs().amax(-1) / top
    y = x / torch.where(scale > 0, scale, torch.ones_like(scale))[..., None]
    return (y.round().to(torch.int8) if dtype == torch.int8 else y.to(dtype)), scale


def slots(h, table, starts, counts):
    """[(b, t, page, slot)] of every token of the spans."""
    page = h.cfg.page_size
    return [(b, t, int(table[b, (s + t) // page]), (s + t) % page) for b, (s, m) in enumerate(zip(starts, counts)) for t in range(m)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("src", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,H,D,page,starts,n,counts", [
    (1, 1, 8, 1, [0], 1, None), (2, 3, 64, 16, [0, 37], 5, None), (3, 2, 128, 24, [0, 23, 100], 30, [0, 30, 7]),
    (2, 8, 80, 7, [13, 0], 16, [16, 1]), (1, 20, 96, 64, [1], 129, None),
])
def test_write_and_read(dtype, src, B, H, D, page, starts, n, counts):
    h, layer, table, start, g = make(B, 2 * H, H, D, dtype, page, starts, n, seed=n + D)
    count = None if counts is None else torch.tensor(counts, dtype=torch.int32, device=DEV)
    packed = normal(g, B, n, 4 * H, D).mul(torch.exp(2 * normal(g, B, n, 4 * H, 1))).to(src)
    k, v = packed[:, :, 2 * H:3 * H], packed[:, :, 3 * H:]
    before = {m: getattr(layer, m).view(torch.uint8).clone() for m in ("k", "v")}
    assert h.write(layer, k, v, table, start, count) is None
    where = slots(h, table.cpu(), starts, counts or [n] * B)
    b, t, p, s = (torch.tensor(x, device=DEV) for x in zip(*where))
    for name, x in (("k", k), ("v", v)):
        cache, x = getattr(layer, name), x[b, t].float()      # [tokens, H, D]
        got = cache.view(torch.uint8).unflatten(3, (D, -1))[p, :, s]
        if dtype == torch.bfloat16:
            held, scale = x.bfloat16(), None
        else:
            held, scale = quantised(x, dtype)
            assert torch.equal(getattr(layer, name + "_scale")[p, :, s], scale)
        assert torch.equal(got, held.contiguous().view(torch.uint8).unflatten(2, (D, -1)))
        # nothing else was touched
        after = cache.view(torch.uint8).clone()
        after.view(*cache.shape[:3], -1)[p, :, s] = before[name].view(*cache.shape[:3], -1)[p, :, s]
        assert torch.equal(after, before[name])
    for out in (torch.bfloat16, torch.float32):
        for name, y in zip(("k", "v"), h.read(layer, table, start, n, count, dtype=out)):
            want = torch.zeros(B, n, H, D, device=DEV)
            x = (k if name == "k" else v)[b, t].float()
            if dtype == torch.bfloat16:
                want[b, t] = x.bfloat16().float()
            else:
                held, scale = quantised(x, dtype)
                want[b, t] = held.float() * scale[..., None]
            assert torch.equal(y, want.to(out))
    assert h.sync() == sjd.SJD_OK


@pytest.mark.parametrize("dtype", TYPES)
def test_write_turns_keys_and_queries(dtype):
    B, n, H, D, starts = 2, 11, 3, 96, [5, 70]
    h, layer, table, start, g = make(B, 4 * H, H, D, dtype, 16, starts, n)
    for interleaved in (False, True):
        rope = kv.Rope.sections((12, 20, 8), interleaved=interleaved)
        axis = [0] * 12 + [1] * 20 + [2] * 8
        freq = [10000.0 ** (-i / m) for m in (12, 20, 8) for i in range(m)]
        packed = normal(g, B, n, 6 * H, D)
        q, k, v = packed[:, :, :4 * H], packed[:, :, 4 * H:5 * H], packed[:, :, 5 * H:]
        positions = torch.randint(0, 9000, (B, n, 3), device=DEV, generator=g).int()
        q_out = h.write(layer, k, v, table, start, rope=rope, positions=positions, q=q)
        assert torch.equal(q_out, rope.rotate(q, positions))
        assert h.write(layer, k, v, table, start, rope=rope, positions=positions) is None
        back, vback = h.read(layer, table, start, n, dtype=torch.float32)
        want = rotated(k.double(), positions, freq, axis, interleaved)
        size = want.abs().amax(-1, keepdim=True)
        step = want.abs() * 2.0 ** -8 if dtype == torch.bfloat16 else size / 127 / 2 if dtype == torch.int8 else \
            torch.maximum(want.abs() * 2.0 ** -4, size / 448 * 2.0 ** -10)
        assert ((back.double() - want).abs() <= step * 1.001 + 2e-6 * size).all()
        if dtype != torch.bfloat16:
            held, scale = quantised(v, dtype)
            assert torch.equal(vback, held.float() * scale[..., None])


@pytest.mark.parametrize("dtype", TYPES)
def test_vectors_of_zeros_infinities_and_nan(dtype):
    h, layer, table, start, g = make(1, 2, 2, 16, dtype, 4, [0], 8)
    x = normal(g, 1, 8, 2, 16)
    x[0, 0, 0] = 0.0
    x[0, 1, 0, 3] = math.inf
    x[0, 2, 1, 5] = -math.inf
    x[0, 3, 0, 0] = math.nan
    x[0, 4] = 1e-44                  # a scale that rounds to zero
    x[0, 5] *= 1e30
    h.write(layer, x, x, table, start)
    k, v = h.read(layer, table, start, 8, dtype=torch.float32)
    assert torch.equal(k.nan_to_num(7.0), v.nan_to_num(7.0))
    if dtype == torch.bfloat16:
        assert torch.equal(k.nan_to_num(7.0), x.bfloat16().float().nan_to_num(7.0))
    else:
        assert (k[0, 0, 0] == 0).all() and (k[0, 4] == 0).all()
        for t, head in ((1, 0), (2, 1), (3, 0)):
            assert k[0, t, head].isnan().all() and not k[0, t, 1 - head].isnan().any()
        held, scale = quantised(x[0, 5:], dtype)
        assert torch.equal(k[0, 5:], held.float() * scale[..., None])


# --- attention ----------------------------------------------------------------

def attention(h, layer, q, table, starts, counts, mask, scale):
    """(o, lse, size, spread): the definition in f64; size = sum_j p_j |v_j|,
    spread = the largest scale * sum_i |q_i k_ij| of a row."""
    c = h.cfg
    B, n, G = q.shape[0], q.shape[1], c.heads // c.kv_heads
    o = torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    size = torch.zeros_like(o)
    lse = torch.full(q.shape[:3], -math.inf, dtype=torch.float64, device=DEV)
    spread = torch.zeros_like(lse)
    for b in range(B):
        s, m = starts[b], counts[b]
        if m == 0:
            continue
        rows = torch.arange(s + m, device=DEV)
        page, slot = table[b].long()[rows // c.page_size], rows % c.page_size
        keys = []
        for name in ("k", "v"):
            cache = getattr(layer, name)
            x = cache.view(torch.uint8).unflatten(3, (c.head_dim, -1))[page, :, slot].contiguous().view(cache.dtype).flatten(2).double()
            if getattr(layer, name + "_scale") is not None:
                x = x * getattr(layer, name + "_scale")[page, :, slot].double()[..., None]
            keys.append(x)                                     # [T, Hkv, D]
        k, v = keys
        seen = torch.ones(m, s + m, dtype=torch.bool, device=DEV)
        if isinstance(mask, str):
            seen = seen.tril(s)
        elif mask is not None:
            seen[:, s:] = mask[b if mask.shape[0] > 1 else 0, :m, :m].bool()
        for head in range(c.heads):
            x = q[b, :m, head].double()
            score = (x @ k[:, head // G].T * scale).masked_fill(~seen, -math.inf)
            top = score.amax(-1, keepdim=True)
            top = torch.where(top == -math.inf, torch.zeros_like(top), top)
            w = (score - top).exp()
            total = w.sum(-1, keepdim=True)
            p = torch.where(total > 0, w / total, torch.zeros_like(w))
            value = v[:, head // G]
            for t in range(m):                                 # keys a row does not see take no part
                at = seen[t]
                o[b, t, head] = p[t, at] @ value[at]
                size[b, t, head] = p[t, at] @ value[at].abs()
            lse[b, :m, head] = (top + total.log())[:, 0]
            spread[b, :m, head] = ((x.abs() @ k[:, head // G].abs().T) * scale).masked_fill(~seen, 0).amax(-1)
    return o, lse, size, spread


def check(got, got_lse, want):
    o, lse, size, spread = want
    wrong = 2.0 ** -17 * spread + 2e-6
    fine = o.isfinite() & size.isfinite()
    assert torch.equal(got.isfinite(), o.isfinite())
    tol = 2.0 ** -8 * 1.05 * (size + o.abs()) + 2 * wrong[..., None] * size
    off = (got.double() - o).abs()
    assert (off <= tol)[fine].all(), (off - tol)[fine].max()
    # many roundings of one sign are no accident
    if fine.sum() > 1000:
        assert (got.double() - o)[fine].norm() <= 0.004 * o[fine].norm()
    if got_lse is not None:
        some = lse.isfinite()
        assert torch.equal(got_lse == -math.inf, lse == -math.inf)
        assert ((got_lse.double() - lse).abs() <= wrong + 1e-6 * lse.abs())[some].all()


def filled(h, layer, table, starts, n, g, sharp=1.0):
    """Writes keys and values of every token before and in the chunk."""
    c = h.cfg
    B, most = c.batch, max(starts) + n
    zero = torch.zeros(B, dtype=torch.int32, device=DEV)
    whole = kv.KV(B, c.heads, c.kv_heads, c.head_dim, c.n_pages, c.page_size, c.max_pages, most, h.dtype)
    k = normal(g, B, most, c.kv_heads, c.head_dim).mul(sharp)
    v = normal(g, B, most, c.kv_heads, c.head_dim) * torch.exp(normal(g, B, most, 1, 1))
    count = torch.tensor([s + n for s in starts], dtype=torch.int32, device=DEV)
    whole.write(kv.Layer(layer.k, layer.v, layer.k_scale, layer.v_scale), k, v, table, zero, count)
    assert whole.sync() == sjd.SJD_OK


def chunk_mask(kind, B, n, g):
    if kind in ("causal", None):
        return kind
    m = torch.rand(1 if kind == "shared" else B, n, n, device=DEV, generator=g) < 0.4
    if kind == "empty":
        m[:, ::2] = False                                      # rows that see nothing of the chunk
    return m


CASES = [  # B, heads, kv_heads, D, page, starts, n, counts, mask
    (1, 1, 1, 8, 1, [0], 1, None, "causal"),
    (1, 4, 1, 64, 16, [0], 1, None, "causal"),
    (2, 8, 2, 128, 16, [127, 128], 1, None, "causal"),
    (3, 6, 6, 64, 24, [0, 129, 300], 1, [1, 0, 1], None),
    (2, 32, 8, 128, 64, [1000, 617], 16, None, "causal"),
    (2, 8, 8, 96, 7, [250, 3], 5, [5, 2], "causal"),
    (1, 128, 1, 128, 32, [77], 3, None, "causal"),
    (2, 14, 2, 80, 40, [0, 511], 33, None, "causal"),
    (1, 4, 4, 64, 128, [0], 128, None, "causal"),
    (1, 4, 4, 128, 128, [0], 129, None, "causal"),
    (2, 3, 1, 120, 8, [100, 0], 200, [200, 131], "causal"),
    (1, 8, 4, 128, 64, [1500], 700, None, "causal"),
    (2, 5, 5, 64, 24, [200, 0], 50, None, "own"),
    (2, 8, 2, 128, 16, [0, 100], 37, [37, 20], "empty"),
    (3, 4, 2, 64, 16, [0, 5, 130], 140, None, "shared"),
    (2, 4, 2, 128, 64, [60, 0], 64, None, None),
    (2, 2, 2, 128, 64, [20000, 4096], 1, None, "causal"),
    (17, 4, 2, 64, 16, [31 * i for i in range(17)], 2, None, "causal"),
    (40, 2, 1, 64, 16, [5 * i for i in range(40)], 3, [i % 4 for i in range(40)], "causal"),
    (9, 2, 1, 64, 16, [30000] + [3] * 8, 1, None, "causal"),       # one sequence has nearly all blocks
    (9, 8, 8, 64, 16, [30000] + [3] * 8, 4, [4] * 8 + [0], "causal"),
    (3, 32, 8, 128, 32, [2500, 70, 0], 8, [8, 0, 3], "causal"),    # 32 rows
    (3, 32, 8, 128, 32, [2500, 70, 0], 9, [9, 0, 9], None),        # 36
    (2, 64, 4, 96, 16, [1300, 1], 4, None, "own"),                 # 64
    (2, 64, 4, 96, 16, [1300, 1], 5, None, "own"),                 # 80
    (1, 16, 2, 72, 16, [5000], 4, None, "empty"),                  # vectors of 72 codes
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", range(len(CASES)))
def test_attend(case, dtype):
    B, heads, kv_heads, D, page, starts, n, counts, kind = CASES[case]
    h, layer, table, start, g = make(B, heads, kv_heads, D, dtype, page, starts, n, seed=case)
    filled(h, layer, table, starts, n, g, sharp=1.0 if case % 2 else 2.5)
    q = normal(g, B, n, heads + 2 * kv_heads, D).bfloat16()[:, :, :heads]
    count = None if counts is None else torch.tensor(counts, dtype=torch.int32, device=DEV)
    mask = chunk_mask(kind, B, n, g)
    scale = 0.11 if case % 3 == 0 else None
    o, lse = h.attend(layer, q, table, start, count, mask=mask, scale=scale, lse=True)
    assert h.sync() == sjd.SJD_OK, h.last_error()
    want = attention(h, layer, q, table, starts, counts or [n] * B, mask, scale or D ** -0.5)
    check(o, lse, want)
    again = h.attend(layer, q, table, start, count, mask=mask, scale=scale)
    assert torch.equal(again, o)


def test_attend_scores_of_any_size():
    """Sharp rows: the running maximum moves by hundreds, up and down."""
    h, layer, table, start, g = make(1, 4, 2, 64, torch.bfloat16, 16, [700], 40)
    filled(h, layer, table, [700], 40, g, sharp=30.0)
    q = (normal(g, 1, 40, 4, 64) * 10).bfloat16()
    o, lse = h.attend(layer, q, table, start, lse=True)
    want = attention(h, layer, q, table, [700], [40], "causal", 64 ** -0.5)
    check(o, lse, want)
    for scale in (0.0, -0.5):
        o, lse = h.attend(layer, q, table, start, scale=scale, lse=True)
        want = attention(h, layer, q, table, [700], [40], "causal", scale)
        check(o, lse, (want[0], want[1], want[2], want[3].abs() + 100 * abs(scale)))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads,n", [(2, 3), (2, 40), (8, 30), (4, 200)])
@pytest.mark.parametrize("size", [1e2, 1e6, 1e12])
def test_attend_scores_beyond_every_exponent(dtype, heads, n, size):
    """Queries that are one key each, many times over: the row's weight is on
    that key alone, by a margin of hundreds to 10^13 powers of e, and its
    result the key's value."""
    D, context = 128, 400
    h, layer, table, start, g = make(1, heads, 2, D, dtype, 16, [context], n)
    filled(h, layer, table, [context], n, g)
    zero = torch.zeros_like(start)
    whole = kv.KV(1, heads, 2, D, h.cfg.n_pages, 16, h.cfg.max_pages, context + n, dtype)
    k, v = whole.read(kv.Layer(layer.k, layer.v, layer.k_scale, layer.v_scale), table, zero, context + n, dtype=torch.float32)
    at = torch.randint(0, context, (n, heads), device=DEV, generator=g)
    head = torch.arange(heads, device=DEV) * 2 // heads
    q = (k[0, at, head] * size).bfloat16()[None].contiguous()
    o, lse = h.attend(layer, q, table, start, lse=True)
    assert ((o[0].float() - v[0, at, head]).abs() <= 2.0 ** -7 * v[0, at, head].abs() + 1e-6).all()
    want = (q[0].double() * k[0, at, head].double()).sum(-1) * D ** -0.5
    assert ((lse[0].double() - want).abs() <= 1e-5 * want.abs()).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["causal", "given"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_unseen_keys_have_no_effect_whatever_they_hold(dtype, kind, bad):
    """A NaN or infinity in the keys or values of chunk token 3 reaches the
    rows that see it and no others."""
    B, n, heads, kv_heads, D = 1, 9, 4, 2, 64
    starts = [133]
    h, layer, table, start, g = make(B, heads, kv_heads, D, dtype, 16, starts, n)
    filled(h, layer, table, starts, n, g)
    q = normal(g, B, n, heads, D).bfloat16()
    mask = "causal"
    if kind == "given":
        mask = torch.eye(n, device=DEV).bool()[None].clone()
        mask[0, 6, 3] = True
    rows = torch.arange(n, device=DEV)
    sees = rows >= 3 if kind == "causal" else (rows == 3) | (rows == 6)
    k, v = h.read(layer, table, start, n, dtype=torch.float32)
    h.write(layer, k, v, table, start)
    clean = h.attend(layer, q, table, start, mask=mask)
    for which in ("k", "v"):
        x = (k if which == "k" else v).clone()
        x[0, 3, 1, 5] = bad
        args = (x, v) if which == "k" else (k, x)
        h.write(layer, *args, table, start)
        o, lse = h.attend(layer, q, table, start, mask=mask, lse=True)
        group1 = slice(heads // kv_heads, heads)
        assert torch.equal(o[:, ~sees, group1], clean[:, ~sees, group1])
        assert torch.equal(o[:, :, :2], clean[:, :, :2])           # the other key head
        assert lse[:, ~sees].isfinite().all()
        hit = o[0, sees][:, group1].float()
        if which == "v" and dtype == torch.bfloat16:
            assert torch.equal(hit[..., :5], clean[0, sees][:, group1][..., :5].float())
            assert (hit[..., 5].isnan() if math.isnan(bad) else hit[..., 5] == bad).all()
        elif which == "v" or math.isnan(bad) or dtype != torch.bfloat16:
            assert hit.isnan().any(-1).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["causal", None, "given"])
@pytest.mark.parametrize("heads,n", [(4, 9), (2, 200)])
def test_context_keys_that_hold_nan(dtype, kind, heads, n):
    """A NaN in a key or value of the context, in the tile where the chunk
    begins and in one before it, reaches every row of its head; with mask
    None one of the chunk does too."""
    starts, D = [300], 64
    h, layer, table, start, g = make(1, heads, 2, D, dtype, 16, starts, n)
    filled(h, layer, table, starts, n, g)
    q = normal(g, 1, n, heads, D).bfloat16()
    mask = torch.eye(n, device=DEV).bool()[None] if kind == "given" else kind
    one = torch.ones(1, dtype=torch.int32, device=DEV)
    for where in [298, 20] + ([299 + n] if kind is None else []):
        at = torch.tensor([where], dtype=torch.int32, device=DEV)
        k, v = h.read(layer, table, at, 1, dtype=torch.float32)
        for which in ("k", "v"):
            x = (k if which == "k" else v).clone()
            x[0, 0, 1, 7] = math.nan
            h.write(layer, *((x, v) if which == "k" else (k, x)), table, at, one)
            o = h.attend(layer, q, table, start, mask=mask)
            assert o[:, :, :heads // 2].isfinite().all()
            hit = o[:, :, heads // 2:]
            if which == "v" and dtype == torch.bfloat16:
                assert hit[..., 7].isnan().all() and hit[..., :7].isfinite().all() and hit[..., 8:].isfinite().all()
            else:
                assert hit.isnan().all()
            h.write(layer, k, v, table, at, one)
    assert h.attend(layer, q, table, start, mask=mask).isfinite().all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.int8])
def test_offsets_past_32_bits(dtype):
    """A cache of more than 2^32 elements: its last pages, written, read and
    attended to."""
    kv_heads, D, page = 8, 128, 64
    total = 2 ** 32 // (kv_heads * D * page) + 40
    h = kv.KV(1, 8, kv_heads, D, total, page, 8, 100, dtype)
    layer = h.new_layer()
    table = torch.tensor([[total - 1 - 3 * i for i in range(8)]], dtype=torch.int32, device=DEV)
    start = torch.tensor([300], dtype=torch.int32, device=DEV)
    g = gen(3)
    zero = torch.zeros(1, dtype=torch.int32, device=DEV)
    k, v = normal(g, 1, 400, kv_heads, D), normal(g, 1, 400, kv_heads, D)
    for s in range(0, 400, 100):
        h.write(layer, k[:, s:s + 100], v[:, s:s + 100], table, zero + s)
    kb, vb = h.read(layer, table, zero, 400, dtype=torch.float32)
    assert (kb - k).abs().max() <= 0.03 and (vb - v).abs().max() <= 0.03
    q = normal(g, 1, 100, 8, D).bfloat16()
    o, lse = h.attend(layer, q, table, start, lse=True)
    check(o, lse, attention(h, layer, q, table, [300], [100], "causal", D ** -0.5))
    assert h.sync() == sjd.SJD_OK


# --- calls --------------------------------------------------------------------

def test_calls_on_another_stream_are_ordered():
    side = torch.cuda.Stream()
    starts, n = [500], 8
    h, layer, table, start, g = make(1, 4, 2, 64, torch.bfloat16, 16, starts, n)
    filled(h, layer, table, starts, n, g)
    q = normal(g, 1, n, 4, 64).bfloat16()
    kvs = normal(g, 2, 1, n, 2, 64).bfloat16()
    h.write(layer, kvs[0], kvs[1], table, start)
    want = h.attend(layer, q, table, start)
    for t in range(20):
        with torch.cuda.stream(side):
            big = torch.randn(3000, 3001, device=DEV)
            for _ in range(5):
                big = big * 1.0001
            x = kvs.clone()
            mine = q.clone()
            h.write(layer, x[0], x[1], table, start)
            got = h.attend(layer, mine, table, start)
            assert torch.equal(got, want)
    torch.cuda.synchronize()


def test_calls_back_to_back_wait_for_each_other():
    """Kernels that start while the one before drains: a chain of calls, each
    on the last one's result, against the same chain with waits between."""
    starts, n, D = [300, 40], 8, 64
    h, layer, table, start, g = make(2, 8, 2, D, torch.int8, 16, starts, n)
    filled(h, layer, table, starts, n, g)
    rope = kv.Rope.sections((16, 16))
    positions = torch.randint(0, 500, (2, n, 2), device=DEV, generator=g).int()
    x0 = normal(g, 2, n, 8, D).bfloat16()

    def chain(wait):
        x = x0.clone()
        for _ in range(60):
            q = rope.rotate(x, positions)
            wait()
            turned = h.write(layer, x[:, :, :2], x[:, :, 2:4], table, start, rope=rope, positions=positions, q=q)
            wait()
            k, v = h.read(layer, table, start, n)
            wait()
            o = h.attend(layer, turned, table, start)
            wait()
            x = rope.rotate(o, positions, inverse=True)
            wait()
            x = torch.cat([k, v, x[:, :, 4:]], 2) * 1.5    # a kernel of another library between
        return x

    want = chain(torch.cuda.synchronize)
    for _ in range(3):
        assert torch.equal(chain(lambda: None), want)


def test_captured_calls_follow_the_device_positions():
    """A captured write and attention replayed as the sequence grows."""
    starts, n, D = [250], 4, 64
    h, layer, table, start, g = make(1, 4, 2, D, torch.float8_e4m3fn, 16, [400], n)
    filled(h, layer, table, [400], n, g)
    start.fill_(starts[0])
    rope = kv.Rope.sections((16, 16))
    k, v = normal(g, 1, n, 2, D), normal(g, 1, n, 2, D)
    q = normal(g, 1, n, 4, D)
    positions = torch.zeros(1, n, 2, dtype=torch.int32, device=DEV)

    def step():
        turned = h.write(layer, k, v, table, start, rope=rope, positions=positions, q=q)
        return h.attend(layer, turned.bfloat16(), table, start)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    h2 = kv.KV(1, 4, 2, D, h.cfg.n_pages, 16, h.cfg.max_pages, n, torch.float8_e4m3fn, stream=side)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        turned = h2.write(layer, k, v, table, start, rope=rope, positions=positions, q=q)
        out = h2.attend(layer, turned.bfloat16(), table, start)
    for t in range(3):
        start.fill_(250 + 60 * t)
        positions.fill_(7 * t)
        graph.replay()
        got = out.clone()
        assert torch.equal(got, step())


def test_device_errors_are_latched_and_cleared():
    n, page = 4, 16
    h, layer, table, start, g = make(2, 4, 2, 64, torch.int8, page, [20, 40], n)
    filled(h, layer, table, [20, 40], n, g)
    q = normal(g, 2, n, 4, 64).bfloat16()
    x = normal(g, 2, n, 2, 64)
    good = h.attend(layer, q, table, start)
    room = table.shape[1] * page

    def bits():
        return [getattr(layer, m).view(torch.uint8).clone() for m in ("k", "v", "k_scale", "v_scale")]

    before = bits()
    for bad in (-1, room - n + 1, 2 ** 31 - 1, -2 ** 31):
        s = torch.tensor([bad, 40], dtype=torch.int32, device=DEV)
        o = h.attend(layer, q, table, s)
        assert h.sync() == sjd.SJD_ERR_PAGE and h.last_error()
        assert (o[0] == 0).all() and torch.equal(o[1], good[1])
        k, v = h.read(layer, table, s, n)
        assert h.sync() == sjd.SJD_ERR_PAGE and (k[0] == 0).all() and (k[1] != 0).any()
    for bad in (-1, n + 1):
        c = torch.tensor([bad, n], dtype=torch.int32, device=DEV)
        o = h.attend(layer, q, table, start, c)
        assert h.sync() == sjd.SJD_ERR_PAGE and (o[0] == 0).all() and torch.equal(o[1], good[1])
        h.write(layer, x[:1].expand(2, -1, -1, -1), x[:1].expand(2, -1, -1, -1), table, start, torch.zeros_like(c) + bad)
        assert h.sync() == sjd.SJD_ERR_PAGE
    assert all(torch.equal(a, b) for a, b in zip(before, bits()))
    for bad in (-1, h.cfg.n_pages, 2 ** 31 - 1):
        t = table.clone()
        t[0, 1] = bad
        s = torch.tensor([20, 40], dtype=torch.int32, device=DEV)
        o = h.attend(layer, q, t, s)
        assert h.sync() == sjd.SJD_ERR_PAGE and o.isfinite().all() and torch.equal(o[1], good[1])
        one = torch.tensor([n, 0], dtype=torch.int32, device=DEV)
        h.write(layer, x, x, t, s, one)
        assert h.sync() == sjd.SJD_ERR_PAGE
    assert all(torch.equal(a, b) for a, b in zip(before, bits()))
    assert h.sync() == sjd.SJD_OK


def test_arguments_are_refused():
    h, layer, table, start, g = make(2, 4, 2, 64, torch.int8, 16, [20, 40], 4)
    q = normal(g, 2, 4, 4, 64).bfloat16()
    x = normal(g, 2, 4, 2, 64)
    rope = kv.Rope.sections((16, 16))
    positions = torch.zeros(2, 4, 2, dtype=torch.int32, device=DEV)
    mask = torch.ones(2, 4, 4, dtype=torch.bool, device=DEV)
    for call in (
            lambda: h.attend(layer, q.float(), table, start), lambda: h.attend(layer, q[:, :, :3], table, start),
            lambda: h.attend(layer, q.cpu(), table, start), lambda: h.attend(layer, q, table.long(), start),
            lambda: h.attend(layer, q, table[:, :1], start), lambda: h.attend(layer, q, table, start[:1]),
            lambda: h.attend(layer, q, table, start, mask=mask[:, :3]), lambda: h.attend(layer, q, table, start, mask=mask.float()),
            lambda: h.attend(layer, q, table, start, mask="all"), lambda: h.attend(layer, q, table, start, out=q.float()),
            lambda: h.attend(kv.Layer(layer.k, layer.v), q, table, start),
            lambda: h.attend(kv.Layer(layer.k.float(), layer.v, layer.k_scale, layer.v_scale), q, table, start),
            lambda: h.write(layer, x.half(), x.half(), table, start), lambda: h.write(layer, x, x.bfloat16(), table, start),
            lambda: h.write(layer, x, x[:, :3], table, start), lambda: h.write(layer, x, x, table, start, count=start.long()),
            lambda: h.write(layer, x, x, table, start, rope=rope, positions=positions[..., :1]),
            lambda: h.read(layer, table, start, 4, dtype=torch.float16),
            lambda: rope.rotate(x.half(), positions), lambda: rope.rotate(x, positions.long()),
            lambda: rope.rotate(x.transpose(2, 3), positions), lambda: rope.rotate(x[0], positions),
            lambda: kv.Rope([1.0] * 3, [0] * 3), lambda: kv.Rope([1.0] * 4, [0, 0, 0, 8]),
            lambda: kv.KV(2, 4, 2, 64, 4, 16, 4, 4, torch.float16)):
        with pytest.raises(ValueError):
            call()
    many = torch.cat([x, x], 1)
    odd = normal(g, 2, 4, 4 * 64 + 1).bfloat16()[:, :, 1:].unflatten(2, (4, 64))
    for call in (
            lambda: h.write(layer, many, many, table, start),      # more than max_new
            lambda: h.attend(layer, odd, table, start),            # rows off 16-byte boundaries
            lambda: h.attend(layer, q, table, start, scale=math.nan),
            lambda: h.read(layer, table, start, table.shape[1] * 16 + 1), lambda: h.read(layer, table, start, 0),
            lambda: rope.rotate(normal(g, 2, 4, 2, 24), positions), lambda: rope.rotate(normal(g, 2, 4, 2, 60), positions),
            lambda: h.write(layer, x, x, table, start, q=q.float()),
            lambda: h.write(layer, x, x, table, start, rope=kv.Rope([1.0] * 36, [0] * 36), positions=positions[..., :1].contiguous()),
            lambda: kv.KV(2, 4, 3, 64, 4, 16, 4, 4), lambda: kv.KV(2, 4, 2, 60, 4, 16, 4, 4), lambda: kv.KV(2, 4, 2, 136, 4, 16, 4, 4),
            lambda: kv.KV(0, 4, 2, 64, 4, 16, 4, 4), lambda: kv.KV(2, 4, 2, 64, 4, 0, 4, 4),
            lambda: kv.KV(2, 4, 2, 64, 4, 2 ** 20, 2 ** 12, 4), lambda: kv.KV(2, 258, 2, 64, 4, 16, 4, 4)):
        with pytest.raises(sjd.SJDError) as e:
            call()
        assert e.value.code == sjd.SJD_ERR_ARG
    assert h.sync() == sjd.SJD_OK
