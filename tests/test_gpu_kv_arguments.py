"""The operators' arguments at the edges of what they take: scales of the
scores, strides of dimensions of one element, vectors of subnormal numbers,
tables on other devices and streams, tensors that want a gradient."""

import math

import numpy as np
import pytest
import torch

import test_gpu_kv as base
from paper_2603_18599_gb300 import kv, sjd

pytestmark = pytest.mark.gpu

DEV = "cuda"


# --- rotary tables ------------------------------------------------------------

def test_a_rope_of_another_device_or_without_positions_is_refused():
    h, layer, table, start, g = base.make(2, 4, 2, 64, torch.int8, 16, [20, 40], 4)
    x = base.normal(g, 2, 4, 2, 64)
    q = base.normal(g, 2, 4, 4, 64)
    positions = torch.zeros(2, 4, 2, dtype=torch.int32, device=DEV)
    rope = kv.Rope.sections((16, 16))
    before = layer.k.clone()
    with pytest.raises(ValueError):
        h.write(layer, x, x, table, start, rope=rope)
    with pytest.raises(ValueError):
        h.write(layer, x, x, table, start, rope=rope, positions=positions, q_out=q)
    rope.device = torch.device("cuda", 1)          # (as one made there)
    with pytest.raises(ValueError):
        h.write(layer, x, x, table, start, rope=rope, positions=positions)
    assert torch.equal(layer.k, before)


def test_a_rope_may_go_while_its_last_call_runs():
    """Tables made on one stream, used on another and given back: their memory
    is not handed out before the call has read them."""
    side = torch.cuda.Stream()
    g = base.gen(1)
    x = base.normal(g, 1, 64, 4, 64)
    positions = torch.arange(64, dtype=torch.int32, device=DEV).view(1, 64, 1)
    want = kv.Rope([0.1 * i for i in range(32)], [0] * 32).rotate(x, positions)
    h = kv.KV(1, 4, 4, 64, 8, 16, 8, 64, torch.bfloat16, stream=side)
    layer = h.new_layer()
    table = torch.arange(8, dtype=torch.int32, device=DEV)[None]
    start = torch.zeros(1, dtype=torch.int32, device=DEV)
    big = torch.randn(4000, 4000, device=DEV)
    torch.cuda.synchronize()
    for call in ("rotate", "write"):
        rope = kv.Rope([0.1 * i for i in range(32)], [0] * 32)
        sizes = [(t.shape, t.dtype) for t in (rope._turns, rope._axis)]
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for _ in range(20):
                big = (big @ big).clamp(-1, 1)
            y = rope.rotate(x, positions) if call == "rotate" else h.write(layer, x, x, table, start, rope=rope, positions=positions, q=x)
        del rope
        mine = [torch.zeros(shape, dtype=dtype, device=DEV) for shape, dtype in sizes for _ in range(4)]
        torch.cuda.synchronize()
        assert torch.equal(y, want), call
        del mine


# --- gradients ----------------------------------------------------------------

def test_tensors_that_want_a_gradient_are_refused():
    """No call records one: it says so, unless gradients are off."""
    h, layer, table, start, g = base.make(1, 4, 2, 64, torch.bfloat16, 16, [20], 4)
    base.filled(h, layer, table, [20], 4, g)
    rope = kv.Rope.sections((16, 16))
    positions = torch.zeros(1, 4, 2, dtype=torch.int32, device=DEV)
    x, q = base.normal(g, 1, 4, 2, 64).bfloat16(), base.normal(g, 1, 4, 4, 64).bfloat16()
    leaf = lambda t: t.clone().requires_grad_()
    calls = (lambda: rope.rotate(leaf(q), positions), lambda: rope.rotate(q, positions, out=leaf(q)),
             lambda: h.write(layer, leaf(x), x, table, start), lambda: h.write(layer, x, leaf(x), table, start),
             lambda: h.write(layer, x, x, table, start, rope=rope, positions=positions, q=leaf(q)),
             lambda: h.attend(layer, leaf(q), table, start))
    for call in calls:
        with pytest.raises(ValueError, match="gradient"):
            call()
    with torch.no_grad():
        assert torch.equal(h.attend(layer, leaf(q), table, start), h.attend(layer, q, table, start))
        assert torch.equal(rope.rotate(leaf(q), positions), rope.rotate(q, positions))
        h.write(layer, leaf(x), leaf(x), table, start)


# --- quantising vectors of subnormal numbers ----------------------------------

@pytest.mark.parametrize("dtype", [torch.float8_e4m3fn, torch.int8])
def test_codes_of_subnormal_vectors_keep_their_signs(dtype):
    """Scales below 2^-126 are rounded to few bits, and a quotient may pass
    the largest code: it is held to it."""
    D, tops = 16, list(range(100, 700, 7)) + [3000, 100000]
    n = len(tops)
    h, layer, table, start, g = base.make(1, 2, 2, D, dtype, 16, [0], n)
    x = np.zeros((1, n, 2, D), dtype=np.float32)
    for t, top in enumerate(tops):
        for head in range(2):
            x[0, t, head] = np.ldexp(np.float32(1.0), -149) * np.rint(np.linspace(-top, top, D)).astype(np.float32)
    x[:, :, 1] *= -1.0
    xs = torch.from_numpy(x).to(DEV)
    h.write(layer, xs, xs, table, start)
    got, _ = h.read(layer, table, start, n, dtype=torch.float32)
    most = np.float32(base.MOST[dtype])
    scale = np.abs(x).max(-1, keepdims=True) / most
    y = np.clip(np.divide(x, scale, out=np.zeros_like(x), where=scale > 0), -most, most)
    codes = np.rint(y) if dtype == torch.int8 else torch.from_numpy(y).to(dtype).float().numpy()
    assert (np.abs(codes) == most).any()
    np.testing.assert_array_equal(got.cpu().numpy(), (codes * scale).astype(np.float32))


# --- strides ------------------------------------------------------------------

@pytest.mark.parametrize("dtype", base.TYPES)
def test_strides_of_dimensions_of_one_element_mean_nothing(dtype):
    for B, n, heads in ((1, 1, 4), (1, 3, 1), (2, 1, 1), (1, 1, 1)):
        starts = [37, 60][:B]
        h, layer, table, start, g = base.make(B, heads, 1, 64, dtype, 16, starts, n)
        base.filled(h, layer, table, starts, n, g)
        q = base.normal(g, B, n, heads, 64).bfloat16()
        want = h.attend(layer, q, table, start)
        strides = [s if m > 1 else s + 3 for m, s in zip(q.shape, q.stride())]
        odd = torch.as_strided(q, q.shape, strides)
        assert torch.equal(h.attend(layer, odd, table, start), want)


# --- scales of the scores -----------------------------------------------------

@pytest.mark.parametrize("dtype", base.TYPES)
@pytest.mark.parametrize("heads,n", [(2, 3), (2, 40), (8, 30), (4, 200)])
def test_scales_next_to_the_largest_number(dtype, heads, n):
    """1.5e38 with queries as small: as 1 with queries of their usual size. A
    scale whose product with log2(e) is no fp32 number is refused."""
    starts = [300]
    h, layer, table, start, g = base.make(1, heads, 2, 64, dtype, 16, starts, n)
    base.filled(h, layer, table, starts, n, g)
    q = base.normal(g, 1, n, heads, 64).bfloat16()
    up = 2.0 ** 126
    want, want_lse = h.attend(layer, q, table, start, scale=0.125, lse=True)
    small = (q.double() * 2.0 ** -100).bfloat16()
    o, lse = h.attend(layer, small, table, start, scale=0.125 * 2.0 ** 100, lse=True)
    assert torch.equal(o, want) and (lse - want_lse).abs().max() <= 1e-4
    o = h.attend(layer, (q.double() * 2.0 ** -40).bfloat16(), table, start, scale=up)
    assert o.isfinite().all()
    for scale in (3e38, -3e38):
        with pytest.raises(sjd.SJDError) as e:
            h.attend(layer, q, table, start, scale=scale)
        assert e.value.code == sjd.SJD_ERR_ARG


@pytest.mark.parametrize("dtype", base.TYPES)
@pytest.mark.parametrize("heads,n", [(2, 3), (2, 40), (8, 30), (4, 200)])
def test_scaled_scores_past_the_largest_number(dtype, heads, n):
    """Scores that are numbers and whose product with the scale is none: the
    weight is on the largest, here a key that the query points to."""
    D, context = 64, 300
    h, layer, table, start, g = base.make(1, heads, 2, D, dtype, 16, [context], n)
    base.filled(h, layer, table, [context], n, g)
    whole = kv.KV(1, heads, 2, D, h.cfg.n_pages, 16, h.cfg.max_pages, context + n, dtype)
    k, v = whole.read(kv.Layer(*layer._t), table, torch.zeros_like(start), context + n, dtype=torch.float32)
    score = torch.einsum("thd,shd->hts", k[0], k[0])
    at = torch.randint(0, context, (n, heads), device=DEV, generator=g)
    head = torch.arange(heads, device=DEV) * 2 // heads
    q = (k[0, at, head] * 1e25).bfloat16()[None].contiguous()
    o = h.attend(layer, q, table, start, scale=1e15)
    best = score[head[None, :].expand(n, -1), at].topk(2, -1)         # [n, heads, 2]: a key that wins by far
    some = (best.indices[..., 0] == at) & (best.values[..., 1] < 0.9 * best.values[..., 0])
    assert some.float().mean() > 0.8
    assert o.isfinite().all()
    off = (o[0].float() - v[0, at, head]).abs() - 2.0 ** -7 * v[0, at, head].abs() - 1e-6
    assert (off[some] <= 0).all()
