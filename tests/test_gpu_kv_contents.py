"""Attention over caches with contents that are not numbers: slots of a span
that nobody has written, codes that stand for NaN, scales and values that
are infinite. What a row does not see has no effect on it; what it sees
reaches it as the definition has it (a weight is above 0: an infinity stays
one, two of both signs and a NaN give NaN).
"""

import math

import pytest
import torch

import test_gpu_kv as base
from paper_2603_18599_gb300 import kv, sjd

pytestmark = pytest.mark.gpu

DEV = "cuda"
D = 64
ROWS = [(8, 2, 7), (8, 2, 12), (8, 2, 30), (4, 2, 140)]   # 32, 64, 128 and more rows of a key head


def place(table, page, at):
    return int(table[0, at // page]), at % page


@pytest.mark.parametrize("dtype", [torch.float8_e4m3fn, torch.int8])
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("code,scale", [(0xff, 1.0), (0x7f, math.nan), (0xff, math.inf), (0x55, math.inf), (0x7f, 0.0)])
def test_a_slot_that_nobody_sees(dtype, rows, code, scale):
    """A chunk token that no row sees, its slot never written: codes and
    scales of any bits change nothing (but the last bits, where fp16's unit moves)."""
    heads, kv_heads, n = rows
    s, hole = 333, n // 2
    h, layer, table, start, g = base.make(1, heads, kv_heads, D, dtype, 16, [s], n)
    base.filled(h, layer, table, [s], n, g)
    q = base.normal(g, 1, n, heads, D).bfloat16()
    mask = torch.ones(1, n, n, dtype=torch.bool, device=DEV).tril()
    mask[:, :, hole] = False
    want, want_lse = h.attend(layer, q, table, start, mask=mask, lse=True)
    page, slot = place(table, 16, s + hole)
    for name in ("k", "v"):
        getattr(layer, name).view(torch.uint8)[page, :, slot] = code
        getattr(layer, name + "_scale")[page, :, slot] = scale
    o, lse = h.attend(layer, q, table, start, mask=mask, lse=True)
    assert h.sync() == sjd.SJD_OK
    assert o.isfinite().all() and torch.equal(lse, want_lse)
    assert (o.double() - want.double()).norm() <= 0.003 * want.double().norm()


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("where", ["context", "chunk"])
def test_a_code_that_stands_for_nan(rows, where):
    """One e4m3 code in one column of one key: NaN there in the rows that see
    the key, and nowhere else."""
    heads, kv_heads, n = rows
    s = 333
    h, layer, table, start, g = base.make(1, heads, kv_heads, D, torch.float8_e4m3fn, 16, [s], n)
    base.filled(h, layer, table, [s], n, g)
    q = base.normal(g, 1, n, heads, D).bfloat16()
    want = h.attend(layer, q, table, start)
    at = 40 if where == "context" else s + n // 2
    page, slot = place(table, 16, at)
    for code in (0x7f, 0xff):
        layer.v.view(torch.uint8)[page, 1, slot, 5] = code
        o = h.attend(layer, q, table, start)
        sees = torch.arange(n, device=DEV) >= at - s
        G = heads // kv_heads
        assert o[:, sees, G:, 5].isnan().all()
        o[:, sees, G:, 5] = want[:, sees, G:, 5]
        assert (o.double() - want.double()).norm() <= 0.003 * want.double().norm()


@pytest.mark.parametrize("dtype", [torch.float8_e4m3fn, torch.int8])
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("where", ["context", "chunk"])
def test_an_infinite_scale_that_is_seen(dtype, rows, where):
    """Infinite in the rows that see the key, with the codes' signs, NaN where
    the code is 0; the other rows do not change."""
    heads, kv_heads, n = rows
    s = 333
    h, layer, table, start, g = base.make(1, heads, kv_heads, D, dtype, 16, [s], n)
    base.filled(h, layer, table, [s], n, g)
    q = base.normal(g, 1, n, heads, D).bfloat16()
    at = 40 if where == "context" else s + n // 2
    page, slot = place(table, 16, at)
    layer.v.view(torch.uint8)[page, 1, slot, 3] = 0
    want = h.attend(layer, q, table, start)
    layer.v_scale[page, 1, slot] = math.inf
    o = h.attend(layer, q, table, start)
    sees = torch.arange(n, device=DEV) >= at - s
    G = heads // kv_heads
    row = layer.v.view(torch.uint8)[page, 1, slot].view(dtype).float() * math.inf
    hit = o[0, sees][:, G:].float()
    assert torch.equal(hit.nan_to_num(nan=7.0), row.expand_as(hit).nan_to_num(nan=7.0))
    o[:, sees, G:] = want[:, sees, G:]
    assert (o.double() - want.double()).norm() <= 0.003 * want.double().norm()


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("at", [[40], [300], [40, 200]])
def test_infinite_values_that_every_row_sees(rows, at):
    """A 16-bit cache: an infinity stays one, two of both signs give NaN."""
    heads, kv_heads, n = rows
    s = 333
    h, layer, table, start, g = base.make(1, heads, kv_heads, D, torch.bfloat16, 16, [s], n)
    base.filled(h, layer, table, [s], n, g)
    q = base.normal(g, 1, n, heads, D).bfloat16()
    want = h.attend(layer, q, table, start)
    for i, key in enumerate(at):
        page, slot = place(table, 16, key)
        layer.v[page, 1, slot, 5] = -math.inf
        layer.v[page, 1, slot, 9] = math.inf if i == 0 else -math.inf
    o = h.attend(layer, q, table, start)
    G = heads // kv_heads
    assert (o[:, :, G:, 5] == -math.inf).all()
    assert (o[:, :, G:, 9] == math.inf).all() if len(at) == 1 else o[:, :, G:, 9].isnan().all()
    for column in (5, 9):
        o[:, :, G:, column] = want[:, :, G:, column]
    assert torch.equal(o, want)
