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
