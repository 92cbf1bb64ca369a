"""The window forward with weights in 8-bit codes, inside the decode loop,
against the same model computed plainly in 64 bits over the whole sequence,
with the values that the codes of its weights stand for.

Tolerances (2-norm of a row's logits): what goes into a product is rounded to
codes, off by 1 / sqrt(12) of a step of max / 127 (rms). The largest of 512
normal values is about 3.2 rms: 0.0073 of the rms, and products keep it; silu's
output is uneven, its largest of 1024 about 6 rms: 0.014. In two layers and the
head that is 7 products of the one kind and 2 of the other, which add up as squares: 2.7 %
at most, were all of the logits made of the branches. With the forward's
roundings to bf16 (0.8 %) and an s8 cache's (0.6 %): 2.9 %; 6 % is held to.
"""

import pytest
import torch

from test_gpu_window_model import plain_logits

from paper_2603_18599_gb300 import dense, sjd
from paper_2603_18599_gb300.window_model import CACHES, WindowModel

pytestmark = pytest.mark.gpu

TOLERANCE = 0.06


class Plain:
    """The model with the values of the codes for its weights."""

    def __init__(self, m):
        self.__dict__.update(m.__dict__)

        def values(w):
            codes, scale = dense.quantise(w.T.contiguous())
            return (codes.double() * scale.double()[:, None]).T

        self.layers = [{k: values(w) for k, w in layer.items()} for layer in m.layers]
        self.head = values(m.head)


@pytest.mark.parametrize("cache", ["bf16", "s8"])
def test_forwards_of_a_decode(cache):
    B, W, V, grid = 2, 16, 512, 8
    prompts = [23, 5, 1, 2]
    m = WindowModel(B, W, prompts, grid, V, cache=CACHES[cache], page_size=24, weights="s8")
    plain = Plain(m)
    m.prefill()
    ctx = sjd.SJD(sjd.make_config(B, W, V, cfg_scale=1.5, top_k=50, seed=3))
    cond, uncond = (torch.empty(B, W, V, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    seen = []

    def forward(window, prev, abs_pos, c, u):
        m.forward(window, prev, abs_pos, c, u)
        seen.append(tuple(t.clone() for t in (window, abs_pos, c, u)))

    tokens, accepted, steps = ctx.decode_loop(forward, grid * grid, cond, uncond)
    assert ctx.sync() == sjd.SJD_OK and m.cache.sync() == sjd.SJD_OK
    assert all(w.sync() == sjd.SJD_OK for layer in m.packed for w in layer.values()) and m.packed_head.sync() == sjd.SJD_OK
    checked = 0
    for window, abs_pos, c, u in seen[::5]:
        for b in range(B):
            at = int(abs_pos[b])
            if at + W > grid * grid:
                continue
            for branch, logits in enumerate((c, u)):
                s = branch * B + b
                inputs = torch.cat([V + torch.arange(prompts[s], device="cuda"), tokens[b, :at].long(), window[b, :-1].long()])
                want = plain_logits(plain, inputs, s)[-W:]
                off = (logits[b].double() - want).norm(dim=-1) / want.norm(dim=-1)
                assert (off <= TOLERANCE).all(), (at, branch, off.max())
                checked += 1
    assert checked >= 8
    # the same decode again gives the same tokens
    ctx2 = sjd.SJD(sjd.make_config(B, W, V, cfg_scale=1.5, top_k=50, seed=3))
    m.prefill()
    again, _, steps2 = ctx2.decode_loop(m.forward, grid * grid, cond, uncond)
    assert steps2 == steps and torch.equal(again, tokens)


def test_weights_of_other_kinds_are_refused():
    with pytest.raises(ValueError):
        WindowModel(1, 4, [2, 2], 4, 64, layers=1, heads=1, kv_heads=1, weights="e4m3")
