"""The window forward on the library's operators, inside the decode loop,
against the same model computed plainly in 64 bits over the whole sequence.

Tolerances (2-norm of a row's logits): a forward rounds to bf16 about 20
times between the embedding and the logits (2 layers), each rounding off by
0.0017 (rms) of its value, and the residual stream keeps those apart: 0.0017 *
sqrt(20) = 0.8 %; 2.5 % is held to. An s8 vector is off by 1/127/sqrt(12) of
its largest element (about 2.7 rms of 64 normal ones): 0.6 % more; an e4m3
value by 2^-4/sqrt(12) of itself at most: 1.8 % more in the values and as much
through the scores, twice: 8 % is held to.
"""

import pytest
import torch

from paper_2603_18599_gb300 import sjd
from paper_2603_18599_gb300.window_model import CACHES, WindowModel

pytestmark = pytest.mark.gpu

TOLERANCE = {"bf16": 0.025, "s8": 0.03, "e4m3": 0.08}


def plain_logits(m, tokens, b):
    """Logits [n, vocab] of sequence b holding `tokens` from position 0 on, f64."""
    n = tokens.numel()
    at = torch.arange(n, device=tokens.device)
    image = at - int(m.first[b])
    row = torch.where(image >= 0, image.div(m.grid, rounding_mode="floor"), at)
    pos = torch.stack([at, row, torch.where(image >= 0, image % m.grid, at)], 1).double()
    pairs = m.head_dim // 2
    side = pairs // 8 * 3
    axis = [0] * (pairs - 2 * side) + [1] * side + [2] * side
    freq = [10000.0 ** (-i / k) for k in (pairs - 2 * side, side, side) for i in range(k)]
    angle = pos[:, axis] * torch.tensor(freq, dtype=torch.float64, device=tokens.device)
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]

    def turned(x):
        y = torch.complex(x[..., :pairs], x[..., pairs:]) * turn
        return torch.cat([y.real, y.imag], -1)

    def norm(x):
        return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)

    h, g, d = m.heads, m.kv_heads, m.head_dim
    x = m.embed[tokens].double()
    for w in m.layers:
        qkv = (norm(x) @ w["qkv"].double()).view(n, h + 2 * g, d)
        q, k, v = turned(qkv[:, :h]), turned(qkv[:, h:h + g]), qkv[:, h + g:]
        s = torch.einsum("thd,shd->hts", q, k.repeat_interleave(h // g, 1)) * d ** -0.5
        s = s.masked_fill(~torch.ones(n, n, dtype=torch.bool, device=s.device).tril(), -float("inf"))
        o = torch.einsum("hts,shd->thd", s.softmax(-1), v.repeat_interleave(h // g, 1)).reshape(n, h * d)
        x = x + o @ w["o"].double()
        x = x + torch.nn.functional.silu(norm(x) @ w["up"].double()) @ w["down"].double()
    return norm(x) @ m.head.double()


@pytest.mark.parametrize("cache", sorted(CACHES))
def test_forwards_of_a_decode(cache):
    """Every fifth forward of a decode: the window's logits against the plain
    model on the committed tokens and the window's drafts, for both branches
    of two images that commit at their own pace."""
    B, W, V, grid = 2, 16, 512, 9
    prompts = [23, 5, 1, 2]
    m = WindowModel(B, W, prompts, grid, V, cache=CACHES[cache], page_size=24)
    m.prefill()
    ctx = sjd.SJD(sjd.make_config(B, W, V, cfg_scale=1.5, top_k=50, seed=3))
    cond, uncond = (torch.empty(B, W, V, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    seen = []

    def forward(window, prev, abs_pos, c, u):
        m.forward(window, prev, abs_pos, c, u)
        seen.append(tuple(t.clone() for t in (window, abs_pos, c, u)))

    tokens, accepted, steps = ctx.decode_loop(forward, grid * grid, cond, uncond)
    assert ctx.sync() == sjd.SJD_OK and m.cache.sync() == sjd.SJD_OK
    assert ((tokens >= 0) & (tokens < V)).all()
    # (a window may reach past the image: what it commits there is not in `tokens`)
    checked = 0
    for window, abs_pos, c, u in seen[::5]:
        for b in range(B):
            at = int(abs_pos[b])
            if at + W > grid * grid:
                continue
            for branch, logits in enumerate((c, u)):
                s = branch * B + b
                inputs = torch.cat([V + torch.arange(prompts[s], device="cuda"), tokens[b, :at].long(), window[b, :-1].long()])
                want = plain_logits(m, inputs, s)[-W:]
                off = (logits[b].double() - want).norm(dim=-1) / want.norm(dim=-1)
                assert (off <= TOLERANCE[cache]).all(), (cache, at, branch, off.max())
                checked += 1
    assert checked >= 8
    # the same decode again gives the same tokens
    ctx2 = sjd.SJD(sjd.make_config(B, W, V, cfg_scale=1.5, top_k=50, seed=3))
    m.prefill()
    again, _, steps2 = ctx2.decode_loop(m.forward, grid * grid, cond, uncond)
    assert steps2 == steps and torch.equal(again, tokens)
