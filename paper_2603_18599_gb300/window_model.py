"""A small decoder whose forward of the Jacobi window runs on the library's
operators, and a decode of one image with it (random weights: the tokens mean
nothing, the calls are those of a real model).

Every image has two sequences in the cache, one behind the conditional prompt
and one behind the unconditional one. Sequence b holds its prompt at
positions 0 .. prompt[b] - 2 and then the inputs of the image's positions: the
prompt's last token for position 0, image token j - 1 for position j. A
forward writes the keys and values of the window's W inputs over those of the
step before (a rejected draft's are replaced at once), attends with W queries
to everything before each of them, and gives the logits of W positions. Where
the window stands is read from device arrays: no step waits for the host.

    python -m paper_2603_18599_gb300.window_model --cache e4m3 --grid 24
"""

import argparse
import time

import torch

from . import kv, sjd

CACHES = {"bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "s8": torch.int8}


class WindowModel:
    """vocab image tokens, `layers` layers of `heads` query and `kv_heads`
    key heads of `head_dim`; positions on three axes: of the sequence, and row
    and column in the image's grid."""

    def __init__(self, images, window, prompts, grid, vocab=8192, layers=2, heads=8, kv_heads=2, head_dim=64, page_size=32,
                 cache=torch.bfloat16, seed=0, device="cuda"):
        self.images, self.window, self.grid, self.vocab, self.device = images, window, grid, vocab, device
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim
        dim = heads * head_dim
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)

        def weight(n_in, n_out):
            return (torch.randn(n_in, n_out, device=device, generator=gen) * n_in ** -0.5).bfloat16()

        # image tokens, then the prompts' own tokens (each prompt position has one)
        self.prompt = list(prompts)                            # [2 * images] lengths, the last token opens the image
        self.embed = torch.randn(vocab + max(prompts), dim, device=device, generator=gen).bfloat16()
        self.layers = [{"qkv": weight(dim, (heads + 2 * kv_heads) * head_dim), "o": weight(dim, dim),
                        "up": weight(dim, 2 * dim), "down": weight(2 * dim, dim)} for _ in range(layers)]
        self.head = weight(dim, vocab)
        pairs = head_dim // 2
        side = pairs // 8 * 3
        self.rope = kv.Rope.sections((pairs - 2 * side, side, side), device=device)

        sequences, longest = 2 * images, max(prompts) + grid * grid + window
        pages = -(-longest // page_size)
        self.cache = kv.KV(sequences, heads, kv_heads, head_dim, n_pages=sequences * pages, page_size=page_size, max_pages=pages,
                           max_new=max(window, max(prompts)), dtype=cache, device=device)
        self.held = [self.cache.new_layer() for _ in range(layers)]
        self.table = torch.randperm(sequences * pages, device=device, generator=gen).int().view(sequences, pages)
        self.first = torch.tensor(prompts, dtype=torch.int32, device=device) - 1   # the position of the image's first input
        self._zero = torch.zeros(sequences, dtype=torch.int32, device=device)

    def positions(self, at):
        """[B, n, 3] of sequence positions at [B, n]: prompt tokens stand on
        the diagonal, image inputs in their grid."""
        image = at - self.first[:, None]
        inside = image >= 0
        row = torch.where(inside, image.div(self.grid, rounding_mode="floor"), at)
        return torch.stack([at, row, torch.where(inside, image % self.grid, at)], 2).int()

    @staticmethod
    def norm(x):
        y = x.float()
        return (y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype)

    def hidden(self, tokens, start, count=None):
        """The last layer's output for `tokens` [2 * images, n] at positions
        start[b] .. of their sequences, whose keys and values are written."""
        B, n = tokens.shape
        h, g, d = self.heads, self.kv_heads, self.head_dim
        positions = self.positions(start[:, None] + torch.arange(n, device=self.device))
        x = self.embed[tokens]
        for w, held in zip(self.layers, self.held):
            qkv = (self.norm(x) @ w["qkv"]).view(B, n, h + 2 * g, d)
            q = self.cache.write(held, qkv[:, :, h:h + g], qkv[:, :, h + g:], self.table, start, count, rope=self.rope,
                                 positions=positions, q=qkv[:, :, :h])
            o = self.cache.attend(held, q, self.table, start, count)
            x = x + o.view(B, n, h * d) @ w["o"]
            x = x + torch.nn.functional.silu(self.norm(x) @ w["up"]) @ w["down"]
        return x

    def prefill(self):
        """The prompts, but for their last tokens, into the cache: one chunk,
        every sequence as long as its prompt."""
        n = max(self.prompt) - 1
        if n > 0:
            tokens = self.vocab + torch.arange(n, device=self.device).expand(2 * self.images, n)
            self.hidden(tokens, self._zero, self.first)

    def forward(self, window, prev, abs_pos, cond, uncond):
        """The target forward of sjd_decode_loop: logits [images, W, vocab]
        of both branches. (The loop goes on until the slowest image is done;
        the others stay at their end.)"""
        abs_pos = abs_pos.clamp(max=self.grid * self.grid)
        opening = self.vocab + self.first.view(2, -1)                       # [branch, image]
        last = torch.where(abs_pos == 0, opening, prev.expand(2, -1))
        tokens = torch.cat([last[:, :, None], window[:, :-1].expand(2, -1, -1)], 2).view(2 * self.images, -1)
        x = self.hidden(tokens, self.first + abs_pos.repeat(2))
        logits = (self.norm(x) @ self.head).view(2, self.images, self.window, self.vocab)
        cond.copy_(logits[0])
        uncond.copy_(logits[1])


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--cache", choices=sorted(CACHES), default="e4m3")
    ap.add_argument("--images", type=int, default=2)
    ap.add_argument("--window", type=int, default=16)
    ap.add_argument("--grid", type=int, default=24, help="image tokens per row and column")
    ap.add_argument("--vocab", type=int, default=8192)
    args = ap.parse_args()
    B, W, V = args.images, args.window, args.vocab
    prompts = [20 + 7 * b for b in range(B)] + [1] * B                       # conditional, unconditional
    model = WindowModel(B, W, prompts, args.grid, V, cache=CACHES[args.cache])
    cfg = sjd.make_config(B, W, V, cfg_scale=3.0, top_k=2000, seed=0)
    ctx = sjd.SJD(cfg)
    cond, uncond = (torch.empty(B, W, V, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    model.prefill()
    torch.cuda.synchronize()
    begun = time.perf_counter()
    tokens, accepted, steps = ctx.decode_loop(model.forward, args.grid ** 2, cond, uncond)
    seconds = time.perf_counter() - begun
    if model.cache.sync() != sjd.SJD_OK:
        raise SystemExit("cache: " + model.cache.last_error())
    print("%d images of %d tokens: %d steps, %.2f tokens accepted per step, %.2f ms per step, %s cache" % (
        B, tokens.shape[1], steps, B * tokens.shape[1] / (B * steps), seconds / steps * 1e3, args.cache))


if __name__ == "__main__":
    main()
