"""Workloads that the speed of the window forward's operators is measured on:
rotary positions with several axes, the paged cache (written, quantised on
the way, and read back), and attention of a chunk of new tokens over it.

A case is one call of a decoding program with its sizes and types. Sequences
come in pairs of a conditional and an unconditional branch, every sequence
has its own length, and what a sequence holds is scattered over the cache's
pages. Inputs are made on the GPU from a seed: queries, keys and values are
normal, the magnitude of a token's keys and values differs from token to
token, and they are views of one packed projection, as a model's are.

With `own` false the operators are computed in their plain form, elementary
torch operations in 32 bits, rounded once at the end; with `own` true through
the library.
"""

import math

import torch

own = False

DEVICE = "cuda"

DEFAULTS = {
    "op": "attend",          # rotate | write | read | attend
    "batch": 2, "new": 16, "context": 0,   # sequences, new tokens, tokens before them (of the longest sequence)
    "heads": 32, "kv_heads": 8, "dim": 128,
    "dtype": "bf16",         # of queries, keys and values: bf16 | f32 (rotate and write)
    "cache": "bf16",         # bf16 | e4m3 | s8
    "page": 64,              # tokens of a page
    "mask": "causal",        # causal | tree | all
    "axes": 3, "interleaved": False, "inverse": False, "rope": False,
    "grid": 32,              # image tokens per grid row (the positions' second and third axis)
    "lse": False,            # attend: the logarithm of the sum too
}

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn, "s8": torch.int8}
LARGEST = {"e4m3": 448.0, "s8": 127.0}
TREE_K, TREE_D = 4, 3        # the drafting tree: K children of a node, depth D
TREE_ROWS = sum(TREE_K ** d - 1 for d in range(1, TREE_D))


def _case(name=None, **kw):
    c = dict(DEFAULTS, **kw)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # the queries of a window of one image, both branches, time, row and
        # column axes: a small call, its latency paid in every layer
        _case("rotate_window", op="rotate"),
        # the gradient of a long batch's queries, f32, two axes, neighbouring
        # pairs, a head size that is no power of two
        _case("rotate_gradient_f32", op="rotate", batch=3, new=4097, heads=20, dim=80, dtype="f32", axes=2,
              interleaved=True, inverse=True, grid=90),
        # one token of one image: the smallest write
        _case("write_token_s8", op="write", new=1, context=700, cache="s8", page=16, rope=True),
        # the window of sixteen images, both branches: queries and keys
        # rotated, keys and values quantised, in the middle of long sequences
        _case("write_windows_e4m3", op="write", batch=32, new=64, context=4000, cache="e4m3", rope=True, grid=90),
        # two whole images written at once, f32, pages of no power of two
        _case("write_images_s8_f32", op="write", batch=4, new=8100, kv_heads=16, heads=16, dim=96, dtype="f32", cache="s8",
              page=24, grid=90),
        # ragged sequences taken out of an 8-bit cache
        _case("read_images_e4m3", op="read", batch=16, new=8100, cache="e4m3", page=32),
        # one token over a short sequence: the smallest attention
        _case("attend_token", new=1, context=300, page=16),
        # the window of one image, both branches, over its 32 x 32 grid
        _case("attend_window", new=16, context=1000, lse=True),
        # the windows of sixteen images over 90 x 90 grids, 8-bit cache
        _case("attend_windows_e4m3", batch=32, new=64, context=8100, cache="e4m3", page=128),
        # windows with the full drafting tree's nodes, every head its own
        # keys, odd pages
        _case("attend_trees_s8", batch=8, new=32 + TREE_ROWS, context=2000, heads=16, kv_heads=16, dim=64, cache="s8", page=24,
              mask="tree", lse=True),
        # a long prompt behind a prefix that is in the cache already
        _case("attend_prompt", batch=1, new=4000, context=4100, page=128),
        # one token of many long sequences, 8-bit cache
        _case("attend_long_e4m3", batch=16, new=1, context=32768, heads=64, cache="e4m3", page=64),
    ]


def lengths(c):
    """Tokens before the new ones, per sequence: the longest has them all,
    the others down to half of them."""
    return [int(c["context"] * (1.0 - 0.5 * ((b * 0.6180339887) % 1.0))) for b in range(c["batch"])]


def tree_mask(window, k, depth):
    """mask[i][j]: row i of the chunk sees row j. The window's rows form a
    chain; then every node i >= 1 of the depths 1..D-1 sees itself, its
    ancestors (node 0 of depth d is the window's row d) and row 0."""
    row = {(d, 0): d for d in range(depth)}
    at = window
    for d in range(1, depth):
        for i in range(1, k ** d):
            row[d, i] = at
            at += 1
    mask = torch.zeros(at, at, dtype=torch.bool)
    mask[:window, :window] = torch.ones(window, window).tril().bool()
    for (d, i), r in row.items():
        if r >= window:
            while True:
                mask[r, row[d, i]] = True
                if d == 0:
                    break
                d, i = d - 1, i // k
    return mask


def _visible(c):
    """Pairs of a query and a key that it sees, of one head."""
    n = c["new"]
    if c["mask"] == "tree":
        own_pairs = int(tree_mask(n - TREE_ROWS, TREE_K, TREE_D).sum())
    else:
        own_pairs = n * (n + 1) // 2 if c["mask"] == "causal" else n * n
    return sum(n * s + own_pairs for s in lengths(c))


def work(c):
    b, n, h, g, d = c["batch"], c["new"], c["heads"], c["kv_heads"], c["dim"]
    e = 4 if c["dtype"] == "f32" else 2
    held = g * (d * 2 if c["cache"] == "bf16" else d + 4)      # one token's keys (or values) in the cache
    if c["op"] == "rotate":
        return {"bytes": b * n * (2 * h * d * e + 4 * c["axes"]), "flops": 3 * b * n * h * d}
    if c["op"] == "write":
        turned = 2 * h * d * e + 4 * c["axes"] if c["rope"] else 0
        return {"bytes": b * n * (2 * (g * d * e + 2 * held + g * d * 2) + turned),
                "flops": b * n * (2 * 4 * g * d + (3 * (h + g) * d if c["rope"] else 0))}
    tokens = sum(lengths(c)) + b * n
    if c["op"] == "read":
        tokens = sum(_counts(c))
        return {"bytes": 2 * tokens * (held + g * d * 2), "flops": 2 * tokens * g * d}
    return {"bytes": 2 * tokens * held + b * n * h * (4 * d + (4 if c["lse"] else 0)) + (n * n if c["mask"] == "tree" else 0),
            "flops": 4 * h * d * _visible(c)}


def _counts(c):
    """Tokens to be read of each sequence: the longest has them all."""
    return [max(1, int(c["new"] * (1.0 - 0.5 * ((b * 0.6180339887) % 1.0)))) for b in range(c["batch"])]


def draw(rng):
    """One more case of the ranges above: 1 to 32 sequences, chunks of 1 to
    4097 tokens (8100 written or read), contexts up to 32768, head sizes 64
    to 128, 1 to 16 query heads per key head, all types, pages of 8 to 128."""
    def log_uniform(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    every = listed()
    while True:
        op = rng.choice(["attend", "attend", "attend", "attend", "write", "write", "read", "rotate"])
        kv_heads, group = rng.choice([(8, 4), (8, 8), (16, 1), (32, 1), (4, 7), (2, 16), (1, 8), (5, 4), (4, 3)])
        c = _case(op=op, batch=log_uniform(1, 32), kv_heads=kv_heads, heads=kv_heads * group,
                  dim=rng.choice([64, 64, 80, 112, 128, 128, 128]), cache=rng.choice(["bf16", "e4m3", "s8"]),
                  page=rng.choice([8, 16, 24, 32, 40, 64, 128]), axes=rng.choice([1, 2, 3]),
                  interleaved=rng.random() < 0.4, grid=rng.choice([24, 32, 90]))
        if op == "attend":
            c.update(mask=rng.choice(["causal", "causal", "tree", "all"]), lse=rng.random() < 0.5)
            c.update(new=rng.choice([1, log_uniform(1, 64), log_uniform(2, 64), log_uniform(64, 4097)]),
                     context=rng.choice([0, log_uniform(16, 2048), log_uniform(64, 32768)]))
            if c["mask"] == "tree":
                c["new"] = log_uniform(TREE_D, 64) + TREE_ROWS
        else:
            c.update(new=rng.choice([1, log_uniform(1, 64), log_uniform(64, 8100)]), dtype=rng.choice(["bf16", "bf16", "f32"]))
            if op == "write":
                c.update(context=log_uniform(16, 8100), rope=rng.random() < 0.6)
            if op == "rotate":
                c.update(inverse=rng.random() < 0.4)
            if op == "read":
                c.update(dtype="bf16")
        cost = work(c)
        most = [work(x) for x in every if x["op"] == op]
        if cost["bytes"] > max(w["bytes"] for w in most) or cost["flops"] > max(w["flops"] for w in most):
            continue
        # the plain form holds every pair of a query and a key
        t = max(lengths(c)) + c["new"]
        if op == "attend" and (c["batch"] * c["heads"] * c["new"] * t > 1.1e9 or c["batch"] * c["kv_heads"] * c["dim"] * t > 6e8):
            continue
        return c


def _pairs(c):
    """Each pair's axis and its angle per position, in turns: the pairs are
    shared out among the axes, each with frequencies of its own."""
    half, axes = c["dim"] // 2, c["axes"]
    share = [half // axes + (1 if a < half % axes else 0) for a in range(axes)]
    axis = [a for a in range(axes) for _ in range(share[a])]
    freq = [10000.0 ** (-i / share[a]) for a in range(axes) for i in range(share[a])]
    return axis, freq


def _positions(c, start):
    """[B, n, axes]: a running position, the grid's row and its column."""
    p = torch.arange(c["new"], device=DEVICE)[None, :] + start[:, None]
    return torch.stack([p, p // c["grid"], p % c["grid"]][:c["axes"]], dim=2).int()


def _quantise(x, kind):
    """x [..., dim] in f32 -> values held in the cache's type and the scale
    of each vector (None for a 16-bit cache)."""
    if kind == "bf16":
        return x.bfloat16(), None
    top = torch.full((), LARGEST[kind], device=x.device)
    scale = x.abs().amax(-1) / top
    y = x / torch.where(scale > 0, scale, torch.ones_like(scale))[..., None]
    return (y.round().to(torch.int8) if kind == "s8" else y.to(torch.float8_e4m3fn)), scale


def prepare(case, seed):
    """Inputs of one call: the packed projection, positions, the cache with
    its page table, and the library's handle where that is what runs."""
    c = _case(**case)
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(1000003 * int(seed) + 17)
    b, n, h, g, d = c["batch"], c["new"], c["heads"], c["kv_heads"], c["dim"]

    def normal(*shape):
        return torch.randn(*shape, device=DEVICE, generator=gen)

    s = {"case": c, "start": torch.tensor(lengths(c), dtype=torch.int32, device=DEVICE)}
    if c["op"] != "read":
        width = h if c["op"] == "rotate" else h + 2 * g
        packed = normal(b, n, width, d) * (1.5 if c["op"] == "attend" else 1.0) * torch.exp(0.3 * normal(b, n, 1, 1))
        packed = packed.to(TYPES[c["dtype"]])
        s["q"] = packed[:, :, :h]
        if c["op"] == "write":
            s["k"], s["v"] = packed[:, :, h:h + g], packed[:, :, h + g:]
    if c["op"] == "rotate" or c["rope"]:
        axis, freq = _pairs(c)
        s["positions"] = _positions(c, s["start"])
        s["axis"] = torch.tensor(axis, device=DEVICE)
        turns = [round(f / (2.0 * math.pi) * 2.0 ** 64) for f in freq]
        s["turns"] = torch.tensor([t - 2 ** 64 if t >= 2 ** 63 else t for t in turns], device=DEVICE)
    if c["op"] != "rotate":
        held = [x + n for x in lengths(c)] if c["op"] != "read" else _counts(c)
        pages = [-(-x // c["page"]) for x in held]
        total = sum(pages) + 3
        order = torch.randperm(total, device=DEVICE, generator=gen).int().tolist()
        table, at = [], 0
        for m in pages:
            table.append(order[at:at + m] + [-1] * (max(pages) - m))
            at += m
        s["table"] = torch.tensor(table, dtype=torch.int32, device=DEVICE)
        for name in ("k", "v"):
            values = normal(total, g, c["page"], d) * torch.exp(0.3 * normal(total, g, c["page"], 1))
            s[name + "_cache"], s[name + "_scale"] = _quantise(values, c["cache"])
            del values
    if c["op"] == "read":
        s["count"] = torch.tensor(_counts(c), dtype=torch.int32, device=DEVICE)
        s["zero"] = torch.zeros(b, dtype=torch.int32, device=DEVICE)
    if c["op"] == "attend" and c["mask"] == "tree":
        s["mask"] = tree_mask(n - TREE_ROWS, TREE_K, TREE_D).to(DEVICE)[None]
    if own:
        from paper_2603_18599_gb300 import kv
        if "turns" in s:
            s["rope"] = kv.Rope(freq, axis, interleaved=c["interleaved"], device=DEVICE)
        if c["op"] != "rotate":
            s["handle"] = kv.KV(batch=b, heads=h, kv_heads=g, head_dim=d, n_pages=total, page_size=c["page"],
                                max_pages=s["table"].shape[1], max_new=n, dtype=TYPES[c["cache"]], device=DEVICE)
            s["layer"] = kv.Layer(s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"])
    return s


def _rotated(x, s):
    """Plain rotation: pair i turned by position * frequency, reduced to a
    fraction of a turn in integers."""
    c = s["case"]
    part = (s["positions"].long()[:, :, s["axis"]] * s["turns"]) >> 32
    angle = part.float() * (2.0 * math.pi / 2.0 ** 32)
    cos, sin = torch.cos(angle)[:, :, None], torch.sin(angle)[:, :, None]
    if c["inverse"]:
        sin = -sin
    x = x.float()
    half = c["dim"] // 2
    u, v = (x[..., 0::2], x[..., 1::2]) if c["interleaved"] else (x[..., :half], x[..., half:])
    p, q = u * cos - v * sin, u * sin + v * cos
    return torch.stack([p, q], -1).flatten(-2) if c["interleaved"] else torch.cat([p, q], -1)


def _taken(s, name, last):
    """Plain read: the first `last` tokens of every sequence, [B, Hkv, last, D]
    in f32."""
    c = s["case"]
    table = s["table"][:, :-(-last // c["page"])].clamp(min=0).long()
    cache = s[name + "_cache"]
    bits = cache.view(torch.uint8) if cache.dtype == torch.float8_e4m3fn else cache
    x = bits[table].view(cache.dtype).float()
    if s[name + "_scale"] is not None:
        x = x * s[name + "_scale"][table][..., None]
    return x.permute(0, 2, 1, 3, 4).flatten(2, 3)[:, :, :last]


def _plain_write(s):
    c = s["case"]
    q, k, v = s["q"], s["k"].float(), s["v"].float()
    if c["rope"]:
        q, k = _rotated(q, s).to(s["q"].dtype), _rotated(s["k"], s)
    at = s["start"].long()[:, None] + torch.arange(c["new"], device=DEVICE)
    page, slot = s["table"].long().gather(1, at // c["page"]), at % c["page"]
    back = []
    for name, x in (("k", k), ("v", v)):
        held, scale = _quantise(x, c["cache"])
        if c["cache"] == "e4m3":
            s[name + "_cache"].view(torch.uint8)[page, :, slot] = held.view(torch.uint8)
        else:
            s[name + "_cache"][page, :, slot] = held
        if scale is not None:
            s[name + "_scale"][page, :, slot] = scale
        bits = s[name + "_cache"]
        bits = bits.view(torch.uint8) if c["cache"] == "e4m3" else bits
        y = bits[page, :, slot].view(TYPES[c["cache"]]).float()
        if scale is not None:
            y = y * s[name + "_scale"][page, :, slot][..., None]
        back.append(y.bfloat16())
    return {"q": q if c["rope"] else None, "k": back[0], "v": back[1]}


def _plain_attend(s):
    c = s["case"]
    b, n, h, g, d = c["batch"], c["new"], c["heads"], c["kv_heads"], c["dim"]
    last = s["table"].shape[1] * c["page"]
    key = torch.arange(last, device=DEVICE)
    start = s["start"].long()[:, None, None]
    if c["mask"] == "causal":
        seen = key <= start + torch.arange(n, device=DEVICE)[:, None]
    elif c["mask"] == "all":
        seen = (key < start + n).expand(b, n, last)
    else:
        inside = (key - start).expand(b, n, last)
        seen = (inside < 0) | ((inside < n) & s["mask"].expand(b, n, n).gather(2, inside.clamp(0, n - 1)))
    q = s["q"].float().view(b, n, g, h // g, d).permute(0, 2, 1, 3, 4).reshape(b, g, n * (h // g), d)
    score = (q @ _taken(s, "k", last).transpose(2, 3)).view(b, g, n, h // g, last) * d ** -0.5
    score.masked_fill_(~seen[:, None, :, None], -math.inf)
    top = score.amax(-1, keepdim=True).clamp(min=-3e38)
    score = score.sub_(top).exp_()
    total = score.sum(-1, keepdim=True)
    o = score.view(b, g, n * (h // g), last) @ _taken(s, "v", last)
    o = o.view(b, g, n, h // g, d) / torch.where(total > 0, total, torch.ones_like(total))
    out = {"o": o.permute(0, 2, 1, 3, 4).reshape(b, n, h, d).bfloat16()}
    if c["lse"]:
        out["lse"] = (top + total.log()).squeeze(-1).permute(0, 2, 1, 3).reshape(b, n, h)
    return out


def run(s):
    c = s["case"]
    if c["op"] == "rotate":
        if own:
            return s["rope"].rotate(s["q"], s["positions"], inverse=c["inverse"])
        return _rotated(s["q"], s).to(s["q"].dtype)
    if c["op"] == "write":
        if not own:
            return _plain_write(s)
        rope = {"rope": s["rope"], "positions": s["positions"], "q": s["q"]} if c["rope"] else {}
        q = s["handle"].write(s["layer"], s["k"], s["v"], s["table"], s["start"], **rope)
        k, v = s["handle"].read(s["layer"], s["table"], s["start"], c["new"])
        return {"q": q, "k": k, "v": v}
    if c["op"] == "read":
        if own:
            return s["handle"].read(s["layer"], s["table"], s["zero"], c["new"], count=s["count"])
        inside = (torch.arange(c["new"], device=DEVICE) < s["count"][:, None])[:, :, None, None]
        return tuple((_taken(s, name, c["new"]).transpose(1, 2) * inside).bfloat16() for name in ("k", "v"))
    if not own:
        return _plain_attend(s)
    mask = s.get("mask", "causal" if c["mask"] == "causal" else None)
    o = s["handle"].attend(s["layer"], s["q"], s["table"], s["start"], mask=mask, lse=c["lse"])
    return {"o": o[0], "lse": o[1]} if c["lse"] else {"o": o}


# --- the same from the definitions, in 64 bits ------------------------------

def _nearest(y, kind):
    """The value nearest to y (ties to even) that an 8-bit code stands for."""
    if kind == "s8":
        return y.round().clamp(-127, 127)
    exponent = torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -20))).clamp(min=-6)
    step = torch.exp2(exponent - 3)
    return ((y / step).round() * step).clamp(-448, 448)


def _held(x, kind):
    if kind == "bf16":
        return x.bfloat16().double()
    scale = x.abs().amax(-1, keepdim=True) / LARGEST[kind]
    return _nearest(x / torch.where(scale > 0, scale, torch.ones_like(scale)), kind) * scale


def _turned(x, positions, c):
    axis, freq = _pairs(c)
    where = positions.double()[:, :, torch.tensor(axis, device=DEVICE)]
    angle = where * torch.tensor(freq, dtype=torch.float64, device=DEVICE) * (-1.0 if c["inverse"] else 1.0)
    turn = torch.polar(torch.ones_like(angle), angle)[:, :, None]
    half = c["dim"] // 2
    if c["interleaved"]:
        y = torch.view_as_complex(x.unflatten(-1, (half, 2)).contiguous()) * turn
        return torch.view_as_real(y).flatten(-2)
    y = torch.complex(x[..., :half], x[..., half:]) * turn
    return torch.cat([y.real, y.imag], -1)


def _sequence(s, name, b, head, last):
    """The first `last` tokens of one sequence's head, [last, D] in f64."""
    c = s["case"]
    rows = torch.arange(last, device=DEVICE)
    page, slot = s["table"][b].long()[rows // c["page"]], rows % c["page"]
    cache = s[name + "_cache"]
    x = cache.view(torch.uint8 if cache.element_size() == 1 else cache.dtype)[page, head, slot].view(cache.dtype).double()
    return x if s[name + "_scale"] is None else x * s[name + "_scale"][page, head, slot].double()[:, None]


def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    n, group = c["new"], c["heads"] // c["kv_heads"]
    if c["op"] == "rotate":
        return _turned(s["q"].double(), s["positions"], c)
    if c["op"] == "write":
        k = s["k"].double()
        out = {"q": None}
        if c["rope"]:
            out["q"], k = _turned(s["q"].double(), s["positions"], c), _turned(k, s["positions"], c)
        return dict(out, k=_held(k, c["cache"]), v=_held(s["v"].double(), c["cache"]))
    if c["op"] == "read":
        out = [torch.zeros(c["batch"], n, c["kv_heads"], c["dim"], dtype=torch.float64, device=DEVICE) for _ in range(2)]
        for b, m in enumerate(_counts(c)):
            for head in range(c["kv_heads"]):
                for o, name in zip(out, ("k", "v")):
                    o[b, :m, head] = _sequence(s, name, b, head, m)
        return tuple(out)
    o = torch.zeros(c["batch"], n, c["heads"], c["dim"], dtype=torch.float64, device=DEVICE)
    lse = torch.zeros(c["batch"], n, c["heads"], dtype=torch.float64, device=DEVICE)
    for b, before in enumerate(lengths(c)):
        seen = torch.ones(n, before + n, dtype=torch.bool, device=DEVICE)
        if c["mask"] == "causal":
            seen = seen.tril(before)
        elif c["mask"] == "tree":
            seen[:, before:] = s["mask"][0]
        for head in range(c["heads"]):
            k, v = (_sequence(s, name, b, head // group, before + n) for name in ("k", "v"))
            score = (s["q"][b, :, head].double() @ k.T / math.sqrt(c["dim"])).masked_fill(~seen, -math.inf)
            o[b, :, head] = torch.softmax(score, -1) @ v
            lse[b, :, head] = torch.logsumexp(score, -1)
    return {"o": o, "lse": lse} if c["lse"] else {"o": o}
