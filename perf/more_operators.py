"""Workloads that the speed of the window forward's dense operators is
measured on: the embedding of tokens and its gradient, norms with a residual
and their gradient, and the matrix product in 8-bit integers with scales per
token and channel.

A case is one call of a decoding (or adapting) program with its sizes and
types. Rows are tokens: a window's of every image and branch, a prompt's, a
whole image's. Activations are normal with a magnitude of their own for each
token and some channels that are several times as large, as a model's hidden
states have; weights are quantised channel by channel. Inputs are made on the
GPU from a seed.

With `own` false the operators are computed in their plain form, elementary
torch operations in 32 bits, rounded once at the end; with `own` true through
the library.
"""

import math

import torch

own = False

DEVICE = "cuda"

DEFAULTS = {
    "op": "product",         # product | project | norm | norm_gradient | embed | embed_gradient
    "tokens": 32,            # rows
    "dim": 4096,             # features: of a row, and of a product's input
    "out": 4096,             # channels of a product
    "dtype": "bf16",         # of activations and results: bf16 | f32
    "bias": False, "residual": False,
    "centre": False,         # norm: with the mean taken off (layer norm), else by the root of the mean square alone
    "vocab": 65536,          # rows of the embedding's table
    "table": "bf16",         # its type
    "apart": 0,              # elements between one row and the next, beside the row (views of wider tensors)
}

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6


def _case(name=None, **kw):
    c = dict(DEFAULTS, **kw)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # one token of one image, both branches, queries, keys and values at
        # once: the smallest product, its weight read for two rows
        _case("product_token", tokens=2, out=6144),
        # the window of one image, both branches: attention's output back into
        # the residual stream
        _case("product_window", tokens=32, residual=True),
        # the logits of a window of 64, both branches, f32
        _case("product_logits_f32", tokens=128, out=65536, dtype="f32"),
        # sizes that no tile divides: a ragged vocabulary, 1000 features
        # inside wider rows, a bias
        _case("product_ragged", tokens=333, dim=1000, out=10007, bias=True, apart=7),
        # whole images of 90 x 90 tokens through the wide layer
        _case("product_images", tokens=8100, out=16384),
        # the windows of sixteen images: residual and norm, codes, product
        _case("project_windows", op="project", tokens=2048, out=6144, residual=True),
        # a window's norm: a small call, paid twice in every layer
        _case("norm_window", op="norm", tokens=32, residual=True),
        # two whole images, with mean and bias
        _case("norm_images", op="norm", tokens=16200, dim=1600, centre=True, bias=True),
        # gradients: bf16 with a residual branch's, and f32 with mean and bias
        _case("norm_gradient", op="norm_gradient", tokens=8100, residual=True),
        _case("norm_gradient_f32", op="norm_gradient", tokens=12291, dim=1600, dtype="f32", centre=True, bias=True),
        # the tokens of a window
        _case("embed_window", op="embed", tokens=32),
        # two images' gradient into the table of a large vocabulary, a few
        # ids in most of the places
        _case("embed_gradient", op="embed_gradient", tokens=16200),
    ]


def work(c):
    c = _case(**c)
    t, d, n, v = c["tokens"], c["dim"], c["out"], c["vocab"]
    e = 4 if c["dtype"] == "f32" else 2
    product = d * n + 4 * n + e * t * n + (4 * n if c["bias"] else 0)
    if c["op"] == "product":
        return {"bytes": product + t * d + 4 * t + (e * t * n if c["residual"] else 0), "flops": 2 * t * d * n}
    if c["op"] == "project":
        return {"bytes": product + (3 if c["residual"] else 1) * e * t * d + 4 * d, "flops": 2 * t * d * n + 8 * t * d}
    if c["op"] == "norm":
        return {"bytes": (4 if c["residual"] else 2) * e * t * d + 4 * d * (2 if c["bias"] else 1), "flops": 8 * t * d}
    if c["op"] == "norm_gradient":
        return {"bytes": (4 if c["residual"] else 3) * e * t * d + 4 * d * (3 if c["bias"] else 2), "flops": 16 * t * d}
    if c["op"] == "embed":
        return {"bytes": t * (4 + d * (e + (4 if c["table"] == "f32" else 2))), "flops": t * d}
    return {"bytes": t * (4 + d * e) + 4 * v * d, "flops": 2 * t * d}


def draw(rng):
    """One more case of the ranges above: 1 to 16384 rows of 64 to 16384
    features, products of 16 to 65536 channels, vocabularies of 512 to 65536,
    both types, rows side by side or apart."""
    def log_uniform(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    every = listed()
    while True:
        op = rng.choice(["product", "product", "product", "product", "project", "project", "norm", "norm_gradient", "norm_gradient",
                         "embed", "embed_gradient"])
        c = _case(op=op, tokens=rng.choice([log_uniform(1, 64), log_uniform(1, 512), log_uniform(64, 16384)]),
                  dim=rng.choice([512, 1024, 1600, 2048, 4096, 4096, 5120, 8192, log_uniform(64, 4096), log_uniform(64, 16384)]),
                  out=rng.choice([512, 1024, 4096, 6144, 10007, 16384, 32768, 65536, log_uniform(16, 16384)]),
                  dtype=rng.choice(["bf16", "bf16", "f32"]), bias=rng.random() < 0.4, residual=rng.random() < 0.5,
                  centre=rng.random() < 0.4, vocab=rng.choice([8192, 16384, 65536, 10007, log_uniform(512, 65536)]),
                  table=rng.choice(["bf16", "f32"]), apart=rng.choice([0, 0, 0, 8, 7]))
        if op == "project":
            c["dtype"] = "bf16"      # (codes next to a border differ by one with the order of the norm's sums)
        cost = work(c)
        most = [work(x) for x in every if op in (x["op"], "embed")]
        if cost["bytes"] <= max(w["bytes"] for w in most) and cost["flops"] <= max(w["flops"] for w in most):
            return c


def _quantise(x):
    """Rows in f32 -> codes of 8 bits and a scale for each row."""
    scale = x.abs().amax(-1) / torch.full((), 127.0, device=x.device)
    return (x / torch.where(scale > 0, scale, torch.ones_like(scale))[:, None]).round().to(torch.int8), scale


def prepare(case, seed):
    """Inputs of one call, and the library's packed weight where that is what runs."""
    c = _case(**case)
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(1000003 * int(seed) + 29)
    t, d, n = c["tokens"], c["dim"], c["out"]
    dtype = TYPES[c["dtype"]]

    def normal(*shape):
        return torch.randn(*shape, device=DEVICE, generator=gen)

    def uniform(*shape):
        return torch.rand(*shape, device=DEVICE, generator=gen)

    def hidden(rows):
        large = 1.0 + 5.0 * (uniform(d) < 0.01).float()
        return normal(rows, d) * torch.exp(0.3 * normal(rows, 1)) * large

    def apart(x):
        """The same values as a view of wider rows."""
        if not c["apart"]:
            return x
        wide = torch.zeros(x.shape[0], x.shape[1] + c["apart"], dtype=x.dtype, device=DEVICE)
        wide[:, :x.shape[1]] = x
        return wide[:, :x.shape[1]]

    s = {"case": c}
    if c["op"] in ("product", "project"):
        s["weight"], s["channel_scale"] = _quantise(normal(n, d) * d ** -0.5 * torch.exp(0.2 * normal(n, 1)))
        s["bias"] = 0.1 * normal(n) if c["bias"] else None
        if own:
            from paper_2603_18599_gb300 import dense
            s["packed"] = dense.Weight(s["weight"], s["channel_scale"])
    if c["op"] == "product":
        codes, s["scale"] = _quantise(hidden(t))
        s["codes"] = apart(codes)
        s["residual"] = apart(normal(t, n).to(dtype)) if c["residual"] else None
    if c["op"] in ("project", "norm", "norm_gradient"):
        s["x"] = apart(hidden(t).to(dtype))
        s["gain"] = 1.0 + 0.1 * normal(d)
        s["offset"] = 0.1 * normal(d) if c["bias"] and c["op"] != "project" else None
        s["residual"] = apart(hidden(t).to(dtype)) if c["residual"] else None
    if c["op"] == "norm_gradient":
        s["dy"] = apart(normal(t, d).to(dtype))
    if c["op"] in ("embed", "embed_gradient"):
        # small ids are frequent ones, and one place in twenty is empty (-1)
        tokens = (c["vocab"] * uniform(t) ** 3).long().clamp(max=c["vocab"] - 1).int()
        s["tokens"] = torch.where(uniform(t) < 0.05, torch.full_like(tokens, -1), tokens)
        s["scale"] = d ** 0.5
        if c["op"] == "embed":
            s["table"] = (normal(c["vocab"], d) * d ** -0.5).to(TYPES[c["table"]])
        else:
            s["dy"] = apart(normal(t, d).to(dtype))
    return s


def _product(codes, scale, s, residual):
    y = (codes.float() @ s["weight"].float().T) * scale[:, None] * s["channel_scale"]
    if s["bias"] is not None:
        y = y + s["bias"]
    if residual is not None:
        y = y + residual.float()
    return y.to(TYPES[s["case"]["dtype"]])


def _normed(h, s):
    """h in f32 without its mean (or as it is), and the factor that makes it one in the root of the mean square."""
    u = h - h.mean(-1, keepdim=True) if s["case"]["centre"] else h
    return u, 1.0 / torch.sqrt(u.square().mean(-1, keepdim=True) + EPS)


def _plain_norm(s):
    """The residual stream, and its norm in f32."""
    h = s["x"]
    if s["residual"] is not None:
        h = (h.float() + s["residual"].float()).to(h.dtype)
    u, r = _normed(h.float(), s)
    y = u * r * s["gain"]
    return h, y if s["offset"] is None else y + s["offset"]


def _plain_norm_gradient(s):
    dy = s["dy"].float()
    u, r = _normed(s["x"].float(), s)
    u = u * r
    g = dy * s["gain"]
    dx = g - u * (g * u).mean(-1, keepdim=True)
    if s["case"]["centre"]:
        dx = dx - g.mean(-1, keepdim=True)
    dx = dx * r
    if s["residual"] is not None:
        dx = dx + s["residual"].float()
    out = {"dx": dx.to(s["x"].dtype), "dgain": (dy * u).sum(0)}
    return dict(out, doffset=dy.sum(0)) if s["offset"] is not None else out


def run(s):
    c = s["case"]
    if own:
        from paper_2603_18599_gb300 import dense
    if c["op"] == "product":
        if own:
            return dense.product(s["codes"], s["scale"], s["packed"], bias=s["bias"], residual=s["residual"], dtype=TYPES[c["dtype"]])
        return _product(s["codes"], s["scale"], s, s["residual"])
    if c["op"] == "project":
        if own:
            codes, scale, *h = dense.norm_codes(s["x"], s["gain"], residual=s["residual"], eps=EPS, centre=c["centre"])
            return {"y": dense.product(codes, scale, s["packed"], bias=s["bias"], dtype=TYPES[c["dtype"]]), "h": h[0] if h else None}
        h, y = _plain_norm(s)
        return {"y": _product(*_quantise(y), s, None), "h": h if s["residual"] is not None else None}
    if c["op"] == "norm":
        if own:
            y = dense.norm(s["x"], s["gain"], s["offset"], residual=s["residual"], eps=EPS, centre=c["centre"])
            return {"y": y[0], "h": y[1]} if s["residual"] is not None else {"y": y, "h": None}
        h, y = _plain_norm(s)
        return {"y": y.to(h.dtype), "h": h if s["residual"] is not None else None}
    if c["op"] == "norm_gradient":
        if not own:
            return _plain_norm_gradient(s)
        dx, dgain, doffset = dense.norm_gradient(s["dy"], s["x"], s["gain"], eps=EPS, centre=c["centre"], dh=s["residual"], bias=c["bias"])
        return {"dx": dx, "dgain": dgain, "doffset": doffset} if c["bias"] else {"dx": dx, "dgain": dgain}
    if c["op"] == "embed":
        if own:
            return dense.embed(s["table"], s["tokens"], scale=s["scale"], dtype=TYPES[c["dtype"]])
        inside = (s["tokens"] >= 0)[:, None]
        return (s["table"][s["tokens"].clamp(min=0)].float() * s["scale"] * inside).to(TYPES[c["dtype"]])
    if own:
        return dense.embed_gradient(s["dy"], s["tokens"], c["vocab"], scale=s["scale"])
    # (a row more, for the places that are empty)
    at = torch.where(s["tokens"] < 0, torch.full_like(s["tokens"], c["vocab"]), s["tokens"])
    grad = torch.zeros(c["vocab"] + 1, c["dim"], device=DEVICE)
    return grad.index_add_(0, at, s["dy"].float() * s["scale"])[:-1]


# --- the same from the definitions, in 64 bits ------------------------------

def _exact_norm(s):
    c = s["case"]
    h = s["x"].double()
    if s["residual"] is not None:
        h = (h + s["residual"].double()).to(s["x"].dtype).double()
    mean = h.sum(1) / c["dim"] if c["centre"] else torch.zeros(c["tokens"], dtype=torch.float64, device=DEVICE)
    spread = (h - mean[:, None]).pow(2).sum(1) / c["dim"]
    return h, (h - mean[:, None]) / (spread + EPS).pow(0.5)[:, None], (spread + EPS).pow(-0.5)


def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    if c["op"] in ("product", "project"):
        h = None
        if c["op"] == "product":
            value = s["codes"].double() * s["scale"].double()[:, None]
        else:
            h, u, _ = _exact_norm(s)
            y = u * s["gain"].double()
            step = y.abs().amax(1, keepdim=True) / 127
            value = torch.where(step > 0, (y / step).round() * step, torch.zeros_like(y))
        out = torch.einsum("td,nd->tn", value, s["weight"].double() * s["channel_scale"].double()[:, None])
        if s["bias"] is not None:
            out += s["bias"].double()
        if c["op"] == "project":
            return {"y": out, "h": h if s["residual"] is not None else None}
        return out if s["residual"] is None else out + s["residual"].double()
    if c["op"] == "norm":
        h, u, _ = _exact_norm(s)
        y = u * s["gain"].double()
        return {"y": y if s["offset"] is None else y + s["offset"].double(), "h": h if s["residual"] is not None else None}
    if c["op"] == "norm_gradient":
        branch, s["residual"] = s["residual"], None
        _, u, r = _exact_norm(s)
        dy = s["dy"].double()
        g = dy * s["gain"].double()
        along = torch.einsum("td,td->t", g, u) / c["dim"]
        mean = g.sum(1) / c["dim"] if c["centre"] else torch.zeros_like(along)
        dx = r[:, None] * (g - mean[:, None] - u * along[:, None])
        out = {"dx": dx if branch is None else dx + branch.double(), "dgain": torch.einsum("td,td->d", dy, u)}
        return dict(out, doffset=dy.sum(0)) if c["bias"] else out
    tokens = s["tokens"].long()
    if c["op"] == "embed":
        rows = s["table"].double().index_select(0, tokens.clamp(min=0)) * s["scale"]
        return rows.masked_fill((tokens < 0)[:, None], 0.0)
    grad = torch.zeros(c["vocab"], c["dim"], dtype=torch.float64, device=DEVICE)
    kept = tokens >= 0
    return grad.index_add_(0, tokens[kept], s["dy"][kept].double() * s["scale"])
