"""Python binding of the forward's operators on rows of features (include/sjd.h):
the embedding of tokens and its gradient, norms with a residual and their
gradient, and matrix products of 8-bit integers with a scale for each token and
each channel. Argument marshalling only.

    x = dense.embed(table, tokens)
    up = dense.Weight.quantise(w)                       # [out, in], bf16 or f32
    codes, scale = dense.norm_codes(x, gain)
    y = dense.product(codes, scale, up)
    codes, scale, x = dense.norm_codes(y, gain, residual=x)

Rows are the last dimension; the others are tokens, in any number of
dimensions that can be seen as one, up to 2^31 - 1 of them. Calls run on the caller's current stream, on
the device of their tensors, and take the workspace that they need from torch's
allocator.

No call records a gradient. A tensor that wants one is refused, unless
gradients are off (torch.no_grad), and so is one with a tangent of forward mode;
norm_gradient and embed_gradient are the gradients.
"""

import ctypes
import functools
import struct
from ctypes import c_float, c_int32, c_int64, c_size_t, c_void_p

import torch
from torch.autograd import forward_ad as _forward

from . import sjd
from .kv import _current_device, _raw_stream
from .sjd import SJD_OK, SJDError

_DTYPES = {torch.float32: sjd.SJD_F32, torch.bfloat16: sjd.SJD_BF16}
_ROWS = struct.Struct("Qq")         # sjd_rows
_INF = float("inf")
_MOST = 2 ** 31 - 1                 # rows, places and ids of a call

_empty_like = torch.empty_like

_lib = None


def load():
    global _lib
    if _lib is not None:
        return _lib
    L = sjd.load()
    P, I, F, S = c_void_p, c_int32, c_float, c_size_t
    for name, args, res in (
            ("sjd_quantise", [P, I, I, I, P, P, P], I),
            ("sjd_norm", [P, P, P, P, F, I, I, I, I, P, P, P, P, P], I),
            ("sjd_norm_gradient_workspace_size", [I, I, I], S),
            ("sjd_norm_gradient", [P, P, P, F, I, P, I, I, I, P, P, P, P, S, P], I),
            ("sjd_embed", [P, I, I, P, I, I, F, I, P, P], I),
            ("sjd_embed_gradient_workspace_size", [I, I], S),
            ("sjd_embed_gradient", [P, P, I, I, I, F, I, P, P, S, P], I),
            ("sjd_weight_size", [I, I], S),
            ("sjd_weight_pack", [P, c_int64, P, I, I, P, S, P], I),
            ("sjd_product_workspace_size", [I, I, I], S),
            ("sjd_product", [P, I, I, P, P, I, P, P, I, P, P, S, P], I),
            ("sjd_weight_sync", [P, P], I)):
        f = getattr(L, name)
        f.argtypes, f.restype = args, res
    _lib = L
    return L


def _no_gradient(x, name):
    if x.requires_grad and torch.is_grad_enabled():
        raise ValueError("%s wants a gradient, and no call here records one: detach it, or call under torch.no_grad()" % name)
    if _forward.unpack_dual(x).tangent is not None:
        raise ValueError("%s has a forward-mode tangent, and no call here takes it on: detach it" % name)


def _rows(x, name, dtypes, device=None):
    """x as [rows, features], its last dimension dense."""
    # (most often all is as it should be: calls are short, and what the host does for one counts)
    if x.dim() == 2 and x.dtype in dtypes and x.is_cuda and (device is None or x.device == device) and x.stride(1) == 1 and not x.requires_grad and _forward._current_level < 0:
        return x
    if x.dtype not in dtypes or not x.is_cuda or (device is not None and x.device != device) or x.dim() < 1:
        raise ValueError("%s must be a tensor of %s on %s" % (name, " or ".join(str(d) for d in dtypes), device or "a GPU"))
    if x.requires_grad or _forward._current_level >= 0:   # (no tensor has a tangent outside of forward mode)
        _no_gradient(x, name)
    if x.dim() != 2:
        try:
            x = x.view(-1, x.shape[-1]) if x.numel() else x.reshape(x.shape[:-1].numel(), x.shape[-1])
        except RuntimeError:
            raise ValueError("%s: its dimensions but the last cannot be seen as one" % name) from None
    if x.stride(1) != 1 and x.shape[1] > 1:
        raise ValueError("%s: its last dimension must be dense" % name)
    return x


def _same(x, name, like):
    """x as [rows, features] of the type, shape and device of the tensor `like`."""
    if x.shape != like.shape:
        raise ValueError("%s must have the shape %s" % (name, tuple(like.shape)))
    return _rows(x, name, (like.dtype,), like.device)


def _vector(x, name, n, device):
    if x.dtype != torch.float32 or x.dim() != 1 or x.shape[0] != n or x.device != device or not x.is_contiguous():
        raise ValueError("%s must be a contiguous float32 tensor of shape (%d,) on %s" % (name, n, device))
    if x.requires_grad or _forward._current_level >= 0:   # (no tensor has a tangent outside of forward mode)
        _no_gradient(x, name)
    return x.data_ptr()


def _pack(x):
    return _ROWS.pack(x.data_ptr(), x.stride(0)) if x is not None else None


def _like(x):
    """A new contiguous tensor of x's shape and type."""
    return _empty_like(x) if x.is_contiguous() else torch.empty(x.shape, dtype=x.dtype, device=x.device)


def _features(dim, most):
    if not 1 <= dim <= most:
        raise ValueError("rows have 1 to %d features" % most)


def _count(n, what):
    """(The library takes an int32: more would arrive as another number.)"""
    if n > _MOST:
        raise ValueError("a call has at most 2^31 - 1 %s" % what)


def _tokens(tokens, device):
    if tokens.dtype != torch.int32 or tokens.device != device or not tokens.is_contiguous():
        raise ValueError("tokens must be a contiguous int32 tensor on %s" % (device,))
    return tokens.data_ptr()


def _run(device, name, *args):
    """One call, its last argument the device's current stream, which is returned."""
    call, index = getattr(_lib or load(), name), device.index
    raw = _raw_stream(index)
    if _current_device() == index:
        rc = call(*args, raw)
    else:
        with torch.cuda.device(device):
            rc = call(*args, raw)
    if rc != SJD_OK:
        raise SJDError(rc, "%s failed" % name)
    return raw


@functools.lru_cache(4096)
def _size(index, name, *args):
    """A workspace's size, on the device that it is for (it depends on nothing else)."""
    with torch.cuda.device(index):
        return getattr(load(), name)(*args)


class Weight:
    """A weight [out, in] in 8-bit codes with a scale for each channel, laid
    out for `product`: a byte a code. weight: int8, its last dimension dense;
    scale: float32 [out]. Neither is needed afterwards."""

    def __init__(self, weight, scale):
        if weight.dim() != 2 or weight.dtype != torch.int8 or weight.device.type != "cuda" or (weight.stride(1) != 1 and weight.shape[1] > 1):
            raise ValueError("weight must be an int8 tensor [out, in] on a GPU, its last dimension dense")
        self.out, self.dim = weight.shape
        self.device = weight.device
        at = None if scale is None else _vector(scale, "scale", self.out, self.device)
        size = load().sjd_weight_size(self.out, self.dim) if max(self.out, self.dim) <= _MOST else 0
        if scale is None or size == 0:
            raise ValueError("a weight has 1 to 2^24 channels of 1 to 65536 features, and a scale for each channel")
        self._packed = torch.empty(size, dtype=torch.uint8, device=self.device)
        self._at = self._packed.data_ptr()
        self._streams = {_raw_stream(self.device.index)}   # that the allocator knows the codes to be used on
        _run(self.device, "sjd_weight_pack", weight.data_ptr(), weight.stride(0), at, self.out, self.dim, self._at, size)

    @classmethod
    def quantise(cls, weight):
        """The weight [out, in] (bf16 or f32, rows of up to 16384) in codes."""
        return cls(*quantise(weight))

    def _used_on(self, raw):
        """The codes' memory is not handed out again before a call on another
        stream than the one they were made on has read them."""
        self._streams.add(raw)
        self._packed.record_stream(torch.cuda.current_stream(self.device))

    def sync(self):
        """Returns the device-side status code of the products with this weight
        on the current stream (0 = OK; SJD_ERR_TIMEOUT or, from the
        bounds-checked build, SJD_ERR_BOUNDS: results are not valid) and clears it."""
        with torch.cuda.device(self.device):
            return int(load().sjd_weight_sync(self._at, _raw_stream(self.device.index)))


def product(codes, scale, weight, bias=None, residual=None, dtype=torch.bfloat16):
    """sjd_product: codes int8 [..., in] with scale float32 [...] of their rows,
    times the weight: [..., out] of dtype (bf16 or f32), plus bias float32 [out] and
    residual [..., out] of dtype."""
    if dtype not in _DTYPES:
        raise ValueError("dtype must be bf16 or f32")
    device, shape = weight.device, codes.shape
    x = _rows(codes, "codes", (torch.int8,), device)
    if x.shape[1] != weight.dim:
        raise ValueError("codes have %d features, the weight %d" % (x.shape[1], weight.dim))
    rows, out = x.shape[0], weight.out
    if rows > _MOST:
        _count(rows, "rows")
    if (scale.shape[0] != rows if scale.dim() == 1 == len(shape) - 1 else scale.shape != shape[:-1]):
        raise ValueError("scale must have the shape %s" % (tuple(shape[:-1]),))
    if scale.dim() != 1 and scale.is_contiguous():
        scale = scale.view(-1)
    at = _vector(scale, "scale", rows, device)
    b = None if bias is None else _vector(bias, "bias", out, device)
    y = torch.empty((rows, out) if len(shape) == 2 else (*shape[:-1], out), dtype=dtype, device=device)
    r = None
    if residual is not None:
        r = _same(residual, "residual", y)
    if rows == 0:
        return y
    size = _size(device.index, "sjd_product_workspace_size", rows, out, weight.dim)
    workspace = torch.empty(size, dtype=torch.uint8, device=device) if size else None
    raw = _run(device, "sjd_product", weight._at, out, weight.dim, _pack(x), at, rows, b, _pack(r), _DTYPES[dtype],
         _ROWS.pack(y.data_ptr(), out), workspace.data_ptr() if size else None, size)
    if raw not in weight._streams:
        weight._used_on(raw)
    return y


def quantise(x):
    """sjd_quantise: (codes int8 of x's shape, scale float32 of its rows)."""
    rows = _rows(x, "x", _DTYPES)
    n, dim = rows.shape
    device = x.device
    if not 1 <= dim <= 16384:
        _features(dim, 16384)
    if n > _MOST:
        _count(n, "rows")
    codes = torch.empty(x.shape, dtype=torch.int8, device=device)
    scale = torch.empty(x.shape[:-1], dtype=torch.float32, device=device)
    if n:
        _run(device, "sjd_quantise", _ROWS.pack(rows.data_ptr(), rows.stride(0)), n, dim, _DTYPES[x.dtype], codes.data_ptr(), scale.data_ptr())
    return codes, scale


def _norm(x, gain, bias, residual, eps, centre, coded):
    rows = _rows(x, "x", _DTYPES)
    n, dim = rows.shape
    device, dtype = x.device, x.dtype
    if not 1 <= dim <= 16384:
        _features(dim, 16384)
    if n > _MOST:
        _count(n, "rows")
    if not 0.0 <= eps < _INF:
        raise ValueError("eps must be finite and not negative")
    g = None if gain is None else _vector(gain, "gain", dim, device)
    b = None if bias is None else _vector(bias, "bias", dim, device)
    r = h = hw = yw = c_at = s_at = None
    if residual is not None:
        r = _pack(_same(residual, "residual", x))
        h = _like(x)
        hw = _ROWS.pack(h.data_ptr(), dim)
    if coded:
        codes = torch.empty(x.shape, dtype=torch.int8, device=device)
        scale = torch.empty((n,) if x.dim() == 2 else x.shape[:-1], dtype=torch.float32, device=device)
        c_at, s_at = codes.data_ptr(), scale.data_ptr()
    else:
        y = _like(x)
        yw = _ROWS.pack(y.data_ptr(), dim)
    if n:
        _run(device, "sjd_norm", _ROWS.pack(rows.data_ptr(), rows.stride(0)), r, g, b, eps, 1 if centre else 0, n, dim, _DTYPES[dtype], hw, yw, c_at, s_at)
    if coded:
        return (codes, scale) if h is None else (codes, scale, h)
    return y if h is None else (y, h)


def norm(x, gain=None, bias=None, residual=None, eps=1e-6, centre=False):
    """sjd_norm: the norm of h = x + residual over the last dimension, bf16 or
    f32, by the root of the mean square or, with `centre`, around the mean (layer
    norm). gain and bias: float32 [dim]. Returns y, or (y, h) with a residual."""
    return _norm(x, gain, bias, residual, eps, centre, False)


def norm_codes(x, gain=None, bias=None, residual=None, eps=1e-6, centre=False):
    """The same norm as codes for `product`: (codes, scale), or (codes, scale,
    h) with a residual."""
    return _norm(x, gain, bias, residual, eps, centre, True)


def norm_gradient(dy, x, gain=None, eps=1e-6, centre=False, dh=None, bias=False):
    """sjd_norm_gradient: (dx, dgain, dbias) of norm at x (with a residual: at
    h), dx of x's type, dgain and dbias float32 (dbias None without `bias`). dh:
    the gradient that reaches h otherwise."""
    rows = _rows(x, "x", _DTYPES)
    n, dim = rows.shape
    device, dtype = x.device, x.dtype
    if not 1 <= dim <= 16384:
        _features(dim, 16384)
    if n > _MOST:
        _count(n, "rows")
    if not 0.0 <= eps < float("inf"):
        raise ValueError("eps must be finite and not negative")
    d = _same(dy, "dy", x)
    r = _same(dh, "dh", x) if dh is not None else None
    g = None if gain is None else _vector(gain, "gain", dim, device)
    dx = _like(x)
    made = torch.empty if n else torch.zeros
    dgain = made(dim, dtype=torch.float32, device=device)
    dbias = made(dim, dtype=torch.float32, device=device) if bias else None
    if n:
        size = _size(device.index, "sjd_norm_gradient_workspace_size", n, dim, _DTYPES[dtype])
        workspace = torch.empty(size, dtype=torch.uint8, device=device)
        _run(device, "sjd_norm_gradient", _pack(d), _pack(rows), g, eps, 1 if centre else 0, _pack(r), n, dim, _DTYPES[dtype],
             _ROWS.pack(dx.data_ptr(), dim), dgain.data_ptr(), dbias.data_ptr() if bias else None, workspace.data_ptr(), size)
    return dx, dgain, dbias


def embed(table, tokens, scale=1.0, dtype=None):
    """sjd_embed: scale * table[tokens] of dtype (the table's), zeros where a
    token is outside the table. table [vocab, dim] bf16 or f32, tokens int32 of
    any shape."""
    if table.dim() != 2:
        raise ValueError("table must be [vocab, dim]")
    dtype = table.dtype if dtype is None else dtype
    if dtype not in _DTYPES:
        raise ValueError("dtype must be bf16 or f32")
    t = _rows(table, "table", _DTYPES)
    vocab, dim = t.shape
    if not 1 <= dim <= 65536:
        _features(dim, 65536)
    if vocab < 1:
        raise ValueError("the table has no rows")
    n, device = tokens.numel(), table.device
    if vocab > _MOST or n > _MOST:
        _count(max(vocab, n), "tokens and ids")
    at = _tokens(tokens, device)
    y = torch.empty((*tokens.shape, dim), dtype=dtype, device=device)
    if n:
        _run(device, "sjd_embed", _pack(t), vocab, _DTYPES[table.dtype], at, n, dim, scale, _DTYPES[dtype], _ROWS.pack(y.data_ptr(), dim))
    return y


def embed_gradient(dy, tokens, vocab, scale=1.0):
    """sjd_embed_gradient: the gradient [vocab, dim], float32, of embed's table,
    from dy [..., dim] and the tokens [...]."""
    rows = _rows(dy, "dy", _DTYPES)
    n, dim = rows.shape
    if not 1 <= dim <= 65536:
        _features(dim, 65536)
    if vocab < 1:
        raise ValueError("the table has no rows")
    if vocab > _MOST or n > _MOST:
        _count(max(vocab, n), "rows and ids")
    if tokens.shape != dy.shape[:-1]:
        raise ValueError("tokens must have the shape %s" % (tuple(dy.shape[:-1]),))
    at = _tokens(tokens, dy.device)
    if n == 0:
        return torch.zeros(vocab, dim, dtype=torch.float32, device=dy.device)
    grad = torch.empty(vocab, dim, dtype=torch.float32, device=dy.device)
    size = load().sjd_embed_gradient_workspace_size(n, vocab)
    workspace = torch.empty(size, dtype=torch.uint8, device=dy.device)
    _run(dy.device, "sjd_embed_gradient", _pack(rows), at, n, dim, vocab, scale, _DTYPES[dy.dtype], grad.data_ptr(), workspace.data_ptr(), size)
    return grad
