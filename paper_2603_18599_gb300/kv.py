"""Python binding of the window forward's operators (the sjd_rope, sjd_rotate
and sjd_kv entry points of include/sjd.h): rotary positions with several
axes, a paged cache of keys and values that is quantised as it is written,
and attention of a chunk of new tokens over it. Argument marshalling only.

    rope = kv.Rope.sections((16, 24, 24))               # time, row, column
    cache = kv.KV(batch=2, heads=32, kv_heads=8, head_dim=128, n_pages=256, page_size=64,
                  max_pages=64, max_new=16, dtype=torch.float8_e4m3fn)
    layer = cache.new_layer()
    q = cache.write(layer, k, v, table, start, rope=rope, positions=positions, q=q)
    o = cache.attend(layer, q, table, start)

Calls run on the handle's stream. Where that is not the caller's current
stream, a call first waits for the current one, and the current one for the
call, so that tensors may be made and used on either. A capture cannot wait
for a stream outside it: calls that are captured into a graph need a handle made with
the capture's stream (KV(..., stream=side), torch.cuda.graph(..., stream=side)).

No call records a gradient. A tensor that wants one is refused, unless
gradients are off (torch.no_grad); a rotation's gradient is the rotation with
inverse=True.
"""

import ctypes
import math
import struct
from ctypes import POINTER, byref, c_double, c_float, c_int32, c_int64, c_size_t, c_uint64, c_void_p

import torch

from . import sjd
from .sjd import SJD_OK, SJDError

_DTYPES = {torch.float32: sjd.SJD_F32, torch.bfloat16: sjd.SJD_BF16}
_KV_DTYPES = {torch.bfloat16: sjd.SJD_BF16, torch.float8_e4m3fn: sjd.SJD_E4M3, torch.int8: sjd.SJD_S8}
MASK_CAUSAL, MASK_ALL, MASK_GIVEN = 0, 1, 2


class _config(ctypes.Structure):
    _fields_ = [(n, c_int32) for n in ("batch", "heads", "kv_heads", "head_dim", "page_size", "n_pages", "max_pages",
                                       "max_new", "kv_dtype")]


# The other structures of include/sjd.h, packed for each call (a window's
# calls are short: what the host does for one counts)
_LAYER = struct.Struct("4Q")        # sjd_kv_layer
_VIEW = struct.Struct("Q3q")        # sjd_view
_SPAN = struct.Struct("3Qi4x")      # sjd_kv_span
_ROPE = struct.Struct("2Q3i4x")     # sjd_rope


_lib = None


def load():
    global _lib
    if _lib is not None:
        return _lib
    L = sjd.load()
    P, I = c_void_p, c_int32
    for name, args, res in (
            ("sjd_rope_turns", [POINTER(c_double), I, POINTER(c_uint64)], I),
            ("sjd_rotate", [P, P, P, P, I, I, I, I, I, I, P], I),
            ("sjd_kv_workspace_size", [P], c_size_t),
            ("sjd_kv_init", [P, P, c_size_t, P, POINTER(P)], I),
            ("sjd_kv_write", [P, P, P, I, P, P, P, P, P, P], I),
            ("sjd_kv_read", [P, P, P, I, P, P], I),
            ("sjd_kv_attend", [P, P, P, P, I, P, c_int64, c_int64, c_float, P, P], I),
            ("sjd_kv_sync", [P], I),
            ("sjd_kv_last_error", [P], ctypes.c_char_p),
            ("sjd_kv_destroy", [P], None)):
        f = getattr(L, name)
        f.argtypes, f.restype = args, res
    _lib = L
    return L


# (as torch.cuda.current_stream and current_device, without making an object)
_raw_stream = torch._C._cuda_getCurrentRawStream
_current_device = torch._C._cuda_getDevice


def _device(device):
    device = torch.device(device)
    if device.type == "cuda" and device.index is None:
        device = torch.device("cuda", torch.cuda.current_device())
    return device


def _view_of(x, name, shape, dtype, device):
    if x.shape != shape or x.dtype != dtype or x.device != device or x.stride(3) != 1:
        raise ValueError("%s must be a %s tensor of shape %s on %s, its last dimension dense" % (name, dtype, tuple(shape), device))
    if x.requires_grad and torch.is_grad_enabled():
        raise ValueError("%s wants a gradient, and no call here records one: detach it, or call under torch.no_grad()" % name)
    s = x.stride()
    return _VIEW.pack(x.data_ptr(), s[0], s[1], s[2])


def _array(x, name, shape, device, dtype=torch.int32):
    if x.shape != shape or x.dtype != dtype or x.device != device or not x.is_contiguous():
        raise ValueError("%s must be a contiguous %s tensor of shape %s on %s" % (name, dtype, tuple(shape), device))
    return x.data_ptr()


class Rope:
    """Rotary positions with several axes: pair i turns by positions[axis[i]]
    * freq[i] (radians). Pairs are elements (i, i + pairs), or (2i, 2i + 1)
    where interleaved; the elements after the pairs are kept."""

    def __init__(self, freq, axis, interleaved=False, device="cuda"):
        freq, axis = [float(f) for f in freq], [int(a) for a in axis]
        if len(freq) != len(axis) or not freq or len(freq) % 4:
            raise ValueError("freq and axis need a multiple of 4 entries each")
        if min(axis) < 0 or max(axis) > 7:
            raise ValueError("axes are numbered 0 to 7")
        self.pairs, self.axes, self.interleaved = len(freq), max(axis) + 1, bool(interleaved)
        turns = (c_uint64 * self.pairs)()
        if load().sjd_rope_turns((c_double * self.pairs)(*freq), self.pairs, turns) != SJD_OK:
            raise SJDError(sjd.SJD_ERR_ARG, "frequencies must be finite")
        self.device = _device(device)
        self._turns = torch.tensor([t - 2 ** 64 if t >= 2 ** 63 else t for t in turns], dtype=torch.int64, device=self.device)
        self._axis = torch.tensor(axis, dtype=torch.int32, device=self.device)
        self._c = _ROPE.pack(self._turns.data_ptr(), self._axis.data_ptr(), self.pairs, self.axes, self.interleaved)
        self._streams = {_raw_stream(self.device.index)}   # that the allocator knows the tables to be used on

    @classmethod
    def sections(cls, pairs, theta=10000.0, shared=False, interleaved=False, device="cuda"):
        """pairs[a] pairs for axis a. Each axis has its own frequencies
        theta^(-i / pairs[a]), or with `shared` its section of one spectrum
        theta^(-i / sum(pairs))."""
        axis = [a for a, m in enumerate(pairs) for _ in range(m)]
        if shared:
            freq = [theta ** (-i / len(axis)) for i in range(len(axis))]
        else:
            freq = [theta ** (-i / m) for m in pairs for i in range(m)]
        return cls(freq, axis, interleaved, device)

    def _used_on(self, raw, stream):
        """The tables' memory is not handed out again before a call on another
        stream than the one they were made on has read them."""
        if raw not in self._streams:
            self._streams.add(raw)
            self._turns.record_stream(stream())
            self._axis.record_stream(stream())

    def rotate(self, x, positions, inverse=False, out=None):
        """x [B, n, H, D] (bf16 or f32) turned by positions [B, n, axes]
        int32; with `inverse` by the transpose, which takes the gradient of
        the result to that of x. `out` may be x."""
        dev, dtype = self.device, x.dtype
        if x.dim() != 4 or dtype not in _DTYPES or x.device != dev:
            raise ValueError("x must be a [B, n, H, D] bf16 or f32 tensor on %s" % (dev,))
        shape = B, n, H, D = x.shape
        at = _array(positions, "positions", (B, n, self.axes), dev)
        xw = _view_of(x, "x", shape, dtype, dev)
        if out is None:
            out = torch.empty(shape, dtype=dtype, device=dev)
            ow = _VIEW.pack(out.data_ptr(), n * H * D, H * D, D)
        else:
            ow = _view_of(out, "out", shape, dtype, dev)
        if x.numel() == 0:
            return out
        raw = _raw_stream(dev.index)
        args = (self._c, xw, ow, at, B, n, H, D, _DTYPES[dtype], 1 if inverse else 0, raw)
        if _current_device() == self.device.index:
            rc = load().sjd_rotate(*args)
        else:
            with torch.cuda.device(self.device):
                rc = load().sjd_rotate(*args)
        if rc != SJD_OK:
            raise SJDError(rc, "sjd_rotate failed (dim a multiple of 8 up to 256, 2 * pairs at most dim)")
        self._used_on(raw, lambda: torch.cuda.current_stream(dev))
        return out


class Layer:
    """One layer's cache: k, v [n_pages, kv_heads, page_size, head_dim] and,
    of an 8-bit cache, k_scale, v_scale [n_pages, kv_heads, page_size] f32."""

    __slots__ = ("_t", "_for")

    def __init__(self, k, v, k_scale=None, v_scale=None):
        self._t, self._for = (k, v, k_scale, v_scale), None

    k = property(lambda self: self._t[0])
    v = property(lambda self: self._t[1])
    k_scale = property(lambda self: self._t[2])
    v_scale = property(lambda self: self._t[3])


class KV:
    """One handle: the sizes of a cache, the workspace and the stream that
    the calls of all layers share. dtype: torch.bfloat16, torch.float8_e4m3fn
    or torch.int8."""

    def __init__(self, batch, heads, kv_heads, head_dim, n_pages, page_size, max_pages, max_new, dtype=torch.bfloat16,
                 device="cuda", stream=None):
        self.L = load()
        self.ctx = c_void_p()
        if dtype not in _KV_DTYPES:
            raise ValueError("a cache holds bfloat16, float8_e4m3fn or int8")
        self.cfg = _config(batch, heads, kv_heads, head_dim, page_size, n_pages, max_pages, max_new, _KV_DTYPES[dtype])
        self.dtype = dtype
        size = int(self.L.sjd_kv_workspace_size(byref(self.cfg)))
        if size == 0:
            raise SJDError(sjd.SJD_ERR_ARG, "invalid configuration")
        self.device = _device(device)
        self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        self._raw = self.stream.cuda_stream
        with torch.cuda.device(self.device), torch.cuda.stream(self.stream):
            self.workspace = torch.empty(size, dtype=torch.uint8, device=self.device)
            rc = self.L.sjd_kv_init(byref(self.cfg), self.workspace.data_ptr(), size, self.stream.cuda_stream, byref(self.ctx))
        if rc != SJD_OK:
            self.ctx = c_void_p()
            raise SJDError(rc, "sjd_kv_init failed")
        c = self.cfg
        self._shapes = ((c.n_pages, c.kv_heads, c.page_size, c.head_dim), (c.n_pages, c.kv_heads, c.page_size),
                        (c.batch, c.max_pages), (c.batch,))
        self._scale = 1.0 / math.sqrt(c.head_dim)

    # -- helpers ------------------------------------------------------------
    def _layer_of(self, layer):
        k, v, ks, vs = layer._t
        if layer._for is not self:   # (a handle's sizes and a layer's tensors do not change)
            pages, scales = self._shapes[:2]
            _array(k, "k", pages, self.device, self.dtype)
            _array(v, "v", pages, self.device, self.dtype)
            if self.dtype != torch.bfloat16:
                if ks is None or vs is None:
                    raise ValueError("an 8-bit cache needs k_scale and v_scale")
                _array(ks, "k_scale", scales, self.device, torch.float32)
                _array(vs, "v_scale", scales, self.device, torch.float32)
            layer._for = self
        if self.dtype == torch.bfloat16:
            return _LAYER.pack(k.data_ptr(), v.data_ptr(), 0, 0)
        return _LAYER.pack(k.data_ptr(), v.data_ptr(), ks.data_ptr(), vs.data_ptr())

    def _span(self, table, start, count, n):
        return _SPAN.pack(_array(table, "table", self._shapes[2], self.device), _array(start, "start", self._shapes[3], self.device),
                          0 if count is None else _array(count, "count", self._shapes[3], self.device), n)

    def _run(self, call, args, tensors):
        """call(*args) with the handle's device current, ordered with the
        current stream where that is another one. `tensors`: what it uses."""
        index = self.device.index
        if _raw_stream(index) == self._raw and _current_device() == index:
            rc = call(*args)
        else:
            with torch.cuda.device(self.device):
                here = torch.cuda.current_stream(self.device)
                self.stream.wait_stream(here)
                rc = call(*args)
                here.wait_stream(self.stream)
                for t in tensors:
                    if t is not None:
                        t.record_stream(self.stream)
        if rc != SJD_OK:
            raise SJDError(rc, self.L.sjd_kv_last_error(self.ctx).decode())

    # -- entry points ---------------------------------------------------------
    def new_layer(self):
        """A layer's cache, all zeros."""
        pages, scales = self._shapes[:2]

        def zeros(shape, dtype):
            return torch.zeros(shape, dtype=dtype, device=self.device)

        def held():
            return zeros(pages, torch.uint8 if self.dtype == torch.float8_e4m3fn else self.dtype).view(self.dtype)

        if self.dtype == torch.bfloat16:
            return Layer(held(), held())
        return Layer(held(), held(), zeros(scales, torch.float32), zeros(scales, torch.float32))

    def write(self, layer, k, v, table, start, count=None, rope=None, positions=None, q=None, q_out=None):
        """sjd_kv_write: k, v [B, n, kv_heads, D] (bf16 or f32) become tokens
        start[b] .. start[b] + count[b] - 1 (count None: n) of the sequences
        whose pages are table [B, max_pages]. With rope and positions [B, n,
        axes] the keys are turned first, and q [B, n, heads, D], if given, is
        turned into the result (q_out, or a new tensor), whose rows from
        count[b] on are not written."""
        c = self.cfg
        if k.dim() != 4 or k.dtype not in _DTYPES:
            raise ValueError("k must be a [B, n, kv_heads, D] bf16 or f32 tensor")
        B, n, dt = c.batch, k.shape[1], k.dtype
        shape = (B, n, c.kv_heads, c.head_dim)
        kw, vw = _view_of(k, "k", shape, dt, self.device), _view_of(v, "v", shape, dt, self.device)
        at, span = self._layer_of(layer), self._span(table, start, count, n)
        rope_c = pos = qw = ow = None
        if q is None and q_out is not None:
            raise ValueError("q_out goes with q")
        if rope is not None:
            if rope.device != self.device:
                raise ValueError("rope is on %s, the cache on %s" % (rope.device, self.device))
            if positions is None:
                raise ValueError("rope goes with positions")
            rope_c, pos = rope._c, _array(positions, "positions", (B, n, rope.axes), self.device)
        if q is not None:
            shape = (B, n, c.heads, c.head_dim)
            qw = _view_of(q, "q", shape, dt, self.device)
            if q_out is None:
                q_out = torch.empty(shape, dtype=dt, device=self.device)
                ow = _VIEW.pack(q_out.data_ptr(), n * c.heads * c.head_dim, c.heads * c.head_dim, c.head_dim)
            else:
                ow = _view_of(q_out, "q_out", shape, dt, self.device)
        self._run(self.L.sjd_kv_write, (self.ctx, at, span, _DTYPES[dt], kw, vw, rope_c, pos, qw, ow),
                  (*layer._t, k, v, table, start, count, positions, q, q_out))
        if rope is not None:
            rope._used_on(self._raw, lambda: self.stream)
        return q_out

    def read(self, layer, table, start, n, count=None, dtype=torch.bfloat16):
        """sjd_kv_read: (k, v) [B, n, kv_heads, D] of the spans, zeros from
        count[b] on."""
        c = self.cfg
        if dtype not in _DTYPES:
            raise ValueError("dtype must be bf16 or f32")
        at, span = self._layer_of(layer), self._span(table, start, count, n)
        shape = (c.batch, n, c.kv_heads, c.head_dim)
        k = torch.empty(shape, dtype=dtype, device=self.device)
        v = torch.empty(shape, dtype=dtype, device=self.device)
        self._run(self.L.sjd_kv_read, (self.ctx, at, span, _DTYPES[dtype], k.data_ptr(), v.data_ptr()),
                  (*layer._t, table, start, count, k, v))
        return k, v

    def attend(self, layer, q, table, start, count=None, mask="causal", scale=None, lse=False, out=None):
        """sjd_kv_attend: q [B, n, heads, D] bf16, the chunk's keys and
        values in the cache already. mask: "causal", None (the whole chunk is
        seen) or a bool or uint8 tensor [B or 1, n, n] of what each chunk
        token sees of the chunk. Returns o [B, n, heads, D], or (o, lse
        [B, n, heads] f32)."""
        c = self.cfg
        if q.dim() != 4:
            raise ValueError("q must be a [B, n, heads, D] bf16 tensor")
        B, n = c.batch, q.shape[1]
        qw = _view_of(q, "q", (B, n, c.heads, c.head_dim), torch.bfloat16, self.device)
        at, span = self._layer_of(layer), self._span(table, start, count, n)
        kind, mask_at, mb, mr, given = MASK_CAUSAL, None, 0, 0, None
        if mask is None:
            kind = MASK_ALL
        elif isinstance(mask, torch.Tensor):
            kind, given = MASK_GIVEN, mask
            if mask.dtype not in (torch.bool, torch.uint8) or mask.device != self.device or mask.dim() != 3 or \
                    mask.shape[0] not in (1, B) or mask.shape[1:] != (n, n) or (mask.stride(2) != 1 and n > 1):
                raise ValueError("mask must be a bool or uint8 tensor [%d or 1, %d, %d] on %s, its rows dense" % (B, n, n, self.device))
            mask_at, mb, mr = mask.data_ptr(), mask.stride(0) if mask.shape[0] == B else 0, mask.stride(1)
        elif mask != "causal":
            raise ValueError("mask must be \"causal\", None or a tensor")
        shape = (B, n, c.heads, c.head_dim)
        if out is None:
            out = torch.empty(shape, dtype=torch.bfloat16, device=self.device)
            o_at = out.data_ptr()
        else:
            o_at = _array(out, "out", shape, self.device, torch.bfloat16)
        sums = torch.empty((B, n, c.heads), dtype=torch.float32, device=self.device) if lse else None
        scale = self._scale if scale is None else float(scale)
        self._run(self.L.sjd_kv_attend, (self.ctx, at, span, qw, kind, mask_at, mb, mr, scale, o_at, sums.data_ptr() if lse else None),
                  (*layer._t, q, table, start, count, given, out, sums))
        return (out, sums) if lse else out

    def sync(self):
        """Returns the device-side status code (0 = OK) and clears it."""
        return int(self.L.sjd_kv_sync(self.ctx))

    def last_error(self):
        return self.L.sjd_kv_last_error(self.ctx).decode()

    def close(self):
        if self.ctx:
            self.L.sjd_kv_destroy(self.ctx)
            self.ctx = c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
