"""Host side of the window forward's operators (no GPU compute): argument
checks before the device is touched, and the frequencies as turns."""

import ctypes
import math
from fractions import Fraction

import pytest

from test_abi import libsjd  # noqa: F401  (builds the library if needed)


@pytest.fixture()
def lib(libsjd):  # noqa: F811
    from paper_2603_18599_gb300 import kv
    return kv.load()


def config(**over):
    from paper_2603_18599_gb300 import kv
    d = dict(batch=2, heads=32, kv_heads=8, head_dim=128, page_size=64, n_pages=100, max_pages=50, max_new=16, kv_dtype=1)
    d.update(over)
    return kv._config(*[d[n] for n, _ in kv._config._fields_])


def test_struct_sizes_match_the_header(lib):
    from paper_2603_18599_gb300 import kv
    assert ctypes.sizeof(kv._config) == 36
    assert kv._VIEW.size == 32
    assert kv._SPAN.size == 32
    assert kv._ROPE.size == 32
    assert kv._LAYER.size == 32


def test_workspace_size_validates_configs(lib):
    size = lib.sjd_kv_workspace_size
    assert size(ctypes.byref(config())) > 0
    assert size(None) == 0
    for over in (dict(batch=0), dict(heads=0), dict(kv_heads=0), dict(kv_heads=5), dict(heads=8 * 129), dict(head_dim=0),
                 dict(head_dim=129), dict(head_dim=136), dict(page_size=0), dict(n_pages=0), dict(max_pages=0), dict(max_new=0),
                 dict(kv_dtype=0), dict(kv_dtype=4), dict(page_size=1 << 20, max_pages=(1 << 10) + 1), dict(batch=1 << 20, max_new=1 << 12),
                 dict(n_pages=1 << 20, page_size=512), dict(kv_heads=65537, heads=65537)):
        assert size(ctypes.byref(config(**over))) == 0, over


def test_null_and_bad_arguments_are_refused(lib):
    from paper_2603_18599_gb300 import sjd
    ctx = ctypes.c_void_p()
    good = config()
    n = lib.sjd_kv_workspace_size(ctypes.byref(good))
    assert lib.sjd_kv_init(ctypes.byref(good), None, n, None, ctypes.byref(ctx)) == sjd.SJD_ERR_ARG
    assert lib.sjd_kv_init(ctypes.byref(good), 8, n, None, ctypes.byref(ctx)) == sjd.SJD_ERR_ARG
    assert lib.sjd_kv_init(ctypes.byref(good), 256, n - 1, None, ctypes.byref(ctx)) == sjd.SJD_ERR_CAPACITY
    assert lib.sjd_kv_init(ctypes.byref(config(batch=0)), 256, n, None, ctypes.byref(ctx)) == sjd.SJD_ERR_ARG
    assert lib.sjd_kv_init(ctypes.byref(good), 256, n, None, None) == sjd.SJD_ERR_ARG
    assert lib.sjd_kv_sync(None) == sjd.SJD_ERR_ARG
    assert lib.sjd_kv_write(None, None, None, 0, None, None, None, None, None, None) == sjd.SJD_ERR_ARG
    assert lib.sjd_kv_read(None, None, None, 0, None, None) == sjd.SJD_ERR_ARG
    assert lib.sjd_kv_attend(None, None, None, None, 0, None, 0, 0, 1.0, None, None) == sjd.SJD_ERR_ARG
    assert lib.sjd_rotate(None, None, None, None, 1, 1, 1, 8, 0, 0, None) == sjd.SJD_ERR_ARG
    assert lib.sjd_kv_last_error(None) == b"no handle"
    lib.sjd_kv_destroy(None)


def test_frequencies_as_turns(lib):
    """turns = f / (2 pi) * 2^64 mod 2^64, to double precision."""
    freq = [1.0, 10000.0 ** -0.25, 1e-9, 0.0, -1.0, 100.0, 2 * math.pi * 0.75, 1e-30]
    turns = (ctypes.c_uint64 * len(freq))()
    assert lib.sjd_rope_turns((ctypes.c_double * len(freq))(*freq), len(freq), turns) == 0
    pi = Fraction(3141592653589793238462643383279502884197, 10 ** 39)
    for f, t in zip(freq, turns):
        want = Fraction(f) / (2 * pi)
        off = (Fraction(t, 2 ** 64) - want) % 1
        off = min(off, 1 - off)
        assert off <= abs(want) * Fraction(1, 2 ** 52) + Fraction(1, 2 ** 53), f
    assert turns[3] == 0
    for bad in (math.nan, math.inf, -math.inf, 1e17):
        assert lib.sjd_rope_turns((ctypes.c_double * 1)(bad), 1, turns) == 1
    assert lib.sjd_rope_turns(None, 1, turns) == 1
