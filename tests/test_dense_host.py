"""Host side of the dense operators (no GPU compute): sizes, and argument
checks before the device is touched."""

import ctypes

import pytest
import torch

from test_abi import libsjd  # noqa: F401  (builds the library if needed)


@pytest.fixture()
def lib(libsjd):  # noqa: F811
    from paper_2603_18599_gb300 import dense
    return dense.load()


def rows(data, stride=64):
    from paper_2603_18599_gb300 import dense
    return dense._ROWS.pack(data, stride)


def test_sizes(lib):
    from paper_2603_18599_gb300 import dense
    assert dense._ROWS.size == 16
    size = lib.sjd_weight_size
    # a byte a code, channels and features filled up, and 256 bytes and 8 a channel beside them
    assert size(1, 1) == 256 + 256 * 8 + 256 * 64
    assert size(4096, 4096) == 256 + 4096 * 8 + 4096 * 4096
    assert size(1 << 24, 65536) == 256 + (1 << 27) + (1 << 40)
    for out, dim in ((0, 1), (1, 0), (-1, 5), ((1 << 24) + 1, 1), (1, 65537)):
        assert size(out, dim) == 0, (out, dim)
    # where each id's places begin, the places, and a list of 256 ids and its length for every 256 ids
    assert lib.sjd_embed_gradient_workspace_size(3, 5) == 4 * (5 + 1 + 3) + 16 * 257
    assert lib.sjd_embed_gradient_workspace_size(2 ** 31 - 1, 2 ** 31 - 1) == 4 * (2 ** 32 - 1) + 16 * 2 ** 23 * 257
    assert lib.sjd_embed_gradient_workspace_size(0, 5) == lib.sjd_embed_gradient_workspace_size(5, 0) == 0
    assert lib.sjd_norm_gradient_workspace_size(0, 5, 0) == lib.sjd_norm_gradient_workspace_size(5, 16385, 0) == lib.sjd_norm_gradient_workspace_size(5, 5, 2) == 0
    assert lib.sjd_product_workspace_size(0, 5, 5) == lib.sjd_product_workspace_size(5, 5, 65537) == 0


def test_bad_arguments_are_refused(lib):
    """Addresses are made up: every call has to return before it uses one."""
    arg, at = 1, 1 << 20
    x = rows(at)
    inf, nan = float("inf"), float("nan")

    def refused(name, good, changes):
        call = getattr(lib, name)
        for i, values in changes.items():
            for v in values:
                args = list(good)
                args[i] = v
                assert call(*args) == arg, (name, i, v)

    sizes = (0, -1)
    refused("sjd_quantise", [x, 2, 64, 0, at, at, None],
            {0: (None, rows(0), rows(at + 2)), 1: sizes, 2: (*sizes, 16385), 3: (2, 3, -1), 4: (None,), 5: (None, at + 2)})
    norm = [x, None, at, at, 1e-6, 1, 2, 64, 1, None, x, None, None, None]
    refused("sjd_norm", norm, {0: (None, rows(0), rows(at + 1)), 1: (x, rows(0)), 2: (at + 2,), 3: (at + 1,), 4: (-1e-6, inf, nan),
                               5: (2, -1), 6: sizes, 7: (*sizes, 16385), 8: (2, 3, -1), 9: (x,), 10: (None, rows(0), rows(at + 1)),
                               11: (at,), 12: (at,)})
    codes = list(norm)
    codes[10], codes[11], codes[12] = None, at, at
    refused("sjd_norm", codes, {10: (x,), 11: (None,), 12: (None, at + 2)})
    refused("sjd_norm_gradient", [x, x, at, 1e-6, 1, x, 2, 64, 1, x, at, at, at, 1 << 30, None],
            {0: (None, rows(at + 1)), 1: (None, rows(0)), 2: (at + 2,), 3: (-1.0, nan), 4: (2,), 5: (rows(0), rows(at + 1)), 6: sizes,
             7: (*sizes, 16385), 8: (3,), 9: (None, rows(at + 1)), 10: (None, at + 2), 11: (at + 2,), 12: (None, at + 8)})
    refused("sjd_embed", [x, 10, 0, at, 2, 64, 1.0, 1, x, None],
            {0: (None, rows(at + 2)), 1: sizes, 2: (2,), 3: (None, at + 2), 4: sizes, 5: (*sizes, 65537), 7: (3,), 8: (None, rows(at + 1))})
    refused("sjd_embed_gradient", [x, at, 2, 64, 10, 1.0, 0, at, at, 1 << 30, None],
            {0: (None, rows(at + 2)), 1: (None, at + 2), 2: sizes, 3: (*sizes, 65537), 4: sizes, 6: (2,), 7: (None, at + 2), 8: (None, at + 8)})
    refused("sjd_weight_pack", [at, 64, at, 10, 64, at, 1 << 30, None],
            {0: (None,), 2: (None, at + 2), 3: (*sizes, (1 << 24) + 1), 4: (*sizes, 65537), 5: (None, at + 128)})
    assert lib.sjd_weight_pack(at, 64, at, 10, 64, at, lib.sjd_weight_size(10, 64) - 1, None) == 3
    assert lib.sjd_embed_gradient(x, at, 2, 64, 10, 1.0, 0, at, at, lib.sjd_embed_gradient_workspace_size(2, 10) - 1, None) == 3
    refused("sjd_product", [at, 10, 64, x, at, 2, at, x, 1, x, at, 1 << 30, None],
            {0: (None, at + 128), 1: (*sizes, (1 << 24) + 1), 2: (*sizes, 65537), 3: (None, rows(0)), 4: (None, at + 2), 5: sizes, 6: (at + 2,),
             7: (rows(0), rows(at + 1)), 8: (2,), 9: (None, rows(at + 1)), 10: (at + 128,)})
    assert lib.sjd_weight_sync(None, None) == lib.sjd_weight_sync(at + 8, None) == arg


def test_tensors_that_are_not_on_a_gpu_are_refused(lib):
    from paper_2603_18599_gb300 import dense
    x, tokens = torch.zeros(2, 8), torch.zeros(2, dtype=torch.int32)
    for call in (lambda: dense.quantise(x), lambda: dense.norm(x), lambda: dense.norm_codes(x), lambda: dense.norm_gradient(x, x),
                 lambda: dense.embed(x, tokens), lambda: dense.embed_gradient(x, tokens, 5),
                 lambda: dense.Weight(torch.zeros(4, 8, dtype=torch.int8), torch.zeros(4)), lambda: dense.Weight.quantise(x)):
        with pytest.raises(ValueError):
            call()
    assert ctypes.sizeof(ctypes.c_size_t) == 8
