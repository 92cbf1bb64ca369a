"""The window forward's operators on the bounds-checked build
(libsjd_checked.so): their tests pass on it, so that no index they take from
tables, spans and lengths lies outside its array (one that did would latch
SJD_ERR_BOUNDS, which the tests' syncs turn into a failure); and an index that
is outside is clamped and reported. Run in child processes, so that the
checked library is the one that is loaded."""

import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

HERE = os.path.dirname(os.path.abspath(__file__))
ENV = dict(os.environ, SJD_LIBRARY="checked", PYTHONPATH=os.pathsep.join([os.path.dirname(HERE), HERE]))

CASES = " or ".join(["test_attend", "test_write_and_read", "test_write_turns_keys_and_queries", "test_rotate", "test_offsets_past_32_bits",
                     "test_device_errors_are_latched_and_cleared", "test_calls_back_to_back_wait_for_each_other"])

AXIS = """
import torch
from paper_2603_18599_gb300 import kv, sjd
assert sjd.lib_path().endswith("libsjd_checked.so")
h = kv.KV(1, 4, 2, 64, 8, 16, 8, 8, torch.bfloat16)
layer = h.new_layer()
x = torch.randn(1, 8, 2, 64, device="cuda")
table = torch.arange(8, dtype=torch.int32, device="cuda")[None]
start = torch.zeros(1, dtype=torch.int32, device="cuda")
positions = torch.arange(16, dtype=torch.int32, device="cuda").view(1, 8, 2)
rope = kv.Rope.sections((16, 16))
h.write(layer, x, x, table, start, rope=rope, positions=positions)
assert h.sync() == sjd.SJD_OK
want = layer.k.clone()
rope._axis[16:] = 1000000000          # the second axis: clamped to it
h.write(layer, x, x, table, start, rope=rope, positions=positions)
assert h.sync() == sjd.SJD_ERR_BOUNDS and h.last_error()
assert torch.equal(layer.k, want)
assert h.sync() == sjd.SJD_OK
rope._axis[:16] = -5
assert torch.equal(rope.rotate(x, positions), kv.Rope.sections((16, 16)).rotate(x, positions))
print("clamped and reported")
"""


def test_operators_on_the_bounds_checked_build():
    r = subprocess.run([sys.executable, "-m", "pytest", os.path.join(HERE, "test_gpu_kv.py"), "-m", "gpu", "-k", CASES, "-x", "-q",
                        "-p", "no:cacheprovider"], env=ENV, capture_output=True, text=True, timeout=1800)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-2000:]
    assert " passed" in r.stdout


def test_an_axis_out_of_range_is_clamped_and_reported():
    r = subprocess.run([sys.executable, "-c", AXIS], env=ENV, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0 and "clamped and reported" in r.stdout, r.stdout[-2000:] + r.stderr[-3000:]
