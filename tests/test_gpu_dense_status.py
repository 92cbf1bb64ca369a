"""What a weight's status word tells (its values are written by the host here),
and the dense operators' ways on the bounds-checked build (libsjd_checked.so), where
every product's test asks for the status afterwards: an index outside its array
would show there. Run in a child process, so that the checked library is the one
that is loaded."""

import os
import subprocess
import sys

import pytest
import torch

from paper_2603_18599_gb300 import dense, sjd

pytestmark = pytest.mark.gpu

HERE = os.path.dirname(os.path.abspath(__file__))
ENV = dict(os.environ, SJD_LIBRARY="checked", PYTHONPATH=os.pathsep.join([os.path.dirname(HERE), HERE]))


def test_a_weights_status_tells_what_it_was_and_is_cleared():
    weight = dense.Weight(torch.ones(3, 5, dtype=torch.int8, device="cuda"), torch.ones(3, device="cuda"))
    status = weight._packed[:4].view(torch.int32)
    timeout, bounds = 1 << (sjd.SJD_ERR_TIMEOUT - 1), 1 << (sjd.SJD_ERR_BOUNDS - 1)
    for bits, code in ((0, sjd.SJD_OK), (timeout, sjd.SJD_ERR_TIMEOUT), (bounds, sjd.SJD_ERR_BOUNDS), (timeout | bounds, sjd.SJD_ERR_TIMEOUT)):
        status.fill_(bits)
        assert weight.sync() == code
        assert weight.sync() == sjd.SJD_OK


@pytest.mark.parametrize("file,cases", [("test_gpu_dense_ways.py", "test_ways_of_a_product or 1600"),
                                        ("test_gpu_dense.py", "test_product or test_embed or test_offsets_past_32_bits_in_a_product"),
                                        ("test_gpu_dense_calls.py", "right_before")])
def test_ways_on_the_bounds_checked_build(file, cases):
    r = subprocess.run([sys.executable, "-m", "pytest", os.path.join(HERE, file), "-m", "gpu", "-k", cases, "-x", "-q", "-p", "no:cacheprovider"],
                       env=ENV, capture_output=True, text=True, timeout=1800)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-2000:]
    assert " passed" in r.stdout
