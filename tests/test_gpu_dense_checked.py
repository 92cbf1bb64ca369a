"""The dense operators on the bounds-checked build (libsjd_checked.so): cases of
each give the same there. Run in a child process, so that the checked library is
the one that is loaded."""

import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

HERE = os.path.dirname(os.path.abspath(__file__))
ENV = dict(os.environ, SJD_LIBRARY="checked", PYTHONPATH=os.pathsep.join([os.path.dirname(HERE), HERE]))

CASES = " or ".join(["test_embed", "test_a_chain", "test_sums_beyond", "test_norm_gradient_against", "test_quantise_rows", "test_long_rows",
                     "test_product_of_many_dimensions"])


def test_operators_on_the_bounds_checked_build():
    r = subprocess.run([sys.executable, "-m", "pytest", os.path.join(HERE, "test_gpu_dense.py"), "-m", "gpu", "-k", CASES, "-x", "-q",
                        "-p", "no:cacheprovider"], env=ENV, capture_output=True, text=True, timeout=1800)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-2000:]
    assert " passed" in r.stdout
