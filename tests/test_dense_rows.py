"""The features of a row that each thread of the row's group takes, compiled
for the host: every feature is taken by one thread, once."""

import os
import subprocess

from paper_2603_18599_gb300 import _build

HERE = os.path.dirname(os.path.abspath(__file__))


def groups(d):
    """(threads, pieces, wide) as the kernels take rows of d features; pieces 0: the embedding's loop."""
    wides = (0, 1) if d % 8 == 0 else (0,)
    for wide in wides:
        for pieces in (1, 2, 4):
            lanes = 8 if wide else 32
            while 8 * pieces * lanes < d:
                lanes *= 2
            yield lanes if lanes <= 32 else -(-d // (256 * pieces)) * 32, pieces, wide
        lanes = 8 if wide else 32
        while 32 * lanes < d:
            lanes *= 2
        yield lanes if d <= 1024 else 128, 0, wide


def test_every_feature_is_taken_once(tmp_path):
    exe = str(tmp_path / "rows")
    subprocess.run([_build.nvcc(), *_build._flags(), "-o", exe, os.path.join(HERE, "dense_rows.cu")], check=True)
    dims = [1, 7, 8, 31, 33, 64, 100, 255, 256, 257, 512, 513, 1000, 1023, 1024, 1025, 1030, 1600, 2048, 2049, 4095, 4096, 4097, 5120, 8191, 8192, 8200,
            12289, 16383, 16384, 40001, 65535, 65536]
    cases = [(d, *group) for d in dims for group in groups(d)]
    out = subprocess.run([exe], input="".join("%d %d %d %d\n" % c for c in cases), capture_output=True, text=True, check=True).stdout
    got = [tuple(int(x) for x in line.split()) for line in out.splitlines()]
    assert len(got) == len(cases)
    wrong = [(c, n) for c, n in zip(cases, got) if n != (1, 1, 0)]
    assert not wrong, wrong


def test_every_thread_has_the_first_of_two_pieces():
    """Behind a row's end a thread of the kernels for many rows (513 to 8192
    features, two pieces) looks at its first piece again: every thread has one."""
    for d in range(520, 8193, 8):
        threads = -(-(-(-d // 16)) // 32) * 32
        assert 8 * (threads - 1) < d, d
