"""The numbers that the attention's work is shared out by, compiled for the
host: the key tiles of a sequence, at small sizes and where 32 bits are not
enough for their sum."""

import os
import subprocess

from paper_2603_18599_gb300 import _build

HERE = os.path.dirname(os.path.abspath(__file__))


def tiles(rows, start, count, group, causal):
    """Of every item of `rows` rows, the tiles of 128 keys that some row of it sees."""
    total = 0
    for row0 in range(0, count * group, rows):
        last = min(row0 + rows, count * group) - 1
        total += -(-(start + (last // group + 1 if causal else count)) // 128)
    return total


def test_key_tiles_are_counted_in_64_bits(tmp_path):
    exe = str(tmp_path / "shares")
    subprocess.run([_build.nvcc(), *_build._flags(), "-o", exe, os.path.join(HERE, "attend_shares.cu")], check=True)
    cases = [(rows, start, count, group, causal) for rows in (128, 256) for causal in (0, 1)
             for start, count, group in ((0, 0, 3), (0, 1, 1), (127, 1, 8), (128, 1, 128), (1000, 33, 7), (0, 300, 4), (5, 129, 128),
                                         (2 ** 30 - 4096, 4096, 8),         # a long prefix
                                         (2 ** 30 - 2000000, 1 << 20, 4),
                                         (0, 1 << 20, 128),                 # a million tokens of 128 heads to a key head
                                         (12345, 5900000, 4))]
    out = subprocess.run([exe], input="".join("%d %d %d %d %d\n" % c for c in cases), capture_output=True, text=True, check=True).stdout
    got = [int(x) for x in out.split()]
    assert len(got) == len(cases)
    assert max(tiles(*c) for c in cases) > 2 ** 31
    for c, n in zip(cases, got):
        assert n == tiles(*c), c
