"""The whole attention half of a layer on scales that are refused, in a process of its own: an answer that never comes fails the test and nothing else."""
import subprocess
import sys

import pytest

CALLS = """
import ctypes, sys
sys.path[:0] = ["tests", "."]
import paper_2408_11743_b200 as marlin
from test_attention_host import cache
from test_attention_more_host import append, attend, block, scales
for format in (1, 2):
    c = cache(marlin, format=format)
    for bad in (dict(block_size=2 ** 31 - 1), dict(block_size=2 ** 30 + 1), dict(block_size=-2 ** 31), dict(k=None, block_size=2 ** 31 - 1)):
        # (refused behind the checks of the cache; what it leaves on the stack is an 8-bit cache)
        assert block(marlin, c, scales(marlin), window=-1) == 2
        for call in (block, append, attend):
            assert call(marlin, c, scales(marlin, **bad)) == (1 if "k" in bad else 2), (call, bad)
print("answered")
"""


def test_scales_with_blocks_that_no_shift_reaches_are_refused():
    from paper_2408_11743_b200 import build
    build.build()
    from test_attention_host import NULL, SHAPE
    assert (NULL, SHAPE) == (1, 2)
    try:
        done = subprocess.run([sys.executable, "-c", CALLS], cwd=str(build._ROOT), capture_output=True, text=True, timeout=180)
    except subprocess.TimeoutExpired:
        pytest.fail("a call with a block size that is refused did not return")
    assert done.returncode == 0 and "answered" in done.stdout, done.stderr
