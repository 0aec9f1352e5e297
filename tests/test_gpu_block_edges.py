"""GPU: 8-bit caches with a scale per block of tokens where an edge lies inside of a block."""
import pytest

from blocks_util import BlockCase
from test_gpu_attention_sinks import check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def marlin():
    import torch
    assert torch.cuda.is_available()
    import paper_2408_11743_b200 as m
    m.lib()
    return m


# one warp's rows, rows that warps share, tcgen05, heads of 256; one new token and several; prompts
ROWS = [(4, 128, 1), (4, 128, 3), (20, 64, 1), (48, 128, 1), (48, 128, 3), (12, 256, 2), (8, 128, 30), (16, 64, 20)]


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("page,block", [(4, 2), (4, 4), (8, 2), (8, 4), (8, 8), (16, 8)])
@pytest.mark.parametrize("q_heads,dim,new", ROWS)
def test_windows_that_begin_inside_of_a_block(marlin, kind, page, block, q_heads, dim, new):
    # every residue of the window's edge, with the end of the sinks at some; pages smaller than the sixteen keys that a warp copies
    case = BlockCase([300, 41, 20, 7], new, q_heads, 1, dim, page, kind, block, seed=page + block)
    for sinks in (0, 1, 5):
        for window in range(9, 18):
            check(marlin, case, window=window, sinks=sinks)
