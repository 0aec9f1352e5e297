"""GPU: 8-bit caches with a scale per block of tokens where an edge lies inside of a block, and what is not finite there."""
import pytest

from blocks_util import BlockCase
from test_gpu_attention_sinks import attend, check

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


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("q_heads,dim", [(4, 128), (20, 64), (48, 128), (3, 256)])
@pytest.mark.parametrize("new", [1, 3])
def test_a_scale_that_is_not_finite_under_a_weight_of_nothing(marlin, kind, q_heads, dim, new):
    # a key so far below the others that its weight is 0 in fp32, near the end of the sequence and at the edge of the window: its value's scale
    # reaches the rows that see it, and no others
    import torch
    case = BlockCase([200], new, q_heads, 1, dim, 16, kind, 1, seed=dim)
    case.q[:] = 4
    window = 50
    for odd in (199, 200 - new, 200 - window, 200 - window - new + 1, 170):
        k = case.k_t.clone()
        k.view(torch.uint8)[:] = 0
        d = case.dev(marlin)
        page, slot = int(case.table[0, odd // 16]), odd % 16
        k[page, :, slot] = -100
        d["k_cache"].view(torch.uint8).copy_(k.view(torch.uint8))
        d["k_scale"].fill_(0.03)
        d["v_scale"][page, :, slot] = float("nan")
        got, _ = attend(marlin, case, d, window=window, sinks=2, scale=1.0)  # (a logit of -12 dim)
        for t in range(new):
            p = 200 - new + t
            sees = odd <= p and odd > p - window
            assert got[t].isnan().all() if sees else torch.isfinite(got[t]).all(), (odd, t)
