"""GPU: one long prompt and many sequences with a new token each, and with long contexts, in one call; and which kernel answers prompts."""
import numpy as np
import pytest

from blocks_util import BlockCase
from test_gpu_attention_prompt import check
from test_gpu_attention_sinks import attend

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def marlin():
    import torch
    assert torch.cuda.is_available()
    import paper_2408_11743_b200 as m
    m.lib()
    return m


def mixed(kind, block, q_heads, kv_heads, dim, at, seed=0):
    """A prompt of 900 tokens as sequence `at` of 40, the others with one new token each behind 1 to 5000."""
    rng = np.random.default_rng(seed)
    lengths = np.exp(rng.uniform(0, np.log(5000), 40)).astype(int)
    lengths[[3, 17, 30]] = 5000, 1, 4097
    new = [1] * 40
    lengths[at], new[at] = 1300, 900
    new[5], new[6] = 0, 4
    return BlockCase(list(lengths), new, q_heads, kv_heads, dim, 32, kind, block, seed=seed)


@pytest.mark.parametrize("kind,block", [("fp16", 0), ("e4m3", 0), ("e4m3", 8), ("int8", 16)])
@pytest.mark.parametrize("q_heads,kv_heads,dim", [(16, 2, 128), (8, 1, 64), (4, 2, 256)])
@pytest.mark.parametrize("at", [0, 20, 39])
def test_a_prompt_beside_sequences_with_long_contexts(marlin, kind, block, q_heads, kv_heads, dim, at):
    case = mixed(kind, block, q_heads, kv_heads, dim, at, seed=at)
    check(marlin, case, window=0, sinks=1)
    check(marlin, case, window=600, sinks=70)
    check(marlin, case)


def kernels_of(call):
    """Names of the kernels of the library that a call launches."""
    import torch
    from torch.profiler import ProfilerActivity, profile
    with profile(activities=[ProfilerActivity.CUDA, ProfilerActivity.CPU]) as p:
        call()
        torch.cuda.synchronize()
    return [e.name for e in p.events() if "marlin_b200" in e.name]


@pytest.mark.parametrize("kind,block,q_heads,dim,lengths,new,window,sinks,prompt", [
    ("fp16", 0, 16, 128, [900], [900], 0, 1, True), ("fp16", 0, 16, 64, [900, 50], [900, 1], 200, 4, True), ("fp16", 0, 1, 128, [7000], [6500], 200, 4, True),
    ("fp16", 0, 4, 128, [900], 1, 200, 4, False), ("fp16", 0, 16, 64, [900, 5000], 1, 0, 1, False), ("int8", 8, 32, 128, [900], 1, 0, 0, False)])
def test_prompts_take_the_kernel_for_prompts(marlin, kind, block, q_heads, dim, lengths, new, window, sinks, prompt):
    # (from 128 rows a sequence and key head, and 24 blocks of 256 rows, on; two sides that agree would not tell which of them answered)
    case = BlockCase(lengths, new, q_heads, 1, dim, 32, kind, block)
    d = case.dev(marlin)
    names = kernels_of(lambda: attend(marlin, case, d, window=window, sinks=sinks))
    if not names:
        pytest.skip("the profiler sees no kernels here")
    assert len(names) == 1 and ("attention_prompt_kernel" in names[0]) == prompt, names
