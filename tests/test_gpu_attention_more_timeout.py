"""GPU: the bounded waits of the attention kernels for sinks, scales by block and prompts expire, report, and leave the device usable.

As in test_gpu_attention_timeout.py: a test build of the library with waits of a few milliseconds and a hook by which one CTA leaves out an
arrival when a magic word sits in the workspace.  Nothing is faulted, trapped or hung.
"""
import ctypes

import numpy as np
import pytest

from blocks_util import BlockCase

pytestmark = pytest.mark.gpu

WITHHOLD_MAGIC = 0x57495448


@pytest.fixture(scope="module")
def marlin():
    import torch
    assert torch.cuda.is_available()
    import paper_2408_11743_b200 as m
    m.lib()
    return m


@pytest.fixture(scope="module")
def test_lib(tmp_path_factory):
    from paper_2408_11743_b200 import binding, build
    out = str(tmp_path_factory.mktemp("marlin_test_build") / "libmarlin_b200_testhooks.so")
    build.build(extra_flags=["-DMARLIN_TEST_HOOKS", "-DMARLIN_WAIT_LIMIT_NS=5000000ull"], out=out)
    lib = ctypes.CDLL(out)
    lib.marlin_attention_sinks.argtypes = binding.lib().marlin_attention_sinks.argtypes
    lib.marlin_read_status.argtypes = [ctypes.c_void_p, ctypes.c_void_p]
    return lib


# every kind of kernel; sequences so long that worker 0 has a part of them for certain, or prompts of many blocks
@pytest.mark.parametrize("kind,block,q_heads,lengths,new,window", [
    ("fp16", 0, 4, [130000, 700], 1, 120000), ("int8", 16, 4, [130000, 700], 1, 0), ("e4m3", 8, 4, [130000, 700], 1, 0), ("int8", 64, 16, [130000, 700], 1, 0),
    ("fp16", 0, 16, [130000, 700], 1, 120000), ("int8", 64, 40, [130000, 700], 1, 0), ("fp16", 0, 8, [4000, 900], 900, 700)])
def test_an_expired_wait_is_reported_and_the_next_calls_are_right(marlin, test_lib, kind, block, q_heads, lengths, new, window):
    import torch
    from paper_2408_11743_b200 import binding
    case = BlockCase(lengths, new, q_heads, 1, 128, 64, kind, block, seed=q_heads)
    d = case.dev(marlin)
    q = torch.from_numpy(case.q.reshape(case.T, -1)).cuda()
    k, v = d["k_cache"], d["v_cache"]
    stream = torch.cuda.current_stream().cuda_stream
    cache = binding.KvCache(k=k.data_ptr(), v=v.data_ptr(), stride=(ctypes.c_int64 * 3)(*k.stride()[:3]), table=d["pages"].data_ptr(),
                            table_stride=d["pages"].stride(0), lengths=d["lengths"].data_ptr(), pages=case.pages, max_pages=d["pages"].shape[1],
                            sequences=case.B, kv_heads=1, head_dim=128, page_size=64, format=("fp16", "e4m3", "int8").index(kind))
    scales = None
    if block:
        s = d["k_scale"]
        scales = ctypes.byref(binding.KvScales(k=s.data_ptr(), v=d["v_scale"].data_ptr(), stride=(ctypes.c_int64 * 3)(*s.stride()), block_size=block))
    starts = None if new == 1 else d["starts"].data_ptr()

    def call(ws, out):
        assert test_lib.marlin_attention_sinks(q.data_ptr(), q.stride(0), ctypes.byref(cache), scales, starts, case.T, q_heads, 0.125, window, 5,
                                               out.data_ptr(), ws.data_ptr(), ws.numel(), stream) == 0

    spaces = [torch.zeros_like(d["workspace"]) for _ in range(4)]
    outs = [torch.full_like(q, float("nan")) for _ in spaces]
    for ws in spaces[::2]:
        ws[:32].view(torch.int32)[7] = WITHHOLD_MAGIC
    for ws, out in zip(spaces, outs):  # (calls that give up, and right behind them calls that use the same tensor memory and shared memory)
        call(ws, out)
    ref = case.sinks_ref_on_gpu(0.125, window, 5)
    for i, (ws, out) in enumerate(zip(spaces, outs)):
        assert test_lib.marlin_read_status(ws.data_ptr(), stream) == (0 if i % 2 else 8)
        if i % 2:
            assert np.all(np.abs(out.float().cpu().numpy().reshape(ref[0].shape) - ref[0]) <= case.sinks_bound(ref))
        else:
            rec = ws[:32].cpu().numpy().view(np.int32)
            assert rec[0] == 8 and rec[1] == 0 and rec[6] >= 4000  # worker 0, after 5 ms (in units of 1.024 us)
    spaces[0].zero_()
    call(spaces[0], outs[0])
    assert test_lib.marlin_read_status(spaces[0].data_ptr(), stream) == 0
    assert torch.equal(outs[0], outs[1])
