"""GPU: the bounded waits of the attention kernels expire, report, and leave the device usable.

As for the products (test_gpu_timeout.py): a test build of the library, with waits of a few milliseconds and a hook by which one CTA
leaves out an arrival when a magic word sits in the workspace.  Nothing is faulted, trapped or hung.
"""
import ctypes

import numpy as np
import pytest

from cache_util import Case, attention_bound

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
    vp, i, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
    lib.marlin_attention_decode.argtypes = [vp, ctypes.c_int64, ctypes.POINTER(binding.KvCache), vp, i, i, ctypes.c_float, i, vp, vp, sz, vp]
    lib.marlin_attention_decode.restype = i
    lib.marlin_read_status.argtypes = [vp, vp]
    lib.marlin_read_status.restype = i
    return lib


# every kernel: rows beside the keys, on tcgen05, and there with conversion; several tiles of one sequence for worker 0
@pytest.mark.parametrize("q_heads,eight_bit", [(4, False), (4, True), (16, False), (40, False), (40, True)])
def test_an_expired_wait_is_reported_and_the_next_call_is_correct(marlin, test_lib, q_heads, eight_bit):
    import torch
    from paper_2408_11743_b200 import binding
    case = Case([130000, 700], 1, q_heads, 1, 128, 16, eight_bit, seed=q_heads)  # (so long that worker 0 has a part of it for certain)
    d = case.dev(marlin)
    q = torch.from_numpy(case.q.reshape(case.T, -1)).cuda()
    out = torch.zeros_like(q)
    ws = d["workspace"]
    stream = torch.cuda.current_stream().cuda_stream
    k, v = d["k_cache"], d["v_cache"]
    cache = binding.KvCache(
        k=k.data_ptr(), v=v.data_ptr(), stride=(ctypes.c_int64 * 3)(*k.stride()[:3]), table=d["pages"].data_ptr(),
        table_stride=d["pages"].stride(0), lengths=d["lengths"].data_ptr(),
        k_scale=d["k_scale"].data_ptr() if eight_bit else None, v_scale=d["v_scale"].data_ptr() if eight_bit else None,
        pages=case.pages, max_pages=d["pages"].shape[1], sequences=case.B, kv_heads=1, head_dim=128, page_size=16,
        format=int(eight_bit))

    def call():
        return test_lib.marlin_attention_decode(q.data_ptr(), q.stride(0), ctypes.byref(cache), None, case.T, q_heads, 0.125, 0,
                                                out.data_ptr(), ws.data_ptr(), ws.numel(), stream)

    ref = case.attention_ref(0.125)

    def check(got):
        assert np.all(np.abs(got.float().cpu().numpy().reshape(ref[0].shape) - ref[0]) <= attention_bound(ref))

    assert call() == 0
    assert test_lib.marlin_read_status(ws.data_ptr(), stream) == 0
    check(out)

    ws[:32].view(torch.int32)[7] = WITHHOLD_MAGIC
    assert call() == 0
    torch.cuda.synchronize()  # the kernel returns through its normal control flow
    assert test_lib.marlin_read_status(ws.data_ptr(), stream) == 8  # MARLIN_ERR_DEVICE_TIMEOUT
    rec = ws[:32].cpu().numpy().view(np.int32)
    assert rec[0] == 8 and rec[1] == 0
    assert 0 <= rec[2] < 1024 and rec[5] > 0
    assert rec[6] >= 4000  # (in units of 1.024 us)

    ws.zero_()
    out.fill_(float("nan"))
    assert call() == 0
    assert test_lib.marlin_read_status(ws.data_ptr(), stream) == 0
    check(out)
    ws2 = torch.zeros_like(ws)
    check(marlin.attention_decode(q, k, v, d["pages"], d["lengths"], ws2, scale=0.125, k_scale=d.get("k_scale"), v_scale=d.get("v_scale")))
    assert marlin.read_status(ws2) == 0


@pytest.mark.parametrize("q_heads,dim,eight_bit", [(12, 64, False), (20, 48, False), (64, 64, False), (16, 112, False), (32, 128, False), (64, 80, True)])
def test_products_that_are_under_way_when_a_wait_expires_end_before_the_block(marlin, test_lib, q_heads, dim, eight_bit):
    # Every width of the tcgen05 kernel, three calls of it in a row that give up while products of earlier tiles may be running; calls on other
    # workspaces, queued right behind them, use the same tensor memory and shared memory and have to be right.
    import torch
    from paper_2408_11743_b200 import binding
    case = Case([200000, 700], 1, q_heads, 1, dim, 16, eight_bit, seed=q_heads)  # (worker 0 has more of it than an item costs beside its tiles)
    d = case.dev(marlin)
    q = torch.from_numpy(case.q.reshape(case.T, -1)).cuda()
    k, v = d["k_cache"], d["v_cache"]
    cache = binding.KvCache(
        k=k.data_ptr(), v=v.data_ptr(), stride=(ctypes.c_int64 * 3)(*k.stride()[:3]), table=d["pages"].data_ptr(),
        table_stride=d["pages"].stride(0), lengths=d["lengths"].data_ptr(),
        k_scale=d["k_scale"].data_ptr() if eight_bit else None, v_scale=d["v_scale"].data_ptr() if eight_bit else None,
        pages=case.pages, max_pages=d["pages"].shape[1], sequences=case.B, kv_heads=1, head_dim=dim, page_size=16, format=int(eight_bit))
    stream = torch.cuda.current_stream().cuda_stream
    spaces = [torch.zeros_like(d["workspace"]) for _ in range(6)]
    outs = [torch.full_like(q, float("nan")) for _ in spaces]
    for ws in spaces[::2]:
        ws[:32].view(torch.int32)[7] = WITHHOLD_MAGIC
    for ws, out in zip(spaces, outs):
        assert test_lib.marlin_attention_decode(q.data_ptr(), q.stride(0), ctypes.byref(cache), None, case.T, q_heads, 0.125, 0,
                                                out.data_ptr(), ws.data_ptr(), ws.numel(), stream) == 0
    ref = case.attention_ref(0.125)
    for i, (ws, out) in enumerate(zip(spaces, outs)):
        assert test_lib.marlin_read_status(ws.data_ptr(), stream) == (0 if i % 2 else 8)
        if i % 2:
            assert np.all(np.abs(out.float().cpu().numpy().reshape(ref[0].shape) - ref[0]) <= attention_bound(ref))


def test_a_time_out_and_a_report_of_the_cache_do_not_hide_each_other(marlin, test_lib):
    # a page that is not there is reported and contained; a wait that expires later, on the same workspace, is what the host has to know
    import torch
    from paper_2408_11743_b200 import binding
    case = Case([130000], 1, 4, 1, 128, 16, seed=1)
    d = case.dev(marlin)
    q = torch.from_numpy(case.q.reshape(case.T, -1)).cuda()
    out = torch.zeros_like(q)
    ws = d["workspace"]
    stream = torch.cuda.current_stream().cuda_stream
    k, v, good = d["k_cache"], d["v_cache"], d["pages"]
    bad = good.clone()
    bad[0, 5] = case.pages

    def call(table):
        cache = binding.KvCache(
            k=k.data_ptr(), v=v.data_ptr(), stride=(ctypes.c_int64 * 3)(*k.stride()[:3]), table=table.data_ptr(),
            table_stride=table.stride(0), lengths=d["lengths"].data_ptr(), pages=case.pages, max_pages=table.shape[1], sequences=1,
            kv_heads=1, head_dim=128, page_size=16, format=0)
        assert test_lib.marlin_attention_decode(q.data_ptr(), q.stride(0), ctypes.byref(cache), None, 1, 4, 0.125, 0, out.data_ptr(),
                                                ws.data_ptr(), ws.numel(), stream) == 0
        return test_lib.marlin_read_status(ws.data_ptr(), stream)

    assert call(good) == 0
    assert call(bad) == 9
    assert call(good) == 9  # it stays until the workspace is zeroed
    ws[:32].view(torch.int32)[7] = WITHHOLD_MAGIC
    assert call(good) == 8
    rec = ws[:32].cpu().numpy().view(np.int32)
    assert rec[0] == 8 and rec[1] == 0 and rec[6] >= 4000  # with its record
    ws.zero_()
    ws[:32].view(torch.int32)[7] = WITHHOLD_MAGIC
    assert call(bad) == 8  # both in one call
    ws.zero_()
    assert call(good) == 0
