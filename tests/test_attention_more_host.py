"""Refusals of the calls on 8-bit caches with scales by block, on sinks and on page tables: made before a CUDA call, so none of this needs a GPU."""
import ctypes
import os

import numpy as np
import pytest

from test_attention_host import ALIGN, BAD_CACHES, FAKE, NULL, SHAPE, WORKSPACE, cache


@pytest.fixture(scope="module")
def marlin():
    from paper_2408_11743_b200 import build
    build.build()
    import paper_2408_11743_b200 as m
    return m


def scales(marlin, k=FAKE, v=FAKE, stride=(32, 16, 1), block_size=4):
    s = marlin.KvScales()
    s.k, s.v, s.block_size = k, v, block_size
    for i, x in enumerate(stride):
        s.stride[i] = x
    return s


def ref(x):
    return ctypes.byref(x) if x is not None else None


def append(marlin, c, s, q=FAKE, qs=512, k=FAKE, ks=512, v=FAKE, vs=512, q_out=FAKE, starts=None, tokens=3, q_heads=8, inv=FAKE, rotary=64, ws=FAKE,
           ws_bytes=1 << 30):
    return marlin.lib().marlin_kv_append_scaled(q, qs, k, ks, v, vs, q_out, ref(c), ref(s), starts, tokens, q_heads, inv, rotary, 0, ws, ws_bytes, None)


def attend(marlin, c, s, q=FAKE, qs=512, starts=None, tokens=3, q_heads=8, window=0, sinks=0, out=FAKE, ws=FAKE, ws_bytes=1 << 30):
    return marlin.lib().marlin_attention_sinks(q, qs, ref(c), ref(s), starts, tokens, q_heads, 1.0, window, sinks, out, ws, ws_bytes, None)


def block(marlin, c, s, a=FAKE, w=(FAKE,) * 4, scratch=(FAKE,) * 3, out=FAKE, starts=None, M=3, K=512, q_heads=8, N=512, G=128, inv=FAKE, rotary=64,
          window=0, sinks=0, ws=FAKE, ws_bytes=1 << 30):
    return marlin.lib().marlin_attention_block_sinks(a, *w, *scratch, out, ref(c), ref(s), starts, M, K, q_heads, N, G, inv, rotary, 0, 1.0,
                                                     window, sinks, ws, ws_bytes, None)


EIGHT = dict(format=2)  # two's complement; the strides of `cache` are multiples of 16


@pytest.mark.parametrize("wrong,status", BAD_CACHES)
def test_caches_that_are_refused(marlin, wrong, status):
    assert attend(marlin, cache(marlin, **wrong), None, window=5, sinks=1) == status  # (format 2 without scales among them)
    assert block(marlin, cache(marlin, **wrong), None, window=5, sinks=1) == status
    if "format" in wrong or "k_scale" in wrong or "v_scale" in wrong:
        return
    eight = cache(marlin, **{**EIGHT, **wrong})
    want = ALIGN if wrong.get("stride") and status == ALIGN else status
    for call in (append, attend, block):
        assert call(marlin, eight, scales(marlin)) == want


@pytest.mark.parametrize("format", [1, 2])
def test_scales_that_are_refused(marlin, format):
    c = cache(marlin, format=format)
    for wrong, status in ((dict(k=None), NULL), (dict(v=None), NULL), (dict(k=FAKE + 2), ALIGN), (dict(v=FAKE + 1), ALIGN), (dict(block_size=0), SHAPE),
                          (dict(block_size=3), SHAPE), (dict(block_size=32), SHAPE), (dict(block_size=-4), SHAPE), (dict(stride=(-1, 4, 1)), SHAPE),
                          (dict(stride=(8, -4, 1)), SHAPE), (dict(stride=(8, 4, -1)), SHAPE)):
        for call in (append, attend, block):
            assert call(marlin, c, scales(marlin, **wrong)) == status, wrong
    for call in (append, attend, block):
        assert call(marlin, cache(marlin, format=format, page_size=256, stride=(16384, 16384, 64)), scales(marlin, block_size=256)) == SHAPE
        assert call(marlin, cache(marlin, format=0), scales(marlin)) == SHAPE
        assert call(marlin, cache(marlin, format=format, k_scale=FAKE), scales(marlin)) == SHAPE
        assert call(marlin, cache(marlin, format=format, v_scale=FAKE), scales(marlin)) == SHAPE
    assert append(marlin, c, None) == NULL


def test_arguments_that_are_refused(marlin):
    c, s = cache(marlin, **EIGHT), scales(marlin)
    for call in (append, attend, block):
        assert call(marlin, None, s) == NULL
    for name in ("q", "k", "v", "q_out", "ws"):
        assert append(marlin, c, s, **{name: None}) == NULL and append(marlin, c, s, **{name: FAKE + 8}) == ALIGN
    for name in ("q", "out", "ws"):
        assert attend(marlin, c, s, **{name: None}) == NULL and attend(marlin, c, s, **{name: FAKE + 8}) == ALIGN
    for call in (append, attend):
        assert call(marlin, c, s, tokens=0) == call(marlin, c, s, tokens=4) == call(marlin, c, s, q_heads=7) == SHAPE
        assert call(marlin, c, s, ws_bytes=marlin.attention_workspace_bytes(64) - 1) == WORKSPACE
    assert append(marlin, c, s, inv=None) == append(marlin, c, s, rotary=72) == SHAPE
    for call in (attend, block):
        assert call(marlin, c, s, window=-1) == call(marlin, c, s, sinks=-1) == call(marlin, c, s, sinks=-1, window=4) == SHAPE


def pages(marlin, **more):
    c = marlin.KvPages()
    given = dict(table=FAKE, table_stride=9, lengths=FAKE, free_pages=FAKE, free_count=FAKE, capacity=100, max_pages=9, sequences=3, page_size=16)
    for name, x in {**given, **more}.items():
        setattr(c, name, x)
    return c


def reserve(marlin, c, counts=FAKE, keep=FAKE, tokens=5, starts=FAKE, slots=FAKE, positions=FAKE, ws=FAKE, ws_bytes=8192):
    return marlin.lib().marlin_kv_reserve(ref(c), counts, keep, tokens, starts, slots, positions, ws, ws_bytes, None)


def test_page_tables_that_are_refused(marlin):
    assert reserve(marlin, None) == NULL
    for name in ("table", "lengths", "free_pages", "free_count"):
        assert reserve(marlin, pages(marlin, **{name: None})) == NULL
        assert reserve(marlin, pages(marlin, **{name: FAKE + 2})) == ALIGN
    for wrong in (dict(page_size=0), dict(page_size=12), dict(page_size=-16), dict(max_pages=0), dict(table_stride=8), dict(sequences=0), dict(capacity=0)):
        assert reserve(marlin, pages(marlin, **wrong)) == SHAPE, wrong
    c = pages(marlin)
    assert reserve(marlin, c, ws=None) == NULL and reserve(marlin, c, ws=FAKE + 8) == ALIGN and reserve(marlin, c, ws_bytes=8191) == WORKSPACE
    assert reserve(marlin, c, tokens=-1) == reserve(marlin, c, tokens=2 ** 30 + 1) == SHAPE
    for name in ("counts", "keep", "starts", "positions"):
        assert reserve(marlin, c, **{name: FAKE + 2}) == ALIGN, name
    assert reserve(marlin, c, slots=FAKE + 4) == ALIGN


def test_the_binding_refuses_what_is_not_on_a_gpu(marlin):
    import torch
    x, k = torch.zeros(3, 512, dtype=torch.float16), torch.zeros(4, 2, 16, 64, dtype=torch.int8)
    pages, lengths, ws = torch.zeros(3, 2, dtype=torch.int32), torch.ones(3, dtype=torch.int32), torch.zeros(1 << 20, dtype=torch.uint8)
    s = torch.zeros(4, 2, 4)
    with pytest.raises(TypeError, match="CUDA"):
        marlin.kv_append(x, k, k, pages, lengths, ws, k_scale=s, v_scale=s)
    with pytest.raises(TypeError, match="CUDA"):
        marlin.attention_decode(x, k, k, pages, lengths, ws, k_scale=s, v_scale=s, window=4, sinks=2)
    for wrong in (lengths, None, np.zeros(3)):
        with pytest.raises(TypeError, match="CUDA"):
            marlin.kv_reserve(wrong, pages, lengths, lengths[:1], ws, 16, 3)


def test_the_kernels_read_nothing_through_the_read_only_path():
    # they are resident while the kernel before them still writes what they read
    from paper_2408_11743_b200 import build
    for name in ("kv_append_blocks.cu", "kv_reserve.cu", "attention_warp.cuh", "attention_tc.cuh", "attention_more.cu", "attention_tc_more.cu",
                 "attention_prompt.cu"):
        with open(os.path.join(build.CSRC, name)) as f:
            code = "\n".join(line.split("//")[0] for line in f)
        for word in ("__ldg", "ld.global.nc", "__restrict__"):
            assert word not in code, (name, word)


def test_the_oracle_is_what_it_says():
    import torch
    from oracle import attention_ref, cache_blocks_ref
    rng = np.random.default_rng(0)
    # e4m3 codes and their rounding against torch's
    codes = torch.arange(256, dtype=torch.uint8)
    assert np.array_equal(cache_blocks_ref.E4M3, codes.view(torch.float8_e4m3fn).double().numpy(), equal_nan=True)
    x = torch.from_numpy(rng.standard_normal(20000).astype(np.float32)) * torch.logspace(-4, 2.4, 20000)
    x = x.clamp(-448, 448)  # (beyond that torch gives NaN, the definition 448)
    assert np.array_equal(cache_blocks_ref.to_e4m3(x.numpy()), x.to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    assert list(cache_blocks_ref.to_e4m3([448, 1e9, -np.inf, 17 / 16, 19 / 16, 2.0 ** -10])) == [126, 126, 254, 56, 58, 0]
    assert list(cache_blocks_ref.to_int8([0.5, 1.5, -2.5, 127.4, 1e9, -np.inf, np.nan])) == [0, 2, -2, 127, 127, -127, 0]
    # a block filled at once, and one filled token by token
    new = rng.standard_normal((16, 1, 32)).astype(np.float32)
    c, s = np.zeros((2, 1, 16, 32), np.int8), np.zeros((2, 1, 2), np.float32)
    cache_blocks_ref.append(c, s, new, [1], 0, 8)
    assert np.allclose(s[1, 0], np.abs(new).reshape(2, -1).max(-1) / 127)
    assert np.abs(cache_blocks_ref.expanded(c, s)[1] - new.transpose(1, 0, 2)).max() <= s.max() / 2 * 1.001
    one, t = np.zeros_like(c), np.zeros_like(s)
    for i in range(16):
        cache_blocks_ref.append(one, t, new[i:i + 1], [1], i, 8)
    assert (t[1] >= s[1]).all() and (t[1] < 2 * s[1] * 1.001).all()
    assert np.abs(cache_blocks_ref.expanded(one, t)[1] - new.transpose(1, 0, 2)).max() <= t.max()
    # attention without sinks is the one that was there
    q, k, v = rng.standard_normal((2, 3, 16)), rng.standard_normal((6, 1, 1, 16)), rng.standard_normal((6, 1, 1, 16))
    for window in (0, 2):
        for a, b in zip(cache_blocks_ref.attention(q, k, v, np.arange(6)[None], [6], [0, 2], 0.25, window), attention_ref.attention(q, k, v, np.arange(6)[None], [6], [0, 2], 0.25, window)):
            assert np.allclose(a, b)
    out = cache_blocks_ref.attention(q, k, v, np.arange(6)[None], [6], [0, 2], 0.25, 2, 1)[0]
    for t, at in ((0, [0, 3, 4]), (1, [0, 4, 5])):
        w = np.exp(q[t] @ k[at, 0, 0].T * 0.25)
        assert np.allclose(out[t], (w / w.sum(-1, keepdims=True)) @ v[at, 0, 0])
