"""Refusals of the calls on the paged cache: every one of them is made before a CUDA call, so none of this needs a GPU."""
import ctypes

import numpy as np
import pytest


@pytest.fixture(scope="module")
def marlin():
    from paper_2408_11743_b200 import build
    build.build()
    import paper_2408_11743_b200 as m
    return m


FAKE = 0x1000  # aligned, never dereferenced
NULL, SHAPE, GROUP, ALIGN, WORKSPACE = 1, 2, 3, 4, 5


def cache(marlin, **more):
    c = marlin.KvCache()
    given = dict(k=FAKE, v=FAKE, table=FAKE, table_stride=9, lengths=FAKE, k_scale=None, v_scale=None, pages=100, max_pages=9,
                 sequences=3, kv_heads=2, head_dim=64, page_size=16, format=0)
    given.update(more)
    strides = given.pop("stride", (2048, 1024, 64))
    for name, x in given.items():
        setattr(c, name, x)
    for i, x in enumerate(strides):
        c.stride[i] = x
    return c


def append(marlin, c, q=FAKE, qs=512, k=FAKE, ks=512, v=FAKE, vs=512, q_out=FAKE, starts=None, tokens=3, q_heads=8, inv=FAKE, rotary=64,
           ws=FAKE, ws_bytes=1 << 30):
    return marlin.lib().marlin_kv_append(q, qs, k, ks, v, vs, q_out, ctypes.byref(c) if c else None, starts, tokens, q_heads, inv, rotary,
                                         0, ws, ws_bytes, None)


def attend(marlin, c, q=FAKE, qs=512, starts=None, tokens=3, q_heads=8, scale=1.0, window=0, out=FAKE, ws=FAKE, ws_bytes=1 << 30):
    return marlin.lib().marlin_attention_decode(q, qs, ctypes.byref(c) if c else None, starts, tokens, q_heads, scale, window, out, ws,
                                                ws_bytes, None)


def block(marlin, c, a=FAKE, w=(FAKE,) * 4, scratch=(FAKE,) * 3, out=FAKE, starts=None, M=3, K=512, q_heads=8, N=512, G=128, inv=FAKE,
          rotary=64, window=0, ws=FAKE, ws_bytes=1 << 30):
    return marlin.lib().marlin_attention_block(a, *w, *scratch, out, ctypes.byref(c) if c else None, starts, M, K, q_heads, N, G, inv,
                                               rotary, 0, 1.0, window, ws, ws_bytes, None)


# what is wrong with the cache, and the status of all three calls
BAD_CACHES = [
    (dict(k=None), NULL), (dict(v=None), NULL), (dict(table=None), NULL), (dict(lengths=None), NULL),
    (dict(head_dim=0), SHAPE), (dict(head_dim=72), SHAPE), (dict(head_dim=272), SHAPE), (dict(head_dim=-16), SHAPE),
    (dict(page_size=0), SHAPE), (dict(page_size=24), SHAPE), (dict(page_size=-16), SHAPE), (dict(pages=0), SHAPE),
    (dict(max_pages=0), SHAPE), (dict(table_stride=8), SHAPE), (dict(sequences=0), SHAPE), (dict(sequences=4), SHAPE),
    (dict(kv_heads=0), SHAPE), (dict(kv_heads=3), SHAPE), (dict(format=2), SHAPE), (dict(format=-1), SHAPE),
    (dict(stride=(-2048, 1024, 64)), SHAPE), (dict(k_scale=FAKE), SHAPE), (dict(v_scale=FAKE), SHAPE),
    (dict(k=FAKE + 8), ALIGN), (dict(v=FAKE + 2), ALIGN), (dict(table=FAKE + 2), ALIGN), (dict(lengths=FAKE + 1), ALIGN),
    (dict(stride=(2048, 1024, 68)), ALIGN), (dict(stride=(2048, 1028, 64)), ALIGN), (dict(stride=(2044, 1024, 64)), ALIGN),
    (dict(format=1, stride=(2048, 1024, 72)), ALIGN), (dict(format=1, k_scale=FAKE + 2), ALIGN),
]


@pytest.mark.parametrize("wrong,status", BAD_CACHES)
def test_caches_that_are_refused(marlin, wrong, status):
    assert append(marlin, cache(marlin, **wrong)) == status
    assert attend(marlin, cache(marlin, **wrong)) == status
    # (the block looks at the layers first: with these head_dims they have no shape either)
    assert block(marlin, cache(marlin, **wrong)) == status


def test_arguments_that_are_refused(marlin):
    c = cache(marlin)
    assert append(marlin, None) == attend(marlin, None) == block(marlin, None) == NULL
    for name in ("q", "k", "v", "q_out", "ws"):
        assert append(marlin, c, **{name: None}) == NULL, name
        assert append(marlin, c, **{name: FAKE + 8}) == ALIGN, name
    for name in ("qs", "ks", "vs"):
        assert append(marlin, c, **{name: 516}) == ALIGN, name
        assert append(marlin, c, **{name: -512}) == SHAPE, name
    for name in ("q", "out", "ws"):
        assert attend(marlin, c, **{name: None}) == NULL, name
        assert attend(marlin, c, **{name: FAKE + 8}) == ALIGN, name
    for call in (append, attend):
        assert call(marlin, c, tokens=0) == SHAPE
        assert call(marlin, c, tokens=4) == SHAPE             # one row per sequence without starts
        assert call(marlin, c, starts=FAKE + 2, tokens=4) == ALIGN
        assert call(marlin, c, q_heads=7) == SHAPE            # not a multiple of the key heads
        assert call(marlin, c, q_heads=-2) == SHAPE
        assert call(marlin, c, ws_bytes=marlin.attention_workspace_bytes(64) - 1) == WORKSPACE
        assert call(marlin, c, tokens=2 ** 30, starts=FAKE, q_heads=1024) == SHAPE
    assert append(marlin, c, inv=None) == SHAPE               # queries are rotated or stay where they are
    assert append(marlin, c, inv=FAKE + 1) == ALIGN
    for rotary in (0, 8, 24, 80, -16):
        assert append(marlin, c, rotary=rotary) == SHAPE, rotary
    assert attend(marlin, c, q_heads=0) == SHAPE
    assert attend(marlin, c, window=-1) == SHAPE
    assert attend(marlin, c, qs=516) == ALIGN
    assert attend(marlin, c, qs=-512) == SHAPE


def test_blocks_that_are_refused(marlin):
    c = cache(marlin)
    for i in range(4):
        for x, status in ((None, NULL), (FAKE + 8, ALIGN)):
            assert block(marlin, c, w=tuple(x if j == i else FAKE for j in range(4))) == status
    for i in range(3):
        for x, status in ((None, NULL), (FAKE + 8, ALIGN)):
            assert block(marlin, c, scratch=tuple(x if j == i else FAKE for j in range(3))) == status
    for name in ("a", "out"):
        assert block(marlin, c, **{name: None}) == NULL
        assert block(marlin, c, **{name: FAKE + 8}) == ALIGN
    for wrong in (dict(M=0), dict(M=4), dict(K=500), dict(N=500), dict(q_heads=0), dict(q_heads=7), dict(rotary=8), dict(window=-1),
                  dict(q_heads=1 << 20)):
        assert block(marlin, c, **wrong) == SHAPE, wrong
    assert block(marlin, cache(marlin, head_dim=16, stride=(512, 256, 16)), rotary=16, q_heads=6) == SHAPE  # output layer: K = 96
    assert block(marlin, c, G=96) == GROUP
    need = max(marlin.workspace_bytes(3, 512, 768), marlin.workspace_bytes(3, 512, 512), marlin.attention_workspace_bytes(64))
    assert block(marlin, c, ws_bytes=need - 1) == WORKSPACE


def test_workspace_sizes(marlin):
    sizes = [marlin.attention_workspace_bytes(d) for d in range(16, 257, 16)]
    assert min(sizes) > 8192 and max(sizes) < 64 << 20
    for d in (0, 8, 24, 257, 272, -16):
        with pytest.raises(marlin.MarlinError):
            marlin.attention_workspace_bytes(d)
    assert marlin.lib().marlin_status_string(9).startswith(b"a length")


def test_the_binding_refuses_what_is_not_on_a_gpu(marlin):
    import torch
    x = torch.zeros(3, 512, dtype=torch.float16)
    k = torch.zeros(4, 2, 16, 64, dtype=torch.float16)
    pages, lengths = torch.zeros(3, 2, dtype=torch.int32), torch.ones(3, dtype=torch.int32)
    ws = torch.zeros(1 << 20, dtype=torch.uint8)
    with pytest.raises(TypeError, match="CUDA"):
        marlin.kv_append(x, k, k, pages, lengths, ws)
    with pytest.raises(TypeError, match="CUDA"):
        marlin.attention_decode(x, k, k, pages, lengths, ws)
    with pytest.raises(TypeError, match="CUDA"):
        marlin.attention_block(x, ws, ws, ws, ws, k, k, pages, lengths, 512, 8, 512, 128, ws)
    for wrong in (None, 3, np.zeros(3)):
        with pytest.raises(TypeError, match="CUDA"):
            marlin.attention_decode(x, wrong, k, pages, lengths, ws)


def test_the_oracle_is_softmax_attention_on_a_plain_layout(marlin):
    # one page per token in order: the oracle against a direct formula on small integers
    from oracle import attention_ref as ref
    rng = np.random.default_rng(0)
    k, v = rng.standard_normal((6, 1, 1, 16)), rng.standard_normal((6, 1, 1, 16))
    q = rng.standard_normal((2, 3, 16))
    out = ref.attention(q, k, v, np.arange(6)[None], [6], [0, 2], 0.25)[0]
    for t, n in ((0, 5), (1, 6)):
        for h in range(3):
            w = np.exp(q[t, h] @ k[:n, 0, 0].T * 0.25)
            assert np.allclose(out[t, h], (w / w.sum()) @ v[:n, 0, 0], rtol=1e-12)
    x = rng.standard_normal((1, 16))
    for interleaved in (False, True):
        y = ref.rotate(x, 3, [0.5, 0.0], interleaved)
        i, j = ((0, 1) if interleaved else (0, 2))
        assert np.allclose([y[0, i], y[0, j]], [x[0, i] * np.cos(1.5) - x[0, j] * np.sin(1.5), x[0, j] * np.cos(1.5) + x[0, i] * np.sin(1.5)])
        assert np.array_equal(y[0, 4:], x[0, 4:])
        assert np.allclose((y ** 2).sum(), (x ** 2).sum())


def test_the_kernels_read_nothing_through_the_read_only_path():
    # they are resident while the kernel before them still writes what they read
    import os
    from paper_2408_11743_b200 import build
    for name in ("kv_append.cu", "kv_cache.cuh", "attention.cu", "attention.cuh", "attention_tc.cu"):
        with open(os.path.join(build.CSRC, name)) as f:
            code = "\n".join(line.split("//")[0] for line in f)
        for word in ("__ldg", "ld.global.nc", "__restrict__"):
            assert word not in code, (name, word)
