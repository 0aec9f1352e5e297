"""GPU: attention through a window with sinks, and over 8-bit caches with a scale per block, against the oracle in 64 bits."""
import numpy as np
import pytest

from blocks_util import BlockCase

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def marlin():
    import torch
    assert torch.cuda.is_available()
    import paper_2408_11743_b200 as m
    m.lib()
    return m


def attend(marlin, case, d=None, **more):
    import torch
    d = d or case.dev(marlin)
    q = torch.from_numpy(case.q.reshape(case.T, -1)).cuda()
    out = marlin.attention_decode(q, **{**d, **more})
    torch.cuda.synchronize()
    return out, d


def check(marlin, case, window=0, sinks=0, scale=None):
    scale = case.dim ** -0.5 if scale is None else scale
    out, d = attend(marlin, case, window=window, sinks=sinks, scale=scale)
    assert marlin.read_status(d["workspace"]) == 0
    ref = case.sinks_ref(float(np.float32(scale)), window, sinks)
    got = out.float().cpu().numpy().reshape(ref[0].shape)
    off, bound = np.abs(got - ref[0]), case.sinks_bound(ref)
    bad = ~(off <= bound)
    assert not bad.any(), f"{bad.sum()} of {bad.size} off, the first at {np.argwhere(bad)[0]}: {got[bad][0]} for {ref[0][bad][0]}"
    return out, d


KINDS = [("fp16", 0), ("e4m3", 0), ("e4m3", 8), ("int8", 16), ("int8", 1)]
# rows of a key head from one to many: every kernel
ROWS = [(4, 4, 128, 1), (8, 1, 64, 1), (12, 1, 128, 1), (29, 1, 64, 1), (16, 2, 256, 3), (40, 1, 128, 2), (71, 1, 64, 2), (6, 1, 80, 5), (20, 1, 48, 1)]


@pytest.mark.parametrize("kind,block", KINDS)
@pytest.mark.parametrize("q_heads,kv_heads,dim,new", ROWS)
def test_windows_with_sinks(marlin, kind, block, q_heads, kv_heads, dim, new):
    # lengths around nothing, the sinks, the window and their sum, and far past them; sinks that end inside of a tile and of a page
    case = BlockCase([0, 1, 5, 70, 133, 205, 206, 270, 1000, 4099], new, q_heads, kv_heads, dim, 16, kind, block, seed=dim + new)
    check(marlin, case, window=133, sinks=70)


@pytest.mark.parametrize("kind,block", KINDS)
@pytest.mark.parametrize("window,sinks", [(1, 1), (1, 300), (64, 64), (64, 1), (128, 127), (500, 3), (2000, 100), (7, 5000), (10, 0), (0, 4)])
def test_edges_of_windows_and_sinks(marlin, kind, block, window, sinks):
    case = BlockCase([700, 64, 65, 1027, 3], 3, 8, 2, 64, 32, kind, block, seed=window)
    check(marlin, case, window=window, sinks=sinks)
    case = BlockCase([1500, 700], 9, 16, 1, 128, 64, kind, block, seed=window)
    check(marlin, case, window=window, sinks=sinks)


@pytest.mark.parametrize("kind,block", [("fp16", 0), ("e4m3", 8), ("int8", 4)])
@pytest.mark.parametrize("q_heads,kv_heads,dim", [(8, 1, 128), (4, 4, 64), (6, 2, 256), (29, 1, 64)])
def test_prompts(marlin, kind, block, q_heads, kv_heads, dim):
    # blocks of rows with tiles of their own: a prompt from its beginning, one that goes on, one shorter than everything
    case = BlockCase([500, 900, 40], [500, 333, 40], q_heads, kv_heads, dim, 16, kind, block, seed=dim)
    check(marlin, case, window=100, sinks=5)
    check(marlin, case, window=300, sinks=150)
    check(marlin, case)


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("page,block", [(1, 1), (4, 2), (8, 8), (16, 4), (64, 64), (128, 128), (128, 1), (256, 32)])
@pytest.mark.parametrize("q_heads,dim", [(4, 128), (48, 128), (16, 64), (12, 256)])
def test_blocks_and_pages(marlin, kind, page, block, q_heads, dim):
    check(marlin, BlockCase([0, 1, 63, 300, 515], 1, q_heads, 1, dim, page, kind, block, seed=page + block))


@pytest.mark.parametrize("kind,block", KINDS)
@pytest.mark.parametrize("layout", ["tokens", "wide"])
def test_layouts(marlin, kind, block, layout):
    check(marlin, BlockCase([300, 41, 0], 2, 8, 2, 64, 16, kind, block, layout), window=100, sinks=9)
    check(marlin, BlockCase([300, 41, 0], 2, 32, 1, 128, 16, kind, block, layout), window=100, sinks=9)


def test_scales_with_strides(marlin):
    import torch
    case = BlockCase([300, 41], 2, 8, 2, 64, 16, "int8", 4)
    d = case.dev(marlin)
    want, _ = attend(marlin, case, d)
    for name in ("k_scale", "v_scale"):
        s = d[name]
        big = torch.full((s.shape[2], s.shape[0] + 1, s.shape[1] + 2), float("nan"), device="cuda")
        view = big.permute(1, 2, 0)[1:, 1:-1]
        view.copy_(s)
        d[name] = view
    with pytest.raises(ValueError, match="contiguous"):
        attend(marlin, case, d)
    for name in ("k_scale", "v_scale"):
        s = torch.from_numpy(getattr(case, name)).cuda()
        big = torch.full((s.shape[1] + 2, s.shape[0] + 1, s.shape[2]), float("nan"), device="cuda")
        view = big.transpose(0, 1)[1:, 1:-1]
        view.copy_(s)
        d[name] = view
    got, _ = attend(marlin, case, d)
    assert torch.equal(got, want)


@pytest.mark.parametrize("kind,block", KINDS)
@pytest.mark.parametrize("q_heads,dim", [(4, 128), (40, 128), (20, 64), (12, 256)])
def test_hidden_places_do_not_matter(marlin, kind, block, q_heads, dim):
    # what lies between the sinks and the window, behind the sequences and in pages of nobody: infinities and NaN, scales too
    import torch
    case = BlockCase([700, 300], 1, q_heads, 1, dim, 16, kind, block, seed=3)
    window, sinks = 130, 20
    d = case.dev(marlin)
    want, _ = attend(marlin, case, d, window=window, sinks=sinks)
    hidden = np.ones((case.pages, 16), bool)
    for b, n in enumerate(case.lengths):
        at = np.arange(n)
        at = at[(at > n - 1 - window) | (at < sinks)]
        hidden[case.table[b][at // 16], at % 16] = False
    where = torch.from_numpy(hidden).cuda()[:, None, :, None]
    for x in ("k_cache", "v_cache"):
        if kind == "fp16":
            d[x].masked_fill_(where, float("nan"))
            d[x][:, :, 1::2].masked_fill_(where[:, :, 1::2], float("inf"))
        elif kind == "e4m3":
            d[x].view(torch.uint8).masked_fill_(where, 0x7f)
    if block:
        whole = torch.from_numpy(hidden.reshape(case.pages, -1, block).all(-1)).cuda()[:, None]
        d["k_scale"].masked_fill_(whole, float("nan"))
        d["v_scale"].masked_fill_(whole, float("inf"))
    got, _ = attend(marlin, case, d, window=window, sinks=sinks)
    assert torch.equal(got, want)
    assert marlin.read_status(d["workspace"]) == 0


@pytest.mark.parametrize("kind,block", KINDS)
@pytest.mark.parametrize("q_heads,dim", [(2, 128), (10, 128), (5, 64), (3, 256)])
def test_what_some_rows_see_reaches_these_only(marlin, kind, block, q_heads, dim):
    # seven new tokens: values that are not finite in the newest ones and at the edge of the window
    import torch
    case = BlockCase([700], 7, q_heads, 1, dim, 16, kind, block, seed=4)
    window, sinks = 130, 3
    first = 700 - 7
    d = case.dev(marlin)
    odd = [first + 4, first - window + 3, 5]  # a new token, one that the first two rows see, one that nobody sees
    by_scale = block == 1
    if by_scale:  # (what is not finite has no part in the units of the sums, no more than 0 has)
        for pos in odd:
            d["v_scale"][int(case.table[0][pos // 16]), :, pos % 16] = 0
    clean, _ = attend(marlin, case, d, window=window, sinks=sinks)
    clean = clean.view(7, q_heads, dim)
    for pos in odd:
        page, slot = int(case.table[0][pos // 16]), pos % 16
        if by_scale:
            d["v_scale"][page, :, slot] = float("inf")
        elif kind == "fp16":
            d["v_cache"][page, :, slot, 1] = float("inf")
        elif kind == "e4m3":
            d["v_cache"].view(torch.uint8)[page, :, slot, 1] = 0x7f
        else:
            return  # (two's complement has nothing that is not finite)
    got, _ = attend(marlin, case, d, window=window, sinks=sinks)
    got = got.view(7, q_heads, dim)
    for t in range(7):
        p = first + t
        hit = any(pos <= p and pos > p - window for pos in odd)
        if not hit:
            assert torch.equal(got[t], clean[t])
        elif by_scale:
            assert not torch.isfinite(got[t]).all(-1).any()
        else:
            assert not torch.isfinite(got[t][:, 1]).any()
            assert torch.isfinite(got[t][:, 2:]).all()
    # 0 times such a value must not reach the others: every element but the odd one is as before, up to the order of sums
    if not by_scale:
        assert torch.equal(got[:, :, 2:], clean[:, :, 2:])


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("q_heads,dim", [(4, 128), (48, 128), (12, 64)])
def test_scales_of_very_different_sizes(marlin, kind, q_heads, dim):
    case = BlockCase([2000, 130, 4000], 1, q_heads, 1, dim, 32, kind, 8, seed=5)
    rng = np.random.default_rng(6)
    case.v_scale = (case.v_scale * 2.0 ** rng.integers(-12, 13, case.v_scale.shape)).astype(np.float32)
    case.v_scale[rng.random(case.v_scale.shape) < 0.1] = 0
    case.k_scale[rng.random(case.k_scale.shape) < 0.1] = 0
    check(marlin, case)
    case.v_scale[:] = 0
    out, _ = check(marlin, case)
    assert not out.any()


@pytest.mark.parametrize("scale", [0.0, -0.1])
@pytest.mark.parametrize("kind,block", [("fp16", 0), ("int8", 8)])
@pytest.mark.parametrize("q_heads", [4, 48])
def test_scales_of_logits_that_are_not_positive(marlin, scale, kind, block, q_heads):
    check(marlin, BlockCase([200, 700, 0], 3, q_heads, 1, 128, 16, kind, block), window=150, sinks=10, scale=scale)


@pytest.mark.parametrize("kind,block,q_heads", [("fp16", 0, 16), ("int8", 64, 40), ("e4m3", 64, 48), ("int8", 16, 8)])
def test_long_sequences(marlin, kind, block, q_heads):
    # parts of many CTAs, and more tiles than are summed in one go; all but a few tokens in front of a window of most of them
    case = BlockCase([140001, 20011], 1, q_heads, 1, 128, 128, kind, block, seed=8)
    check(marlin, case)
    check(marlin, case, window=30000, sinks=1000)


@pytest.mark.parametrize("kind,block", KINDS)
def test_rows_of_nobody_are_left_as_they_are_and_calls_repeat(marlin, kind, block):
    import torch
    case = BlockCase([100, 50, 0], [2, 3, 2], 8, 2, 64, 16, kind, block)
    d = case.dev(marlin)
    out, _ = attend(marlin, case, d, window=40, sinks=4)
    q = torch.from_numpy(case.q.reshape(case.T, -1)).cuda()
    more = torch.cat([torch.full((3, q.shape[1]), float("nan"), device="cuda", dtype=q.dtype), q, torch.full((5, q.shape[1]), float("nan"), device="cuda", dtype=q.dtype)])
    marked = torch.full_like(more, 7.0)
    starts = d["starts"] + 3
    for _ in range(3):
        got = marlin.attention_decode(more, **{**d, "starts": starts}, window=40, sinks=4, out=marked)
        assert got is marked
        assert torch.equal(got[3:-5], out) and (got[:3] == 7).all() and (got[-5:] == 7).all()
    assert not out[5:].any()  # (an empty sequence: zeros)
    assert marlin.read_status(d["workspace"]) == 0


@pytest.mark.parametrize("kind,block", [("fp16", 0), ("int8", 8)])
@pytest.mark.parametrize("q_heads,dim", [(4, 64), (32, 128)])
def test_pages_that_are_not_there(marlin, kind, block, q_heads, dim):
    import torch
    case = BlockCase([300, 300], 1, q_heads, 1, dim, 16, kind, block)
    case.table[0, 0] = case.pages  # of the sinks
    case.table[0, 12] = -5         # of the window
    out, d = attend(marlin, case, window=150, sinks=20)
    assert marlin.read_status(d["workspace"]) == 9
    ref = case.sinks_ref(dim ** -0.5, 150, 20)
    assert np.all(np.abs(out.float().cpu().numpy().reshape(ref[0].shape) - ref[0]) <= case.sinks_bound(ref))
    d["workspace"].zero_()
    d["lengths"][1] = -2  # a sequence that kv_reserve has refused
    got, _ = attend(marlin, case, d, window=150, sinks=20)
    assert marlin.read_status(d["workspace"]) == 9
    assert not got[1].any()


@pytest.mark.parametrize("kind,block", [("fp16", 0), ("e4m3", 0), ("int8", 8)])
def test_a_captured_call_on_another_stream_follows_the_lengths(marlin, kind, block):
    import torch
    case = BlockCase([900, 300, 20], 1, 16, 2, 128, 16, kind, block)
    d = case.dev(marlin)
    q = torch.from_numpy(case.q.reshape(case.T, -1)).cuda()
    side = torch.cuda.Stream()
    out = torch.empty_like(q)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        marlin.attention_decode(q, **d, window=64, sinks=4, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        marlin.attention_decode(q, **d, window=64, sinks=4, out=out)
    full = case.lengths.copy()
    for cut in (0, 1, 19):
        d["lengths"].copy_(torch.from_numpy(full - cut))
        graph.replay()
        torch.cuda.synchronize()
        case.lengths = (full - cut).astype(np.int32)
        ref = case.sinks_ref(128 ** -0.5, 64, 4)
        assert np.all(np.abs(out.float().cpu().numpy().reshape(ref[0].shape) - ref[0]) <= case.sinks_bound(ref))
    assert marlin.read_status(d["workspace"]) == 0


def test_without_sinks_or_blocks_it_is_the_call_that_it_was(marlin):
    # e4m3 with scales per key head: the same values through both entries, within the bounds of both
    import torch
    case = BlockCase([900, 33], 1, 8, 2, 128, 16, "e4m3", 0)
    d = case.dev(marlin)
    a, _ = attend(marlin, case, d)
    by_block = {**d, "k_scale": d["k_scale"][None, :, None].repeat(case.pages, 1, 1).contiguous(), "v_scale": d["v_scale"][None, :, None].repeat(case.pages, 1, 1).contiguous()}
    b, _ = attend(marlin, case, by_block)
    ref = case.sinks_ref(128 ** -0.5)
    for x in (a, b):
        assert np.all(np.abs(x.float().cpu().numpy().reshape(ref[0].shape) - ref[0]) <= case.sinks_bound(ref) + 2.0 ** -31 * 0.09 * 448 * 900)


def test_refusals(marlin):
    case = BlockCase([100, 50], 1, 8, 2, 64, 16, "int8", 4)
    d = case.dev(marlin)
    s = d["k_scale"]
    for wrong in (dict(k_scale=None), dict(v_scale=None), dict(k_scale=s[:, :, :3]), dict(k_scale=s[:-1]), dict(k_scale=s[:, :1]), dict(k_scale=s[0, :, 0]),
                  dict(v_scale=s.transpose(0, 1).contiguous().transpose(0, 1)), dict(k_scale=s[:, :, :3], v_scale=s[:, :, :3])):
        with pytest.raises(ValueError):
            attend(marlin, case, d, **wrong)
    with pytest.raises(TypeError):
        attend(marlin, case, d, k_scale=s.double())
    with pytest.raises(marlin.MarlinError):
        attend(marlin, case, d, sinks=-1, window=5)
    with pytest.raises(marlin.MarlinError):
        attend(marlin, case, d, window=-1)
    half = BlockCase([100, 50], 1, 8, 2, 64, 16, "fp16")
    with pytest.raises(ValueError, match="8-bit"):
        attend(marlin, half, None, k_scale=s, v_scale=s)
