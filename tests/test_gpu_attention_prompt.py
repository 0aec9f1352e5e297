"""GPU: attention of prompts (many new tokens of a sequence at a time) through windows with sinks, against the formula in 64 bits."""
import numpy as np
import pytest

from blocks_util import BlockCase
from test_gpu_attention_sinks import attend

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def marlin():
    import torch
    assert torch.cuda.is_available()
    import paper_2408_11743_b200 as m
    m.lib()
    return m


def check(marlin, case, window=0, sinks=0, scale=None):
    scale = case.dim ** -0.5 if scale is None else scale
    out, d = attend(marlin, case, window=window, sinks=sinks, scale=scale)
    assert marlin.read_status(d["workspace"]) == 0
    ref = case.sinks_ref_on_gpu(float(np.float32(scale)), window, sinks)
    got = out.float().cpu().numpy().reshape(ref[0].shape)
    bad = ~(np.abs(got - ref[0]) <= case.sinks_bound(ref))
    assert not bad.any(), f"{bad.sum()} of {bad.size} off, the first at {np.argwhere(bad)[0]}: {got[bad][0]} for {ref[0][bad][0]}"


# 24 blocks of 256 rows at least, 128 rows a sequence and key head: the kernel for prompts
SHAPES = [(8, 1, 128), (1, 1, 128), (24, 8, 64), (29, 1, 64), (71, 1, 48), (12, 4, 80), (5, 1, 112), (16, 1, 16)]


def prompts(q_heads, kv_heads, dim, page, layout="heads", seed=0):
    group = q_heads // kv_heads
    n = max(200, 24 * 256 // (group * kv_heads * 4) + 40)  # tokens of a sequence, about
    lengths = [n, n + 333, 1, 0, 2 * n + 7, 150]
    return BlockCase(lengths, [n, n - 5, 1, 3, 2 * n, 150], q_heads, kv_heads, dim, page, "fp16", 0, layout, seed)


@pytest.mark.parametrize("q_heads,kv_heads,dim", SHAPES)
@pytest.mark.parametrize("window,sinks", [(100, 5), (1, 0), (129, 300), (300, 128)])
def test_windows(marlin, q_heads, kv_heads, dim, window, sinks):
    check(marlin, prompts(q_heads, kv_heads, dim, 16, seed=window), window=window, sinks=sinks)


@pytest.mark.parametrize("q_heads,kv_heads,dim", SHAPES[:5])
def test_without_a_window(marlin, q_heads, kv_heads, dim):
    # (sinks mean nothing then; they choose the entry)
    check(marlin, prompts(q_heads, kv_heads, dim, 64, seed=1), window=0, sinks=1)
    check(marlin, prompts(q_heads, kv_heads, dim, 64, seed=2), window=10 ** 6, sinks=1)


@pytest.mark.parametrize("page", [1, 4, 16, 128, 512])
@pytest.mark.parametrize("layout", ["heads", "tokens", "wide"])
def test_pages_and_layouts(marlin, page, layout):
    check(marlin, prompts(16, 2, 128, page, layout, seed=page), window=200, sinks=30)
    check(marlin, prompts(16, 2, 64, page, layout, seed=page), window=0, sinks=1)


@pytest.mark.parametrize("scale", [0.0, -0.1, 3.0])
def test_scales_of_logits(marlin, scale):
    # (3: logits of some hundreds, bases that move from tile to tile)
    check(marlin, prompts(16, 2, 128, 16, seed=7), window=300, sinks=4, scale=scale)
    check(marlin, prompts(16, 2, 64, 16, seed=8), window=0, sinks=4, scale=scale)


@pytest.mark.parametrize("dim", [128, 64])
def test_logits_that_grow_along_the_keys(marlin, dim):
    # every tile moves the bases of all rows
    import torch
    case = prompts(16, 2, dim, 16, seed=9)
    for b, n in enumerate(case.lengths):
        for p in range(int(n)):
            case.k_t[case.table[b][p // 16], :, p % 16] *= (p + 1) / 200
    case.k_t = case.k_t.to(torch.float16)
    check(marlin, case, window=0, sinks=1)
    check(marlin, case, window=500, sinks=10)


@pytest.mark.parametrize("dim", [128, 64])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_values_that_are_not_finite_reach_the_rows_that_see_them(marlin, dim, value):
    import torch
    case = prompts(16, 2, dim, 16, seed=10)
    window, sinks = 100, 10
    d = case.dev(marlin)
    clean, _ = attend(marlin, case, d, window=window, sinks=sinks)
    n = int(case.lengths[4])
    odd = [3, 40, 257, 300, n - 1]  # a sink, and positions that few see
    for pos in odd:
        d["v_cache"][int(case.table[4][pos // 16]), :, pos % 16, 5] = value
        if pos > sinks:  # (a key that is not finite: rows that see it are lost, others are as they were)
            d["k_cache"][int(case.table[4][pos // 16]), 1, pos % 16, 2] = value
    got, _ = attend(marlin, case, d, window=window, sinks=sinks)
    first = int(case.starts[4])
    assert torch.equal(got[:first], clean[:first]) and torch.equal(got[int(case.starts[5]):], clean[int(case.starts[5]):])
    got, clean = (t[first:int(case.starts[5])].view(-1, 16, dim) for t in (got, clean))
    for t in range(got.shape[0]):
        p = n - got.shape[0] + t
        hit = [o for o in odd if o <= p and (o > p - window or o < sinks)]
        if not hit:
            assert torch.equal(got[t], clean[t]), t
            continue
        assert not torch.isfinite(got[t][:8, 5]).any()
        keep = torch.arange(dim) != 5
        assert torch.equal(got[t][:8][:, keep], clean[t][:8][:, keep]), t
        if any(o > sinks for o in hit) and value != value:
            assert got[t][8:].isnan().all()


def test_hidden_places_do_not_matter_and_calls_repeat(marlin):
    import torch
    case = prompts(16, 2, 128, 16, seed=11)
    d = case.dev(marlin)
    window, sinks = 150, 20
    want, _ = attend(marlin, case, d, window=window, sinks=sinks)
    hidden = np.ones((case.pages, 16), bool)
    for b, n in enumerate(case.lengths):
        n, new = int(n), case.new[b]
        at = np.arange(n)
        at = at[(at > max(n - new, 0) - window) | (at < sinks)]
        hidden[case.table[b][at // 16], at % 16] = False
    where = torch.from_numpy(hidden).cuda()[:, None, :, None]
    for x in ("k_cache", "v_cache"):
        d[x].masked_fill_(where, float("nan"))
    for _ in range(3):
        got, _ = attend(marlin, case, d, window=window, sinks=sinks)
        assert torch.equal(got, want)
    assert marlin.read_status(d["workspace"]) == 0


def test_rows_of_nobody_and_pages_that_are_not_there(marlin):
    import torch
    case = prompts(16, 2, 128, 16, seed=12)
    case.table[0, 1], case.table[4, 20] = case.pages, -1
    d = case.dev(marlin)
    q = torch.from_numpy(case.q.reshape(case.T, -1)).cuda()
    wide = torch.full((case.T + 9, 2 * q.shape[1] + 8), float("nan"), device="cuda", dtype=q.dtype)
    wide[4:-5, 8:8 + q.shape[1]] = q
    marked = torch.full((case.T + 9, q.shape[1]), 7.0, device="cuda", dtype=q.dtype)
    marlin.attention_decode(wide[:, 8:8 + q.shape[1]], **{**d, "starts": d["starts"] + 4}, window=150, sinks=20, out=marked)
    assert marlin.read_status(d["workspace"]) == 9
    assert (marked[:4] == 7).all() and (marked[-5:] == 7).all()
    ref = case.sinks_ref_on_gpu(128 ** -0.5, 150, 20)
    assert np.all(np.abs(marked[4:-5].float().cpu().numpy().reshape(ref[0].shape) - ref[0]) <= case.sinks_bound(ref))


def test_long_prompts_behind_long_contexts(marlin):
    case = BlockCase([33000, 2500], [300, 2500], 16, 2, 128, 128, "fp16", seed=13)
    for window, sinks in ((32000, 700), (1000, 4)):  # most of 32 thousand keys
        check(marlin, case, window, sinks)


def test_both_sides_of_the_choice_agree(marlin):
    # calls with a little too few rows, and ones that see too far, for the kernel for prompts
    for tokens, kv_heads, span in ((760, 8, 100), (780, 8, 100), (780, 8, 32768), (780, 8, 32769), (127, 40, 50), (128, 40, 50)):
        check(marlin, BlockCase([max(1000, tokens)] if span < 1000 else [36000], [tokens], kv_heads, kv_heads, 64, 64, "fp16", seed=tokens), window=span - 1, sinks=1)


def test_captured_on_another_stream(marlin):
    import torch
    case = prompts(16, 2, 128, 16, seed=14)
    d = case.dev(marlin)
    q = torch.from_numpy(case.q.reshape(case.T, -1)).cuda()
    want, _ = attend(marlin, case, d, window=150, sinks=20)
    side, out = torch.cuda.Stream(), torch.empty_like(q)
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        for _ in range(3):
            marlin.attention_decode(q, **d, window=150, sinks=20, out=out)
    out.fill_(float("nan"))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
