"""Attention over the paged cache (marlin_attention_decode) against its definition in 64 bits.  The bound is derived in
cache_util.attention_bound."""
import numpy as np
import pytest

from cache_util import Case, attention_bound

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def marlin():
    import torch
    assert torch.cuda.is_available()
    import paper_2408_11743_b200 as m
    m.lib()
    return m


def run(marlin, case, window=0, scale=None, q=None, d=None, **more):
    import torch
    d = d or case.dev(marlin)
    q = torch.from_numpy(case.q.reshape(case.T, -1)).cuda() if q is None else q
    out = marlin.attention_decode(q, window=window, scale=scale, **d, **more)
    torch.cuda.synchronize()
    assert marlin.read_status(d["workspace"]) == 0
    assert not d["workspace"][256:8192].any()  # counters are left zero
    return out


def check(case, out, window=0, scale=None):
    ref = case.attention_ref(case.dim ** -0.5 if scale is None else scale, window)
    got = out.cpu().numpy().astype(np.float64).reshape(ref[0].shape)
    worst = np.max(np.abs(got - ref[0]) / attention_bound(ref))
    assert worst <= 1.0, worst


EDGES = [0, 1, 2, 15, 16, 17, 48, 63, 64, 65, 100, 127, 128, 129, 700]


@pytest.mark.parametrize("q_heads,kv_heads,dim,page", [
    (4, 4, 128, 16), (8, 1, 128, 16), (16, 2, 64, 32), (29, 1, 64, 8), (71, 1, 64, 16), (3, 3, 80, 16), (4, 2, 16, 4), (6, 2, 48, 64),
    (8, 2, 256, 16), (40, 1, 256, 32), (2, 2, 192, 1), (5, 1, 112, 256), (64, 2, 128, 2), (17, 1, 128, 128), (130, 2, 32, 16),
    (40, 1, 128, 16), (96, 2, 112, 8), (34, 1, 128, 1)])
@pytest.mark.parametrize("eight_bit", [False, True])
def test_single_tokens_at_every_edge_of_the_lengths(marlin, q_heads, kv_heads, dim, page, eight_bit):
    case = Case(EDGES, 1, q_heads, kv_heads, dim, page, eight_bit, seed=q_heads + dim)
    out = run(marlin, case)
    check(case, out)
    assert not out[0].any()  # nothing to see: zeros


@pytest.mark.parametrize("q_heads,kv_heads,dim,new", [
    (8, 8, 128, [3, 0, 5, 1, 2, 4, 6, 0]), (16, 2, 128, [6, 1, 2, 6, 0, 3, 4, 5]), (32, 1, 64, [1, 2, 3, 4, 5, 4, 3, 2]),
    (4, 1, 256, [9, 16, 1, 0, 4, 17, 2, 3]), (7, 1, 80, [40, 1, 70, 3, 5, 64, 2, 1]),
    (24, 2, 128, [9, 1, 3, 5, 6, 4, 2, 8])])
@pytest.mark.parametrize("eight_bit", [False, True])
@pytest.mark.parametrize("window", [0, 1, 37, 64, 150])
def test_several_new_tokens_and_windows(marlin, q_heads, kv_heads, dim, new, eight_bit, window):
    # sequence 0 has fewer tokens than rows: the first of them have no position and see nothing
    case = Case([2, 40, 64, 65, 130, 200, 17, 333], new, q_heads, kv_heads, dim, 16, eight_bit, seed=dim + window)
    out = run(marlin, case, window)
    check(case, out, window)
    if new[0] > 2:
        assert not out[:new[0] - 2].any()


@pytest.mark.parametrize("window", [1, 5, 63, 64, 65, 1000])
def test_windows_of_single_tokens(marlin, window):
    case = Case(EDGES, 1, 8, 2, 128, 16, seed=window)
    check(case, run(marlin, case, window), window)


@pytest.mark.parametrize("layout", ["heads", "tokens", "wide"])
@pytest.mark.parametrize("eight_bit", [False, True])
def test_layouts_of_the_cache(marlin, layout, eight_bit):
    case = Case([5, 64, 200, 91], [2, 1, 3, 1], 8, 4, 64, 8, eight_bit, layout=layout, seed=11)
    check(case, run(marlin, case))


@pytest.mark.parametrize("lengths,q_heads,kv_heads,new,dim", [
    ([33001], 8, 8, 1, 64), ([20000, 3, 9000], 8, 1, 1, 64), ([16384, 16385], 24, 1, [3, 4], 64), ([50] * 700, 2, 2, 1, 64),
    (list(range(1, 300)), 4, 1, 1, 64), ([9000, 40, 12345], 16, 1, [3, 4, 3], 128), ([70] * 300, 40, 1, 1, 128)])
@pytest.mark.parametrize("eight_bit", [False, True])
def test_long_sequences_and_many(marlin, lengths, q_heads, kv_heads, new, dim, eight_bit):
    # parts of one sequence on many CTAs, several sequences on one CTA
    case = Case(lengths, new, q_heads, kv_heads, dim, 16, eight_bit, seed=len(lengths))
    d = case.dev(marlin)
    d["workspace"][8192:] = 0xFF  # slots are written before they are read
    first = run(marlin, case, d=d)
    check(case, first)
    again = run(marlin, case, d=d)
    assert (first == again).all()  # the same bits every time


def test_scale_and_column_ranges(marlin):
    import torch
    case = Case([77, 130, 1], 1, 8, 2, 64, 16, seed=5)
    wide = torch.full((3, 8 * 64 + 72), float("nan"), dtype=torch.float16, device="cuda")
    q = wide[:, 40:40 + 8 * 64]
    q.copy_(torch.from_numpy(case.q.reshape(3, -1)))
    out = torch.full((3, 8 * 64), float("nan"), dtype=torch.float16, device="cuda")
    for scale in (0.0, 0.3, -0.2):
        assert run(marlin, case, scale=scale, q=q, out=out) is out
        check(case, out, scale=scale)


@pytest.mark.parametrize("q_heads", [4, 12, 20, 40])
@pytest.mark.parametrize("eight_bit", [False, True])
@pytest.mark.parametrize("scale", [0.0, -0.2])
def test_scales_that_are_not_positive(marlin, q_heads, eight_bit, scale):
    # what is hidden stays hidden: in the last tile, around the new tokens and at the edge of a window
    for new, window in ((1, 0), ([3, 1, 2, 5], 0), ([3, 1, 2, 5], 30)):
        case = Case([70, 1, 130, 129], new, q_heads, 1, 128, 16, eight_bit, seed=q_heads)
        if eight_bit and scale:  # (a sign of its own)
            case.k_scale = -case.k_scale
        check(case, run(marlin, case, window, scale=scale), window, scale=scale)


@pytest.mark.parametrize("q_heads", [4, 20])
def test_windows_as_long_as_can_be(marlin, q_heads):
    import torch
    case = Case([3, 40, 300], [5, 2, 1], q_heads, 1, 64, 16, seed=q_heads)
    d = case.dev(marlin)
    plain = run(marlin, case, d=d)
    for window in (2 ** 31 - 1, 2 ** 30, case.table.shape[1] * 16):
        assert torch.equal(run(marlin, case, window, d=d), plain)


def test_values_that_no_token_sees_do_not_matter(marlin):
    # everything that is not a key or a value of some sequence is NaN, also behind the last token on its page
    import torch
    for eight_bit in (False, True):
        case = Case([3, 64, 129, 90], 1, 8, 2, 64, 16, eight_bit, seed=3)
        d = case.dev(marlin)
        plain = run(marlin, case, d=d)
        windowed = run(marlin, case, window=20, d=d)
        for window, want in ((0, plain), (20, windowed)):
            k, v = d["k_cache"].clone(), d["v_cache"].clone()
            seen = torch.zeros(case.pages, case.page, dtype=torch.bool)
            for b, n in enumerate(case.lengths):
                at = np.arange(max(0, n - window) if window else 0, n)
                seen[case.table[b][at // case.page], at % case.page] = True
            hide = ~seen.cuda()[:, None, :, None].expand(k.shape)
            for x in (k, v):
                bits = x.view(torch.uint8 if eight_bit else torch.int16)
                bits[hide] = 0x7F if eight_bit else 0x7E00
            got = run(marlin, case, window=window, d={**d, "k_cache": k, "v_cache": v})
            assert torch.equal(got, want)


@pytest.mark.parametrize("eight_bit", [False, True])
@pytest.mark.parametrize("q_heads,dim", [(2, 64), (12, 64), (24, 64), (3, 128), (12, 128)])
def test_infinities_and_nan_reach_the_tokens_that_see_them_alone(marlin, q_heads, dim, eight_bit):
    import torch
    case = Case([40, 80], [5, 4], q_heads, 1, dim, 16, eight_bit, seed=9)
    d = case.dev(marlin)
    want = run(marlin, case, d=d)
    k, v = d["k_cache"].clone(), d["v_cache"].clone()

    def at(b, pos):
        return int(case.table[b][pos // 16]), 0, pos % 16
    nan, inf = float("nan"), float("inf")
    if eight_bit:
        v.view(torch.uint8)[at(0, 38)][7] = 0x7F
        k.view(torch.uint8)[at(1, 79)][:] = 0x7F
    else:
        v[at(0, 38)][7], v[at(0, 37)][8], v[at(0, 38)][9], v[at(0, 37)][10], v[at(0, 39)][10] = nan, inf, -inf, inf, -inf
        k[at(1, 79)][:] = nan
    got = run(marlin, case, d={**d, "k_cache": k, "v_cache": v}).view(9, q_heads, dim)
    want = want.view(9, q_heads, dim).clone()
    # sequence 0 has positions 35 .. 39 in rows 0 .. 4, sequence 1 76 .. 79 in rows 5 .. 8
    want[3:5, :, 7] = nan
    if not eight_bit:
        want[2:5, :, 8], want[3:5, :, 9], want[2:4, :, 10], want[4, :, 10] = inf, -inf, inf, nan
    want[8] = nan
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    fine = ~torch.isnan(want)
    assert torch.equal(got[fine], want[fine])


def test_logits_of_all_sizes(marlin):
    # logits of +-60000, all equal, all -inf, one +inf
    import torch
    case = Case([70, 70, 70, 70], 1, 4, 1, 64, 16, seed=2)
    d = case.dev(marlin)
    q = torch.zeros(4, 4, 64, dtype=torch.float16, device="cuda")
    q[0] = torch.from_numpy(case.q[0]).cuda() * 400
    q[2, :, 0] = float("-inf")
    k = d["k_cache"]
    k[..., 0] = 1.0
    out = run(marlin, case, q=q.view(4, -1), d=d)
    case.q = q.cpu().numpy()
    case.k_t = k.cpu()
    ref = case.attention_ref(0.125)
    got = out.cpu().numpy().astype(np.float64).reshape(ref[0].shape)
    bound = attention_bound(ref)
    for b in (0, 1, 3):
        assert np.all(np.abs(got - ref[0])[b] <= bound[b])
    assert np.isnan(got[2]).all() and np.isnan(ref[0][2]).all()  # -inf - -inf, as the formula has it


def test_rows_of_nobody_are_left_as_they_were(marlin):
    import torch
    case = Case([20, 30], [2, 3], 4, 2, 64, 16, seed=8)
    d = case.dev(marlin)
    d["starts"] = d["starts"] + 2
    q = torch.full((12, 4 * 64), float("nan"), dtype=torch.float16, device="cuda")
    q[2:7] = torch.from_numpy(case.q.reshape(5, -1)).cuda()
    out = torch.full_like(q, 7.0)
    run(marlin, case, q=q, d=d, out=out)
    assert (out[:2] == 7).all() and (out[7:] == 7).all()
    check(case, out[2:7])


def test_what_points_outside_of_the_cache_is_reported(marlin):
    import torch
    case = Case([40, 50], 1, 4, 2, 64, 16, seed=8)
    q = torch.from_numpy(case.q.reshape(2, -1)).cuda()
    for what, value in (("pages", case.pages), ("pages", -1), ("pages", 2 ** 31 - 1), ("lengths", 65), ("lengths", -1)):
        d = case.dev(marlin)
        (d["pages"][0, :1] if what == "pages" else d["lengths"][:1]).fill_(value)
        if what == "lengths" and value == 65:
            d["pages"] = d["pages"][:, :4].clone()
            d["pages"][0] = 0
        out = marlin.attention_decode(q, **d)
        assert marlin.read_status(d["workspace"]) == 9
        ref = case.attention_ref(0.125)
        got = out.cpu().numpy().astype(np.float64).reshape(ref[0].shape)
        assert np.all(np.abs(got - ref[0])[1] <= attention_bound(ref)[1])  # the other sequence is as it was


def test_starts_that_descend_or_point_outside_touch_nothing_else(marlin):
    import torch
    case = Case([40, 50, 60], 1, 4, 2, 64, 16, seed=8)
    q = torch.from_numpy(case.q.reshape(3, -1)).cuda()
    d = case.dev(marlin)
    big = torch.full((9, 256), 7.0, dtype=torch.float16, device="cuda")
    for starts in ([0, 3, 1, 2 ** 31 - 1], [-5, -1, 2, 3], [3, 2, 1, 0], [9, 9, 9, 9]):
        marlin.attention_decode(q, **d, starts=torch.tensor(starts, dtype=torch.int32, device="cuda"), out=big[3:6])
        torch.cuda.synchronize()
        assert (big[:3] == 7).all() and (big[6:] == 7).all()
        assert not d["workspace"][256:8192].any()


def test_offsets_beyond_32_bits(marlin):
    import torch
    case = Case([200, 100], 1, 8, 8, 128, 16, seed=4)
    stride = 16 * 8 * 128
    pages = (1 << 31) // stride + 40  # more than 2^31 elements
    d = case.dev(marlin)
    k = torch.empty(pages, 8, 16, 128, dtype=torch.float16, device="cuda")
    v = torch.empty_like(k)
    k[-case.pages:], v[-case.pages:] = d["k_cache"], d["v_cache"]
    table = torch.where(d["pages"] >= 0, d["pages"] + (pages - case.pages), d["pages"])
    want = run(marlin, case, d=d)
    got = run(marlin, case, d={**d, "k_cache": k, "v_cache": v, "pages": table})
    assert torch.equal(got, want)


def test_captured_calls_follow_the_lengths(marlin):
    # captured with short sequences, replayed with long ones: the work is shared out on the device
    import torch
    case = Case([5000, 3, 1200, 64], 1, 8, 2, 128, 16, seed=6)
    d = case.dev(marlin)
    q = torch.from_numpy(case.q.reshape(4, -1)).cuda()
    lengths = d["lengths"].clone()
    want = run(marlin, case, d=d)
    d["lengths"].fill_(1)
    out = torch.empty_like(want)
    graphs = []
    for _ in range(2):  # two graphs that share a workspace, one after the other
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            marlin.attention_decode(q, **d, out=out)
        graphs.append(graph)
    graphs[0].replay()
    d["lengths"].copy_(lengths)
    for graph in graphs:
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    assert marlin.read_status(d["workspace"]) == 0


def test_another_stream(marlin):
    import torch
    case = Case([900, 30], 1, 8, 2, 128, 16, seed=6)
    d = case.dev(marlin)
    want = run(marlin, case, d=d)
    q = torch.from_numpy(case.q.reshape(2, -1)).cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = marlin.attention_decode(q, **d, stream=side)
    with torch.cuda.stream(side):
        inside = marlin.attention_decode(q, **d)
    side.synchronize()
    assert torch.equal(got, want) and torch.equal(inside, want)
