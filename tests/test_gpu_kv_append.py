"""Appending to the paged cache (marlin_kv_append) against its definition in 64 bits.

A rotated value is a product of two fp32 roundings each of cosine, sine and the products, and rounded once: it may be off by
half a step of its type at its own size (fp16 2^-11, 2^-25 below 2^-14; e4m3 2^-4, 2^-10 below 2^-6) plus 2^-21 of |a| + |c|
(sine and cosine are off by 2^-23 of their largest value after a reduction in 64 bits, the products and their sum by 2^-24 each)."""
import numpy as np
import pytest

from cache_util import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def marlin():
    import torch
    assert torch.cuda.is_available()
    import paper_2408_11743_b200 as m
    m.lib()
    return m


def frequencies(rotary):
    return (10000.0 ** (-np.arange(rotary // 2) * 2.0 / max(rotary, 1))).astype(np.float32)


def want_of(case, rotary, interleaved):
    """(q, {(sequence, position): (k, v)}, size of what is turned) in float64; keys and values in units of the cache."""
    from oracle import attention_ref as ref
    x = case.qkv.astype(np.float64).reshape(case.T, -1, case.dim)
    q = np.zeros((case.T, case.q_heads, case.dim))
    put = {}
    H, K = case.q_heads, case.kv_heads
    for t, b, p in ref.positions(case.lengths, case.starts):
        if p < 0:
            continue
        y = ref.rotate(x[t, :H + K], int(p), frequencies(rotary), interleaved)
        q[t] = y[:H]
        k, v = y[H:], x[t, H + K:]
        if case.eight_bit:
            k, v = k / case.k_scale[:, None].astype(np.float64), v / case.v_scale[:, None].astype(np.float64)
        put[b, int(p)] = k, v
    return q, put


def allowed(want, size, eight_bit):
    if not eight_bit:
        return np.maximum(2.0 ** -11 * np.abs(want), 2.0 ** -25) + 2.0 ** -21 * size
    return np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10) + 2.0 ** -20 * size


CASES = [
    # lengths, new, q_heads, kv_heads, dim, page, rotary, interleaved
    ([1, 16, 17, 300], 1, 32, 32, 128, 16, 128, False),
    ([5, 64, 65], 1, 64, 8, 128, 16, 128, False),
    ([1000000, 2, 129], 1, 4, 2, 64, 4096, 64, True),
    ([9, 40, 3, 77], [3, 0, 2, 40], 8, 2, 64, 8, 32, False),
    ([9, 40, 3, 77], [3, 0, 2, 40], 8, 2, 64, 8, 32, True),
    ([2, 5], [4, 1], 6, 2, 80, 4, 48, False),     # fewer tokens than rows
    ([0, 7, 0], 1, 2, 1, 16, 1, 16, False),       # empty sequences of a padded batch
    ([31, 33], [31, 33], 5, 5, 256, 32, 256, False),
    ([200], [200], 71, 1, 64, 16, 16, True),
    ([8, 9], 1, 130, 2, 192, 2, 96, False),
    ([33] * 300, 1, 2, 2, 32, 16, 32, False),
]


@pytest.mark.parametrize("lengths,new,q_heads,kv_heads,dim,page,rotary,interleaved", CASES)
@pytest.mark.parametrize("eight_bit", [False, True])
@pytest.mark.parametrize("layout", ["heads", "tokens"])
def test_rotated_and_in_its_place(marlin, lengths, new, q_heads, kv_heads, dim, page, rotary, interleaved, eight_bit, layout):
    import torch
    case = Case(lengths, new, q_heads, kv_heads, dim, page, eight_bit, layout, seed=dim + len(lengths))
    d = case.dev(marlin)
    before = [d["k_cache"].float().cpu().numpy(), d["v_cache"].float().cpu().numpy()]
    q = marlin.kv_append(torch.from_numpy(case.qkv).cuda(), **d, inv_freq=torch.from_numpy(frequencies(rotary)).cuda(),
                         interleaved=interleaved)
    torch.cuda.synchronize()
    assert marlin.read_status(d["workspace"]) == 0
    q_want, put = want_of(case, rotary, interleaved)
    got = q.cpu().numpy().astype(np.float64).reshape(q_want.shape)
    most = float(np.abs(case.qkv.astype(np.float64)).max())
    assert np.all(np.abs(got - q_want) <= allowed(q_want, 2 * most, False))
    after = [d["k_cache"].float().cpu().numpy(), d["v_cache"].float().cpu().numpy()]
    touched = np.zeros(before[0].shape, bool)
    for (b, p), kv in put.items():
        at = case.table[b][p // page], slice(None), p % page
        touched[at] = True
        for cache, want, scale in zip(after, kv, (case.k_scale, case.v_scale)):
            size = 2 * most / (scale.min() if eight_bit else 1.0)
            assert np.all(np.abs(cache[at].astype(np.float64) - want) <= allowed(want, size, eight_bit))
    for x, y in zip(before, after):
        assert np.array_equal(x[~touched], y[~touched])  # nothing else is written


def test_far_positions(marlin):
    # one page table row of a billion tokens, of which only the last page is there
    import torch
    n, page = 1_000_000_007, 1 << 20
    case = Case([7], 1, 4, 2, 64, 16, seed=1)
    pages = torch.full((1, n // page + 1), -1, dtype=torch.int32, device="cuda")
    pages[0, -1] = 0
    k = torch.zeros(1, 2, page, 64, dtype=torch.float16, device="cuda")
    v = torch.zeros_like(k)
    ws = torch.zeros(marlin.attention_workspace_bytes(64), dtype=torch.uint8, device="cuda")
    q = marlin.kv_append(torch.from_numpy(case.qkv).cuda(), k, v, pages, torch.tensor([n], dtype=torch.int32, device="cuda"), ws,
                         inv_freq=torch.from_numpy(frequencies(64)).cuda())
    torch.cuda.synchronize()
    assert marlin.read_status(ws) == 0
    case.lengths = np.array([n])
    want, _ = want_of(case, 64, False)
    got = q.cpu().numpy().astype(np.float64).reshape(want.shape)
    # the angle, 10^9 radians in 64 bits, is off by 2^-53 of it at each of three roundings: 3.4e-7
    assert np.all(np.abs(got - want) <= allowed(want, 10.0, False) + 3.4e-7 * 10.0)


def test_without_rotation_the_queries_stay_where_they_are(marlin):
    import torch
    case = Case([9, 17], 1, 8, 2, 64, 16, seed=3)
    d = case.dev(marlin)
    qkv = torch.from_numpy(case.qkv).cuda()
    q = marlin.kv_append(qkv, **d)
    torch.cuda.synchronize()
    assert q.data_ptr() == qkv.data_ptr() and torch.equal(q, qkv[:, :512])
    for b, n in enumerate(case.lengths):
        page, off = int(case.table[b][(n - 1) // 16]), (n - 1) % 16
        assert torch.equal(d["k_cache"][page, :, off], qkv[b, 512:640].view(2, 64))
        assert torch.equal(d["v_cache"][page, :, off], qkv[b, 640:].view(2, 64))


def test_saturation_and_nan_in_eight_bits(marlin):
    import torch
    case = Case([3], 1, 1, 1, 16, 16, eight_bit=True, seed=3)
    d = case.dev(marlin)
    d["k_scale"].fill_(0.5), d["v_scale"].fill_(2.0)
    inf, nan = float("inf"), float("nan")
    x = torch.tensor([0.0, 224.0, 225.0, -230.0, 65504.0, inf, -inf, nan, 1.0, 2.0 ** -9, 2.0 ** -10, 2.0 ** -11, 3 * 2.0 ** -11, -1e-7, 17.0, 18.0])
    qkv = torch.cat([x, x, x])[None].half().cuda()
    marlin.kv_append(qkv, **d)
    torch.cuda.synchronize()
    at = int(case.table[0][0]), 0, 2
    for cache, scale in ((d["k_cache"], 0.5), (d["v_cache"], 2.0)):
        want = (x.half().float() / scale).clamp(-448, 448).to(torch.float8_e4m3fn).float()
        got = cache[at].float().cpu()
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got[~torch.isnan(got)], want[~torch.isnan(want)])


def test_ranges_of_columns_rows_of_nobody_and_a_given_output(marlin):
    import torch
    case = Case([9, 40], [2, 3], 4, 2, 64, 16, seed=3)
    d = case.dev(marlin)
    inv = torch.from_numpy(frequencies(64)).cuda()
    want = marlin.kv_append(torch.from_numpy(case.qkv).cuda(), **d, inv_freq=inv)
    k, v = d["k_cache"].clone(), d["v_cache"].clone()
    e = case.dev(marlin)
    e["starts"] = e["starts"] + 1
    wide = torch.full((9, 512 + 24), float("nan"), dtype=torch.float16, device="cuda")
    wide[1:6, 16:16 + 512] = torch.from_numpy(case.qkv).cuda()
    out = torch.full((9, 256), 7.0, dtype=torch.float16, device="cuda")
    assert marlin.kv_append(wide[:, 16:16 + 512], **e, inv_freq=inv, out=out) is out
    torch.cuda.synchronize()
    assert torch.equal(out[1:6], want) and (out[:1] == 7).all() and (out[6:] == 7).all()
    assert torch.equal(e["k_cache"], k) and torch.equal(e["v_cache"], v)


def test_what_points_outside_of_the_cache_is_reported_and_not_written(marlin):
    import torch
    case = Case([40, 50], 1, 4, 2, 64, 16, seed=8)
    qkv = torch.from_numpy(case.qkv).cuda()
    for what, value in (("pages", case.pages), ("pages", -1), ("lengths", 2 ** 31 - 1), ("lengths", -3)):
        d = case.dev(marlin)
        before = d["k_cache"].clone()
        if what == "pages":
            d["pages"][0] = value
        else:
            d["lengths"][0] = value
        marlin.kv_append(qkv, **d)
        assert marlin.read_status(d["workspace"]) == 9
        changed = (d["k_cache"] != before).any(-1).any(1).nonzero().tolist()
        assert changed == [[int(case.table[1][3]), 1]]  # position 49 of the other sequence alone


def test_captured_steps(marlin):
    # a decode step captured once: lengths grow on the device, the same graph appends and attends at the new positions
    import torch
    case = Case([30, 63], 1, 8, 2, 64, 16, seed=8, spare_pages=9)
    free = [p for p in range(case.pages) if p not in case.table]
    case.table[0, 2:], case.table[1, 4] = free[:3], free[3]
    d = case.dev(marlin)
    inv = torch.from_numpy(frequencies(64)).cuda()
    qkv = torch.from_numpy(case.qkv).cuda()
    e = {k: x.clone() for k, x in d.items()}

    def step(d, qkv):
        q = marlin.kv_append(qkv, **d, inv_freq=inv)
        return marlin.attention_decode(q, **d)
    step(e, qkv)
    torch.cuda.synchronize()
    e = {k: x.clone() for k, x in d.items()}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(d, qkv)
    for i in range(5):
        qkv.copy_(torch.from_numpy(case.qkv * (1 + i)))
        graph.replay()
        want = step(e, qkv.clone())
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(d["k_cache"], e["k_cache"]) and torch.equal(d["v_cache"], e["v_cache"])
        d["lengths"] += 1
        e["lengths"] += 1
    assert marlin.read_status(d["workspace"]) == 0
