"""The paged cache where calls reach its limits."""
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


def bits(x):
    import torch
    return x.view(torch.uint8)


@pytest.mark.parametrize("length", [65, 67, 1000, 2 ** 30 + 1, 2 ** 31 - 1, -1, -2 ** 31])
@pytest.mark.parametrize("new", [1, 5])
@pytest.mark.parametrize("fill", ["pages of its own", "zeros"])
@pytest.mark.parametrize("eight_bit", [False, True])
def test_a_sequence_that_its_table_cannot_hold_has_no_place(marlin, length, new, fill, eight_bit):
    # a row of four pages of 16 tokens, all of them valid (or filled up with page 0, which belongs to the other sequence)
    import torch
    case = Case([64, 49], new, 8, 2, 64, 16, eight_bit, seed=3)
    d = case.dev(marlin)
    table = torch.tensor([[3, 4, 5, 6], [0, 1, 2, 7]], dtype=torch.int32, device="cuda")
    if fill == "zeros":
        table[0, 1:] = 0
    d["pages"] = table
    inv = torch.from_numpy((10000.0 ** (-np.arange(32) / 32.0)).astype(np.float32)).cuda()
    qkv = torch.from_numpy(case.qkv).cuda()
    before = {name: d[name].clone() for name in ("k_cache", "v_cache")}
    lone = {**d, **{name: x.clone() for name, x in before.items()}, "lengths": d["lengths"].clone()}
    lone["lengths"][0] = 0  # what the other sequence has by itself
    q_want = marlin.kv_append(qkv, **lone, inv_freq=inv)
    o_want = marlin.attention_decode(q_want, **{k: x for k, x in lone.items()})
    torch.cuda.synchronize()
    assert marlin.read_status(lone["workspace"]) == 0

    d["lengths"][0] = length
    q = marlin.kv_append(qkv, **d, inv_freq=inv)
    assert marlin.read_status(d["workspace"]) == 9
    for name, x in before.items():
        changed = (bits(d[name]) != bits(x)).view(x.shape[0], 2, 16, -1).any(-1).any(1).nonzero().tolist()
        places = [(int(table[1, p // 16]), p % 16) for p in range(49 - new, 49)]
        assert sorted(map(tuple, changed)) == sorted(places)  # the other sequence's new tokens alone
        assert torch.equal(bits(d[name]), bits(lone[name]))
    assert not q[:new].any() and torch.equal(q[new:], q_want[new:])
    d["workspace"].zero_()
    out = torch.full_like(q, 7.0)
    marlin.attention_decode(q, **d, out=out)
    assert marlin.read_status(d["workspace"]) == 9
    assert not out[:new].any() and torch.equal(out[new:], o_want[new:])


@pytest.mark.parametrize("length", [64, 63, 1, 0])
def test_a_sequence_that_fills_its_table_is_as_any_other(marlin, length):
    import torch
    case = Case([length, 49], 1, 8, 2, 64, 16, seed=3, spare_pages=8)
    d = case.dev(marlin)
    d["pages"] = torch.tensor([[3, 4, 5, 6], [0, 1, 2, 7]], dtype=torch.int32, device="cuda")
    qkv = torch.from_numpy(case.qkv).cuda()
    marlin.kv_append(qkv, **d)
    assert marlin.read_status(d["workspace"]) == 0
    if length:
        page = int(d["pages"][0, (length - 1) // 16])
        assert torch.equal(d["k_cache"][page, :, (length - 1) % 16], qkv[0, 512:640].view(2, 64))


@pytest.mark.parametrize("q_heads,dim", [(12, 16), (20, 48), (12, 80), (24, 112), (48, 80), (40, 16)])
@pytest.mark.parametrize("eight_bit", [False, True])
def test_values_that_are_not_finite_beside_lanes_without_an_element(marlin, q_heads, dim, eight_bit):
    # several new tokens, one of whose values is NaN: rows that see it are summed up lane by lane, and heads that do not fill their
    # tile leave some lanes out
    import torch
    case = Case([40, 300], [5, 3], q_heads, 1, dim, 16, eight_bit, seed=9)
    d = case.dev(marlin)
    q = torch.from_numpy(case.q.reshape(case.T, -1)).cuda()
    want = marlin.attention_decode(q, **d).view(8, q_heads, dim).clone()
    v = d["v_cache"].clone()
    place = int(case.table[0][38 // 16]), 0, 38 % 16
    if eight_bit:
        v.view(torch.uint8)[place][dim - 1] = 0x7F
    else:
        v[place][dim - 1] = float("nan")
    got = marlin.attention_decode(q, **{**d, "v_cache": v}).view(8, q_heads, dim)
    torch.cuda.synchronize()
    assert marlin.read_status(d["workspace"]) == 0
    want[3:5, :, dim - 1] = float("nan")  # positions 38 and 39 of sequence 0
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    fine = ~torch.isnan(want)
    assert torch.equal(got[fine], want[fine])


@pytest.mark.parametrize("q_heads,dim", [(1, 64), (8, 128), (16, 64), (16, 128), (40, 64), (40, 128), (8, 256), (40, 256)])
@pytest.mark.parametrize("eight_bit", [False, True])
def test_many_weights_far_below_the_largest(marlin, q_heads, dim, eight_bit):
    # Sixteen keys have a weight of 1 and the value 0, 131056 others one of 2^-26 and the value 256: the others have 2^-13 of the weights
    # together, and make all of the result, 2^-13 * 256.  (Every warp that multiplies has one of the sixteen.)
    # A weight of 2^-26 of the largest has to survive its rounding to fp16.  All weights are powers of two: what is left is the rounding
    # of the logit (26 to 2^-19 of it in base 2, so 2^-14 of a weight at most), sums in fp32 of equal terms, the sum of the weights,
    # where the small ones may be lost beside a large one (2^-13 of it), and the result's rounding.
    import torch
    n, page, sequences = 1 << 17, 1 << 10, 320   # (more items than CTAs: no CTA has few of their keys)
    kind = torch.float8_e4m3fn if eight_bit else torch.float16
    k = torch.zeros(n // page, 1, page, dim, device="cuda")
    v = torch.full_like(k, 256.0)
    k[0, 0, 0:256:16, 0] = 13.0
    v[0, 0, 0:256:16] = 0.0
    q = torch.zeros(sequences, q_heads, dim, dtype=torch.float16, device="cuda")
    q[:, :, 0] = 2.0
    table = torch.arange(n // page, dtype=torch.int32, device="cuda").repeat(sequences, 1)
    lengths = torch.full((sequences,), n, dtype=torch.int32, device="cuda")
    ws = torch.zeros(marlin.attention_workspace_bytes(dim), dtype=torch.uint8, device="cuda")
    out = marlin.attention_decode(q.view(sequences, -1), k.to(kind), v.to(kind), table, lengths, ws, scale=float(np.float32(np.log(2.0))))
    assert marlin.read_status(ws) == 0
    rest = (n - 16) * np.exp(-26.0 * float(np.float32(np.log(2.0))))
    want = 256.0 * rest / (16.0 + rest)
    off = (out.double() - want).abs().max().item()
    assert off <= want * (2.0 ** -11 + 2.0 ** -14 + 2.0 ** -13 + 2.0 ** -18), (off, want)


@pytest.mark.parametrize("q_heads,kv_heads,sequences,length", [(64, 64, 4000, 1 << 20), (192, 16, 1024, 1 << 23)])
def test_nearly_as_many_tiles_as_32_bits_count(marlin, q_heads, kv_heads, sequences, length):
    # 0.98 * 2^32 tiles of 64 keys with a row each, and 2^30 of 128 keys with 12 rows on the tensor cores' fifth generation (two to
    # four seconds each).  All entries of the table are page 0 but the last of every row, page 1, so that the result is that of two pages, the first
    # counted as often as it is there.
    import torch
    page, dim = 1 << 14, 16
    times = length // page - 1
    gen = torch.Generator(device="cuda").manual_seed(q_heads)
    k, v = (torch.randn(2, kv_heads, page, dim, generator=gen, device="cuda", dtype=torch.float16) for _ in "kv")
    v[1] += 64.0
    q = torch.randn(sequences, q_heads * dim, generator=gen, device="cuda", dtype=torch.float16)
    table = torch.zeros(sequences, length // page, dtype=torch.int32, device="cuda")
    table[:, -1] = 1
    lengths = torch.full((sequences,), length, dtype=torch.int32, device="cuda")
    ws = torch.zeros(marlin.attention_workspace_bytes(dim), dtype=torch.uint8, device="cuda")
    out = torch.full_like(q, float("nan"))
    marlin.attention_decode(q, k, v, table, lengths, ws, scale=0.25, out=out)
    assert marlin.read_status(ws) == 0
    group = q_heads // kv_heads
    # A sum of one warp (or of one CTA on tcgen05, 16 keys at a time) is added up in fp32 over at most length / 16 steps, each off by
    # 2^-24 of the sum so far: all sums have one sign in the weights and are bounded by the spread in the values; numerator and
    # denominator: 2 * length / 16 * 2^-24.  The rest as in cache_util.attention_bound, with |logit| <= 16 |q| |k| * 0.25 < 64.
    relative = 2.0 ** -11 + 2.0 ** -20 + 2 * length / 16 * 2.0 ** -24 + 4 * 32 * 2.0 ** -24 * 64
    times = torch.tensor([times, 1], dtype=torch.float64, device="cuda").repeat_interleave(page)
    for h in range(kv_heads):
        rows = q.view(sequences, kv_heads, group, dim)[:, h].reshape(-1, dim).double()
        got = out.view(sequences, kv_heads, group, dim)[:, h].reshape(-1, dim).double()
        keys, values = k[:, h].reshape(-1, dim).double(), v[:, h].reshape(-1, dim).double()
        for a in range(0, len(rows), 4096):
            s = rows[a:a + 4096] @ keys.T * 0.25
            w = (s - s.amax(-1, keepdim=True)).exp() * times
            w /= w.sum(-1, keepdim=True)
            want, spread = w @ values, w @ values.abs()
            off = (got[a:a + 4096] - want).abs()
            assert bool((off <= 2.0 ** -11 * want.abs() + relative * spread).all())  # (false for NaN)


def test_more_tiles_than_32_bits_count_are_refused(marlin):
    import torch
    q = torch.ones(4100, 64 * 16, dtype=torch.float16, device="cuda")
    k = torch.ones(1, 64, 1 << 14, 16, dtype=torch.float16, device="cuda")
    table = torch.zeros(4100, 64, dtype=torch.int32, device="cuda")
    lengths = torch.full((4100,), 1 << 20, dtype=torch.int32, device="cuda")
    ws = torch.zeros(marlin.attention_workspace_bytes(16), dtype=torch.uint8, device="cuda")
    out = torch.full_like(q, 7.0)
    marlin.attention_decode(q, k, k, table, lengths, ws, out=out)
    assert marlin.read_status(ws) == 9
    assert (out == 7).all() and not ws[256:].any()
    ws.zero_()
    lengths[4:] = 0
    marlin.attention_decode(q, k, k, table, lengths, ws, out=out)
    assert marlin.read_status(ws) == 0
    assert (out[:4] == 1).all() and not out[4:].any()


@pytest.mark.parametrize("q_heads,dim,eight_bit", [(12, 128, False), (20, 112, False), (40, 128, False), (16, 64, False), (64, 64, False),
                                                   (40, 128, True), (64, 80, True)])
@pytest.mark.parametrize("rising", [False, True])
@pytest.mark.parametrize("n", [16384, 16385, 33000, 524299])
def test_sums_over_long_ranges_of_keys(marlin, q_heads, dim, eight_bit, rising, n):
    # More items than CTAs, so that some CTAs have all the keys of an item; values around 1, so that what a sum loses shows; logits that rise
    # with the position, so that bases move after sums were put aside.  Allowed: the result's rounding and that of the weights,
    # 2^-11 each, and what 16384 keys lose one by one, at most 2^-23 of a sum that grows from 0, 2^-24 of it on the average:
    # 2^-10.  (Exponentials, factors and the rest are below 2^-16.)
    import torch
    page, sequences = 1024, 200 if n > 1 << 17 else 300
    kind = torch.float8_e4m3fn if eight_bit else torch.float16
    gen = torch.Generator(device="cuda").manual_seed(n + dim)
    pages = -(-n // page)
    k = torch.randn(pages * page, dim, generator=gen, device="cuda")
    if rising:
        k[:, 0] = torch.arange(pages * page, device="cuda") * (16.0 / n)
    k = k.to(kind)
    v = (torch.rand(pages * page, dim, generator=gen, device="cuda") + 0.5).to(kind)
    q = (torch.randn(q_heads, dim, generator=gen, device="cuda") * 0.7).half()
    if rising:
        q[:, 0] = dim ** 0.5 * 3.0
    table = torch.arange(pages, dtype=torch.int32, device="cuda").repeat(sequences, 1)
    lengths = torch.full((sequences,), n, dtype=torch.int32, device="cuda")
    ws = torch.zeros(marlin.attention_workspace_bytes(dim), dtype=torch.uint8, device="cuda")
    out = marlin.attention_decode(q.repeat(sequences, 1, 1).view(sequences, -1), k.view(pages, 1, page, dim), v.view(pages, 1, page, dim),
                                  table, lengths, ws)
    assert marlin.read_status(ws) == 0
    w = torch.softmax(q.double() @ k[:n].double().T * dim ** -0.5, -1)
    want = w @ v[:n].double()
    off = (out.double().view(sequences, q_heads, dim) - want).abs() / want
    assert bool((off <= 2.0 ** -11 + 2.0 ** -11 + 2.0 ** -10 + 2.0 ** -16).all()), off.max()


@pytest.mark.parametrize("q_heads,dim", [(1, 64), (8, 128), (5, 80), (3, 256), (12, 64), (16, 128), (40, 64), (40, 128), (24, 256)])
@pytest.mark.parametrize("new", [1, 3])
def test_infinite_values_that_every_row_sees(marlin, q_heads, dim, new):
    import torch
    case = Case([70, 300, 9], new, q_heads, 1, dim, 16, seed=dim + new)
    d = case.dev(marlin)
    q = torch.from_numpy(case.q.reshape(case.T, -1)).cuda() * 0.25  # (no weight is below 2^-10 of the largest)
    want = marlin.attention_decode(q, **d).view(3, new, q_heads, dim).clone()
    v = d["v_cache"].clone()
    inf, nan = float("inf"), float("nan")

    def value(b, pos, element, x):
        v[int(case.table[b][pos // 16]), 0, pos % 16, element] = x
    # keys in every part of a tile and of the sequence
    value(0, 3, 1, inf), value(0, 40, 2, -inf), value(0, 5, 3, inf), value(0, 60, 3, inf), value(0, 17, 4, inf), value(0, 18, 4, -inf)
    value(1, 250, 5, inf), value(1, 1, 6, -inf), value(1, 130, 7, nan), value(2, 0, 8, inf)
    got = marlin.attention_decode(q, **{**d, "v_cache": v}).view(3, new, q_heads, dim)
    torch.cuda.synchronize()
    assert marlin.read_status(d["workspace"]) == 0
    want[0, :, :, 1], want[0, :, :, 2], want[0, :, :, 3], want[0, :, :, 4] = inf, -inf, inf, nan
    want[1, :, :, 5], want[1, :, :, 6], want[1, :, :, 7], want[2, :, :, 8] = inf, -inf, nan, inf
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    fine = ~torch.isnan(want)
    assert torch.equal(got[fine], want[fine])