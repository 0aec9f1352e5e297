"""GPU: appending to 8-bit caches with a scale per block, against the oracle: bit for bit without a rotation."""
import numpy as np
import pytest

from blocks_util import BlockCase
from oracle import attention_ref, cache_blocks_ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def marlin():
    import torch
    assert torch.cuda.is_available()
    import paper_2408_11743_b200 as m
    m.lib()
    return m


def bits(t):
    import torch
    return t.contiguous().view(torch.uint8).cpu().numpy()


def oracle_append(case, new_k, new_v):
    """The caches and scales of a case after new_k and new_v [tokens, heads, dim]."""
    done = []
    for t, scale, new in ((case.k_t, case.k_scale, new_k), (case.v_t, case.v_scale, new_v)):
        codes, scales = case.codes(t).copy(), scale.copy()
        for b, (s, e) in enumerate(zip(case.starts[:-1], case.starts[1:])):
            n = int(case.lengths[b])
            first = max(0, n - (e - s))
            if 0 < n <= case.table.shape[1] * case.page:
                cache_blocks_ref.append(codes, scales, new[e - (n - first):e], case.table[b], first, case.block)
        done.append((codes, scales))
    return done


def split(case):
    x = case.qkv.astype(np.float32).reshape(case.T, -1, case.dim)
    return x[:, :case.q_heads], x[:, case.q_heads:case.q_heads + case.kv_heads], x[:, case.q_heads + case.kv_heads:]


def run(marlin, case, inv_freq=None, interleaved=False, d=None, qkv=None):
    import torch
    d = d or case.dev(marlin)
    qkv = torch.from_numpy(case.qkv).cuda() if qkv is None else qkv
    q = marlin.kv_append(qkv, **d, inv_freq=None if inv_freq is None else torch.from_numpy(inv_freq).cuda(), interleaved=interleaved)
    torch.cuda.synchronize()
    return q, d


def check_exact(marlin, case):
    q, d = run(marlin, case)
    assert marlin.read_status(d["workspace"]) == 0
    _, k, v = split(case)
    for (codes, scales), cache, scale in zip(oracle_append(case, k, v), (d["k_cache"], d["v_cache"]), (d["k_scale"], d["v_scale"])):
        assert np.array_equal(scale.cpu().numpy().view(np.uint32), scales.view(np.uint32))
        assert np.array_equal(bits(cache), codes.view(np.uint8))
    assert np.array_equal(q.cpu().numpy().view(np.uint16), case.qkv[:, :case.q_heads * case.dim].view(np.uint16))
    return d


SHAPES = [(8, 2, 128), (2, 2, 64), (1, 1, 16), (3, 1, 80), (4, 2, 256), (32, 32, 128), (71, 1, 64)]


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("q_heads,kv_heads,dim", SHAPES)
@pytest.mark.parametrize("page,block", [(16, 16), (16, 1), (64, 8), (128, 128)])
def test_codes_and_scales_are_the_definitions(marlin, kind, q_heads, kv_heads, dim, page, block):
    # one token each: the first of a block, the last, one in between, the first of all; growing and keeping scales
    case = BlockCase([1, 2, 16, 17, 64, 65, 100, 127, 128, 129, 300], 1, q_heads, kv_heads, dim, page, kind, block, seed=dim + block)
    check_exact(marlin, case)
    # several tokens each, prompts that go on, a whole prompt, nothing
    case = BlockCase([5, 130, 40, 200, 9], [5, 7, 40, 150, 0], q_heads, kv_heads, dim, page, kind, block, "tokens", seed=dim + block + 1)
    check_exact(marlin, case)


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_blocks_that_grow_step_by_step(marlin, kind):
    # ever larger tokens, one a call: scales double, codes are halved, and a code is never off by more than a step of the last scale
    import torch
    case = BlockCase([1, 1, 1], 1, 2, 2, 64, 32, kind, 16, seed=2)
    case.table = np.arange(6, dtype=np.int32).reshape(3, 2)
    d = case.dev(marlin)
    rng = np.random.default_rng(0)
    want = [(case.codes(t).copy(), s.copy()) for t, s in ((case.k_t, case.k_scale), (case.v_t, case.v_scale))]
    held = np.zeros((3, 16, 4, 64), np.float32)
    for n in range(1, 17):
        x = (rng.standard_normal((3, 6 * 64)) * np.array([[1.5 ** n], [1e-4 * 3 ** n], [0 if n < 4 else 40.0 / n]])).astype(np.float16)
        d["lengths"].fill_(n)
        marlin.kv_append(torch.from_numpy(x).cuda(), **d)
        new = x.astype(np.float32).reshape(3, 6, 64)
        held[:, n - 1] = new[:, 2:]
        for (codes, scales), h in zip(want, (2, 4)):
            for b in range(3):
                cache_blocks_ref.append(codes, scales, new[b:b + 1, h:h + 2], case.table[b], n - 1, 16)
    for i, ((codes, scales), cache, scale) in enumerate(zip(want, (d["k_cache"], d["v_cache"]), (d["k_scale"], d["v_scale"]))):
        assert np.array_equal(scale.cpu().numpy(), scales) and np.array_equal(bits(cache), codes.view(np.uint8))
        got = cache_blocks_ref.expanded(codes, scales)[case.table[:, 0], :, :16]
        x = held[:, :, 2 * i:2 * i + 2].transpose(0, 2, 1, 3)
        s = scales[case.table[:, 0], :, 0][:, :, None, None]
        # e4m3: half a last place, 2^-4, once; steps of 2^-9 below 2^-6, a step in all as in two's complement
        assert np.all(np.abs(got - x) <= (s * 1.001 if kind == "int8" else 2.0 ** -4 * np.abs(x) * 1.001 + s * 2.0 ** -9))


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_values_and_scales_that_are_not_finite(marlin, kind):
    case = BlockCase([40, 8, 16, 24], [40, 3, 1, 24], 2, 2, 64, 16, kind, 8, seed=3)
    x = case.qkv.reshape(case.T, 6, 64)
    x[3, 2, 5], x[3, 2, 6], x[9, 4, 0], x[41, 3, 7] = np.inf, np.nan, -np.inf, np.nan
    x[44:52, 2:] = 0               # a block of nothing but zeros
    x[52:60, 2] = np.inf           # of nothing but infinities
    x[60:68, 3] = np.float16(6e-8) # of the smallest numbers
    case.k_scale[case.table[1][0], 0] = np.nan
    case.v_scale[case.table[1][0], 0] = -1
    case.v_scale[case.table[2][0], 1] = np.inf
    check_exact(marlin, case)


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("q_heads,kv_heads,dim,rotary,interleaved", [(8, 2, 128, 128, False), (8, 2, 128, 64, True), (3, 1, 80, 80, False), (4, 2, 256, 256, True),
                                                                     (4, 2, 256, 16, False), (1, 1, 16, 16, True)])
@pytest.mark.parametrize("lengths,new,page,block", [([100, 33, 0, 5000], 1, 16, 16), ([70, 260, 9], [70, 200, 4], 128, 128), ([70, 260, 9], [70, 200, 4], 32, 2)])
def test_rotated(marlin, kind, q_heads, kv_heads, dim, rotary, interleaved, lengths, new, page, block):
    import torch
    case = BlockCase(lengths, new, q_heads, kv_heads, dim, page, kind, block, "wide" if block == 2 else "heads", seed=rotary)
    inv_freq = (10000.0 ** (-2.0 * np.arange(rotary // 2) / rotary)).astype(np.float32)
    before = [cache_blocks_ref.expanded(case.codes(t), s) for t, s in ((case.k_t, case.k_scale), (case.v_t, case.v_scale))]
    q, d = run(marlin, case, inv_freq, interleaved)
    assert marlin.read_status(d["workspace"]) == 0
    x = case.qkv.astype(np.float64).reshape(case.T, -1, dim)
    q = q.float().cpu().numpy().reshape(case.T, q_heads, dim)
    after = []
    for cache, scale in ((d["k_cache"], d["k_scale"]), (d["v_cache"], d["v_scale"])):
        codes = bits(cache)
        after.append((cache_blocks_ref.expanded(codes.view(np.int8) if kind == "int8" else codes, scale.cpu().numpy()), scale.cpu().numpy()))
    touched = np.zeros((case.pages, page), bool)
    for t, b, p in attention_ref.positions(case.lengths, case.starts):
        if p < 0:
            assert not q[t].any()
            continue
        y = attention_ref.rotate(x[t, :q_heads + kv_heads], p, inv_freq, interleaved)
        # the products and the angle in fp32 (2^-22 of a pair's length), and half a last place of fp16
        length = np.abs(x[t]).max() * 2
        assert np.all(np.abs(q[t] - y[:q_heads]) <= 2.0 ** -11 * np.abs(y[:q_heads]) + 2.0 ** -20 * length)
        number, slot = case.table[b][p // page], p % page
        touched[number, slot // block * block:slot // block * block + block] = True
        for (got, scale), want in zip(after, (y[q_heads:], x[t, q_heads + kv_heads:])):
            s = scale[number, :, slot // block][:, None]
            half = s * 0.5 if kind == "int8" else np.maximum(2.0 ** -4 * np.abs(want), s * 2.0 ** -10)
            assert np.all(np.abs(got[number, :, slot] - want) <= half * 1.001 + 2.0 ** -20 * length)
            assert np.all(np.abs(want).max(-1) <= s[:, 0] * (127 if kind == "int8" else 448) * 1.0001)
    for (got, _), old in zip(after, before):  # other blocks are as they were
        same = (got == old) | (np.isnan(got) & np.isnan(old))
        assert same.transpose(0, 2, 1, 3)[~touched].all()


def test_scales_with_strides_rows_of_nobody_and_pages_that_are_not_there(marlin):
    import torch
    case = BlockCase([40, 8, 20], [40, 3, 2], 2, 2, 64, 16, "int8", 4, seed=5)
    case.table[1, 0] = case.pages + 3
    want = case.dev(marlin)
    run(marlin, case, d=want)
    assert marlin.read_status(want["workspace"]) == 9
    d = case.dev(marlin)
    for name in ("k_scale", "v_scale"):
        big = torch.full((4, case.pages + 1, 4), float("nan"), device="cuda")
        view = big.transpose(0, 1)[1:, 1:3]
        view.copy_(d[name])
        d[name], d[name + "_all"] = view, big
    bigs = [d.pop("k_scale_all"), d.pop("v_scale_all")]
    qkv = torch.full((case.T + 9, case.qkv.shape[1]), float("nan"), device="cuda", dtype=torch.float16)
    qkv[4:-5] = torch.from_numpy(case.qkv).cuda()
    d["starts"] = d["starts"] + 4
    inv_freq = torch.full((32,), 0.0, device="cuda")
    out = torch.full((case.T + 9, 128), 7.0, device="cuda", dtype=torch.float16)
    q = marlin.kv_append(qkv, **d, inv_freq=inv_freq, out=out)
    assert q is out and (out[:4] == 7).all() and (out[-5:] == 7).all()
    assert np.array_equal(out[4:-5].cpu().numpy(), case.qkv[:, :128])
    for name in ("k_cache", "v_cache", "k_scale", "v_scale"):
        assert torch.equal(d[name], want[name]), name
    for big in bigs:
        assert big[0].isnan().all() and big[3].isnan().all() and big[:, 0].isnan().all()


def test_a_sequence_that_is_refused_and_the_whole_of_the_table(marlin):
    import torch
    case = BlockCase([32, 32, 20], 1, 2, 1, 64, 16, "e4m3", 8, seed=6)
    case.table = case.table[:, :2]
    d = case.dev(marlin)
    d["pages"] = d["pages"].contiguous()
    d["lengths"][1] = 33
    d["lengths"][2] = -21
    before = {n: d[n].clone() for n in ("k_cache", "v_cache", "k_scale", "v_scale")}
    q, _ = run(marlin, case, np.zeros(32, np.float32), d=d)
    assert marlin.read_status(d["workspace"]) == 9
    assert not q[1:].any() and q[0].any()
    page = int(case.table[0, 1])
    for n, x in before.items():
        y = d[n].view(torch.uint8).cpu() != x.view(torch.uint8).cpu()
        y[page] = False
        assert not y.any(), n


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_steps_as_a_loop_makes_them_captured_and_replayed(marlin, kind):
    # reserve, append and attend in one captured step, replayed: lengths, tables and scales grow on the GPU
    import torch
    B, heads, kv, dim, page, block, pages = 5, 8, 2, 64, 16, 8, 40
    rng = np.random.default_rng(1)
    lengths = torch.tensor([0, 14, 31, 90, 3], dtype=torch.int32, device="cuda")
    table = torch.full((B, 9), -1, dtype=torch.int32, device="cuda")
    free = torch.from_numpy(rng.permutation(pages).astype(np.int32)).cuda()
    count = torch.tensor([pages], dtype=torch.int32, device="cuda")
    ws = torch.zeros(marlin.attention_workspace_bytes(dim), dtype=torch.uint8, device="cuda")
    dtype = torch.int8 if kind == "int8" else torch.float8_e4m3fn
    k, v = (torch.zeros(pages, kv, page, dim, device="cuda").to(dtype) for _ in range(2))
    ks, vs = (torch.zeros(pages, kv, page // block, device="cuda") for _ in range(2))
    had = lengths.clone()
    lengths.zero_()
    # the tokens that are there already, as prompts
    starts, slots, positions = marlin.kv_reserve(lengths, table, free, count, ws, page, 138, counts=had)
    prompt = torch.from_numpy(rng.standard_normal((138, (heads + 2 * kv) * dim)).astype(np.float16)).cuda()
    cache = dict(k_cache=k, v_cache=v, pages=table, lengths=lengths, workspace=ws, k_scale=ks, v_scale=vs)
    marlin.kv_append(prompt, **cache, starts=starts)
    qkv = torch.empty(B, (heads + 2 * kv) * dim, device="cuda", dtype=torch.float16)
    out = torch.empty(B, heads * dim, device="cuda", dtype=torch.float16)
    given = dict(starts=torch.empty(B + 1, dtype=torch.int32, device="cuda"), slots=torch.empty(B, dtype=torch.int64, device="cuda"),
                 positions=torch.empty(B, dtype=torch.int32, device="cuda"))

    def step():
        marlin.kv_reserve(lengths, table, free, count, ws, page, B, **given)
        q = marlin.kv_append(qkv, **cache)
        marlin.attention_decode(q, **cache, window=20, sinks=2, out=out)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    codes = [x.view(torch.uint8).cpu().numpy() for x in (k, v)]
    want = [((c.view(np.int8) if kind == "int8" else c).copy(), s.cpu().numpy().copy()) for c, s in zip(codes, (ks, vs))]
    for i in range(20):
        x = (rng.standard_normal(qkv.shape) * 1.2 ** i).astype(np.float16)
        qkv.copy_(torch.from_numpy(x))
        graph.replay()
        torch.cuda.synchronize()
        n, t = lengths.cpu().numpy(), table.cpu().numpy()
        assert np.array_equal(n, had.cpu().numpy() + i + 1)
        new = x.astype(np.float32).reshape(B, -1, dim)
        for (c, s), h in zip(want, (heads, heads + kv)):
            for b in range(B):
                cache_blocks_ref.append(c, s, new[b:b + 1, h:h + kv], t[b], int(n[b]) - 1, block)
        for (c, s), cache_t, scale_t in zip(want, (k, v), (ks, vs)):
            assert np.array_equal(cache_t.view(torch.uint8).cpu().numpy(), c.view(np.uint8)) and np.array_equal(scale_t.cpu().numpy(), s)
        at = given["positions"].cpu().numpy()
        assert np.array_equal(at, n - 1)
        assert np.array_equal(given["slots"].cpu().numpy(), t[np.arange(B), at // page].astype(np.int64) * page + at % page)
        case = BlockCase.__new__(BlockCase)
        case.block, case.kind, case.v_scale = block, kind, want[1][1]
        ref = cache_blocks_ref.attention(x[:, :heads * dim].reshape(B, heads, dim), *(cache_blocks_ref.expanded(c, s) for c, s in want), t, n,
                                         np.arange(B + 1), dim ** -0.5, 20, 2)
        assert np.all(np.abs(out.float().cpu().numpy().reshape(ref[0].shape) - ref[0]) <= case.sinks_bound(ref))
    assert marlin.read_status(ws) == 0


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_the_attention_half_of_a_layer(marlin, kind):
    # attention_block with scales by block and sinks is its four calls one after the other
    import torch
    from gpu_util import to_dev
    from paper_2408_11743_b200 import inputs
    M, K, q_heads, kv, dim, N, G = 3, 512, 8, 2, 64, 512, 128
    case = BlockCase([100, 9, 300], 1, q_heads, kv, dim, 16, kind, 8)
    a, b = inputs.make_dense(M, K, (q_heads + 2 * kv) * dim, G, seed=1), inputs.make_dense(M, q_heads * dim, N, G, seed=2)
    (wq, sq), (wo, so) = (marlin.pack(to_dev(x.q_kpacked), to_dev(x.S), G) for x in (a, b))
    ws_bytes = max(marlin.workspace_bytes(M, K, 768), marlin.workspace_bytes(M, 512, N), marlin.attention_workspace_bytes(dim))
    inv_freq = torch.from_numpy((10000.0 ** (-np.arange(32) / 32.0)).astype(np.float32)).cuda()
    A = to_dev(a.A)
    one, two = case.dev(marlin), case.dev(marlin)
    for d in (one, two):
        d["workspace"] = torch.zeros(ws_bytes, dtype=torch.uint8, device="cuda")
    got = marlin.attention_block(A, wq, sq, wo, so, K=K, q_heads=q_heads, N=N, group_size=G, inv_freq=inv_freq, window=64, sinks=4, **one)
    qkv = marlin.gemm(A, wq, sq, K, 768, G, two["workspace"])
    q = marlin.kv_append(qkv, **two, inv_freq=inv_freq)
    o = marlin.attention_decode(q, **two, window=64, sinks=4)
    want = marlin.gemm(o, wo, so, 512, N, G, two["workspace"])
    assert torch.equal(got, want)
    for name in ("k_cache", "v_cache", "k_scale", "v_scale"):
        assert torch.equal(one[name].view(torch.uint8), two[name].view(torch.uint8))
    assert marlin.read_status(one["workspace"]) == 0
    # sinks alone, over fp16
    case = BlockCase([100, 9, 300], 1, q_heads, kv, dim, 16, "fp16")
    one, two = case.dev(marlin), case.dev(marlin)
    for d in (one, two):
        d["workspace"] = torch.zeros(ws_bytes, dtype=torch.uint8, device="cuda")
    got = marlin.attention_block(A, wq, sq, wo, so, K=K, q_heads=q_heads, N=N, group_size=G, inv_freq=inv_freq, window=64, sinks=4, **one)
    q = marlin.kv_append(marlin.gemm(A, wq, sq, K, 768, G, two["workspace"]), **two, inv_freq=inv_freq)
    want = marlin.gemm(marlin.attention_decode(q, **two, window=64, sinks=4), wo, so, 512, N, G, two["workspace"])
    assert torch.equal(got, want) and torch.equal(one["k_cache"], two["k_cache"])


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
def test_zeros_under_a_scale_whose_inverse_is_not_finite(marlin, kind):
    # a block that was begun under 1e-40, and tokens of nothing but zeros: no code but 0
    import torch
    case = BlockCase([21, 5], [1, 2], 2, 2, 64, 32, kind, 16, seed=31)
    case.qkv[:] = 0
    d = case.dev(marlin)
    d["k_scale"].fill_(1e-40), d["v_scale"].fill_(1e-40)
    run(marlin, case, d=d)
    for cache, scale in ((d["k_cache"], d["k_scale"]), (d["v_cache"], d["v_scale"])):
        for b, (s, e) in enumerate(zip(case.starts[:-1], case.starts[1:])):
            for at in range(int(case.lengths[b]) - int(e - s), int(case.lengths[b])):
                page = int(case.table[b, at // 32])
                assert not bits(cache[page, :, at % 32]).any()
                assert (scale[page, :, at % 32 // 16] == scale.new_tensor(1e-40)).all()


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
def test_begins_that_descend_are_contained(marlin, kind):
    # (which they must not: what becomes of these sequences is open, but nothing else is touched)
    import torch
    case = BlockCase([300, 300, 300, 40], [100, 50, 50, 3], 2, 2, 64, 32, kind, 16, seed=32)
    d = case.dev(marlin)
    d["starts"].copy_(torch.tensor([0, 100, 50, 200, 203]))
    before = [bits(d[x]).copy() for x in ("k_cache", "v_cache")]
    q, _ = run(marlin, case, d=d)
    mine = set(int(x) for b in range(4) for x in case.table[b, :-(-int(case.lengths[b]) // 32)])
    others = [x for x in range(case.pages) if x not in mine]
    for was, x in zip(before, ("k_cache", "v_cache")):
        assert np.array_equal(bits(d[x])[others], was[others])
    # the sequence behind them has what it asked for
    assert np.array_equal(q[200:203].cpu().numpy().view(np.uint16), case.qkv[200:203, :case.q_heads * case.dim].view(np.uint16))


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
def test_many_values_against_elementary_operations(marlin, kind):
    # scales and codes of whole prompts bit for bit: amax times the fp32 number nearest to 1 / L, values times the fp32 inverse of that
    import torch
    case = BlockCase([1000, 777, 1500], [1000, 777, 1500], 16, 16, 128, 64, kind, 4, seed=33)
    _, d = run(marlin, case)
    x = torch.from_numpy(case.qkv).cuda().float().view(case.T, -1, 128)
    for cache, scale, first in ((d["k_cache"], d["k_scale"], 16), (d["v_cache"], d["v_scale"], 32)):
        for b, (s, e) in enumerate(zip(case.starts[:-1], case.starts[1:])):
            at = torch.arange(int(e - s), device="cuda")
            page = torch.from_numpy(case.table[b]).cuda().long()[at // 64]
            new = x[int(s):int(e), first:first + 16]
            runs = torch.nn.functional.pad(new, (0, 0, 0, 0, 0, -len(at) % 4)).unflatten(0, (-1, 4))
            top = runs.abs().amax((1, 3)) * (torch.ones((), device="cuda") / (127 if kind == "int8" else 448))
            assert torch.equal(scale[page, :, at % 64 // 4], top[at // 4])
            y = new * (1 / top)[at // 4][..., None]
            want = y.round().to(torch.int8) if kind == "int8" else y.to(torch.float8_e4m3fn)
            assert torch.equal(cache[page, :, at % 64].view(torch.uint8), want.view(torch.uint8))
