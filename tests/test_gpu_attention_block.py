"""The attention half of a decoder layer (marlin_attention_block) and runs of its operators as a decoding loop makes them.

Each step is compared with the definition applied to what the step before it left on the GPU (the qkv layer with the layer's
oracle, append and attention with the definition in 64 bits, the output layer with the layer's oracle again), so that every
comparison has the tolerance of its own operator.
"""
import numpy as np
import pytest

from paper_2408_11743_b200 import inputs
from cache_util import attention_bound
from gpu_util import to_dev, to_host

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def marlin():
    import torch
    assert torch.cuda.is_available()
    import paper_2408_11743_b200 as m
    m.lib()
    return m


class Block:
    def __init__(self, marlin, M, K, q_heads, kv_heads, dim, N, G, page, max_pages, sequences, eight_bit, seed):
        import torch
        self.K, self.N, self.G, self.q_heads, self.kv_heads, self.dim = K, N, G, q_heads, kv_heads, dim
        columns, q_cols = (q_heads + 2 * kv_heads) * dim, q_heads * dim
        self.qkv_case = inputs.make_dense(M, K, columns, G, seed=seed)
        self.o_case = inputs.make_dense(M, q_cols, N, G, seed=seed + 1)
        self.w_qkv, self.s_qkv = marlin.pack(to_dev(self.qkv_case.q_kpacked), to_dev(self.qkv_case.S), G)
        self.w_o, self.s_o = marlin.pack(to_dev(self.o_case.q_kpacked), to_dev(self.o_case.S), G)
        kind = torch.float8_e4m3fn if eight_bit else torch.float16
        self.k_cache, self.v_cache = (torch.zeros(sequences * max_pages + 1, kv_heads, page, dim, device="cuda").to(kind) for _ in "kv")
        self.table = torch.randperm(sequences * max_pages, generator=torch.Generator().manual_seed(seed)).int().view(sequences, max_pages).cuda()
        need = max(marlin.workspace_bytes(M, K, columns), marlin.workspace_bytes(M, q_cols, N), marlin.attention_workspace_bytes(dim))
        self.ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
        self.inv = torch.tensor(10000.0 ** (-np.arange(dim // 2) * 2.0 / dim), dtype=torch.float32, device="cuda")
        self.scales = {}
        if eight_bit:
            self.scales = dict(k_scale=torch.linspace(0.02, 0.04, kv_heads, device="cuda"), v_scale=torch.linspace(0.03, 0.02, kv_heads, device="cuda"))

    def args(self):
        return (self.w_qkv, self.s_qkv, self.w_o, self.s_o, self.k_cache, self.v_cache, self.table)


def check_step(marlin, oracle_lib, blk, A, lengths, starts, QKV, Q, O, C, rotated, window):
    from oracle import attention_ref
    T, D = A.shape[0], blk.dim
    ref = oracle_lib.gemm(A, blk.qkv_case.q_kpacked, blk.qkv_case.S, blk.qkv_case.G)
    bad, worst, _ = oracle_lib.check_tolerance(to_host(QKV), ref)
    assert bad == 0, worst
    x = to_host(QKV).astype(np.float64).reshape(T, -1, D)
    H, n = blk.q_heads, blk.kv_heads
    k_host, v_host = blk.k_cache.float().cpu().numpy(), blk.v_cache.float().cpu().numpy()
    table = to_host(blk.table)
    page = k_host.shape[2]
    ks = to_host(blk.scales["k_scale"]).astype(np.float64)[:, None] if blk.scales else 1.0
    vs = to_host(blk.scales["v_scale"]).astype(np.float64)[:, None] if blk.scales else 1.0
    step, least = (2.0 ** -4, 2.0 ** -10) if blk.scales else (2.0 ** -11, 2.0 ** -25)
    most = np.abs(x).max()
    for t, b, p in attention_ref.positions(lengths, starts):
        y = attention_ref.rotate(x[t, :H + n], int(p), to_host(blk.inv) if rotated else [], False)
        q = to_host(Q).astype(np.float64).reshape(T, H, D)[t]
        assert np.all(np.abs(q - y[:H]) <= np.maximum(2.0 ** -11 * np.abs(y[:H]), 2.0 ** -25) + 2.0 ** -20 * most)
        at = table[b][p // page], slice(None), p % page
        for got, want in ((k_host[at], y[H:] / ks), (v_host[at], x[t, H + n:] / vs)):
            size = 2.0 ** -20 * most / (0.02 if blk.scales else 1.0)
            assert np.all(np.abs(got - want) <= np.maximum(step * np.abs(want), least) + size)
    q = to_host(Q).reshape(T, H, D)
    ref = attention_ref.attention(q, k_host, v_host, table, lengths, starts, D ** -0.5, window,
                                  to_host(blk.scales["k_scale"]) if blk.scales else None, to_host(blk.scales["v_scale"]) if blk.scales else None)
    got = to_host(O).astype(np.float64).reshape(T, H, D)
    assert np.all(np.abs(got - ref[0]) <= attention_bound(ref))
    ref = oracle_lib.gemm(to_host(O), blk.o_case.q_kpacked, blk.o_case.S, blk.o_case.G)
    bad, worst, _ = oracle_lib.check_tolerance(to_host(C), ref)
    assert bad == 0, worst


# rows up to 16 (warp-level kernel), above (tcgen05 kernel); prompt, single tokens, drafted tokens; both formats
@pytest.mark.parametrize("K,q_heads,kv_heads,dim,N,G,eight_bit,rotated,window", [
    (512, 8, 2, 64, 512, 128, False, True, 0), (1024, 4, 4, 128, 256, 128, True, True, 0),
    (512, 16, 1, 32, 256, -1, False, False, 9), (256, 8, 8, 64, 320, 128, True, False, 0)])
def test_a_prompt_then_steps(marlin, oracle_lib, K, q_heads, kv_heads, dim, N, G, eight_bit, rotated, window):
    import torch
    news = [[20, 1, 11], [1, 1, 1], [1, 1, 1], [3, 0, 2], [1, 1, 1], [16, 4, 7]]
    most = max(sum(n) for n in news)
    blk = Block(marlin, most, K, q_heads, kv_heads, dim, N, G, 8, 9, 3, eight_bit, seed=dim)
    rng = np.random.default_rng(1)
    lengths = np.zeros(3, np.int32)
    for new in news:
        T = sum(new)
        lengths = lengths + np.asarray(new, np.int32)
        starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        A = (rng.standard_normal((T, K))).astype(np.float16)
        QKV = torch.empty(T, (q_heads + 2 * kv_heads) * dim, dtype=torch.float16, device="cuda")
        Q, O = (torch.empty(T, q_heads * dim, dtype=torch.float16, device="cuda") for _ in "qo")
        one_each = all(n == 1 for n in new)
        C = marlin.attention_block(to_dev(A), *blk.args(), to_dev(lengths), K, q_heads, N, G, blk.ws, inv_freq=blk.inv if rotated else None,
                                   window=window, starts=None if one_each else to_dev(starts), QKV=QKV, Q=Q, O=O, **blk.scales)
        torch.cuda.synchronize()
        assert marlin.read_status(blk.ws) == 0
        check_step(marlin, oracle_lib, blk, A, lengths, starts, QKV, Q if rotated else QKV[:, :q_heads * dim].contiguous(), O, C, rotated, window)
    # the scratch from torch's allocator: the same bits (the last step again: it writes the same places)
    again = marlin.attention_block(to_dev(A), *blk.args(), to_dev(lengths), K, q_heads, N, G, blk.ws, inv_freq=blk.inv if rotated else None,
                                   window=window, starts=to_dev(starts), **blk.scales)
    assert torch.equal(again, C)
    assert not blk.ws[256:8192].any()


def test_the_parts_called_one_by_one_give_the_same(marlin):
    import torch
    blk = Block(marlin, 4, 512, 8, 2, 64, 512, 128, 16, 40, 4, False, seed=3)
    blk.k_cache.normal_()
    blk.v_cache.normal_()
    A = torch.randn(4, 512, device="cuda").half()
    lengths = torch.tensor([1, 600, 17, 64], dtype=torch.int32, device="cuda")
    want = marlin.attention_block(A, *blk.args(), lengths, 512, 8, 512, 128, blk.ws, inv_freq=blk.inv)
    cache = (blk.k_cache, blk.v_cache, blk.table, lengths, blk.ws)
    for _ in range(3):  # the launches overlap at their edges
        qkv = marlin.gemm(A, blk.w_qkv, blk.s_qkv, 512, 768, 128, blk.ws)
        q = marlin.kv_append(qkv, *cache, inv_freq=blk.inv)
        o = marlin.attention_decode(q, *cache)
        got = marlin.gemm(o, blk.w_o, blk.s_o, 512, 512, 128, blk.ws)
        assert torch.equal(got, want)
    assert marlin.read_status(blk.ws) == 0


def test_a_decoding_loop_in_a_graph_is_the_prompt_at_once(marlin):
    # twelve tokens one at a time through one captured step, with the lengths growing on the device, against all at once:
    # the caches hold the same keys and values up to the order of sums in the layers (fp16 tolerance of the layer)
    import torch
    steps = 12
    one = Block(marlin, 2 * steps, 512, 8, 2, 64, 512, 128, 4, 5, 2, False, seed=5)
    A = torch.randn(2, steps, 512, device="cuda").half()
    lengths = torch.full((2,), steps, dtype=torch.int32, device="cuda")
    starts = torch.tensor([0, steps, 2 * steps], dtype=torch.int32, device="cuda")
    whole = marlin.attention_block(A.view(-1, 512), *one.args(), lengths, 512, 8, 512, 128, one.ws, inv_freq=one.inv, starts=starts)
    k, v = one.k_cache.clone(), one.v_cache.clone()
    one.k_cache.zero_(), one.v_cache.zero_()
    x = torch.zeros(2, 512, dtype=torch.float16, device="cuda")
    lengths.fill_(1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = marlin.attention_block(x, *one.args(), lengths, 512, 8, 512, 128, one.ws, inv_freq=one.inv)
    got = []
    for i in range(steps):
        x.copy_(A[:, i])
        graph.replay()
        got.append(y.clone())
        lengths += 1
    torch.cuda.synchronize()
    assert marlin.read_status(one.ws) == 0
    got = torch.stack(got, 1).view(-1, 512).float()
    for a, b in ((one.k_cache, k), (one.v_cache, v)):
        a, b = a.float(), b.float()
        rms = b[b != 0].square().mean().sqrt()
        # twice the layer's tolerance 5e-3 (|x| + rms), and for a rotated key that of both of its pair: sqrt(2) of the larger
        assert ((a - b).abs() <= 1.5 * 2 * 5e-3 * (b.abs().amax(-1, keepdim=True) + rms)).all()
    assert (got - whole.float()).abs().max() <= 0.05 * whole.float().abs().max()


def test_the_binding_refuses(marlin):
    import torch
    blk = Block(marlin, 4, 512, 8, 2, 64, 512, 128, 16, 4, 4, False, seed=3)
    A = torch.zeros(4, 512, device="cuda").half()
    q = torch.zeros(4, 512, device="cuda").half()
    qkv = torch.zeros(4, 768, device="cuda").half()
    lengths = torch.ones(4, dtype=torch.int32, device="cuda")
    k, v, pages, ws = blk.k_cache, blk.v_cache, blk.table, blk.ws
    inv = blk.inv

    def bad(error, fn, *args, **more):
        with pytest.raises(error):
            fn(*args, **more)
    for fn, x in ((marlin.kv_append, qkv), (marlin.attention_decode, q)):
        bad(TypeError, fn, x.float(), k, v, pages, lengths, ws)
        bad(TypeError, fn, x.cpu(), k, v, pages, lengths, ws)
        bad(ValueError, fn, x[0], k, v, pages, lengths, ws)
        bad(ValueError, fn, x[:, :-8], k, v, pages, lengths, ws)
        bad(ValueError, fn, x.t(), k, v, pages, lengths, ws)
        bad(ValueError, fn, x[:1].expand(4, -1), k, v, pages, lengths, ws)
        bad(TypeError, fn, x, k.float(), v.float(), pages, lengths, ws)
        bad(ValueError, fn, x, k, v[1:], pages, lengths, ws)
        bad(ValueError, fn, x, k, v.to(torch.float8_e4m3fn), pages, lengths, ws)
        bad(ValueError, fn, x, k, v.transpose(1, 2).contiguous().transpose(1, 2), pages, lengths, ws)
        bad(ValueError, fn, x, k[0], v[0], pages, lengths, ws)
        bad(ValueError, fn, x, k[:1].expand(9, -1, -1, -1), v[:1].expand(9, -1, -1, -1), pages, lengths, ws)
        bad(ValueError, fn, x, k[..., ::2], v[..., ::2], pages, lengths, ws)
        bad(TypeError, fn, x, k, v, pages.long(), lengths, ws)
        bad(TypeError, fn, x, k, v, pages, lengths.long(), ws)
        bad(ValueError, fn, x, k, v, pages[:3], lengths, ws)
        bad(ValueError, fn, x, k, v, pages, lengths[None], ws)
        bad(TypeError, fn, x, k, v, pages, lengths, ws.int())
        bad(ValueError, fn, x, k, v, pages, lengths, ws, starts=lengths)
        bad(TypeError, fn, x, k, v, pages, lengths, ws, starts=torch.zeros(5, dtype=torch.int64, device="cuda"))
        bad(ValueError, fn, x, k, v, pages, lengths, ws, k_scale=torch.ones(2, device="cuda"))
        bad(marlin.MarlinError, fn, x[:3], k, v, pages, lengths, ws)
        bad(marlin.MarlinError, fn, x[:0], k, v, pages, lengths, ws, starts=torch.zeros(5, dtype=torch.int32, device="cuda"))
        bad(marlin.MarlinError, fn, x, k, v, pages, lengths, ws[:4096])
        bad(marlin.MarlinError, fn, x, k[:, :, :3], v[:, :, :3], pages, lengths, ws)
        bad(marlin.MarlinError, fn, torch.zeros(4, 776, device="cuda").half()[:, 4:4 + x.shape[1]], k, v, pages, lengths, ws)
    bad(ValueError, marlin.attention_decode, q, k, v, pages, lengths, ws, out=q[:3])
    bad(TypeError, marlin.attention_decode, q, k, v, pages, lengths, ws, out=q.float())
    bad(marlin.MarlinError, marlin.attention_decode, q, k, v, pages, lengths, ws, window=-1)
    bad(TypeError, marlin.attention_decode, q, k, v, pages, lengths, ws, scale="x")
    bad(marlin.MarlinError, marlin.attention_decode, q[:, :64 * 7].contiguous(), k, v, pages, lengths, ws)
    bad(ValueError, marlin.kv_append, qkv[:, :128].contiguous(), k, v, pages, lengths, ws)
    bad(ValueError, marlin.kv_append, qkv, k, v, pages, lengths, ws, out=q)
    bad(TypeError, marlin.kv_append, qkv, k, v, pages, lengths, ws, inv_freq=inv.half())
    bad(ValueError, marlin.kv_append, qkv, k, v, pages, lengths, ws, inv_freq=torch.ones(33, device="cuda"))
    bad(marlin.MarlinError, marlin.kv_append, qkv, k, v, pages, lengths, ws, inv_freq=inv[:7])
    args = (A, *blk.args(), lengths, 512, 8, 512, 128)
    bad(ValueError, marlin.attention_block, A[:, :256], *args[1:], ws)
    bad(ValueError, marlin.attention_block, *args[:10], 9, 512, 128, ws)
    bad(ValueError, marlin.attention_block, *args, ws, QKV=q)
    bad(marlin.MarlinError, marlin.attention_block, *args, ws[:1 << 20])
    torch.cuda.synchronize()
    assert marlin.read_status(ws) == 0 and not ws.any()
    # keys alone: a layer of 2 kv_heads has no queries
    out = marlin.kv_append(qkv[:, 512:], k, v, pages, lengths, ws, inv_freq=inv)
    assert tuple(out.shape) == (4, 0)
