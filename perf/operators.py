"""What is timed of the paged key-value cache: appending new tokens (with the position rotation) and attention over it.

Every case is one call as a decoding loop makes it between the qkv layer and the output layer of a decoder layer.  The head
layouts are those of the layers that this repository benchmarks: 32 query and 32 key heads of 128 (hidden size 4096: a qkv layer
of 12288 columns) and 64 query heads on 8 key heads of 128 (hidden size 8192), and a generic one of 29 query heads per key head
of 64.  Activations are fp16, caches fp16 or e4m3 with a scale per key head.

`run` with `own` false is the plain form in elementary torch operations; with `own` true it calls the library.
"""
import math

import torch

own = False

WORKSPACE_BYTES = 64 << 20  # what a user allocates once; not less than the library asks for in any of these cases


def _case(name, op, seqs, shortest, longest, heads, kv_heads, dim, page, new=1, ragged=False, cache="fp16", window=0, rotary=0,
          interleaved=False, prompt=False):
    case = dict(op=op, seqs=seqs, shortest=shortest, longest=longest, heads=heads, kv_heads=kv_heads, dim=dim, page=page, new=new,
                ragged=ragged, cache=cache, window=window, rotary=rotary, interleaved=interleaved, prompt=prompt)
    return dict(name=name, **case) if name else case


def listed():
    return [
        # one sequence decodes: the smallest call, where only its latency counts
        _case("append 1 token", "append", 1, 700, 700, 32, 32, 128, 16, rotary=128),
        # a decode step of a full batch, grouped heads, sequences of all lengths
        _case("append 64 tokens", "append", 64, 5, 4099, 64, 8, 128, 16, rotary=128),
        # several drafted tokens per sequence into an 8-bit cache; half of each head is rotated, pairs side by side
        _case("append drafts e4m3", "append", 33, 100, 3001, 64, 8, 128, 32, new=5, ragged=True, cache="e4m3", rotary=64,
              interleaved=True),
        # prompts of five sequences in one batch
        _case("append prompts", "append", 5, 301, 4099, 32, 32, 128, 64, new=4099, prompt=True, rotary=128),
        # the smallest attention: one short sequence
        _case("attend 1 x 129", "attend", 1, 129, 129, 32, 32, 128, 16),
        # batch 16, a key head per query head, a thousand tokens
        _case("attend 16 x 1k", "attend", 16, 500, 1531, 32, 32, 128, 16),
        # a full batch of ragged sequences with grouped heads; one of them has nothing yet
        _case("attend 64 ragged gqa", "attend", 64, 0, 8191, 64, 8, 128, 16),
        # one very long sequence: all of the GPU works on one row of heads
        _case("attend 1 x 128k gqa", "attend", 1, 131009, 131009, 64, 8, 128, 64),
        # an 8-bit cache
        _case("attend 32 x 4k e4m3", "attend", 32, 2000, 4099, 64, 8, 128, 32, cache="e4m3"),
        # drafted tokens that the target checks: up to six queries per sequence, 48 rows per key head
        _case("attend drafts", "attend", 16, 1000, 4099, 64, 8, 128, 16, new=6, ragged=True),
        # heads of 64, 29 query heads per key head, a sliding window over long sequences
        _case("attend windows", "attend", 24, 900, 16001, 232, 8, 64, 32, window=2048),
        # the largest: a batch of long sequences with a key head per query head
        _case("attend 64 x 4k", "attend", 64, 2000, 4096, 32, 32, 128, 16),
    ]


HEADS = [(32, 32, 128), (64, 8, 128), (32, 8, 128), (40, 40, 128), (232, 8, 64), (71, 1, 64), (16, 4, 80), (16, 2, 256), (12, 12, 64)]
MOST_BYTES = 3 << 30


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    while True:
        heads, kv_heads, dim = rng.choice(HEADS)
        op = rng.choice(["append", "attend", "attend"])
        cache = rng.choice(["fp16", "fp16", "e4m3"])
        page = rng.choice([8, 16, 32, 64, 128])
        seqs = _spread(rng, 1, 128)
        longest = _spread(rng, 8, 140000 if op == "attend" else 8000)
        shortest = rng.randint(1, longest) if op == "append" else rng.randint(0, longest)
        rotary = rng.choice([dim, dim, 16 * max(1, dim // 32)]) if op == "append" else 0
        new = rng.choice([1, 1, rng.randint(2, 8)])
        prompt = op == "append" and rng.random() < 0.25
        window = rng.choice([0, 0, _spread(rng, 8, 5000)]) if op == "attend" else 0
        case = _case(None, op, seqs, shortest, longest, heads, kv_heads, dim, page, longest if prompt else new,
                     not prompt and new > 1 and rng.random() < 0.5, cache, window, rotary, rng.random() < 0.5 and op == "append", prompt)
        cached = seqs * (longest + page) * kv_heads * dim * (4 if cache == "fp16" else 2)  # as the plain form lays it out
        tokens = sum(n for _, n in _sequences(case))
        if cached <= MOST_BYTES and tokens * (heads + 2 * kv_heads) * dim * 4 <= MOST_BYTES // 4:
            if op == "append" or new * seqs * heads * longest <= 1 << 28:
                return case


def _sequences(case):
    """(length, new tokens) of every sequence: spread evenly from the shortest to the longest, the same for every seed."""
    pairs = []
    for i in range(case["seqs"]):
        part = (1 - i * 0.6180339887498949) % 1.0 if i else 1.0
        length = case["shortest"] + int(round((case["longest"] - case["shortest"]) * part)) if i else case["longest"]
        if i == 1:
            length = case["shortest"]
        new = length if case["prompt"] else (1 + i * 7 % case["new"] if case["ragged"] else case["new"])
        pairs.append((length, new if case["new"] == 1 else min(new, length)))
    return pairs


def _counts(case):
    """Keys that have to be read, and (query token, key) pairs."""
    keys = seen = 0
    for length, new in _sequences(case):
        if new == 0 or length == 0:
            continue
        first = length - new  # position of the first new token
        window = case["window"] or length + 1
        keys += length - max(0, first - window + 1)
        seen += sum(min(p + 1, window) for p in range(first, length)) if new < 64 else new * length
    return keys, seen


def work(case):
    dim, heads, kv_heads = case["dim"], case["heads"], case["kv_heads"]
    size = 2 if case["cache"] == "fp16" else 1
    tokens = sum(n for _, n in _sequences(case))
    if case["op"] == "append":
        return {"bytes": tokens * dim * (2 * (heads + 2 * kv_heads) + 2 * heads + 2 * size * kv_heads),
                "flops": 3 * tokens * (heads + kv_heads) * case["rotary"]}
    keys, seen = _counts(case)
    return {"bytes": 2 * keys * kv_heads * dim * size + 4 * tokens * heads * dim, "flops": 4 * dim * heads * seen}


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dim, heads, kv_heads, page = case["dim"], case["heads"], case["kv_heads"], case["page"]
    order = torch.randperm(case["seqs"], generator=gen, device="cuda").tolist()
    pairs = _sequences(case)
    pairs = [pairs[i] for i in order]
    used = [-(-length // page) for length, _ in pairs]
    width = max(max(used), 1) + 1
    pages = sum(used) + 3
    free = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)  # pages are handed out in no order
    table = torch.zeros(case["seqs"], width, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(used):
        table[b, :n] = free[at:at + n]
        at += n
    tokens = sum(n for _, n in pairs)

    def cache(spread):
        x = torch.randn(pages, kv_heads, page, dim, generator=gen, device="cuda", dtype=torch.float16) * spread
        return x if case["cache"] == "fp16" else x.clamp(-448, 448).to(torch.float8_e4m3fn)

    eight = case["cache"] == "e4m3"
    state = dict(case=case, tokens=tokens, page=page, dim=dim, heads=heads, kv_heads=kv_heads, window=case["window"],
                 k_cache=cache(16.0 if eight else 1.0), v_cache=cache(16.0 if eight else 1.0), table=table,
                 lengths=torch.tensor([length for length, _ in pairs], dtype=torch.int32, device="cuda"),
                 starts=None, k_scale=None, v_scale=None,
                 workspace=torch.zeros(WORKSPACE_BYTES, dtype=torch.uint8, device="cuda"))
    if case["new"] > 1:
        starts = [0]
        for _, n in pairs:
            starts.append(starts[-1] + n)
        state["starts"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
    if eight:
        state["k_scale"] = torch.empty(kv_heads, device="cuda").uniform_(0.04, 0.09, generator=gen)
        state["v_scale"] = torch.empty(kv_heads, device="cuda").uniform_(0.04, 0.09, generator=gen)
    if case["op"] == "append":
        state["qkv"] = torch.randn(tokens, (heads + 2 * kv_heads) * dim, generator=gen, device="cuda", dtype=torch.float16)
        half = torch.arange(case["rotary"] // 2, dtype=torch.float64, device="cuda")
        state["inv_freq"] = (10000.0 ** (-2.0 * half / case["rotary"])).float()
        state["interleaved"] = case["interleaved"]
    else:
        state["q"] = torch.randn(tokens, heads * dim, generator=gen, device="cuda", dtype=torch.float16) * 1.5
        state["scale"] = dim ** -0.5
    return state


def _starts(state):
    if state["starts"] is not None:
        return state["starts"].long()
    return torch.arange(state["lengths"].numel() + 1, device="cuda")


def _positions(state):
    """(sequence, position) of every token."""
    starts = _starts(state)
    token = torch.arange(state["tokens"], device="cuda")
    seq = torch.searchsorted(starts, token, right=True) - 1
    return seq, state["lengths"].long()[seq] - (starts[seq + 1] - token)


def _plain_append(state):
    dim, heads, kv_heads, page = state["dim"], state["heads"], state["kv_heads"], state["page"]
    x = state["qkv"].float().view(state["tokens"], heads + 2 * kv_heads, dim)
    seq, position = _positions(state)
    turned, half = x[:, :heads + kv_heads], state["inv_freq"].numel()
    angle = position.double()[:, None] * state["inv_freq"].double()
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    if state["interleaved"]:
        a, c = turned[..., 0:2 * half:2], turned[..., 1:2 * half:2]
        head = torch.stack((a * cos - c * sin, c * cos + a * sin), -1).flatten(-2)
    else:
        a, c = turned[..., :half], turned[..., half:2 * half]
        head = torch.cat((a * cos - c * sin, c * cos + a * sin), -1)
    turned = torch.cat((head, turned[..., 2 * half:]), -1)
    k, v = turned[:, heads:], x[:, heads + kv_heads:]
    if state["k_scale"] is not None:
        k = (k / state["k_scale"][:, None]).clamp(-448, 448)
        v = (v / state["v_scale"][:, None]).clamp(-448, 448)
    where = state["table"].long()[seq, position // page], slice(None), position % page
    for cache, new in ((state["k_cache"], k), (state["v_cache"], v)):
        new = new.to(cache.dtype)
        if cache.dtype == torch.float8_e4m3fn:
            cache, new = cache.view(torch.uint8), new.view(torch.uint8)
        cache[where] = new
    return turned[:, :heads].to(torch.float16).reshape(state["tokens"], heads * dim), state["k_cache"], state["v_cache"]


def _gathered(cache, table, scale):
    """Pages of every sequence side by side, in 32 bits: [sequences, heads, tokens, dim]."""
    x = cache.view(torch.uint8)[table.long()].view(cache.dtype) if cache.dtype == torch.float8_e4m3fn else cache[table.long()]
    x = x.float().transpose(1, 2).flatten(2, 3)
    return x if scale is None else x * scale[:, None, None]


def _plain_attend(state):
    dim, heads, kv_heads = state["dim"], state["heads"], state["kv_heads"]
    starts, lengths = _starts(state), state["lengths"].long()
    seqs, most = lengths.numel(), state["case"]["new"]
    seq, position = _positions(state)
    rank = torch.arange(state["tokens"], device="cuda") - starts[seq]
    q = torch.zeros(seqs, most, heads * dim, device="cuda")
    q[seq, rank] = state["q"].float()
    q = q.view(seqs, most, kv_heads, heads // kv_heads, dim).permute(0, 2, 1, 3, 4).flatten(2, 3)
    k = _gathered(state["k_cache"], state["table"], state["k_scale"])
    v = _gathered(state["v_cache"], state["table"], state["v_scale"])
    logits = q @ k.transpose(2, 3) * state["scale"]  # [sequences, key heads, new * group, tokens]
    place = torch.full((seqs, most), -1, dtype=torch.long, device="cuda")
    place[seq, rank] = position
    token = torch.arange(k.shape[2], device="cuda")
    visible = token <= place[..., None]
    if state["window"]:
        visible &= token > place[..., None] - state["window"]
    visible = visible.repeat_interleave(heads // kv_heads, 1)[:, None]
    top = logits.masked_fill(~visible, -math.inf).amax(-1, keepdim=True).clamp_min(-3e38)
    weight = ((logits - top).exp()).masked_fill(~visible, 0.0)
    total = weight.sum(-1, keepdim=True)
    out = weight @ v / torch.where(total > 0, total, 1.0)
    out = out.view(seqs, kv_heads, most, heads // kv_heads, dim).permute(0, 2, 1, 3, 4).reshape(seqs, most, heads * dim)
    return out[seq, rank].to(torch.float16)


def run(state):
    if own:
        import paper_2408_11743_b200 as marlin
        if state["case"]["op"] == "append":
            q = marlin.kv_append(state["qkv"], state["k_cache"], state["v_cache"], state["table"], state["lengths"], state["workspace"],
                                 inv_freq=state["inv_freq"], interleaved=state["interleaved"], starts=state["starts"],
                                 k_scale=state["k_scale"], v_scale=state["v_scale"])
            return q, state["k_cache"], state["v_cache"]
        return marlin.attention_decode(state["q"], state["k_cache"], state["v_cache"], state["table"], state["lengths"],
                                       state["workspace"], scale=state["scale"], window=state["window"], starts=state["starts"],
                                       k_scale=state["k_scale"], v_scale=state["v_scale"])
    return _plain_append(state) if state["case"]["op"] == "append" else _plain_attend(state)


def exact(case, seed):
    """The definition, token by token or sequence by sequence, in 64 bits."""
    state = prepare(case, seed)
    dim, heads, kv_heads, page = case["dim"], case["heads"], case["kv_heads"], case["page"]
    lengths = state["lengths"].tolist()
    starts = state["starts"].tolist() if state["starts"] is not None else list(range(len(lengths) + 1))
    size = state["k_cache"].numel() * 8
    if size > 24 << 30 and case["op"] == "append":
        return None
    group = heads // kv_heads
    if case["op"] == "attend":
        out = torch.zeros(state["tokens"], heads, dim, dtype=torch.float64, device="cuda")
        for b, length in enumerate(lengths):
            if length == 0:
                continue
            mine = state["table"][b, :-(-length // page)].tolist()
            both = []
            for cache, scale in ((state["k_cache"], state["k_scale"]), (state["v_cache"], state["v_scale"])):
                x = torch.cat([cache[p].float() for p in mine], 1)[:, :length].double() if len(mine) < 64 else \
                    cache.view(torch.uint8 if cache.dtype == torch.float8_e4m3fn else cache.dtype)[mine].view(cache.dtype) \
                    .double().permute(1, 0, 2, 3).reshape(kv_heads, -1, dim)[:, :length]
                both.append(x if scale is None else x * scale.double().view(-1, 1, 1))
            k, v = both
            for t in range(starts[b], starts[b + 1]):
                last = length - (starts[b + 1] - t)
                first = max(0, last - case["window"] + 1) if case["window"] else 0
                q = state["q"][t].double().view(kv_heads, group, dim)
                weight = torch.softmax(torch.einsum("hgd,hjd->hgj", q, k[:, first:last + 1]) * state["scale"], -1)
                out[t] = torch.einsum("hgj,hjd->hgd", weight, v[:, first:last + 1]).reshape(heads, dim)
        return out.view(state["tokens"], heads * dim)
    x = state["qkv"].double().view(state["tokens"], heads + 2 * kv_heads, dim)
    half = case["rotary"] // 2
    position = torch.cat([torch.arange(n - (e - s), n) for n, s, e in zip(lengths, starts, starts[1:])]).cuda()
    first = torch.arange(half, device="cuda") * 2 if case["interleaved"] else torch.arange(half, device="cuda")
    second = first + 1 if case["interleaved"] else first + half
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), position.double().outer(state["inv_freq"].double()))
    y = x.clone()
    z = torch.complex(x[:, :heads + kv_heads, first], x[:, :heads + kv_heads, second]) * turn[:, None]
    y[:, :heads + kv_heads, first], y[:, :heads + kv_heads, second] = z.real, z.imag
    k, v = y[:, heads:heads + kv_heads], y[:, heads + kv_heads:]
    if state["k_scale"] is not None:
        k, v = k / state["k_scale"].double().view(-1, 1), v / state["v_scale"].double().view(-1, 1)
    k_cache, v_cache = state["k_cache"].double(), state["v_cache"].double()
    seq = torch.cat([torch.full((e - s,), b) for b, (s, e) in enumerate(zip(starts, starts[1:]))]).cuda()
    at = state["table"].long()[seq, position // page]
    k_cache[at, :, position % page], v_cache[at, :, position % page] = k, v
    return y[:, :heads].reshape(state["tokens"], heads * dim), k_cache, v_cache
