"""What is timed of a paged key-value cache that looks after itself: its page tables and slot maps made on the GPU from the lengths of the
requests, 8-bit keys and values with a scale for each block of tokens and key head (appended and attended), and attention through a
window with a few first tokens that stay visible.

Every case is one call (or, of the tables, a step and the step that takes it back) as a serving loop makes it around the qkv layer and
the output layer of a decoder layer.  The head layouts are those of `operators.py` beside this file: 32 query and 32 key heads of 128, 64 query heads on
8 key heads of 128, and 29 query heads per key head of 64.  Queries are fp16; caches fp16, int8 or e4m3.

`run` with `own` false is the plain form in elementary torch operations; with `own` true it calls the library.
"""
import math

import torch

own = False

WORKSPACE_BYTES = 64 << 20  # what a user allocates once; not less than the library asks for in any of these cases
LARGEST = {"int8": 127.0, "e4m3": 448.0}  # the code that the largest value of a block gets


def _named(name, case):
    return dict(name=name, **case) if name else case


def _tables(name, seqs, shortest, longest, page, least, most, ending):
    """A step of a batch: `ending` of a hundred sequences end, the others get `least` to `most` new tokens."""
    return _named(name, dict(op="reserve", seqs=seqs, shortest=shortest, longest=longest, page=page, least=least, most=most, ending=ending))


def _case(name, op, seqs, shortest, longest, heads, kv_heads, dim, page, block=0, new=1, ragged=False, cache="fp16", window=0, sinks=0,
          rotary=0, interleaved=False, prompt=False):
    return _named(name, dict(op=op, seqs=seqs, shortest=shortest, longest=longest, heads=heads, kv_heads=kv_heads, dim=dim, page=page,
                             block=block, new=new, ragged=ragged, cache=cache, window=window, sinks=sinks, rotary=rotary,
                             interleaved=interleaved, prompt=prompt))


def listed():
    return [
        # a decode step: a page for every sixteenth sequence, some requests end
        _tables("tables 64 x 1", 64, 5, 4099, 16, 1, 1, 5),
        # a thousand requests of which most begin: prompts of up to 700 tokens, a table row and a slot for each of them
        _tables("tables 1000 prompts", 1000, 0, 2001, 32, 1, 700, 20),
        # one sequence decodes: the smallest call, where only its latency counts
        _case("append 1 token e4m3", "append", 1, 700, 700, 32, 32, 128, 16, block=16, cache="e4m3", rotary=128),
        # a decode step of a full batch, grouped heads.  (The forms round a rotation differently in its last bit, and a code on a border may then
        # be either of two.  Whole numbers are compared exactly: so int8 codes are appended without a rotation here.)
        _case("append 64 tokens int8", "append", 64, 5, 4099, 64, 8, 128, 32, block=32, cache="int8"),
        # prompts of five sequences in one batch
        _case("append prompts e4m3", "append", 5, 301, 4099, 32, 32, 128, 64, block=64, new=4099, cache="e4m3", prompt=True, rotary=128),
        # the smallest attention: one short sequence
        _case("attend 1 x 129 int8", "attend", 1, 129, 129, 32, 32, 128, 16, block=16, cache="int8"),
        # a full batch of ragged sequences with grouped heads; one of them has nothing yet
        _case("attend 64 ragged int8", "attend", 64, 0, 8191, 64, 8, 128, 16, block=16, cache="int8"),
        # drafted tokens that the target checks: up to six queries per sequence, 48 rows per key head
        _case("attend drafts e4m3", "attend", 16, 1000, 4099, 64, 8, 128, 32, block=8, new=6, ragged=True, cache="e4m3"),
        # a conversation far past what the layer sees: four first tokens and the last four thousand of 131 thousand
        _case("sinks 1 x 128k", "attend", 1, 131009, 131009, 64, 8, 128, 64, window=4096, sinks=4),
        # heads of 64, 29 query heads per key head, a batch of long sequences
        _case("sinks 24 ragged", "attend", 24, 900, 16001, 232, 8, 64, 32, window=2048, sinks=100),
        # the next 700 tokens of three prompts at once
        _case("sinks prompts", "attend", 3, 701, 2600, 64, 8, 128, 16, new=700, window=512, sinks=4),
        # the largest: a batch of long sequences with a key head per query head
        _case("attend 64 x 4k int8", "attend", 64, 2000, 4096, 32, 32, 128, 64, block=64, cache="int8"),
    ]


HEADS = [(32, 32, 128), (64, 8, 128), (32, 8, 128), (40, 40, 128), (232, 8, 64), (71, 1, 64), (16, 4, 80), (16, 2, 256), (12, 12, 64)]
MOST_BYTES = 3 << 30


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    while True:
        op = rng.choice(["reserve", "append", "attend", "attend", "attend"])
        page = rng.choice([8, 16, 32, 64, 128])
        if op == "reserve":
            most = rng.choice([1, rng.randint(2, 8), _spread(rng, 8, 1000)])
            longest = _spread(rng, 8, 20000)
            case = _tables(None, _spread(rng, 1, 3000), rng.randint(0, longest), longest, page, rng.randint(0, 1), most, rng.choice([0, 3, 30]))
            if case["seqs"] * most <= 400000 and case["seqs"] * longest <= page << 20:
                return case
            continue
        heads, kv_heads, dim = rng.choice(HEADS)
        cache = rng.choice(["int8", "e4m3"] if op == "append" or rng.random() < 0.6 else ["fp16"])
        block = 0 if cache == "fp16" else 1 << rng.randint(0, min(page.bit_length() - 1, 6))
        seqs = _spread(rng, 1, 128)
        longest = _spread(rng, 8, 140000 if op == "attend" else 8000)
        shortest = rng.randint(1, longest) if op == "append" else rng.randint(0, longest)
        rotary = rng.choice([dim, 16 * max(1, dim // 32)]) if op == "append" and cache == "e4m3" else 0
        new = rng.choice([1, 1, rng.randint(2, 8)])
        prompt = op == "append" and rng.random() < 0.25
        window = sinks = 0
        if op == "attend" and (cache == "fp16" or rng.random() < 0.4):
            window, sinks = _spread(rng, 8, 5000), _spread(rng, 1, 200)
            if rng.random() < 0.25:
                new = min(longest, _spread(rng, 9, 1000))
        case = _case(None, op, seqs, shortest, longest, heads, kv_heads, dim, page, block, longest if prompt else new,
                     not prompt and new > 1 and rng.random() < 0.5, cache, window, sinks, rotary, rng.random() < 0.5 and op == "append", prompt)
        cached = seqs * (longest + page) * kv_heads * dim * (4 if cache == "fp16" else 2)  # as the plain form lays it out
        tokens = sum(n for _, n in _sequences(case))
        if cached <= MOST_BYTES and tokens * (heads + 2 * kv_heads) * dim * 4 <= MOST_BYTES // 4:
            if (op == "append" or new * seqs * heads * longest <= 1 << 28) and work(case)["bytes"] <= 1.5e9 and work(case)["flops"] <= 3e10:
                return case


def _spaced(i):
    """A number from 0 to 1 for each sequence, spread evenly, 1 first and 0 second."""
    return 1.0 if i == 0 else 0.0 if i == 1 else (1 - i * 0.6180339887498949) % 1.0


def _sequences(case):
    """(length, new tokens) of every sequence: spread evenly from the shortest to the longest, the same for every seed."""
    pairs = []
    for i in range(case["seqs"]):
        length = case["shortest"] + int(round((case["longest"] - case["shortest"]) * _spaced(i)))
        new = length if case["prompt"] else (1 + i * 7 % case["new"] if case["ragged"] else case["new"])
        pairs.append((length, new if case["new"] == 1 else min(new, length)))
    return pairs


def _steps(case):
    """(length, kept, new tokens) of every sequence of a step; one that ends keeps nothing and gets nothing."""
    steps = []
    for i in range(case["seqs"]):
        length = case["shortest"] + int(round((case["longest"] - case["shortest"]) * _spaced(i)))
        ends = i * 37 % 100 < case["ending"] and i > 0
        new = case["least"] + i * 7919 % (case["most"] - case["least"] + 1)
        steps.append((length, 0, 0) if ends else (length, length, new))
    return steps


def _counts(case):
    """Keys that have to be read, and (query token, key) pairs."""
    keys = seen = 0
    for length, new in _sequences(case):
        if new == 0 or length == 0:
            continue
        first = max(0, length - new)  # position of the first new token
        window, sinks = case["window"] or length + 1, case["sinks"]
        low = max(0, first - window + 1)
        keys += length - low + min(sinks, low)
        for p in range(first, length):
            low = max(0, p - window + 1)
            seen += p + 1 - low + min(sinks, low)
    return keys, seen


def work(case):
    if case["op"] == "reserve":
        page, steps = case["page"], _steps(case)
        tokens = sum(n for _, _, n in steps)
        back = sum(length - kept for length, kept, _ in steps)
        moved = sum(abs(-(-(kept + n) // page) - -(-length // page)) for length, kept, n in steps)
        # of both steps: length, kept, count and begin of each sequence, a slot and a position for each token, a page number read and written
        return {"bytes": 2 * 20 * case["seqs"] + 12 * (tokens + back) + 2 * 8 * moved, "flops": 0}
    dim, heads, kv_heads = case["dim"], case["heads"], case["kv_heads"]
    size = 2 if case["cache"] == "fp16" else 1
    tokens = sum(n for _, n in _sequences(case))
    if case["op"] == "append":
        turned = heads if case["rotary"] else 0
        scales = sum(length // case["block"] - max(0, length - n) // case["block"] + 1 for length, n in _sequences(case)) * kv_heads * 16
        return {"bytes": tokens * dim * (4 * turned + 2 * 2 * kv_heads + 2 * size * kv_heads) + scales,
                "flops": tokens * (3 * (turned + kv_heads) * case["rotary"] + 4 * kv_heads * dim)}
    keys, seen = _counts(case)
    return {"bytes": 2 * keys * kv_heads * dim * size + (8 * keys * kv_heads // case["block"] if case["block"] else 0) + 4 * tokens * heads * dim,
            "flops": 4 * dim * heads * seen}


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _pages(lengths, page, gen, spare):
    """Pages handed out in no order: (table, its unused pages as a stack, how many pages there are)."""
    used = [-(-n // page) for n in lengths]
    pages = sum(used) + spare
    free = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    return used, pages, free


def _prepare_tables(case, gen):
    steps = _steps(case)
    order = torch.randperm(case["seqs"], generator=gen, device="cuda").tolist()
    steps = [steps[i] for i in order]
    page = case["page"]
    longest = max(max(length, kept + n) for length, kept, n in steps)
    spare = sum(max(0, -(-(kept + n) // page) - -(-length // page)) for length, kept, n in steps) + 7
    used, pages, order = _pages([length for length, _, _ in steps], page, gen, spare)
    width = -(-longest // page) + 1
    owner = torch.repeat_interleave(torch.arange(case["seqs"], device="cuda"), _ints(used).long())
    entry = torch.arange(sum(used), device="cuda") - (_ints(used).long().cumsum(0) - _ints(used))[owner]
    table = torch.zeros(case["seqs"], width, dtype=torch.int32, device="cuda")
    table[owner, entry] = order[:sum(used)]
    free = torch.full((pages,), -1, dtype=torch.int32, device="cuda")
    free[:pages - sum(used)] = order[sum(used):]
    after = [kept + n for _, kept, n in steps]
    return dict(case=case, page=page, table=table, free=free, free_count=_ints([pages - sum(used)]),
                lengths=_ints([length for length, _, _ in steps]),
                steps=[dict(keep=_ints([kept for _, kept, _ in steps]), counts=_ints([n for _, _, n in steps]), tokens=sum(n for _, _, n in steps)),
                       dict(keep=_ints([kept for _, kept, _ in steps]), counts=_ints([length - kept for length, kept, _ in steps]),
                            tokens=sum(length - kept for length, kept, _ in steps))],
                most=max(after + [1]), workspace=torch.zeros(1 << 20, dtype=torch.uint8, device="cuda"))


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    if case["op"] == "reserve":
        return _prepare_tables(case, gen)
    dim, heads, kv_heads, page, block = case["dim"], case["heads"], case["kv_heads"], case["page"], case["block"]
    order = torch.randperm(case["seqs"], generator=gen, device="cuda").tolist()
    pairs = _sequences(case)
    pairs = [pairs[i] for i in order]
    used, pages, free = _pages([length for length, _ in pairs], page, gen, 3)
    width = max(max(used), 1) + 1
    table = torch.zeros(case["seqs"], width, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(used):
        table[b, :n] = free[at:at + n]
        at += n
    tokens = sum(n for _, n in pairs)

    def cache():
        x = torch.randn(pages, kv_heads, page, dim, generator=gen, device="cuda", dtype=torch.float16)
        if case["cache"] == "fp16":
            return x
        if case["cache"] == "int8":
            return (x * 38).round().clamp(-127, 127).to(torch.int8)
        return (x * 120).clamp(-448, 448).to(torch.float8_e4m3fn)

    def scales():
        if case["cache"] == "fp16":
            return None
        x = torch.empty(pages, kv_heads, page // block, device="cuda").uniform_(2.0, 4.5, generator=gen)
        return x / LARGEST[case["cache"]]

    state = dict(case=case, tokens=tokens, page=page, dim=dim, heads=heads, kv_heads=kv_heads, window=case["window"], sinks=case["sinks"],
                 block=block, k_cache=cache(), v_cache=cache(), k_scale=scales(), v_scale=scales(), table=table,
                 lengths=_ints([length for length, _ in pairs]), starts=None,
                 workspace=torch.zeros(WORKSPACE_BYTES, dtype=torch.uint8, device="cuda"))
    if case["new"] > 1:
        starts = [0]
        for _, n in pairs:
            starts.append(starts[-1] + n)
        state["starts"] = _ints(starts)
    if case["op"] == "append":
        state["qkv"] = torch.randn(tokens, (heads + 2 * kv_heads) * dim, generator=gen, device="cuda", dtype=torch.float16)
        half = torch.arange(case["rotary"] // 2, dtype=torch.float64, device="cuda")
        state["inv_freq"] = (10000.0 ** (-2.0 * half / case["rotary"])).float() if case["rotary"] else None
        state["interleaved"] = case["interleaved"]
        # blocks that get new tokens: how many there are is known as the number of tokens is
        state["runs"] = sum((length - 1) // block - (length - n) // block + 1 for length, n in pairs if n)
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


def _plain_reserve(state, step):
    lengths, table, free, page = state["lengths"], state["table"], state["free"], state["page"]
    old = torch.where(lengths < 0, ~lengths, lengths).long()
    counts = step["counts"].long().clamp_min(0)
    base = torch.minimum(step["keep"].long().clamp_min(0), old)
    held, after = -(-old // page), -(-(base + counts) // page)
    ends = counts.cumsum(0)
    fits = (after <= table.shape[1]) & (ends <= step["tokens"])
    need = (after - held).clamp_min(0) * fits
    upto, there = need.cumsum(0), state["free_count"].long()
    served = fits & ((need == 0) | (upto <= there))
    taken = (upto * (served & (need > 0))).amax()
    # new entries of the rows, from the top of the stack
    entry = torch.arange(table.shape[1], device="cuda")
    nth = (upto - need)[:, None] + entry - held[:, None]
    grows = (served & (need > 0))[:, None] & (entry >= held[:, None]) & (entry < after[:, None])
    table.copy_(torch.where(grows, free[(there - 1 - nth).clamp(0, free.numel() - 1)], table))
    # entries that are given back, in the order in which they would be taken again
    back = (held - after).clamp_min(0) * served
    gone, before = back.sum(), back.cumsum(0) - back
    now = there - taken + gone
    nth = before[:, None] + entry - after[:, None]
    shrinks = (back > 0)[:, None] & (entry >= after[:, None]) & (entry < held[:, None])
    to = torch.where(shrinks, now - 1 - nth, free.numel()).clamp(0, free.numel())
    free.copy_(torch.cat((free, free[:1])).scatter(0, to.flatten(), table.flatten())[:-1])
    state["free_count"].copy_(now)
    lengths.copy_(torch.where(served, base + counts, ~old))
    starts = torch.cat((ends[:1] * 0, ends))
    token = torch.arange(step["tokens"], device="cuda")
    seq = torch.searchsorted(starts, token, right=True) - 1
    mine = (seq >= 0) & (seq < counts.numel())
    seq = seq.clamp(0, counts.numel() - 1)
    mine &= served[seq]
    position = torch.where(mine, base[seq] + token - starts[seq], -1)
    number = table[seq, (position // page).clamp_min(0)].long()
    slot = torch.where(mine & (number >= 0), number * page + position % page, -1)
    return starts.int(), slot, position.int()


def _plain_append(state):
    dim, heads, kv_heads, page, block = state["dim"], state["heads"], state["kv_heads"], state["page"], state["block"]
    x = state["qkv"].float().view(state["tokens"], heads + 2 * kv_heads, dim)
    seq, position = _positions(state)
    turned = x[:, :heads + kv_heads]
    if state["inv_freq"] is not None:
        half = state["inv_freq"].numel()
        angle = position.double()[:, None] * state["inv_freq"].double()
        cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
        if state["interleaved"]:
            a, c = turned[..., 0:2 * half:2], turned[..., 1:2 * half:2]
            head = torch.stack((a * cos - c * sin, c * cos + a * sin), -1).flatten(-2)
        else:
            a, c = turned[..., :half], turned[..., half:2 * half]
            head = torch.cat((a * cos - c * sin, c * cos + a * sin), -1)
        turned = torch.cat((head, turned[..., 2 * half:]), -1)
    # the tokens of one block of one sequence are a run
    token = torch.arange(state["tokens"], device="cuda")
    first = (position % block == 0) | (token == _starts(state)[seq])
    run = first.cumsum(0) - 1
    lead = torch.zeros(state["runs"], dtype=torch.long, device="cuda").scatter_reduce_(0, run, token, "amin", include_self=False)
    there = position[lead] % block  # tokens that the block has already
    number, part = state["table"].long()[seq[lead], position[lead] // page], position[lead] % page // block
    slot = torch.arange(block, device="cuda") + (part * block)[:, None]
    largest = LARGEST[state["case"]["cache"]]
    for cache, scale, new in ((state["k_cache"], state["k_scale"], turned[:, heads:]), (state["v_cache"], state["v_scale"], x[:, heads + kv_heads:])):
        top = torch.zeros(state["runs"], kv_heads, device="cuda").scatter_reduce_(0, run[:, None].expand(-1, kv_heads), new.abs().amax(-1), "amax")
        need = top / largest
        old = scale[number, :, part]
        begun = (there > 0)[:, None] & (old > 0)
        doublings = (need.double() / torch.where(begun, old, 1.0).double()).log2().ceil().clamp_min(0) * begun
        now = torch.where(begun, old * torch.exp2(doublings).float(), need)
        scale[number, :, part] = now
        inverse = torch.where(now > 0, 1 / now, 0.0)
        codes = cache.view(torch.uint8) if cache.dtype == torch.float8_e4m3fn else cache

        def rounded(y):
            if cache.dtype == torch.float8_e4m3fn:
                return y.clamp(-448, 448).to(cache.dtype).view(torch.uint8)
            return y.round().clamp(-127, 127).to(cache.dtype)

        held = codes[number[:, None], :, slot]  # [runs, block, heads, dim]
        shrunk = held.view(cache.dtype).float() * torch.where(begun, torch.exp2(-doublings).float(), 0.0)[:, None, :, None]
        kept = torch.arange(block, device="cuda") < there[:, None]
        codes[number[:, None], :, slot] = torch.where(kept[:, :, None, None], rounded(shrunk), held)
        codes[state["table"].long()[seq, position // page], :, position % page] = rounded(new * inverse[run][..., None])
    q = turned[:, :heads].to(torch.float16).reshape(state["tokens"], heads * dim)
    return q, state["k_cache"], state["v_cache"], state["k_scale"], state["v_scale"]


def _gathered(cache, table, scale, block):
    """Pages of every sequence side by side, in 32 bits: [sequences, heads, tokens, dim]."""
    x = cache.view(torch.uint8)[table.long()].view(cache.dtype) if cache.dtype == torch.float8_e4m3fn else cache[table.long()]
    x = x.float().transpose(1, 2)  # [sequences, heads, pages, page, dim]
    if scale is not None:
        x = x * scale[table.long()].transpose(1, 2).repeat_interleave(block, -1)[..., None]
    return x.flatten(2, 3)


def _plain_attend(state):
    dim, heads, kv_heads = state["dim"], state["heads"], state["kv_heads"]
    starts, lengths = _starts(state), state["lengths"].long()
    seqs, most = lengths.numel(), state["case"]["new"]
    seq, position = _positions(state)
    rank = torch.arange(state["tokens"], device="cuda") - starts[seq]
    q = torch.zeros(seqs, most, heads * dim, device="cuda")
    q[seq, rank] = state["q"].float()
    q = q.view(seqs, most, kv_heads, heads // kv_heads, dim).permute(0, 2, 1, 3, 4).flatten(2, 3)
    k = _gathered(state["k_cache"], state["table"], state["k_scale"], state["block"])
    v = _gathered(state["v_cache"], state["table"], state["v_scale"], state["block"])
    logits = q @ k.transpose(2, 3) * state["scale"]  # [sequences, key heads, new * group, tokens]
    place = torch.full((seqs, most), -1, dtype=torch.long, device="cuda")
    place[seq, rank] = position
    token = torch.arange(k.shape[2], device="cuda")
    visible = token <= place[..., None]
    if state["window"]:
        visible &= (token > place[..., None] - state["window"]) | (token < state["sinks"])
    visible = visible.repeat_interleave(heads // kv_heads, 1)[:, None]
    top = logits.masked_fill(~visible, -math.inf).amax(-1, keepdim=True).clamp_min(-3e38)
    weight = ((logits - top).exp()).masked_fill(~visible, 0.0)
    total = weight.sum(-1, keepdim=True)
    out = weight @ v / torch.where(total > 0, total, 1.0)
    out = out.view(seqs, kv_heads, most, heads // kv_heads, dim).permute(0, 2, 1, 3, 4).reshape(seqs, most, heads * dim)
    return out[seq, rank].to(torch.float16)


def run(state):
    op = state["case"]["op"]
    if op == "reserve":
        outs = []
        for step in state["steps"]:
            if own:
                import paper_2408_11743_b200 as marlin
                outs += marlin.kv_reserve(state["lengths"], state["table"], state["free"], state["free_count"], state["workspace"],
                                          state["page"], step["tokens"], counts=step["counts"], keep=step["keep"])
            else:
                outs += _plain_reserve(state, step)
        return outs + [state["lengths"], state["table"], state["free"], state["free_count"]]
    if own:
        import paper_2408_11743_b200 as marlin
        if op == "append":
            q = marlin.kv_append(state["qkv"], state["k_cache"], state["v_cache"], state["table"], state["lengths"], state["workspace"],
                                 inv_freq=state["inv_freq"], interleaved=state["interleaved"], starts=state["starts"],
                                 k_scale=state["k_scale"], v_scale=state["v_scale"])
            return q, state["k_cache"], state["v_cache"], state["k_scale"], state["v_scale"]
        return marlin.attention_decode(state["q"], state["k_cache"], state["v_cache"], state["table"], state["lengths"],
                                       state["workspace"], scale=state["scale"], window=state["window"], sinks=state["sinks"],
                                       starts=state["starts"], k_scale=state["k_scale"], v_scale=state["v_scale"])
    return _plain_append(state) if op == "append" else _plain_attend(state)


def _exact_attend(case, state, lengths, starts):
    dim, heads, kv_heads, page = case["dim"], case["heads"], case["kv_heads"], case["page"]
    if case["new"] * case["seqs"] * heads * case["longest"] > 1 << 29:
        return None
    out = torch.zeros(state["tokens"], heads, dim, dtype=torch.float64, device="cuda")
    for b, length in enumerate(lengths):
        new = starts[b + 1] - starts[b]
        if length == 0 or new == 0:
            continue
        mine = state["table"][b, :-(-length // page)].long()
        both = []
        for cache, scale in ((state["k_cache"], state["k_scale"]), (state["v_cache"], state["v_scale"])):
            x = (cache.view(torch.uint8)[mine].view(cache.dtype) if case["cache"] == "e4m3" else cache[mine]).double()
            if scale is not None:
                x = x.unflatten(2, (-1, case["block"])) * scale[mine].double()[..., None, None]
                x = x.flatten(2, 3)
            both.append(x.permute(1, 0, 2, 3).reshape(kv_heads, -1, dim)[:, :length])
        k, v = both
        step = max(1, (1 << 27) // (heads * length))  # rows at a time
        for t in range(0, new, step):
            n = min(step, new - t)
            last = torch.arange(length - new + t, length - new + t + n, device="cuda")
            key = torch.arange(length, device="cuda")
            seen = key[None] <= last[:, None]
            if case["window"]:
                seen &= (key[None] > last[:, None] - case["window"]) | (key[None] < case["sinks"])
            q = state["q"][starts[b] + t:starts[b] + t + n].double().view(n, kv_heads, heads // kv_heads, dim)
            logits = torch.einsum("thgd,hjd->thgj", q, k) * state["scale"]
            weight = torch.softmax(torch.where(seen[:, None, None], logits, -math.inf), -1)
            out[starts[b] + t:starts[b] + t + n] = torch.einsum("thgj,hjd->thgd", weight, v).reshape(n, heads, dim)
    return out.view(state["tokens"], heads * dim)


def exact(case, seed):
    """The definition, sequence by sequence or block by block, in 64 bits; nothing in the place of codes that are whole numbers."""
    if case["op"] == "reserve":
        return None
    state = prepare(case, seed)
    dim, heads, kv_heads, page, block = case["dim"], case["heads"], case["kv_heads"], case["page"], case["block"]
    lengths = state["lengths"].tolist()
    starts = state["starts"].tolist() if state["starts"] is not None else list(range(len(lengths) + 1))
    if case["op"] == "attend":
        return _exact_attend(case, state, lengths, starts)
    if state["k_cache"].numel() * 8 > 24 << 30 or state["runs"] > 3000:
        return None
    x = state["qkv"].double().view(state["tokens"], heads + 2 * kv_heads, dim)
    position = torch.cat([torch.arange(n - (e - s), n) for n, s, e in zip(lengths, starts, starts[1:])]).cuda()
    y = x.clone()
    if case["rotary"]:
        half = case["rotary"] // 2
        one = torch.arange(half, device="cuda") * 2 if case["interleaved"] else torch.arange(half, device="cuda")
        two = one + 1 if case["interleaved"] else one + half
        turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), position.double().outer(state["inv_freq"].double()))
        z = torch.complex(x[:, :heads + kv_heads, one], x[:, :heads + kv_heads, two]) * turn[:, None]
        y[:, :heads + kv_heads, one], y[:, :heads + kv_heads, two] = z.real, z.imag
    table = state["table"].tolist()
    whole, found = case["cache"] == "int8", []
    for cache, scale, new in ((state["k_cache"], state["k_scale"], y[:, heads:heads + kv_heads]), (state["v_cache"], state["v_scale"], y[:, heads + kv_heads:])):
        codes, scales = None if whole else cache.double(), scale.double()
        for b, length in enumerate(lengths):
            at = length - (starts[b + 1] - starts[b])
            while at < length:
                end = min(length, at // block * block + block)
                number, part = table[b][at // page], at % page // block
                rows = new[starts[b + 1] - (length - at):starts[b + 1] - (length - end)]  # [tokens, heads, dim]
                need, old = rows.abs().amax((0, 2)) / LARGEST[case["cache"]], scales[number, :, part].clone()
                if at % block:
                    times = torch.exp2((need / old).log2().ceil().clamp_min(0))
                    scales[number, :, part] = old * times
                    if not whole:
                        codes[number, :, part * block:at % page] /= times[:, None, None]
                else:
                    scales[number, :, part] = need
                if not whole:
                    codes[number, :, at % page:at % page + end - at] = (rows / scales[number, :, part][:, None]).transpose(0, 1)
                at = end
        found.append((codes, scales))
    return y[:, :heads].reshape(state["tokens"], heads * dim), found[0][0], found[1][0], found[0][1], found[1][1]
