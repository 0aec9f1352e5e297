"""GPU: page tables and slot maps from lengths, against an oracle that goes through the sequences one after the other."""
import numpy as np
import pytest

from oracle import cache_blocks_ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def marlin():
    import torch
    assert torch.cuda.is_available()
    import paper_2408_11743_b200 as m
    m.lib()
    return m


class Pages:
    def __init__(self, lengths, page, max_pages, spare, seed=0):
        import torch
        rng = np.random.default_rng(seed)
        self.page = page
        self.lengths = np.asarray(lengths, np.int32)
        used = -(-self.lengths // page)
        pages = int(used.sum()) + spare
        order = rng.permutation(pages).astype(np.int32)
        self.table = rng.integers(-9, -1, (len(lengths), max_pages)).astype(np.int32)
        at = 0
        for b, n in enumerate(used):
            self.table[b, :n] = order[at:at + n]
            at += n
        self.free = np.full(pages, -99, np.int32)
        self.free[:spare] = order[at:]
        self.count = spare
        self.put(torch.cuda.current_device())

    def put(self, device):
        import torch
        self.dev = [torch.from_numpy(x.copy()).cuda() for x in (self.lengths, self.table, self.free, np.array([self.count], np.int32))]
        self.ws = torch.zeros(8192, dtype=torch.uint8, device="cuda")

    def step(self, marlin, tokens, counts=None, keep=None, status=0):
        import torch
        dev = lambda x: None if x is None else torch.from_numpy(np.asarray(x, np.int32)).cuda()  # noqa: E731
        got = marlin.kv_reserve(*self.dev, self.ws, self.page, tokens, counts=dev(counts), keep=dev(keep))
        assert marlin.read_status(self.ws) == status
        want = cache_blocks_ref.reserve(self.lengths, self.table, self.free, self.count, self.page, tokens, counts, keep)
        self.lengths, self.table, self.free, self.count = want[:4]
        names = ("lengths", "table", "free", "count", "starts", "slots", "positions")
        for name, x, y in zip(names, [t.cpu().numpy() for t in self.dev] + [t.cpu().numpy() for t in got], want):
            assert np.array_equal(x, np.asarray(y).reshape(x.shape)), name
        return got


def test_one_sequence_from_nothing_on(marlin):
    p = Pages([0], 4, 5, 6)
    for n in range(1, 21):
        p.step(marlin, 1)
    assert p.lengths[0] == 20
    p.step(marlin, 1, status=9)  # its row is full
    assert p.lengths[0] == -21
    p.ws.zero_()
    p.step(marlin, 0, counts=[0])  # the length again
    assert p.lengths[0] == 20
    p.step(marlin, 0, counts=[0], keep=[0])
    assert p.lengths[0] == 0 and p.count == 6


@pytest.mark.parametrize("page", [1, 16, 128])
@pytest.mark.parametrize("sequences", [1, 7, 511, 512, 513, 2000])
def test_random_steps(marlin, page, sequences):
    rng = np.random.default_rng(page + sequences)
    p = Pages(rng.integers(0, 300, sequences), page, -(-500 // page), 40 + sequences * 30 // page, seed=page)
    free = 0
    for i in range(8):
        counts = rng.integers(0, (2, 6, 120)[i % 3], sequences)
        keep = [None, np.maximum(0, np.where(p.lengths < 0, ~p.lengths, p.lengths) - rng.integers(0, 9, sequences)),
                np.where(rng.random(sequences) < 0.3, 0, 10 ** 6)][i % 3]
        now = np.where(p.lengths < 0, ~p.lengths, p.lengths) if keep is None else np.minimum(keep, np.where(p.lengths < 0, ~p.lengths, p.lengths))
        counts = np.minimum(counts, 500 // page * page - now)
        p.step(marlin, int(counts.sum()) + (i % 2) * 5, counts, keep)
        free += p.count
    held = -(-np.where(p.lengths < 0, ~p.lengths, p.lengths) // page)
    every = np.concatenate([p.table[b, :n] for b, n in enumerate(held)] + [p.free[:p.count]])
    assert len(np.unique(every)) == len(every) == len(p.free)  # every page is in one place


def test_a_step_taken_back_leaves_everything_as_it_was(marlin):
    rng = np.random.default_rng(3)
    lengths = rng.integers(0, 100, 40)
    p = Pages(lengths, 8, 40, 300)
    free, count = p.free.copy(), p.count
    held = p.table.copy()
    keep, counts = np.where(rng.random(40) < 0.2, 0, lengths), rng.integers(0, 90, 40)
    p.step(marlin, int(counts.sum()), counts, keep)
    p.step(marlin, int((lengths - keep).sum()), lengths - keep, keep)
    assert np.array_equal(p.lengths, lengths) and p.count == count and np.array_equal(p.free[:count], free[:count])
    for b, n in enumerate(-(-lengths // 8)):
        assert np.array_equal(p.table[b, :n], held[b, :n])


def test_many_tokens(marlin):
    # several blocks of the grid, prompts that lie in two of them, more rows than tokens
    rng = np.random.default_rng(4)
    p = Pages(rng.integers(0, 50, 700), 32, 1300, 60000)
    counts = rng.integers(0, 300, 700)
    counts[5] = 40000
    p.step(marlin, int(counts.sum()) + 20000, counts)
    p.step(marlin, 0, counts * 0, rng.integers(0, 60, 700))
    p.step(marlin, int(counts.sum()), counts)


def test_too_few_pages(marlin):
    # those in front are served, those that need none too; the others are marked, and served when there is room
    p = Pages([16, 15, 30, 32, 8, 16], 16, 6, 3)
    p.step(marlin, 60, [1, 1, 40, 1, 3, 1])
    assert list(p.lengths) == [17, 16, -31, -33, 11, -17]
    p.step(marlin, 40, [0, 0, 40, 0, 0, 0], keep=[0, 99, 99, 99, 99, 99])
    assert list(p.lengths) == [0, 16, -31, 32, 11, 16]  # (what a call gives back is handed out from the next one on)
    p.step(marlin, 40, [0, 0, 40, 0, 0, 0])
    assert list(p.lengths) == [0, 16, 70, 32, 11, 16]


def test_bad_numbers_are_contained(marlin):
    import torch
    p = Pages([16, 5, 30, 3], 16, 4, 20)
    p.step(marlin, 10, [1, -5, 2, 100], status=9)         # a negative count; more rows than there are
    assert list(p.lengths) == [17, -6, 32, -4]
    p.ws.zero_()
    p.step(marlin, 200, [1, 1, 50, 100], status=9)        # rows of the table that are too short
    p.ws.zero_()
    p.step(marlin, 8, [2 ** 31 - 1, 2 ** 31 - 1, 1, 1], [-7, -2 ** 31, 5, 99], status=9)
    p.ws.zero_()
    # a count of free pages that is out of range, and a table whose pages would overflow the stack
    p.dev[3].fill_(10 ** 6)
    p.count = len(p.free)
    p.free[:] = np.arange(len(p.free))
    p.dev[2].copy_(torch.from_numpy(p.free))
    p.step(marlin, 0, [0, 0, 0, 0], [0, 0, 0, 0], status=9)
    # lengths that no row can hold
    p.ws.zero_()
    p.lengths[:] = [2 ** 31 - 1, -2 ** 31, 65, 3]
    p.count = 4
    p.dev[0].copy_(torch.from_numpy(p.lengths))
    p.dev[3].fill_(4)
    p.step(marlin, 4, status=9)
    assert list(p.lengths[:3]) == [-2 ** 31, -2 ** 31, -66]


def test_given_outputs_strided_tables_streams_and_refusals(marlin):
    import torch
    p = Pages([3, 17], 16, 4, 9)
    wide = torch.full((2, 9), -3, dtype=torch.int32, device="cuda")
    wide[:, 2:6] = p.dev[1]
    p.dev[1] = wide[:, 2:6]
    outs = [torch.full((n,), 5, dtype=t, device="cuda") for n, t in ((3, torch.int32), (40, torch.int64), (40, torch.int32))]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    counts = torch.tensor([30, 5], dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    got = marlin.kv_reserve(*p.dev, p.ws, 16, 40, counts=counts, starts=outs[0], slots=outs[1], positions=outs[2], stream=side)
    assert all(x is y for x, y in zip(got, outs))
    side.synchronize()
    want = cache_blocks_ref.reserve(p.lengths, p.table, p.free, p.count, 16, 40, [30, 5], None)
    assert np.array_equal(wide[:, 2:6].cpu().numpy(), want[1]) and (wide[:, :2] == -3).all() and (wide[:, 6:] == -3).all()
    for x, y in zip(outs, want[4:]):
        assert np.array_equal(x.cpu().numpy(), y)
    d = dict(zip(("lengths", "pages", "free_pages", "free_count", "workspace", "page_size", "tokens"), (*p.dev, p.ws, 16, 40)))
    for wrong in (dict(lengths=p.dev[0][:1]), dict(free_count=p.dev[2]), dict(counts=counts[:1]), dict(keep=counts[:1]), dict(starts=outs[0][:2]),
                  dict(slots=outs[1][:3]), dict(tokens=-1), dict(pages=p.dev[1].t())):
        with pytest.raises(ValueError):
            marlin.kv_reserve(**{**d, **wrong})
    for wrong in (dict(page_size=24), dict(page_size=0), dict(workspace=p.ws[:8176])):
        with pytest.raises(marlin.MarlinError):
            marlin.kv_reserve(**{**d, **wrong})
    for wrong in (dict(lengths=p.dev[0].cpu()), dict(counts=counts.long()), dict(slots=outs[2])):
        with pytest.raises(TypeError):
            marlin.kv_reserve(**{**d, **wrong})
    assert marlin.read_status(p.ws) == 0


def test_sums_that_run_full(marlin):
    # more rows than numbers of 32 bits hold, in the first and in a later one of the chunks that are summed at a time
    for at in (0, 700):
        p = Pages(np.full(1200, 5), 16, 4, 300)
        counts = np.zeros(1200, np.int64)
        counts[at], counts[at + 1], counts[at + 3] = 2 ** 31 - 1, 2 ** 31 - 1, 7
        counts[:at:3] = 12
        p.step(marlin, 5000, counts, np.where(np.arange(1200) % 5 == 0, 0, 99), status=9)
