"""GPU tests of octopus_pages_update, octopus_pages_compact, octopus_pages_rename and octopus_pages_copy: whole numbers and bytes, equal to a sequential
model's (tests/pages_model.py)."""
import numpy as np
import pytest

from paper_2605_21226_amd import binding
from pages_model import TILE, Pages, ceil

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

DEV = "cuda:0"
JUNK = -77


def ints(x):
    return None if x is None else torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


class Server:
    """A model's state and the same in device memory, with pools that hold each page's contents."""

    def __init__(self, refs, table, lens, pool_bytes=(16, 48)):
        self.model = Pages(refs, table, lens)
        self.refs, self.table, self.lens = ints(refs), ints(table), ints(lens)
        n_pages, (n_seq, per) = len(self.model.refs), self.model.table.shape
        self.moves = torch.full((2 + 2 * max(n_seq, n_pages // 2),), JUNK, dtype=torch.int32, device=DEV)
        self.map = torch.full((n_pages,), JUNK, dtype=torch.int32, device=DEV)
        self.ws = torch.full((binding.octopus_pages_workspace(n_pages, n_seq, per),), 0xA5, dtype=torch.uint8, device=DEV)
        g = torch.Generator().manual_seed(n_pages)
        self.contents = [torch.randint(0, 256, (n_pages, b), generator=g, dtype=torch.uint8) for b in pool_bytes]
        self.on_device = [c.to(DEV) for c in self.contents]
        self.pools = binding.page_pools(self.on_device)

    def copy(self, stream=None):
        binding.octopus_pages_copy(self.pools, self.moves, stream=stream)
        for c in self.contents:
            before = c.clone()
            for a, b in self.model.moves:
                c[b] = before[a]

    def compare(self, second):
        got = self.moves.cpu().numpy()
        n = len(self.model.moves)
        assert got[0] == n and got[1] == second
        assert got[2:2 + 2 * n].tolist() == [x for pair in self.model.moves for x in pair]
        assert np.all(got[2 + 2 * n:] == JUNK)
        assert np.array_equal(self.refs.cpu().numpy(), self.model.refs)
        assert np.array_equal(self.table.cpu().numpy(), self.model.table)
        assert np.array_equal(self.lens.cpu().numpy(), self.model.lens)
        for a, b in zip(self.contents, self.on_device):
            assert torch.equal(a, b.cpu())

    def update(self, new_lens, source=None, keep_lens=None, stream=None):
        self.moves.fill_(JUNK)
        self.model.update(new_lens, source, keep_lens)
        binding.octopus_pages_update(self.refs, self.table, self.lens, ints(new_lens), self.moves, self.ws, source=ints(source),
                                     keep_lens=ints(keep_lens), stream=stream)
        self.copy(stream)
        torch.cuda.synchronize()
        self.compare(self.model.missing)

    def compact(self, others=()):
        self.moves.fill_(JUNK)
        page_map = self.model.compact()
        self.model.rename(page_map)
        binding.octopus_pages_compact(self.refs, self.map, self.moves, self.ws)
        self.copy()
        binding.octopus_pages_rename(self.map, self.table, self.lens)
        for table, lens in others:
            binding.octopus_pages_rename(self.map, table, lens)
        torch.cuda.synchronize()
        assert self.map.cpu().tolist() == page_map
        self.compare(self.model.used)
        assert np.all(self.model.refs[:self.model.used] > 0) and not np.any(self.model.refs[self.model.used:] > 0)


def server(n_seq, per, n_pages, lens, seed=0, **more):
    """Slots of the given lengths on pages of their own, anywhere in the pool."""
    rng = np.random.default_rng(seed)
    table = rng.integers(-5, n_pages + 5, size=(n_seq, per))        # (entries past a slot's pages mean nothing)
    ids, at, refs = rng.permutation(n_pages), 0, np.zeros(n_pages, dtype=np.int64)
    for s, n in enumerate(lens):
        table[s, :ceil(n)] = ids[at:at + ceil(n)]
        refs[ids[at:at + ceil(n)]] = 1
        at += ceil(n)
    return Server(refs, table, lens, **more)


@pytest.mark.parametrize("n_seq,per,n_pages", [(1, 1, 1), (1, 3, 5), (7, 4, 40), (64, 9, 700), (1024, 8, 9000), (1024, 9, 5000), (33, 300, 9000),
                                               (1025, 2, 3000), (2100, 3, 7000)])
@pytest.mark.parametrize("with_source", [False, True])
def test_steps(n_seq, per, n_pages, with_source):
    """Growth, trims, forks, slots that move, end and begin, at random, one after the other, until pages run out and after."""
    rng = np.random.default_rng(n_seq + n_pages)
    x = server(n_seq, per, n_pages, [int(n) for n in rng.integers(0, min(per * TILE, n_pages * TILE // n_seq) + 1, size=n_seq)], seed=n_seq)
    for step in range(12):
        lens, most = x.model.lens, per * TILE
        kind = rng.integers(0, 6, size=n_seq)
        new = np.choose(kind, [lens, lens + 1, lens + rng.integers(0, 130, size=n_seq), lens - rng.integers(0, 70, size=n_seq),
                               np.where(rng.random(n_seq) < 0.5, 0, lens), rng.integers(0, most + 1, size=n_seq)])
        keep = None if step % 3 == 0 else np.where(rng.random(n_seq) < 0.5, lens, lens - rng.integers(0, 9, size=n_seq))
        source = None
        if with_source:
            source = np.where(rng.random(n_seq) < 0.6, np.arange(n_seq), rng.integers(-1, n_seq + 1, size=n_seq))
            own = np.where((source >= 0) & (source < n_seq), lens[np.clip(source, 0, n_seq - 1)], 0)
            new = np.where(rng.random(n_seq) < 0.7, own + rng.integers(0, 3, size=n_seq), new)
        x.update(new, source, keep)
        x.model.check()
        if step % 4 == 3:
            x.compact()
            x.model.check()


def test_page_borders():
    """Lengths around a page's end; a token more, none more, to the border exactly, and past it."""
    lens = [0, 1, 63, 64, 65, 127, 128, 129]
    x = server(8, 4, 60, lens)
    for grow in ([1] * 8, [0] * 8, [1, 63, 1, 0, 63, 1, 64, 127], [64] * 8):
        x.update(x.model.lens + grow)
        x.model.check()
    x.update([0] * 8)
    assert not np.any(x.model.refs) and np.all(x.model.lens == 0)


@pytest.mark.parametrize("n_seq", [2, 33, 1025])
@pytest.mark.parametrize("tokens", [1, 63, 64, 100, 1000])
def test_samples_of_one_prompt(n_seq, tokens):
    """Every slot goes on from slot 1: all but it copy the page in which the prompt ends, and none where it ends with one."""
    x = server(n_seq, ceil(tokens) + 1, ceil(tokens) + 2 * n_seq, [0, tokens] + [0] * (n_seq - 2))
    x.update([tokens + 1] * n_seq, source=[1] * n_seq)
    x.model.check()
    assert len(x.model.moves) == (n_seq - 1 if tokens % TILE else 0)
    whole = tokens // TILE
    assert np.all(x.model.refs[x.model.table[0, :whole]] == n_seq)
    x.update([tokens + 2] * n_seq)                            # every page that is written into is a slot's own by now
    assert not x.model.moves
    x.model.check()


def test_beams_that_live_on_keep_their_page_and_the_same_call_again_changes_nothing():
    n, tokens = 8, 200
    x = server(n, 6, 60, [tokens] * n, seed=3)
    source, keep = [2, 2, 2, 5, 5, 5, 6, 2], [tokens] * n
    x.update([tokens + 5] * n, source, keep)
    x.model.check()
    assert {pair[0] for pair in x.model.moves} == {int(x.model.table[2, 3]), int(x.model.table[5, 3])} and len(x.model.moves) == 5
    before = x.model.table.copy(), x.model.refs.copy(), list(x.model.moves)
    x.update([tokens + 5] * n, source, keep)
    assert np.array_equal(before[0], x.model.table) and np.array_equal(before[1], x.model.refs) and before[2] == x.model.moves


def test_first_writer_keeps_and_readers_make_all_copy():
    x = server(4, 3, 20, [70, 0, 0, 0])
    x.update([71, 71, 70, 0], source=[0, 0, 0, 0])            # slot 2 reads on: both writers copy
    assert len(x.model.moves) == 2
    y = server(4, 3, 20, [70, 0, 0, 0])
    y.update([0, 71, 71, 0], source=[-1, 0, 0, 7])            # the source leaves: the first of the two keeps the page
    assert y.model.moves == [(int(y.model.table[1, 1]), int(y.model.table[2, 1]))]
    x.model.check()
    y.model.check()


def test_a_page_that_something_else_holds_is_copied_and_never_given_away():
    x = server(3, 3, 9, [100, 64, 10])
    pinned = np.zeros(9, dtype=np.int64)
    pinned[x.model.table[0, 1]] = 2
    pinned[x.model.table[1, 0]] = 1
    x.model.refs += pinned
    x.refs += ints(pinned)
    x.update([101, 65, 11])
    assert x.model.moves[0][0] in np.nonzero(pinned)[0] and len(x.model.moves) == 1
    x.model.check(pinned)
    x.update([0, 0, 0])
    x.model.check(pinned)
    others = np.nonzero(pinned)[0]
    held = ints(others)
    x.compact(others=[(held, ints([2 * TILE])), (held.clone(), None)])
    assert held.cpu().tolist() == [x.map.cpu().tolist()[p] for p in others] and sorted(held.cpu().tolist()) == [0, 1]


@pytest.mark.parametrize("spare", [0, 1, 2, 3])
def test_too_few_pages(spare):
    """Two pages are asked for, one of them for a copy: with fewer nobody grows; a page that the same call releases counts."""
    x = server(4, 4, 3 + 1 + spare, [70, 64, 0, 64], seed=spare)
    x.update([71, 65, 71, 0], source=[0, 1, 0, 3])            # slot 3 releases one: 1 + spare are free, 2 are needed
    x.model.check()
    assert x.model.missing == max(0, 2 - (1 + spare))
    x.update([71, 65, 190, 64])
    x.model.check()


def test_clamped_numbers():
    """Counts below zero and above what a row holds, sources that are none, page numbers outside the pool."""
    big, low = 2 ** 31 - 1, -2 ** 31
    x = Server([1, 1, 1, 0, 0, 0, 0, 0, 0, 0], [[-9, 4], [1, 0], [99, 0]], [64, 10, 3], pool_bytes=(16,))
    x.model.refs[9] = 1
    x.model.refs[2] = 0
    x.refs.copy_(ints(x.model.refs))
    x.update([64, 11, 4])
    x.update([big, low, 5], source=[0, 1, low], keep_lens=[big, big, big])
    assert x.model.lens.tolist() == [128, 0, 5]
    x.update([big, big, big], source=[big, 1, 2], keep_lens=[3, low, -1])
    assert x.model.lens.tolist() == [128, 128, 128]
    y = Server([1] + [0] * 5, [[0, 0]], [big])       # a slot that says it holds more than a row: as much as a row
    y.model.lens[0], y.model.refs[0] = 128, 2
    y.lens.fill_(big)
    y.refs.copy_(ints(y.model.refs))
    y.update([100])


@pytest.mark.parametrize("n_pages,used", [(1, 0), (1, 1), (2, 1), (17, 9), (4096, 2000), (16385, 9000), (20000, 1), (65536, 30000), (65537, 40000), (70001, 70001),
                                          (200000, 90000)])
def test_compaction(n_pages, used):
    rng = np.random.default_rng(n_pages + used)
    refs = np.zeros(n_pages, dtype=np.int64)
    refs[rng.permutation(n_pages)[:used]] = rng.integers(1, 5, size=used)
    refs[(refs == 0) & (rng.random(n_pages) < 0.1)] = -3      # as free as 0
    per = max(1, min(used, 50))
    held = np.nonzero(refs > 0)[0][:per]
    table = np.full((2, per), n_pages + 3)
    table[0, :len(held)] = held
    x = Server(refs, table, [TILE * len(held), 0], pool_bytes=(16,))
    x.compact()
    x.compact()
    assert not x.model.moves


def test_compaction_of_the_largest_pool():
    """2^24 pages, a third of them in use: the pairs, the counts and the map as the definition has them."""
    n_pages = 1 << 24
    used = torch.rand(n_pages, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV) < 0.33
    ids = torch.arange(n_pages, dtype=torch.int32, device=DEV)
    refs = torch.where(used, ids % 5 + 1, 0).int()
    before = refs.clone()
    page_map, moves = torch.zeros_like(refs), torch.zeros(2 + n_pages, dtype=torch.int32, device=DEV)
    ws = torch.empty(binding.octopus_pages_workspace(n_pages, 1, 1), dtype=torch.uint8, device=DEV)
    binding.octopus_pages_compact(refs, page_map, moves, ws)
    n = int(used.sum())
    high, low = ids[n:][used[n:]].flip(0), ids[:n][~used[:n]]
    assert moves[:2].tolist() == [len(high), n] and len(high) == len(low) > 1000000
    assert torch.equal(moves[2:2 + 2 * len(high)].view(-1, 2), torch.stack([high, low], dim=1))
    want_map, want_refs = ids.clone(), before.clone()
    want_map[high.long()] = low
    want_refs[low.long()], want_refs[high.long()] = before[high.long()], 0
    assert torch.equal(page_map, want_map) and torch.equal(refs, want_refs)


def test_free_pages_at_the_end_of_the_largest_pool():
    n_pages = 1 << 24
    refs = torch.ones(n_pages, dtype=torch.int32, device=DEV)
    refs[[0, 5, n_pages - 3, n_pages - 1]] = 0
    refs[5] = -7
    table, lens = torch.zeros((2, 4), dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV)
    moves = torch.zeros(6, dtype=torch.int32, device=DEV)
    ws = torch.empty(binding.octopus_pages_workspace(n_pages, 2, 4), dtype=torch.uint8, device=DEV)
    binding.octopus_pages_update(refs, table, lens, ints([1, 200]), moves, ws)
    assert moves[:2].tolist() == [0, 1] and lens.tolist() == [0, 0] and int((refs == 1).sum()) == n_pages - 4
    binding.octopus_pages_update(refs, table, lens, ints([1, 190]), moves, ws)
    assert moves[:2].tolist() == [0, 0] and table.tolist() == [[0, 0, 0, 0], [5, n_pages - 3, n_pages - 1, 0]] and bool((refs == 1).all())


def test_the_largest_table():
    """32 rows of 2^25 - 1 entries (4 GiB): forks and growth in the last rows; slots that ask for 2^31 tokens each are told how many pages are missing."""
    n_seq, per, n_pages = 32, (2 ** 31 - 1) // 64, 64
    table = torch.zeros((n_seq, per), dtype=torch.int32, device=DEV)
    ws = torch.empty(binding.octopus_pages_workspace(n_pages, n_seq, per), dtype=torch.uint8, device=DEV)
    refs, lens = torch.zeros(n_pages, dtype=torch.int32, device=DEV), torch.zeros(n_seq, dtype=torch.int32, device=DEV)
    moves = torch.zeros(2 + 2 * n_seq, dtype=torch.int32, device=DEV)
    source = torch.arange(n_seq, dtype=torch.int32, device=DEV)
    new = torch.zeros_like(lens)
    new[31] = 200
    binding.octopus_pages_update(refs, table, lens, new, moves, ws)
    assert table[31, :4].tolist() == [0, 1, 2, 3]
    source[29], new[29] = 31, 201
    new[31] = 201
    binding.octopus_pages_update(refs, table, lens, new, moves, ws, source=source)
    assert table[29, :4].tolist() == [0, 1, 2, 4] and moves[:4].tolist() == [1, 0, 3, 4] and refs[:5].tolist() == [2, 2, 2, 1, 1]
    new.fill_(2 ** 31 - 1)
    binding.octopus_pages_update(refs, table, lens, new, moves, ws)
    assert moves[:2].tolist() == [0, n_seq * per - 8 - (n_pages - 5)] and lens.tolist() == [0] * 29 + [201, 0, 201]


@pytest.mark.parametrize("bytes_of", [(16,), (16, 32, 48, 16400), (1 << 14, 1 << 17), tuple(16 * (1 + i % 9) for i in range(150))])
def test_copies_of_every_size_and_number_of_pools(bytes_of):
    rng = np.random.default_rng(len(bytes_of))
    n_pages, n = 40, 13
    ids = rng.permutation(n_pages)[:2 * n]
    pairs = ids.reshape(n, 2)
    pools = [torch.from_numpy(rng.integers(0, 256, size=(n_pages, b), dtype=np.uint8)).to(DEV) for b in bytes_of]
    want = [p.clone() for p in pools]
    for p in want:
        p[pairs[:, 1]] = p[pairs[:, 0]]
    moves = ints([n, 99] + pairs.reshape(-1).tolist() + [3, 4])      # (a pair past the count)
    binding.octopus_pages_copy(binding.page_pools(pools), moves)
    assert all(torch.equal(a, b) for a, b in zip(pools, want))


def test_copies_that_count_and_pages_that_are_there():
    """A count past the room is cut, one below zero is none; pairs outside the pool are left out."""
    pool = torch.arange(8, device=DEV, dtype=torch.int64)[:, None].repeat(1, 2)
    pools = binding.page_pools([pool])
    binding.octopus_pages_copy(pools, ints([2 ** 31 - 1, 0, 0, 5, 8, 1, -1, 2, 3, 8, 4, -2, 1, 6]), max_moves=5)
    assert pool[:, 0].tolist() == [0, 1, 2, 3, 4, 0, 6, 7]
    binding.octopus_pages_copy(pools, ints([-5, 0, 0, 1]))
    binding.octopus_pages_copy(pools, ints([1, 0, 0, 1]), max_moves=0)
    assert pool[:, 0].tolist() == [0, 1, 2, 3, 4, 0, 6, 7]


def test_pools_of_more_than_4_gib():
    """Page numbers times page bytes past 32 bits."""
    n_pages, b = 70, 1 << 26
    pool = torch.empty((n_pages, b), dtype=torch.uint8, device=DEV)
    pool[66:] = 7
    pool[1], pool[2], pool[66] = 1, 2, 66
    binding.octopus_pages_copy(binding.page_pools([pool]), ints([2, 0, 1, 69, 66, 2]))
    assert bool((pool[69] == 1).all()) and bool((pool[2] == 66).all()) and bool((pool[67:69] == 7).all()) and bool((pool[1] == 1).all())


def test_another_stream_and_a_captured_step():
    """A step of growing, trimming and forking, captured once and replayed with its counts changed in place, against the model."""
    side = torch.cuda.Stream()
    n_seq, per, n_pages = 12, 8, 120
    x = server(n_seq, per, n_pages, [60 + 7 * s for s in range(n_seq)], seed=5)
    torch.cuda.synchronize()
    x.update(x.model.lens + 3, stream=side)
    new, keep, source = x.lens.clone(), x.lens.clone(), torch.arange(n_seq, dtype=torch.int32, device=DEV)

    def step():
        binding.octopus_pages_update(x.refs, x.table, x.lens, new, x.moves, x.ws, source=source, keep_lens=keep)
        binding.octopus_pages_copy(x.pools, x.moves)
        binding.octopus_pages_update(x.refs, x.table, x.lens, new, x.moves, x.ws)        # another call with the same workspace
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    rng = np.random.default_rng(1)
    for replay in range(6):
        lens = x.model.lens
        s = np.where(rng.random(n_seq) < 0.5, np.arange(n_seq), rng.integers(0, n_seq, size=n_seq))
        k = lens[s] - rng.integers(0, 40, size=n_seq)
        n = k + rng.integers(0, 90, size=n_seq)
        new.copy_(ints(n))
        keep.copy_(ints(k))
        source.copy_(ints(s))
        x.moves.fill_(JUNK)
        graph.replay()
        torch.cuda.synchronize()
        x.model.update(n, s, k)
        first = list(x.model.moves)
        for c in x.contents:
            before = c.clone()
            for a, b in first:
                c[b] = before[a]
        x.model.update(n)
        assert not x.model.moves
        assert x.moves[:2].tolist() == [0, 0] and x.moves[2:2 + 2 * len(first)].tolist() == [v for pair in first for v in pair]
        assert np.array_equal(x.refs.cpu().numpy(), x.model.refs) and np.array_equal(x.table.cpu().numpy(), x.model.table)
        assert all(torch.equal(a, b.cpu()) for a, b in zip(x.contents, x.on_device))
        x.model.check()


@pytest.mark.parametrize("n_seq,per", [(9, 5), (64, 200)])
def test_two_captured_graphs_of_one_workspace(n_seq, per):
    """Two servers' steps, captured with the same workspace, replayed in turns with eager calls with it in between."""
    n_pages = n_seq * per * 2
    pair = [server(n_seq, per, n_pages, [1 + (37 * s + 11 * i) % (TILE * (per - 2)) for s in range(n_seq)], seed=i) for i in range(2)]
    x, y = pair
    y.ws = x.ws
    rng = np.random.default_rng(8)
    sources = [rng.integers(0, n_seq, size=n_seq) for _ in pair]
    told = [(ints(s), torch.zeros(n_seq, dtype=torch.int32, device=DEV)) for s in sources]
    graphs = []
    torch.cuda.synchronize()
    for z, (source, new) in zip(pair, told):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            binding.octopus_pages_update(z.refs, z.table, z.lens, new, z.moves, z.ws, source=source)
            binding.octopus_pages_copy(z.pools, z.moves)
        graphs.append(graph)
    for turn in range(6):
        i = turn % 2
        z, (source, new) = pair[i], told[i]
        want = np.minimum(z.model.lens[sources[i]] + rng.integers(-30, 60, size=n_seq), TILE * per)
        want = np.maximum(want, 0)
        new.copy_(ints(want))
        z.moves.fill_(JUNK)
        graphs[i].replay()
        torch.cuda.synchronize()
        z.model.update(want, sources[i])
        for c in z.contents:
            before = c.clone()
            for a, b in z.model.moves:
                c[b] = before[a]
        z.compare(z.model.missing)
        other = pair[1 - i]
        other.update(np.minimum(other.model.lens + 5, TILE * per))      # eager, with the same workspace
    for z in pair:
        z.model.check()
