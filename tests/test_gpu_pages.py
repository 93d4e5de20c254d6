"""Page tables and slot maps against a simulation on lists: every number has to be the same."""
import random

import pytest

from oracle import operators_oracle as oracle

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible: these tests need a real MI355X")
    return torch


@pytest.fixture(scope="module")
def Pages(torch):
    from paper_2307_05740_amd.pages import ArrowPages
    return ArrowPages


class Both:
    """The operator and the simulation, side by side."""

    def __init__(self, torch, Pages, pages, page, window, sinks, batch, columns):
        self.torch = torch
        self.op = Pages(pages, page, window, sinks)
        self.table, self.held, self.free = self.op.state(batch, columns)
        self.sim = oracle.Pages(pages, page, window, sinks, batch, columns)

    def ints(self, x, dtype="int32"):
        return self.torch.tensor(x, dtype=getattr(self.torch, dtype), device="cuda")

    def compare(self):
        assert self.table.tolist() == self.sim.table
        assert self.held.tolist() == self.sim.held
        free = self.free.tolist()
        assert free[0] == len(self.sim.stack) and free[1:1 + free[0]] == self.sim.stack

    def step(self, lengths, tokens):
        """`tokens` new ones of each sequence."""
        want = self.sim.step(lengths, [tokens] * len(lengths))
        got = self.op.step(self.table, self.held, self.free, self.ints(lengths), tokens)
        assert (got is None) == (tokens == 0)
        if tokens:
            assert got.tolist() == want
        self.compare()

    def ragged(self, lengths, fresh, before=0, behind=0):
        """New tokens of each sequence, with rows that none has before and behind them."""
        want = self.sim.step(lengths, fresh)
        offsets = [before]
        for n in fresh:
            offsets.append(offsets[-1] + n)
        total = offsets[-1] + behind
        got = self.op.step(self.table, self.held, self.free, self.ints(lengths), total, self.ints(offsets), self.torch.full((total,), 77, device="cuda"))
        flat = [-1] * before + [s for own in want for s in own] + [-1] * behind
        assert (got.tolist() if total else []) == flat
        self.compare()


@pytest.mark.parametrize("page", [1, 16, 64])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (40, 4), (100, 70), (64, 200), (5000, 3)])
@pytest.mark.parametrize("batch", [1, 7, 70])
def test_a_life_of_sequences(torch, Pages, page, window, sinks, batch):
    """Sequences that come, grow by a token, by drafts that are taken back, by prompts, and go, in a pool that runs out now and then."""
    rng = random.Random(page * 1000 + window + batch)
    columns = -(-600 // page)
    both = Both(torch, Pages, max(4, batch * columns // 3), page, window, sinks, batch, columns)
    lengths = [0] * batch
    for turn in range(12):
        kind = rng.choice(("one", "drafts", "prompts", "end", "ragged"))
        if kind == "one":
            lengths = [n + 1 if n else 0 for n in lengths]
            both.step(lengths, 1)
        elif kind == "drafts":
            more = rng.randint(2, 9)
            both.step([n + more for n in lengths], more)
            lengths = [n + rng.randint(0, more) for n in lengths]
            both.step(lengths, 0)
        elif kind == "prompts":
            fresh = [rng.randint(0, 300) if n == 0 or rng.random() < 0.3 else 0 for n in lengths]
            lengths = [min(600, n + f) for n, f in zip(lengths, fresh)]
            both.ragged(lengths, fresh, rng.randint(0, 3), rng.randint(0, 3))
        elif kind == "end":
            lengths = [0 if rng.random() < 0.4 else n for n in lengths]
            both.step(lengths, 0)
        else:
            fresh = [rng.randint(0, 40) for _ in lengths]
            lengths = [n + f for n, f in zip(lengths, fresh)]     # (some beyond the table's row)
            both.ragged(lengths, fresh)
    both.step([0] * batch, 0)


@pytest.mark.parametrize("batch,most", [(1, 9000), (3, 20000), (1024, 9), (1025, 9), (1300, 40), (5000, 3), (200, 2000)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (33, 20)])
def test_steps_of_one_launch_and_of_several(torch, Pages, batch, most, window, sinks):
    rng = random.Random(batch)
    page = 16
    lengths = [rng.randint(0, most) for _ in range(batch)]
    both = Both(torch, Pages, sum(-(-n // page) for n in lengths) + batch, page, window, sinks, batch, -(-most // page) + 1)
    both.ragged(lengths, lengths, 2, 5)
    lengths = [n + 1 for n in lengths]
    both.step(lengths, 1)
    lengths = [n + rng.randint(-min(3, n), 9) for n in lengths]
    both.step(lengths, 9)
    both.step([0 if rng.random() < 0.5 else n for n in lengths], 0)
    both.step([0] * batch, 0)
    free = both.free.tolist()                                     # (all pages, in the order that they came back in)
    assert free[0] == both.op.pages and sorted(free[1:]) == list(range(both.op.pages))


@pytest.mark.parametrize("batch,columns", [(1, 2048), (1, 5000), (3, 5461), (7, 2341), (130, 100), (1, 30000), (40, 2100), (600, 1100)])
@pytest.mark.parametrize("short", [False, True])
def test_long_rows_come_and_go(torch, Pages, batch, columns, short):
    """Rows of more columns than one wavefront goes through, and pages of many rows that one workgroup gives back, with a pool for all and one that leaves holes."""
    rng = random.Random(batch)
    page, room = 2, 2 * columns
    lengths = [rng.randint(room // 2, room) for _ in range(batch)]
    if batch == 3:
        lengths = [2 * 1024, 2 * 1024 + 1, 2 * 4096]              # (at and beyond the ends of what a wavefront has)
    pages = sum(-(-n // page) for n in lengths)
    both = Both(torch, Pages, pages * 3 // 4 if short else pages, page, 0, 0, batch, columns)
    both.ragged(lengths, lengths, 1, 1)
    both.step([n // 3 if rng.random() < 0.5 else n for n in lengths], 0)
    both.step([min(room, n + 1) for n in lengths], 1)
    both.step([0] * batch, 0)


def test_there_and_back(torch, Pages):
    """The list is as it was, in order too."""
    both = Both(torch, Pages, 500, 16, 0, 0, 8, 100)
    lengths = [100, 3, 0, 77, 160, 16, 15, 17]
    both.ragged(lengths, lengths)
    table, free = both.table.clone(), both.free.clone()
    for more in (1, 5, 40):
        both.step([n + more for n in lengths], more)
        both.step(lengths, 0)
        assert torch.equal(both.table, table) and torch.equal(both.free, free)


def test_numbers_out_of_range(torch, Pages):
    """Lengths, entries and a list that are not what they should be are cut to what there is: nothing outside is touched."""
    op = Pages(20, 16)
    room = torch.full((3, 6 + 2), 77, dtype=torch.int32, device="cuda")
    table = torch.full((3, 6), -1, dtype=torch.int32, device="cuda")
    held = torch.tensor([2**31 - 1, -7, 40], dtype=torch.int32, device="cuda")
    table[0] = torch.tensor([5, 99, -3, 6, 2**31 - 1, 7])
    free = torch.tensor([1000] + list(range(20)), dtype=torch.int32, device="cuda")
    n = torch.tensor([-2**31, 2**31 - 1, 30], dtype=torch.int32, device="cuda")
    slots = op.step(table, held, free, n, 3)
    assert bool((slots[:2] == -1).all()) and 0 <= int(free[0]) <= 20
    assert bool((table[0] == -1).all()) and held.tolist() == n.tolist()
    for offsets in ([-5, 3, 2**31 - 1, 9], [9, 2, 1, 0], [100, 100, 100, 100]):
        got = op.step(table, held, free, torch.tensor([10, 20, 30], dtype=torch.int32, device="cuda"), 7, torch.tensor(offsets, dtype=torch.int32, device="cuda"))
        assert got.shape == (7,) and bool((got >= -1).all()) and bool((got < 20 * 16).all())
    assert bool((room == 77).all())


def test_captured(torch, Pages):
    """A graph of a token for each sequence, replayed, beside eager steps of the same."""
    both = Both(torch, Pages, 400, 16, 48, 4, 5, 60)
    lengths = [30, 0, 47, 100, 16]
    both.ragged(lengths, lengths)
    other = [t.clone() for t in (both.table, both.held, both.free)]
    n, slots = both.ints(lengths), torch.zeros(5, 1, dtype=torch.int64, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        n += 1
        both.op.step(both.table, both.held, both.free, n, 1, slots=slots)
    for _ in range(70):
        graph.replay()
        lengths = [x + 1 for x in lengths]
        got = both.op.step(*other, both.ints(lengths), 1)
        assert slots.tolist() == got.tolist() == both.sim.step(lengths, [1] * 5)
        both.compare()


def test_nothing_to_do(torch, Pages):
    op = Pages(10, 16)
    table, held, free = op.state(0, 5)
    assert op.step(table, held, free, held.clone(), 0) is None
    assert op.step(table, held, free, held.clone(), 4).shape == (0, 4)
    assert op.step(table, held, free, held.clone(), 3, torch.zeros(1, dtype=torch.int32, device="cuda")).tolist() == [-1, -1, -1]
    table, held, free = op.state(3, 0)
    assert op.step(table, held, free, torch.tensor([1, 2, 3], dtype=torch.int32, device="cuda"), 1).tolist() == [[-1]] * 3
    none = Pages(0, 16)
    table, held, free = none.state(2, 3)
    assert none.step(table, held, free, torch.tensor([5, 0], dtype=torch.int32, device="cuda"), 1).tolist() == [[-1]] * 2 and int(free[0]) == 0


@pytest.mark.parametrize("ragged", [False, True])
def test_more_new_tokens_than_2_to_the_30(torch, Pages, ragged):
    """Of a step that names far more new tokens than the sequence has, its own are the last ones.  (Slots of 8.6 GB.)"""
    op, n = Pages(8, 16), 2**30 + 64
    table, held, free = op.state(1, 4)
    length = torch.tensor([40], dtype=torch.int32, device="cuda")
    offsets = torch.tensor([0, n], dtype=torch.int32, device="cuda") if ragged else None
    slots = op.step(table, held, free, length, n, offsets).flatten()
    assert slots[-40:].tolist() == list(range(40)) and bool((slots[:-40] == -1).all())
    assert table.tolist() == [[0, 1, 2, -1]] and held.tolist() == [40] and free[:6].tolist() == [5, 7, 6, 5, 4, 3]
    for length in (-5, -2**31):
        slots = op.step(table, held, free, torch.tensor([length], dtype=torch.int32, device="cuda"), n, offsets)
        assert bool((slots == -1).all()) and int(free[0]) == 8


@pytest.mark.parametrize("batch,columns,tokens", [(1, 4, 3), (5, 40, 1), (100, 100, 20), (1000, 60, 8), (60, 30, 200), (1000, 2, 40), (1100, 30, 3), (700, 700, 2), (3, 30_000, 5), (2000, 40, 0), (9, 20, 0)])
def test_nothing_outside_is_touched(torch, Pages, batch, columns, tokens):
    """State, lengths, offsets and slots as pieces of one tensor each with numbers between them, and any numbers in them, in one launch, two and several."""
    g = random.Random(batch)
    op, pages, gap = Pages(batch * columns // 2 + 3, 16, g.choice((0, 100)), 5), batch * columns // 2 + 3, 37
    sizes = {"table": batch * columns, "held": batch, "free": 1 + pages, "lengths": batch, "offsets": batch + 1}

    def any_of(n, low, high):
        x = torch.randint(low, high, (n,), generator=torch.Generator().manual_seed(g.randrange(2**31)))
        wild = torch.tensor([-2**31, -1, 2**31 - 1, 1 << 26, columns * 16, 0])[torch.randint(0, 6, (n,), generator=torch.Generator().manual_seed(g.randrange(2**31)))]
        return torch.where(torch.rand(n, generator=torch.Generator().manual_seed(g.randrange(2**31))) < 0.2, wild, x).int()

    for ragged in (False, True):
        rows = batch * tokens
        room = torch.full((sum(sizes.values()) + gap * (len(sizes) + 1),), 1234567, dtype=torch.int32, device="cuda")
        places = torch.full((rows + 2 * gap,), 1234567, dtype=torch.int64, device="cuda")
        part, own, at = {}, torch.zeros_like(room, dtype=torch.bool), gap
        for name, n in sizes.items():
            part[name], own[at:at + n] = room[at:at + n], True
            at += n + gap
        for _ in range(3):
            part["table"].copy_(any_of(batch * columns, -2, pages + 2))
            part["held"].copy_(any_of(batch, 0, columns * 16))
            part["free"].copy_(any_of(1 + pages, 0, pages))
            part["lengths"].copy_(any_of(batch, 0, columns * 16))
            part["offsets"].copy_(any_of(batch + 1, 0, rows + 1).sort()[0] if g.random() < 0.5 else any_of(batch + 1, 0, rows + 1))
            keep = {name: part[name].clone() for name in ("lengths", "offsets")}
            slots = places[gap:gap + rows]
            op.step(part["table"].view(batch, columns), part["held"], part["free"], part["lengths"], rows if ragged else tokens, part["offsets"] if ragged else None,
                    slots if ragged else slots.view(batch, tokens))
            assert bool((room[~own] == 1234567).all()) and bool((places[:gap] == 1234567).all()) and bool((places[gap + rows:] == 1234567).all())
            assert all(torch.equal(part[name], x) for name, x in keep.items()) and torch.equal(part["held"], part["lengths"])
            assert 0 <= int(part["free"][0]) <= pages
            assert bool(((slots >= -1) & (slots < pages * 16)).all())
