"""The cache in 4 bits against the definitions in 64 bits: what is written is what the oracle makes of it, bit by bit; the attention over it is held to the bounds of
oracle/attention_oracle.py for the values that the cache holds."""
import math

import pytest

from oracle import attention_oracle, operators_oracle as oracle

pytestmark = pytest.mark.gpu

TYPES = ("bfloat16", "float16")


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible: these tests need a real MI355X")
    return torch


@pytest.fixture(scope="module")
def Packed(torch):
    from paper_2307_05740_amd.packed import ArrowPackedAttention
    return ArrowPackedAttention


def normal(torch, seed, dtype, *shape, by=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * by).to(getattr(torch, dtype)).cuda()


def same(torch, got, want):
    got = got.double()
    ok = (got == want) | (got.isnan() & want.isnan())
    assert bool(ok.all()), (int((~ok).sum()), ok.numel(), got[~ok][:4], want[~ok][:4])


def unpacked(torch, pool, page, dim, slots):
    """Keys and values of places, from the bytes."""
    block = pool[slots // page].cpu().int()
    t = (slots % page).cpu()
    i, h = torch.arange(len(t)), pool.shape[1]
    levels = torch.tensor(oracle.LEVELS, dtype=torch.float64)
    at = block[:, :, :page * dim // 2].view(-1, h, page, dim // 2)[i, :, t]
    values = block[:, :, page * dim // 2:page * dim].view(-1, h, page // 4, 16, 4, dim // 32)[i, :, t // 4, :, t % 4].flatten(-2)
    ks = block[:, :, page * dim:page * (dim + dim // 32)].view(-1, h, page, dim // 32)[i, :, t]
    vs = block[:, :, page * (dim + dim // 32):].view(-1, h, page // 4, dim // 32, 4)[i, :, t // 4, :, t % 4]
    out = []
    for codes, scales in ((at, ks), (values, vs)):
        code = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
        x = levels[(code & 7).long()] * torch.where(code >= 8, -1.0, 1.0)
        s = torch.where(scales == 255, math.nan, torch.exp2(scales.double() - 127))
        out.append(x * s.repeat_interleave(32, -1))
    return out


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [32, 64, 128])
def test_every_value_of_the_type(torch, Packed, dtype, dim):
    """All 65,536 of them, each beside others of its size, in three mixtures, among them blocks of zeros, of the largest and the smallest, and with what is not finite."""
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16)
    order = torch.argsort((bits.int() & 0x7fff) * 2 + (bits < 0), stable=True)
    g = torch.Generator().manual_seed(1)
    mixed = torch.randperm(65536, generator=g)
    near = (torch.arange(65536) + torch.randint(-700, 700, (65536,), generator=g)).clamp(0, 65535)
    x = torch.stack([bits[order], bits[mixed], bits[order][near]]).view(getattr(torch, dtype)).view(-1, 2, dim)
    x = torch.cat([x, torch.zeros(1, 2, dim, dtype=x.dtype)]).cuda()
    n, op, page = x.shape[0], Packed(), 32
    pool = op.pool(-(-n // page), page, 2, dim)
    slots = torch.randperm(pool.shape[0] * page, generator=g)[:n].cuda()
    op.append(x, x.flip(0), pool, slots)
    want = oracle.packed(x)
    k, v = unpacked(torch, pool, page, dim, slots)
    same(torch, k.cuda(), want)
    same(torch, v.cuda(), want.flip(0))
    k, v = op.read(pool, slots, dim, x.dtype, torch.full_like(x, 7.0), torch.full_like(x, 7.0))
    same(torch, k, want)
    same(torch, v, want.flip(0))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [32, 64, 128])
@pytest.mark.parametrize("page", [16, 64])
def test_places(torch, Packed, dtype, dim, page):
    """Slots in any order, some of them nowhere; what is not written keeps its bytes; views with other steps."""
    op, heads, pages = Packed(), 3, 9
    g = torch.Generator().manual_seed(1)
    room = torch.randint(0, 256, (pages, heads + 1, page * (dim + dim // 16) + 16), dtype=torch.uint8, generator=g).cuda()
    pool = room[:, 1:, :page * (dim + dim // 16)]
    keep = room.clone()
    for n in (0, 1, 3, 4, 5, 101):
        slots = torch.randperm(pages * page, generator=g)[:n].cuda()
        slots[::4] = torch.tensor([-1, pages * page, 2**40, -2**62], device="cuda").repeat(26)[:len(slots[::4])]
        both = normal(torch, n, dtype, n, 2 * heads + 1, dim, by=3.0)
        k, v = both[:, :heads], both[:, heads:2 * heads]
        op.append(k, v, pool, slots)
        there = (slots >= 0) & (slots < pages * page)
        out = torch.full((n, 2 * heads + 1, dim), 7.0, dtype=both.dtype, device="cuda")
        op.read(pool, slots, dim, both.dtype, out[:, 1:heads + 1], out[:, heads + 1:])
        for got, x in ((out[:, 1:heads + 1], k), (out[:, heads + 1:], v)):
            same(torch, got, torch.where(there[:, None, None], oracle.packed(x), 0.0) if n else x.double())
        assert bool((out[:, 0] == 7).all())
    op = Packed()
    assert torch.equal(room[:, 0], keep[:, 0]) and torch.equal(room[:, :, -16:], keep[:, :, -16:])
    # a token's bytes, and no others
    keep = room.clone()
    op.append(both[:1, :heads], both[:1, heads:2 * heads], pool, torch.tensor([3 * page + 6], device="cuda"))
    changed = (room != keep).nonzero()
    assert bool((changed[:, 0] == 3).all()) and len(changed) <= heads * (dim + dim // 16)


def filled(torch, op, dtype, lengths, page, kv, dim, seed=1, hole=None):
    """A pool with the sequences' keys and values, (tokens, heads, dim) each, as the cache holds them."""
    g = torch.Generator().manual_seed(seed)
    columns = max(1, -(-max(lengths) // page))
    need = [-(-n // page) for n in lengths]
    pages = sum(need) + 2
    order = torch.randperm(pages, generator=g)
    pool = torch.randint(0, 256, (pages, kv, page * (dim + dim // 16)), dtype=torch.uint8, generator=g).cuda()
    table = torch.full((len(lengths), columns), -1, dtype=torch.int32)
    keys, values, first = [], [], 0
    for b, n in enumerate(lengths):
        table[b, :need[b]] = order[first:first + need[b]].int()
        first += need[b]
        t = torch.arange(n)
        slots = (table[b][t // page].long() * page + t % page).cuda()
        k, v = normal(torch, seed + 10 * b + 1, dtype, n, kv, dim), normal(torch, seed + 10 * b + 2, dtype, n, kv, dim)
        op.append(k, v, pool, slots)
        k, v = op.read(pool, slots, dim, k.dtype)
        keys.append(k)
        values.append(v)
    return pool, table.cuda(), torch.tensor(lengths, dtype=torch.int32, device="cuda"), keys, values


def check(torch, op, o, q, keys, values, seen=None):
    kv = keys[0].shape[1]
    for b in range(q.shape[0]):
        for h in range(q.shape[1]):
            k, v = keys[b][:, h * kv // q.shape[1]], values[b][:, h * kv // q.shape[1]]
            if len(k) == 0:
                assert not bool(o[b, h].any())
                continue
            want, bound = attention_oracle.attention(q[b, h][None], k, v, op.window, op.sinks, op.scale, seen=None if seen is None else seen[b])
            off = (o[b, h].double() - want["o"][0]).abs()
            assert bool((off <= bound["o"][0]).all()), (b, h, float((off / bound["o"][0].clamp(min=1e-300)).max()))


MASKS = [(0, 0), (1, 0), (1, 1), (17, 0), (64, 4), (100, 65), (128, 200), (1000, 5)]


@pytest.mark.parametrize("window,sinks", MASKS)
@pytest.mark.parametrize("dim", [32, 64, 128])
@pytest.mark.parametrize("page", [16, 32, 256])
def test_lengths_and_masks(torch, Packed, window, sinks, dim, page):
    dtype = TYPES[(window + dim // 32) % 2]
    op = Packed(window, sinks)
    lengths = [1, 0, 2, 15, 16, 17, 31, 33, 64, 100, 127, 128, 129, 255, 300, 517, 1025]
    pool, table, n, keys, values = filled(torch, op, dtype, lengths, page, 2, dim)
    q = normal(torch, 3, dtype, len(lengths), 6, dim, by=2.0)
    check(torch, op, op.decode(q, pool, table, n), q, keys, values)
    check(torch, op, op.decode(q, pool, table, n, 1025, o=torch.full_like(q, math.nan)), q, keys, values)
    check(torch, op, op.decode(q, pool, table, n, 10), q, keys, values)         # (how the work is split, no more)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads,kv", [(1, 1), (4, 4), (6, 2), (8, 1), (15, 1), (16, 1), (17, 1), (64, 2)])
def test_head_layouts(torch, Packed, dtype, heads, kv):
    op = Packed(200, 3, scale=0.15)
    for dim in (32, 64, 128):
        pool, table, n, keys, values = filled(torch, op, dtype, [700, 1, 40], 16, kv, dim)
        both = normal(torch, 3, dtype, 3, heads + 2, dim)
        q, out = both[:, 1:1 + heads], torch.full_like(both, math.nan)
        o = op.decode(q, pool, table, n, o=out[:, 2:2 + heads])
        check(torch, op, o, q, keys, values)
        assert bool(out[:, :2].isnan().all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("window,sinks", [(0, 0), (3000, 20)])
def test_long_caches_in_stretches(torch, Packed, dtype, window, sinks):
    op = Packed(window, sinks)
    pool, table, n, keys, values = filled(torch, op, dtype, [9000, 37, 5000], 64, 2, 128)
    q = normal(torch, 3, dtype, 3, 8, 128, by=3.0)
    o = op.decode(q, pool, table, n)
    check(torch, op, o, q, keys, values)
    assert all(torch.equal(o, op.decode(q, pool, table, n)) for _ in range(3))


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("batch,kv", [(1, 2), (7, 8), (8, 8), (19, 8), (20, 8), (24, 8), (48, 8), (64, 8), (96, 8), (97, 8)])
@pytest.mark.parametrize("longest", [512, 513, 1024, 1025, 2000, 2001, 6000, 6001, 12001, 30000])
def test_splits_by_rows_and_lengths(torch, Packed, dim, batch, kv, longest):
    """Around the numbers of rows and keys from which the keys are cut otherwise: how they are goes by the longest length that is named, not by those that there are."""
    op = Packed()
    g = torch.Generator().manual_seed(batch)
    lengths = torch.randint(0, 300, (batch,), generator=g).tolist()
    lengths[0] = 1100
    pool, table, n, keys, values = filled(torch, op, TYPES[batch % 2], lengths, 32, kv, dim)
    wide = torch.full((batch, 1000), -1, dtype=torch.int32, device="cuda")
    wide[:, :table.shape[1]] = table
    q = normal(torch, 3, TYPES[batch % 2], batch, 2 * kv, dim, by=2.0)
    o = op.decode(q, pool, wide, n, longest)
    part = slice(0, batch, 9)
    check(torch, op, o[part], q[part], keys[part], values[part])


@pytest.mark.parametrize("dim", [32, 64, 128])
@pytest.mark.parametrize("batch,kv", [(48, 4), (200, 1), (47, 4), (193, 4)])
def test_many_rows_under_a_window(torch, Packed, dim, batch, kv):
    """Around the numbers of rows that have workgroups of eight wavefronts."""
    op = Packed(300, 5)
    g = torch.Generator().manual_seed(batch)
    lengths = torch.randint(0, 900, (batch,), generator=g).tolist()
    pool, table, n, keys, values = filled(torch, op, TYPES[batch % 2], lengths, 32, kv, dim)
    q = normal(torch, 3, TYPES[batch % 2], batch, 2 * kv, dim, by=2.0)
    o = op.decode(q, pool, table, n, 900)
    part = slice(0, batch, 5)
    check(torch, op, o[part], q[part], keys[part], values[part])


@pytest.mark.parametrize("dim", [32, 64, 128])
def test_new_tokens(torch, Packed, dim):
    """k and v go to their place first; those without one (an idle sequence, a page that is not there, a row of the table that is too short) nowhere."""
    op, page = Packed(), 16
    lengths = [1, 16, 17, 300, 0, 64, 33]
    pool, table, n, keys, values = filled(torch, op, "bfloat16", lengths, page, 2, dim)
    q, k, v = normal(torch, 3, "bfloat16", 7, 4, dim), normal(torch, 4, "bfloat16", 7, 2, dim, by=2.0), normal(torch, 5, "bfloat16", 7, 2, dim)
    table[6, 2] = -1                                              # the new token's page
    n[5] = table.shape[1] * page + 1                              # beyond the table's row
    keep = pool.clone()
    o = op.decode(q, pool, table, n, k=k, v=v)
    kq, vq = oracle.packed(k).to(k.dtype), oracle.packed(v).to(v.dtype)
    seen = [None] * 7
    for b in range(4):
        keys[b] = torch.cat([keys[b][:-1], kq[b:b + 1]])
        values[b] = torch.cat([values[b][:-1], vq[b:b + 1]])
        seen[b] = torch.ones(1, len(keys[b]), dtype=torch.bool, device="cuda")
    for b in (5, 6):
        have = 64 if b == 5 else 32
        seen[b] = torch.ones(1, have, dtype=torch.bool, device="cuda")
        keys[b], values[b] = keys[b][:have], values[b][:have]
    check(torch, op, o, q, keys, values, seen)
    slots = torch.tensor([int(table[b, (m - 1) // page]) * page + (m - 1) % page for b, m in enumerate(lengths[:4])], device="cuda")
    got = op.read(pool, slots, dim, k.dtype)
    assert torch.equal(got[0], kq[:4]) and torch.equal(got[1], vq[:4])
    others = [int(p) for b in (5,) for p in table[b] if p >= 0]
    assert torch.equal(pool[others], keep[others])
    assert torch.equal(o, op.decode(q, pool, table, n))


def test_what_is_not_there(torch, Packed):
    """Pages outside the pool hide their keys; an idle sequence, an empty pool and an empty table give zeros."""
    op, page = Packed(), 16
    pool, table, n, keys, values = filled(torch, op, "bfloat16", [200, 77], page, 1, 64)
    q = normal(torch, 3, "bfloat16", 2, 4, 64)
    table[0, 3], table[0, 5], table[1, 0] = -1, pool.shape[0], 2**31 - 1
    seen = [torch.ones(1, m, dtype=torch.bool, device="cuda") for m in (200, 77)]
    seen[0][:, 48:64] = seen[0][:, 80:96] = seen[1][:, :16] = False
    check(torch, op, op.decode(q, pool, table, n), q, keys, values, seen)
    assert not bool(op.decode(q, pool, torch.full_like(table, -1), n).any())
    assert not bool(op.decode(q, pool[:0], table, n).any())
    assert not bool(op.decode(q, pool, table[:, :0].contiguous(), n).any())
    assert not bool(op.decode(q, pool, table, torch.tensor([0, -5], dtype=torch.int32, device="cuda")).any())
    assert op.decode(q[:0], pool, table[:0], n[:0]).shape == (0, 4, 64)
    kept = pool[:0]
    op.append(normal(torch, 1, "bfloat16", 3, 1, 64), normal(torch, 2, "bfloat16", 3, 1, 64), kept, torch.zeros(3, dtype=torch.int64, device="cuda"))
    k, v = op.read(kept, torch.zeros(3, dtype=torch.int64, device="cuda"), 64, torch.bfloat16)
    assert not bool(k.any()) and not bool(v.any())


@pytest.mark.parametrize("dtype", TYPES)
def test_what_is_not_finite(torch, Packed, dtype):
    """NaN in the cache is NaN in the result where it is seen, and nothing where it is not."""
    op = Packed(40, 2)
    pool, table, n, keys, values = filled(torch, op, dtype, [100, 100, 100], 16, 1, 128)
    q = normal(torch, 3, dtype, 3, 4, 128)
    want = op.decode(q, pool, table, n)
    t = lambda b, i: int(table[b, i // 16]) * 16 + i % 16   # noqa: E731
    bad = torch.full((4, 1, 128), math.nan, dtype=q.dtype, device="cuda")
    bad[1:, :, 64:] = 0
    bad[2:] = bad[2:].nan_to_num(math.inf)
    zero = torch.zeros_like(bad)
    # sequence 0: places that nobody sees; 1: a key; 2: the first half of a value's columns
    op.append(bad, bad, pool, torch.tensor([t(0, 2), t(0, 30), t(0, 59), t(0, 40)], device="cuda"))
    op.append(bad[:1], zero[:1], pool, torch.tensor([t(1, 61)], device="cuda"))
    op.append(zero[:1], bad[1:2], pool, torch.tensor([t(2, 1)], device="cuda"))
    o = op.decode(q, pool, table, n)
    assert torch.equal(o[0], want[0]) and bool(o[1].isnan().all())
    assert bool(o[2, :, :64].isnan().all()) and bool(o[2, :, 64:].isfinite().all())
    # rows behind a sequence's end
    bad = torch.full((12, 1, 128), math.nan, dtype=q.dtype, device="cuda")
    op.append(bad, bad, pool, torch.tensor([t(0, i) for i in range(100, 112)], device="cuda"))
    assert torch.equal(op.decode(q, pool, table, n)[0], want[0])


def test_captured(torch, Packed):
    """Two graphs, replayed in turn, with eager work between."""
    op = Packed(500, 4)
    pool, table, n, keys, values = filled(torch, op, "bfloat16", [2000, 900, 33], 32, 2, 64)
    q = normal(torch, 3, "bfloat16", 3, 8, 64)
    k, v = normal(torch, 4, "bfloat16", 3, 2, 64), normal(torch, 5, "bfloat16", 3, 2, 64)
    op.decode(q, pool, table, n, k=k, v=v)
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            o = op.decode(q, pool, table, n, k=k, v=v)
        graphs.append((graph, o))
    for seed in range(4):
        q.copy_(normal(torch, seed, "bfloat16", 3, 8, 64))
        k.copy_(normal(torch, seed + 10, "bfloat16", 3, 2, 64))
        n -= 1
        for graph, o in graphs:
            graph.replay()
        torch.cuda.synchronize()
        want = op.decode(q, pool, table, n, k=k, v=v)
        assert all(torch.equal(o, want) for _, o in graphs)


def test_offsets_beyond_32_bits(torch, Packed):
    """A pool of 6 GB: a sequence at both ends of it."""
    op, page, kv, dim = Packed(), 256, 8, 128
    pages = 6 * 2**30 // (kv * page * (dim + dim // 16))
    pool = torch.zeros(pages, kv, page * (dim + dim // 16), dtype=torch.uint8, device="cuda")
    table = torch.tensor([[pages - 1, 0, pages - 2, pages // 2]], dtype=torch.int32, device="cuda")
    t = torch.arange(1000, device="cuda")
    slots = table[0][t // page].long() * page + t % page
    k, v = normal(torch, 1, "bfloat16", 1000, kv, dim), normal(torch, 2, "bfloat16", 1000, kv, dim)
    op.append(k, v, pool, slots)
    keys, values = op.read(pool, slots, dim, k.dtype)
    same(torch, keys, oracle.packed(k))
    q = normal(torch, 3, "bfloat16", 1, 8, dim)
    check(torch, op, op.decode(q, pool, table, torch.tensor([1000], dtype=torch.int32, device="cuda")), q, [keys], [values])


@pytest.mark.parametrize("dtype,p_unit", [("bfloat16", 2.0 ** -16), ("float16", 2.0 ** -22)])
@pytest.mark.parametrize("dim", [32, 64, 128])
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 7)])
def test_probabilities_are_not_rounded_to_the_type(torch, Packed, dtype, p_unit, dim, window, sinks):
    """What they are off by goes with their own two numbers, not with one of the type: values that cancel each other show it."""
    op = Packed(window, sinks)
    pool, table, n, keys, values = filled(torch, op, dtype, [2, 3, 7, 16, 33, 70, 200, 1500], 16, 2, dim)
    q = normal(torch, 3, dtype, 8, 6, dim)
    for longest in (1500, None):
        o = op.decode(q, pool, table, n, longest)
        for b in range(8):
            for h in range(6):
                want, bound = attention_oracle.attention(q[b, h][None], keys[b][:, h // 3], values[b][:, h // 3], window, sinks, p_unit=p_unit)
                off = (o[b, h].double() - want["o"][0]).abs()
                assert bool((off <= bound["o"][0]).all()), (b, h, float((off / bound["o"][0].clamp(min=1e-300)).max()))


def test_views_of_one_tensor(torch, Packed):
    """Queries, the new token's key and value, and results as views of one tensor; keys and values read into one."""
    op, page = Packed(), 16
    pool, table, n, keys, values = filled(torch, op, "bfloat16", [40, 1, 700], page, 2, 64)
    x = normal(torch, 3, "bfloat16", 3, 4 + 2 + 2 + 4, 64)
    q, k, v, o = x.split((4, 2, 2, 4), 1)
    got = op.decode(q, pool, table, n, k=k, v=v, o=o)
    assert got.data_ptr() == o.data_ptr()
    want = op.decode(q.contiguous(), pool, table, n)
    assert torch.equal(o, want)
    slots = torch.tensor([int(table[2, 3]) * page + 5, int(table[0, 0]) * page, -1], device="cuda")
    both = torch.full((3, 5, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    op.read(pool, slots, 64, torch.bfloat16, both[:, ::2][:, :2], both[:, 1::2])
    k, v = op.read(pool, slots, 64, torch.bfloat16)
    assert torch.equal(both[:, ::2][:, :2], k) and torch.equal(both[:, 1::2], v) and bool((both[:, 4] == 7).all())


def test_more_tokens_than_a_launch_has(torch, Packed):
    """33,554,428 tokens of 8 heads of 128 are the most that a launch writes or reads.  (Keys and values that overlap are 0.5 GB; what is read is 69 GB each.)"""
    op, page, kv, dim, n, border = Packed(), 16, 8, 128, 33_554_500, 33_554_428
    x = normal(torch, 1, "bfloat16", 1 << 20).repeat(-(-(n * 8 + kv * dim + 64) // (1 << 20)))
    k, v = x.as_strided((n, kv, dim), (8, dim, 1)), x.as_strided((n, kv, dim), (8, dim, 1), 64)
    slots = torch.full((n,), -1, dtype=torch.int64, device="cuda")
    some = torch.cat([torch.arange(5), torch.arange(border - 6, border + 9), torch.arange(n - 5, n)]).cuda()
    slots[some] = torch.randperm(2 * page, generator=torch.Generator().manual_seed(1))[:len(some)].cuda()
    pool, want = op.pool(2, page, kv, dim), op.pool(2, page, kv, dim)
    op.append(k, v, pool, slots)
    op.append(k[some], v[some], want, slots[some])
    assert torch.equal(pool, want)
    if torch.cuda.mem_get_info()[0] < 160 * 2**30:
        pytest.skip("the card has not the 138 GB of keys and values")
    got = op.read(pool, slots, dim, torch.bfloat16)
    for a, b in zip(got, op.read(pool, slots[some], dim, torch.bfloat16)):
        assert torch.equal(a[some], b)
    for at in (slice(1000, 2000), slice(border + 100, None), slice(border - 1000, border - 6)):
        assert not any(bool(a[at][slots[at] < 0].any()) for a in got)
    del got
    torch.cuda.empty_cache()
