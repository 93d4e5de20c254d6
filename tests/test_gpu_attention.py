"""Attention under an arrow-shaped mask against the 64-bit oracle: forward, gradients, single tokens over a cache in pages.  The bounds are the oracle's:
what the roundings of the operands' type may do."""
import math

import pytest

from oracle import attention_oracle as oracle

pytestmark = pytest.mark.gpu

TYPES = ("bfloat16", "float16")


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible: these tests need a real MI355X")
    return torch


@pytest.fixture(scope="module")
def Attention(torch):
    from paper_2307_05740_amd.attention import ArrowAttention
    return ArrowAttention


def normal(torch, seed, dtype, *shape, by=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * by).to(getattr(torch, dtype)).cuda()


def within(torch, name, got, want, bound):
    got = got.double()
    same = (got == want) | ((got - want).abs() <= bound)
    if not bool(same.all()):
        off = torch.where(same, 0.0, torch.nan_to_num((got - want).abs() / bound.clamp(min=1e-300), nan=math.inf, posinf=math.inf))
        at = int(off.argmax())
        raise AssertionError(f"{name}: {int((~same).sum())} of {same.numel()} values off, the worst {float(off.max()):.3g} times the bound: "
                             f"{float(got.flatten()[at])} for {float(want.flatten()[at])} at {at}")


def check_sequence(torch, got, q, k, v, window, sinks, scale=None, d_o=None):
    """One sequence, (tokens, heads, dim): got holds o, lse (heads, tokens) and the gradients there are."""
    heads, kv = q.shape[1], k.shape[1]
    grads = {}
    for h in range(heads):
        want, bound = oracle.attention(q[:, h], k[:, h * kv // heads], v[:, h * kv // heads], window, sinks, scale, None if d_o is None else d_o[:, h])
        within(torch, f"o of head {h}", got["o"][:, h], want["o"], bound["o"])
        within(torch, f"lse of head {h}", got["lse"][h], want["lse"], bound["lse"])
        if d_o is not None:
            within(torch, f"dq of head {h}", got["dq"][:, h], want["dq"], bound["dq"])
            for n in ("dk", "dv"):
                a, b = grads.setdefault((n, h * kv // heads), [0, 0])
                grads[n, h * kv // heads] = [a + want[n], b + bound[n]]
    for (n, h), (a, b) in grads.items():
        within(torch, f"{n} of head {h}", got[n][:, h], a, b + oracle.UNIT[q.dtype] * a.abs())


def run(torch, op, q, k, v, d_o=None, **ragged):
    o, lse = op.forward(q, k, v, o=torch.full_like(q, math.nan), **ragged)
    got = {"o": o, "lse": lse}
    if d_o is not None:
        nan = [torch.full_like(t, math.nan) for t in (q, k, v)]
        got["dq"], got["dk"], got["dv"] = op.backward(d_o, q, k, v, o, lse, *nan, **ragged)
    return got


# queries, keys: one token to several tiles and odd numbers of them; more queries than keys leave rows empty
LENGTHS = [(1, 1), (1, 64), (1, 300), (2, 2), (31, 31), (33, 33), (64, 64), (65, 65), (127, 130), (128, 128), (129, 129), (200, 200), (257, 321),
           (300, 300), (7, 0), (50, 20), (300, 130), (3, 700)]
MASKS = [(0, 0), (1, 0), (1, 1), (17, 0), (64, 4), (100, 65), (128, 200), (1000, 5)]


@pytest.mark.parametrize("queries,keys", LENGTHS)
@pytest.mark.parametrize("window,sinks", MASKS)
def test_lengths_and_masks(torch, Attention, queries, keys, window, sinks):
    dtype = TYPES[(queries + window) % 2]
    q, d_o = (normal(torch, s, dtype, 1, queries, 2, 64, by=b) for s, b in ((1, 2.0), (4, 1.0)))
    k, v = (normal(torch, s, dtype, 1, keys, 1, 64) for s in (2, 3))
    got = run(torch, Attention(window, sinks), q, k, v, d_o)
    check_sequence(torch, {n: t[0] for n, t in got.items()}, q[0], k[0], v[0], window, sinks, d_o=d_o[0])
    if keys < queries:
        empty = queries - keys
        assert bool((got["o"][0, :empty] == 0).all()) and bool((got["lse"][0, :, :empty] == -math.inf).all()) and bool((got["dq"][0, :empty] == 0).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [8, 24, 64, 72, 80, 96, 128])
@pytest.mark.parametrize("heads,kv", [(1, 1), (4, 4), (6, 2), (8, 1)])
def test_head_layouts(torch, Attention, dtype, dim, heads, kv):
    q, d_o = (normal(torch, s, dtype, 2, 150, heads, dim) for s in (1, 4))
    k, v = (normal(torch, s, dtype, 2, 170, kv, dim) for s in (2, 3))
    for window, sinks in ((0, 0), (70, 3)):
        got = run(torch, Attention(window, sinks, scale=0.2), q, k, v, d_o)
        for b in range(2):
            check_sequence(torch, {n: t[b] for n, t in got.items()}, q[b], k[b], v[b], window, sinks, 0.2, d_o[b])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [40, 64, 80, 128])
@pytest.mark.parametrize("queries,keys", [(400, 400), (385, 700), (430, 250)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 1), (90, 5), (200, 130)])
def test_many_heads(torch, Attention, dtype, dim, queries, keys, window, sinks):
    """Enough rows for wavefronts to share tiles of keys."""
    q, d_o = (normal(torch, s, dtype, 3, queries, 12, dim, by=b) for s, b in ((1, 2.0), (4, 1.0)))
    k, v = (normal(torch, s, dtype, 3, keys, 4, dim) for s in (2, 3))
    got = run(torch, Attention(window, sinks), q, k, v, d_o)
    for b in range(3):
        check_sequence(torch, {n: t[b] for n, t in got.items()}, q[b], k[b], v[b], window, sinks, d_o=d_o[b])


@pytest.mark.parametrize("window,sinks", [(0, 0), (150, 4), (64, 300)])
def test_long_sequences_in_parts(torch, Attention, window, sinks):
    """Enough tiles for keys that all queries see to be cut into parts, and for the loads to go round both halves of their room."""
    q, d_o = (normal(torch, s, "bfloat16", 1, 1500, 4, 128) for s in (1, 4))
    k, v = (normal(torch, s, "bfloat16", 1, 1700, 2, 128) for s in (2, 3))
    got = run(torch, Attention(window, sinks), q, k, v, d_o)
    check_sequence(torch, {n: t[0] for n, t in got.items()}, q[0], k[0], v[0], window, sinks, d_o=d_o[0])


@pytest.mark.parametrize("dtype", TYPES)
def test_ragged_batches(torch, Attention, dtype):
    lengths, keys = [5, 0, 1, 200, 64, 0, 131], [5, 0, 90, 210, 64, 33, 100]
    nq, nk = sum(lengths) + 9, sum(keys) + 4                     # some tokens belong to no sequence
    q, d_o = (normal(torch, s, dtype, nq, 4, 64) for s in (1, 4))
    k, v = (normal(torch, s, dtype, nk, 2, 64) for s in (2, 3))
    offsets = {n: torch.tensor([sum(x[:i]) for i in range(len(x) + 1)], dtype=torch.int32, device="cuda") for n, x in (("q_offsets", lengths), ("k_offsets", keys))}
    for window, sinks in ((0, 0), (40, 3)):
        for limits in ({}, {"q_len": 200, "k_len": 210}):
            got = run(torch, Attention(window, sinks), q, k, v, d_o, **offsets, **limits)
            a = b = 0
            for n, m in zip(lengths, keys):
                one = {x: got[x][a:a + n] for x in ("o", "dq")}
                one.update({x: got[x][b:b + m] for x in ("dk", "dv")}, lse=got["lse"][:, a:a + n])
                check_sequence(torch, one, q[a:a + n], k[b:b + m], v[b:b + m], window, sinks, d_o=d_o[a:a + n])
                a, b = a + n, b + m
            assert bool(got["o"][a:].isnan().all()) and bool(got["dq"][a:].isnan().all()) and bool(got["dk"][b:].isnan().all()), "no sequence's"


def test_offsets_that_lie_are_cut_to_what_there_is(torch, Attention):
    q, k, v = (normal(torch, s, "bfloat16", 40, 2, 64) for s in (1, 2, 3))
    offsets = torch.tensor([-5, 20, 10, 4000], dtype=torch.int32, device="cuda")
    o, _ = Attention().forward(q, k, v, q_offsets=offsets, k_offsets=offsets)
    want, bound = oracle.attention(q[:20, 0], k[:20, 0], v[:20, 0])
    within(torch, "o", o[:20, 0].double()[:10], want["o"][:10], bound["o"][:10])      # (sequence 2 begins at 10)


def test_strides(torch, Attention):
    """Operands and results within larger tensors: one for queries, keys and values together, heads before tokens, heads that are one head."""
    both = normal(torch, 1, "bfloat16", 2, 100, 3, 4, 64)
    q, k, v = both.unbind(2)
    d_o = normal(torch, 2, "bfloat16", 2, 4, 100, 64).transpose(1, 2)
    out = torch.full_like(both, math.nan)
    op = Attention(30, 2)
    o = torch.empty_strided(q.shape, (100 * 4 * 64, 64, 100 * 64, 1), dtype=q.dtype, device="cuda")
    o, lse = op.forward(q, k, v, o=o)
    dq, dk, dv = op.backward(d_o, q, k, v, o, lse, *out.unbind(2))
    for b in range(2):
        got = {"o": o[b], "lse": lse[b], "dq": out[b, :, 0], "dk": out[b, :, 1], "dv": out[b, :, 2]}
        check_sequence(torch, got, q[b], k[b], v[b], 30, 2, d_o=d_o[b])
    one_k, one_v = k[:, :, :1].expand(-1, -1, 4, -1), v[:, :, :1].expand(-1, -1, 4, -1)
    o1, _ = op.forward(q, one_k, one_v)
    o2, _ = op.forward(q, k[:, :, :1], v[:, :, :1])
    assert torch.equal(o1, o2)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_what_is_not_seen_does_not_count(torch, Attention, bad):
    """NaN and infinities in keys and values ahead of a query, behind its window, and beyond a sequence's end."""
    q, k, v = (normal(torch, s, "bfloat16", 1, 300, 1, 64) for s in (1, 2, 3))
    window, sinks = 50, 4
    want, bound = oracle.attention(q[0, :, 0], k[0, :, 0], v[0, :, 0], window, sinks)
    k[0, 100:102], v[0, 100:102] = bad, bad
    o, lse = Attention(window, sinks).forward(q, k, v)
    rows = [i for i in range(300) if not (100 <= i < 151)]
    within(torch, "o", o[0, rows, 0], want["o"][rows], bound["o"][rows])
    within(torch, "lse", lse[0, 0, rows], want["lse"][rows], bound["lse"][rows])
    offsets = torch.tensor([0, 100], dtype=torch.int32, device="cuda")
    o, _ = Attention(window, sinks).forward(q[0], k[0], v[0], q_offsets=offsets, k_offsets=offsets)
    within(torch, "o of a sequence that ends there", o[:100, 0], want["o"][:100], bound["o"][:100])


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_what_is_not_seen_does_not_count_for_many_heads(torch, Attention, bad):
    """The same where wavefronts share tiles of keys; a row is the same for every head."""
    q, k, v = (normal(torch, s, "bfloat16", 1, 300, 1, 64) for s in (1, 2, 3))
    window, sinks = 50, 4
    want, bound = oracle.attention(q[0, :, 0], k[0, :, 0], v[0, :, 0], window, sinks)
    k[0, 100:102], v[0, 100:102] = bad, bad
    o, lse = Attention(window, sinks).forward(q.expand(-1, -1, 60, -1), k, v)
    rows = [i for i in range(300) if not (100 <= i < 151)]
    for h in (0, 59):
        within(torch, "o", o[0, rows, h], want["o"][rows], bound["o"][rows])
        within(torch, "lse", lse[0, h, rows], want["lse"][rows], bound["lse"][rows])
    assert all(torch.equal(o[:, :, 0].view(torch.int16), o[:, :, h].view(torch.int16)) for h in range(60))


def test_large_scores(torch, Attention):
    """Scores far beyond what exp holds, and rows whose maximum comes last."""
    q = normal(torch, 1, "bfloat16", 1, 200, 1, 64, by=30.0)
    k, v = (normal(torch, s, "bfloat16", 1, 200, 1, 64) for s in (2, 3))
    k[0] *= torch.linspace(0.1, 8, 200, device="cuda")[:, None, None].to(k.dtype)
    got = run(torch, Attention(), q, k, v)
    check_sequence(torch, {n: t[0] for n, t in got.items()}, q[0], k[0], v[0], 0, 0)


def test_gradients_against_differences(torch, Attention):
    """Central differences of <o, d_o> in 64 bits along random directions; the gradient may be off by what its bound allows along them."""
    q, k, v, d_o = (normal(torch, s, "float16", 1, 90, 2 if s in (1, 4) else 1, 64) for s in (1, 2, 3, 4))
    window, sinks = 33, 2
    got = run(torch, Attention(window, sinks), q, k, v, d_o)

    def loss(q, k, v):
        p = 0.0
        for h in range(2):
            s = (q[:, h] @ k[:, 0].T / 8.0).masked_fill(~oracle.visible(90, 90, window, sinks, "cuda"), -math.inf)
            p = p + ((torch.softmax(s, -1) @ v[:, 0]) * d_o[0, :, h].double()).sum()
        return float(p)

    x = {"q": q[0].double(), "k": k[0].double(), "v": v[0].double()}
    for name in x:
        g = torch.Generator().manual_seed(9)
        to = torch.randn(x[name].shape, generator=g).cuda().double()
        eps = 1e-5
        diff = (loss(**{**x, name: x[name] + eps * to}) - loss(**{**x, name: x[name] - eps * to})) / (2 * eps)
        along = float((got["d" + name][0].double() * to).sum())
        room = 0.0
        for h in range(2):
            _, bound = oracle.attention(q[0, :, h], k[0, :, 0], v[0, :, 0], window, sinks, None, d_o[0, :, h])
            room += float((bound["d" + name] * (to[:, h] if name == "q" else to[:, 0]).abs()).sum())
        assert abs(along - diff) <= room + 1e-6 * abs(diff), (name, along, diff, room)


def test_results_are_the_same_every_time(torch, Attention):
    q, d_o = (normal(torch, s, "bfloat16", 1, 1000, 4, 64) for s in (1, 4))
    k, v = (normal(torch, s, "bfloat16", 1, 1000, 2, 64) for s in (2, 3))
    op = Attention(100, 4)
    first = run(torch, op, q, k, v, d_o)
    for _ in range(3):
        again = run(torch, op, q, k, v, d_o)
        assert all(torch.equal(first[n], again[n]) for n in first)


def test_captured_and_on_another_stream(torch, Attention):
    q, d_o = (normal(torch, s, "bfloat16", 1, 500, 4, 64) for s in (1, 4))
    k, v = (normal(torch, s, "bfloat16", 1, 500, 2, 64) for s in (2, 3))
    op = Attention(100, 4)
    want = run(torch, op, q, k, v, d_o)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        there = run(torch, op, q, k, v, d_o)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(want[n], there[n]) for n in want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o, lse = op.forward(q, k, v)
        grads = op.backward(d_o, q, k, v, o, lse)
    for seed in (7, 8, 9):
        q.copy_(normal(torch, seed, "bfloat16", 1, 500, 4, 64))
        graph.replay()
        want = run(torch, op, q, k, v, d_o)
        torch.cuda.synchronize()
        assert torch.equal(o, want["o"]) and all(torch.equal(a, want[n]) for a, n in zip(grads, ("dq", "dk", "dv")))


# ---- a cache in pages --------------------------------------------------------------------------------------------------------------
def paged(torch, dtype, lengths, page, kv, dim, spare=3, columns=None, fill=math.nan):
    """Pools whose unwritten places hold `fill`, a table in which pages lie in any order (-1 where there is none), and the keys and values of
    each sequence."""
    columns = max(1, max(-(-n // page) for n in lengths)) if columns is None else columns
    need = sum(-(-n // page) for n in lengths)
    g = torch.Generator().manual_seed(5)
    order = torch.randperm(need + spare, generator=g).tolist()
    table = torch.full((len(lengths), columns), -1, dtype=torch.int32)
    pools = [torch.full((need + spare, page, kv, dim), fill, dtype=getattr(torch, dtype), device="cuda") for _ in range(2)]
    rows = []
    for b, n in enumerate(lengths):
        own = [normal(torch, 100 * b + s, dtype, n, kv, dim) for s in (1, 2)]
        rows.append(own)
        for c in range(-(-n // page)):
            table[b, c] = order.pop()
            for pool, x in zip(pools, own):
                part = x[c * page:(c + 1) * page]
                pool[table[b, c], :part.shape[0]] = part
    return pools, table.cuda(), torch.tensor(lengths, dtype=torch.int32, device="cuda"), rows


def check_tokens(torch, o, q, rows, window, sinks, scale=None):
    for b, (k, v) in enumerate(rows):
        if k.shape[0] == 0:
            assert bool((o[b] == 0).all())
            continue
        for h in range(q.shape[1]):
            kv = h * k.shape[1] // q.shape[1]
            want, bound = oracle.attention(q[b, h][None], k[:, kv], v[:, kv], window, sinks, scale)
            within(torch, f"o of sequence {b}, head {h}", o[b, h][None], want["o"], bound["o"])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("page", [1, 8, 16, 64, 256])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (50, 4), (33, 70), (128, 1)])
def test_single_tokens(torch, Attention, dtype, page, window, sinks):
    lengths = [1, 0, 31, 32, 33, 200, 700]
    (kp, vp), table, n, rows = paged(torch, dtype, lengths, page, 2, 64)
    q = normal(torch, 3, dtype, len(lengths), 6, 64, by=2.0)
    o = Attention(window, sinks).decode(q, kp, vp, table, n, max(lengths), o=torch.full_like(q, math.nan))
    check_tokens(torch, o, q, rows, window, sinks)


@pytest.mark.parametrize("dim", [8, 72, 96, 128])
@pytest.mark.parametrize("heads,kv", [(1, 1), (16, 1), (17, 1), (40, 1), (12, 4)])
def test_single_tokens_head_layouts(torch, Attention, dim, heads, kv):
    lengths = [5, 300]
    (kp, vp), table, n, rows = paged(torch, "bfloat16", lengths, 16, kv, dim)
    q = normal(torch, 3, "bfloat16", 2, heads, dim)
    for max_len in (None, 300, 1, 100000):                       # whatever is said of the longest
        o = Attention(scale=0.3).decode(q, kp, vp, table, n, max_len)
        check_tokens(torch, o, q, rows, 0, 0, 0.3)


def test_single_tokens_over_a_long_cache(torch, Attention):
    lengths = [9000, 4097, 1]
    (kp, vp), table, n, rows = paged(torch, "bfloat16", lengths, 64, 2, 128)
    q = normal(torch, 3, "bfloat16", 3, 16, 128)
    for window, sinks in ((0, 0), (3000, 100)):
        o = Attention(window, sinks).decode(q, kp, vp, table, n, 9000)
        check_tokens(torch, o, q, rows, window, sinks)


@pytest.mark.parametrize("heads", [4, 40])
def test_the_new_token_is_written_first(torch, Attention, heads):
    lengths = [1, 0, 32, 33, 500]
    (kp, vp), table, n, rows = paged(torch, "bfloat16", lengths, 16, 2, 64)
    q, k, v = normal(torch, 3, "bfloat16", 5, heads, 64), *(normal(torch, s, "bfloat16", 5, 2, 64) for s in (4, 5))
    want_k, want_v = kp.clone(), vp.clone()
    for b, m in enumerate(lengths):
        if m:
            rows[b][0][-1], rows[b][1][-1] = k[b], v[b]
            want_k[table[b, (m - 1) // 16], (m - 1) % 16] = k[b]
            want_v[table[b, (m - 1) // 16], (m - 1) % 16] = v[b]
    o = Attention(40, 3).decode(q, kp, vp, table, n, 500, k=k, v=v)
    check_tokens(torch, o, q, rows, 40, 3)
    assert torch.equal(kp.view(torch.int16), want_k.view(torch.int16)) and torch.equal(vp.view(torch.int16), want_v.view(torch.int16)), "nothing else is written"


def test_pages_that_are_not_there_are_not_seen(torch, Attention):
    """Entries outside the pool, and lengths beyond the table: neither read nor written."""
    lengths = [100]
    (kp, vp), table, n, rows = paged(torch, "float16", lengths, 16, 1, 64)
    table[0, 1], table[0, 3] = -1, 10_000
    gone = [i for i in range(100) if i // 16 in (1, 3)]
    q, k, v = normal(torch, 3, "float16", 1, 2, 64), *(normal(torch, s, "float16", 1, 1, 64) for s in (4, 5))
    seen = torch.ones(1, 100, dtype=torch.bool, device="cuda")
    seen[0, gone] = False
    o = Attention().decode(q, kp, vp, table, n, 100)
    for h in range(2):
        want, bound = oracle.attention(q[0, h][None], rows[0][0][:, 0], rows[0][1][:, 0], seen=seen)
        within(torch, "o", o[0, h][None], want["o"], bound["o"])
    before = kp.clone()
    o = Attention().decode(q, kp, vp, table, torch.tensor([20], dtype=torch.int32, device="cuda"), 100, k=k, v=v)
    assert torch.equal(kp.view(torch.int16), before.view(torch.int16))
    o = Attention().decode(q, kp, vp, table, torch.tensor([2_000_000_000], dtype=torch.int32, device="cuda"), 100)
    assert o.shape == q.shape
    o = Attention().decode(q, kp, vp, table, torch.tensor([-3], dtype=torch.int32, device="cuda"), 100)
    assert bool((o == 0).all())


def test_prompts_are_appended(torch, Attention):
    lengths = [40, 3, 0, 17]
    (kp, vp), table, n, rows = paged(torch, "bfloat16", lengths, 8, 2, 72)
    blank = [torch.zeros_like(kp), torch.zeros_like(vp)]
    new = [normal(torch, s, "bfloat16", 4, 20, 2, 72) for s in (7, 8)]
    Attention().append(*new, *blank, table, n)
    for pool, x in zip(blank, new):
        want = torch.zeros_like(pool)
        for b, m in enumerate(lengths):
            for t in range(20):
                j = m - 20 + t
                if j >= 0:
                    want[table[b, j // 8], j % 8] = x[b, t]
        assert torch.equal(pool, want)


def test_pools_of_heads_before_tokens(torch, Attention):
    lengths = [50, 9]
    (kp, vp), table, n, rows = paged(torch, "bfloat16", lengths, 16, 2, 64)
    q = normal(torch, 3, "bfloat16", 2, 4, 64)
    want = Attention().decode(q, kp, vp, table, n)
    other = [p.transpose(1, 2).contiguous().transpose(1, 2) for p in (kp, vp)]
    assert torch.equal(Attention().decode(q, *other, table, n), want)


def test_single_tokens_agree_with_whole_sequences(torch, Attention):
    """The last row of the forward call, and a captured step that is replayed as the sequence grows."""
    op = Attention(60, 4)
    k, v = (normal(torch, s, "bfloat16", 1, 120, 2, 64) for s in (1, 2))
    q = normal(torch, 3, "bfloat16", 1, 120, 4, 64)
    whole, _ = op.forward(q, k, v)
    pools = [torch.zeros(8, 16, 2, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    table = torch.arange(8, dtype=torch.int32, device="cuda").flip(0)[None].contiguous()
    n = torch.zeros(1, dtype=torch.int32, device="cuda")
    now = [torch.empty(1, t.shape[2], 64, dtype=torch.bfloat16, device="cuda") for t in (q, k, v)]
    now[0].zero_()
    out = torch.empty_like(now[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        n.add_(1)
        op.decode(now[0], *pools, table, n, 120, k=now[1], v=now[2], o=out)
    n.zero_()
    for t in range(120):
        for to, x in zip(now, (q, k, v)):
            to.copy_(x[:, t])
        graph.replay()
        if t % 13 == 0 or t == 119:
            for h in range(4):
                want, bound = oracle.attention(q[0, t, h][None], k[0, :t + 1, h // 2], v[0, :t + 1, h // 2], 60, 4)
                within(torch, "o", out[0, h][None], want["o"], bound["o"])
                within(torch, "o of the whole", whole[0, t, h][None], want["o"], bound["o"])


def test_offsets_beyond_32_bits(torch, Attention):
    """Sequences 2^31 elements apart, heads 2^31 elements apart, and pages whose places pass 2^32 bytes and 2^31 elements."""
    far = 1 << 31
    room = torch.empty(far + 40_000, dtype=torch.bfloat16, device="cuda")
    q, k, v = (torch.as_strided(room, (2, 100, 1, 64), (far, 64, 0, 1), 8000 * i) for i in range(3))
    d_o = normal(torch, 5, "bfloat16", 2, 100, 1, 64)
    for i, t in enumerate((q, k, v)):
        t.copy_(normal(torch, i, "bfloat16", 2, 100, 1, 64))
    op = Attention(30, 2)
    o, lse = op.forward(q, k, v)
    grads = op.backward(d_o, q, k, v, o, lse)
    for b in range(2):
        got = dict(zip(("dq", "dk", "dv"), (g[b] for g in grads)), o=o[b], lse=lse[b])
        check_sequence(torch, got, q[b], k[b], v[b], 30, 2, d_o=d_o[b])
    q = torch.as_strided(room, (1, 100, 2, 64), (0, 64, far, 1))
    o, lse = op.forward(q, q, q)
    check_sequence(torch, {"o": o[0], "lse": lse[0]}, q[0], q[0], q[0], 30, 2)
    del room, q, k, v
    pages, page = 280_000, 16                                    # 2.3 G elements, 4.6 GB
    pools = [torch.empty(pages, page, 8, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    table = torch.tensor([[pages - 1, 0, pages - 7, 263_000]], dtype=torch.int32, device="cuda")
    rows = [[normal(torch, s, "bfloat16", 60, 8, 64) for s in (1, 2)]]
    n = torch.tensor([60], dtype=torch.int32, device="cuda")
    op = Attention()
    op.append(*(x[None] for x in rows[0]), *pools, table, n)
    q = normal(torch, 3, "bfloat16", 1, 8, 64)
    check_tokens(torch, op.decode(q, *pools, table, n, 60), q, rows, 0, 0)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("heads,kv,dim,window,sinks", [(1, 1, 64, 50, 4), (60, 1, 64, 50, 4), (1, 1, 128, 0, 0), (60, 1, 128, 50, 4), (60, 60, 64, 0, 0),
                                                       (60, 60, 128, 20, 0), (8, 2, 72, 100, 100)])
def test_gradients_of_what_is_not_seen(torch, Attention, heads, kv, dim, window, sinks, bad):
    """Keys and values that are not finite leave the gradients of queries that do not see them alone, and queries and gradients of results that
    are not finite those of keys that they do not see.  The rest is as it would be without them."""
    n, last = 300, heads // kv
    q, d_o = (normal(torch, s, "bfloat16", n, heads, dim) for s in (1, 4))
    k, v = (normal(torch, s, "bfloat16", n, kv, dim) for s in (2, 3))
    op = Attention(window, sinks)
    seen = oracle.visible(n, n, window, sinks)
    want = [oracle.attention(q[:, h], k[:, -1], v[:, -1], window, sinks, d_o=d_o[:, h]) for h in range(heads - last, heads)]    # of the last key head

    def check_keys(got, name, keys, columns):
        total, bound = (sum(w[i][name] for w in want) for i in (0, 1))
        bound = bound + oracle.UNIT[q.dtype] * total.abs()
        within(torch, name, got[name][0, :, -1][keys][:, columns], total[keys][:, columns], bound[keys][:, columns])

    at = [150, 151]
    bad_k, bad_v = k.clone(), v.clone()
    bad_k[at], bad_v[at] = bad, bad
    got = run(torch, op, q[None], bad_k[None], bad_v[None], d_o[None])
    rows = [i for i in range(n) if not seen[i, at].any()]
    assert len(rows) >= 148
    for h in (0, -1):
        within(torch, "dq", got["dq"][0, rows, heads - last if h == 0 else -1], want[h][0]["dq"][rows], want[h][1]["dq"][rows])

    bad_q, bad_do = q.clone(), d_o.clone()
    bad_q[at[0]], bad_do[at] = bad, bad
    got = run(torch, op, bad_q[None], k[None], v[None], bad_do[None])
    keys = [j for j in range(n) if not seen[at, j].any()]
    assert len(keys) >= 148
    for name in ("dk", "dv"):
        check_keys(got, name, keys, list(range(dim)))

    bad_do = d_o.clone()                                         # one column of a gradient that some keys do see
    bad_do[at[0], -1, 5] = bad
    got = run(torch, op, q[None], k[None], v[None], bad_do[None])
    check_keys(got, "dv", list(range(n)), [i for i in range(dim) if i != 5])
    assert torch.equal(torch.isfinite(got["dv"][0, :, -1, 5]).cpu(), ~seen[at[0]])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [64, 80, 96, 128])
@pytest.mark.parametrize("queries,keys,window,sinks", [(300, 300, 0, 0), (290, 333, 70, 5), (300, 130, 64, 0), (65, 257, 100, 100)])
def test_workgroups_of_128_queries(torch, Attention, dtype, dim, queries, keys, window, sinks):
    """So many heads that no tile is shared out further; three query heads to a key head, of which the first, the last and one in between are checked."""
    heads, kv = 600, 200
    q, d_o = (normal(torch, s, dtype, 1, queries, heads, dim) for s in (1, 4))
    k, v = (normal(torch, s, dtype, 1, keys, kv, dim) for s in (2, 3))
    got = run(torch, Attention(window, sinks), q, k, v, d_o)
    for g in (0, 77, kv - 1):
        of, at = slice(3 * g, 3 * g + 3), slice(g, g + 1)
        part = {n: got[n][0, :, of] for n in ("o", "dq")} | {n: got[n][0, :, at] for n in ("dk", "dv")} | {"lse": got["lse"][0, of]}
        check_sequence(torch, part, q[0, :, of], k[0, :, at], v[0, :, at], window, sinks, d_o=d_o[0, :, of])


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("dim,window,sinks", [(64, 50, 4), (96, 0, 0), (128, 50, 4)])
def test_what_is_not_seen_by_workgroups_of_128_queries(torch, Attention, dim, window, sinks, bad):
    test_gradients_of_what_is_not_seen(torch, Attention, 240, 240, dim, window, sinks, bad)
    q, k, v = (normal(torch, s, "bfloat16", 1, 300, 1, dim) for s in (1, 2, 3))
    want, bound = oracle.attention(q[0, :, 0], k[0, :, 0], v[0, :, 0], window, sinks)
    k[0, 100:102], v[0, 100:102] = bad, bad
    o, lse = Attention(window, sinks).forward(q.expand(-1, -1, 240, -1), k, v)
    rows = [i for i in range(300) if not oracle.visible(300, 300, window, sinks)[i, 100:102].any()]
    for h in (0, 239):
        within(torch, "o", o[0, rows, h], want["o"][rows], bound["o"][rows])
        within(torch, "lse", lse[0, h, rows], want["lse"][rows], bound["lse"][rows])


def test_gradients_that_lie_anywhere(torch, Attention):
    """What autograd hands over as the gradient of o: one value for all, a part of a larger tensor at an odd address, transposed."""
    q, k, v = (normal(torch, s, "bfloat16", 1, 70, 2, 64) for s in (1, 2, 3))
    op = Attention(30, 2)
    w = normal(torch, 4, "bfloat16", 1, 70, 2, 64)
    uses = {"sum": (lambda o: o.sum(), torch.ones_like(w)), "odd": (lambda o: (torch.cat([o[..., :3], o], -1)[..., 3:] * w).sum(), w),
            "flat": (lambda o: (torch.cat([torch.zeros(3, dtype=o.dtype, device="cuda"), o.flatten()])[3:] * w.flatten()).sum(), w),
            "across": (lambda o: (o.transpose(1, 3).contiguous() * w.transpose(1, 3).contiguous()).sum(), w)}
    for name, (use, d_o) in uses.items():
        x = [t.clone().requires_grad_() for t in (q, k, v)]
        o = op(*x)
        use(o).backward()
        got = dict(zip(("dq", "dk", "dv"), (t.grad[0] for t in x)), o=o[0].detach(), lse=op.forward(q, k, v)[1][0])
        check_sequence(torch, got, q[0], k[0], v[0], 30, 2, d_o=d_o[0])


@pytest.mark.parametrize("dim", [40, 64, 80, 128])
def test_keys_that_their_scores_rule_out(torch, Attention, dim):
    """A key of minus infinity where queries are positive has no weight, first or last columns alike."""
    n, at = 90, 40
    for column in (0, dim - 1):
        (kp, vp), table, lens, rows = paged(torch, "bfloat16", [n], 16, 1, dim)
        k, v = rows[0]
        q = normal(torch, 3, "bfloat16", 1, n, 1, dim)
        q[..., column] = q[..., column].abs() + 0.5
        seen = oracle.visible(n, n, 0, 0, "cuda")
        seen[:, at] = False
        want, bound = oracle.attention(q[0, :, 0], k[:, 0], v[:, 0], seen=seen)
        k[at, 0, column] = -math.inf
        kp[table[0, at // 16], at % 16, 0, column] = -math.inf
        o, _ = Attention().forward(q, k[None], v[None])
        within(torch, "o", o[0, :, 0], want["o"], bound["o"])
        o = Attention().decode(q[:, -1], kp, vp, table, lens, n)
        within(torch, "o of the last token", o[0], want["o"][-1:], bound["o"][-1:])


@pytest.mark.parametrize("heads", [1, 60, 240])
@pytest.mark.parametrize("dim", [64, 128])
def test_rows_without_keys_next_to_values_that_are_not_finite(torch, Attention, heads, dim):
    """More queries than keys: the first ones see nothing, their results and gradients are 0 whatever keys and values hold."""
    q, d_o = (normal(torch, s, "bfloat16", 1, 200, heads, dim) for s in (1, 4))
    k, v = (normal(torch, s, "bfloat16", 1, 130, 1, dim) for s in (2, 3))
    k[0, 3], v[0, 3] = math.nan, math.inf
    got = run(torch, Attention(), q, k, v, d_o)
    for name in ("o", "dq"):
        assert bool((got[name][0, :70] == 0).all()), name
    assert bool((got["lse"][0, :, :70] == -math.inf).all()) and bool(torch.isfinite(got["o"][0, 70:73]).all())


# queries, keys, heads, key heads, dim, window, sinks: few queries of many keys
CUT = [(1, 5000, 4, 2, 128, 0, 0), (16, 9000, 4, 1, 128, 0, 0), (33, 3000, 2, 2, 64, 0, 0), (64, 2500, 3, 3, 80, 2200, 7), (20, 700, 2, 1, 64, 600, 3),
       (5, 20000, 1, 1, 96, 0, 0), (40, 2100, 1, 1, 128, 0, 0)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("queries,keys,heads,kv,dim,window,sinks", CUT)
def test_few_queries_of_many_keys(torch, Attention, dtype, queries, keys, heads, kv, dim, window, sinks):
    """Keys that are cut over several workgroups, also where some sequences of a batch have few or none."""
    q = normal(torch, 1, dtype, queries, heads, dim, by=2.0)
    k, v = (normal(torch, s, dtype, keys, kv, dim) for s in (2, 3))
    op = Attention(window, sinks)
    got = run(torch, op, q[None], k[None], v[None])
    check_sequence(torch, {n: t[0] for n, t in got.items()}, q, k, v, window, sinks)
    again = run(torch, op, q[None], k[None], v[None])
    assert all(torch.equal(got[n], again[n]) for n in got)
    lengths = [(queries, keys - 300), (0, 40), (1, 1), (2, 0), (queries, 130)]
    q_offsets, k_offsets = (torch.tensor([0] + [sum(x[i] for x in lengths[:n + 1]) for n in range(len(lengths))], dtype=torch.int32, device="cuda") for i in (0, 1))
    nq, nk = (sum(x[i] for x in lengths) for i in (0, 1))
    q = normal(torch, 1, dtype, nq + 3, heads, dim)
    k, v = (normal(torch, s, dtype, nk + 3, kv, dim) for s in (2, 3))
    got = run(torch, op, q, k, v, q_offsets=q_offsets, k_offsets=k_offsets, q_len=queries + 1, k_len=keys)
    for b in range(len(lengths)):
        i, j = slice(int(q_offsets[b]), int(q_offsets[b + 1])), slice(int(k_offsets[b]), int(k_offsets[b + 1]))
        check_sequence(torch, {"o": got["o"][i], "lse": got["lse"][:, i]}, q[i], k[j], v[j], window, sinks)
    assert bool(torch.isnan(got["o"][nq:]).all())


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_few_queries_of_many_keys_of_which_some_are_not_seen(torch, Attention, bad):
    q = normal(torch, 1, "bfloat16", 1, 40, 2, 128)
    k, v = (normal(torch, s, "bfloat16", 1, 6000, 2, 128) for s in (2, 3))
    op = Attention(4000, 4)
    k[0, 100:1900], v[0, 100:1900] = bad, bad                    # behind all windows
    k[0, 5990], v[0, 5990] = bad, bad                            # ahead of the first 30
    got = op.forward(q, k, v)[0]
    for h in range(2):
        k2, v2 = torch.where(torch.isfinite(k), k, 0.0), torch.where(torch.isfinite(v), v, 0.0)
        exact, bound = oracle.attention(q[0, :30, h], k2[0, :5990, h], v2[0, :5990, h], 4000, 4)
        within(torch, "o", got[0, :30, h], exact["o"], bound["o"])
    assert not bool(torch.isfinite(got[0, 30:]).any())


@pytest.mark.parametrize("length,window", [(64, 0), (64, 20), (6000, 0)])
def test_a_new_token_beyond_the_table_is_left_out(torch, Attention, length, window):
    """The table is full: the last token's key and value stay, and are the ones that count."""
    page = 16
    (kp, vp), table, n, rows = paged(torch, "bfloat16", [length, length // 2], page, 2, 64, columns=length // page)
    q, k, v = normal(torch, 3, "bfloat16", 2, 4, 64), *(normal(torch, s, "bfloat16", 2, 2, 64) for s in (4, 5))
    half = length // 2                                           # (the other sequence has room)
    rows[1][0][-1], rows[1][1][-1] = k[1], v[1]
    want = [p.clone() for p in (kp, vp)]
    for pool, x in zip(want, (k, v)):
        pool[table[1, (half - 1) // page], (half - 1) % page] = x[1]
    op = Attention(window, 2)
    for more in (length + 1, 2_000_000_000):
        n[0] = more
        o = op.decode(q, kp, vp, table, n, length, k=k, v=v)
        check_tokens(torch, o, q, rows, window, 2)
        for pool, x in zip((kp, vp), want):
            assert torch.equal(pool.view(torch.int16), x.view(torch.int16)), "the token was written over another one"


def test_tokens_that_no_sequence_has_take_no_part_in_training(torch, Attention):
    """Room at the end of a ragged batch, and a sequence cut to q_len and k_len: zeros in o and in the gradients, whatever memory held before."""
    def junk():
        return [torch.full((200, 2, 64), math.nan, dtype=torch.bfloat16, device="cuda") for _ in range(8)]

    offsets = torch.tensor([0, 30, 30, 95], dtype=torch.int32, device="cuda")
    op = Attention(20, 2)
    for limits, end in (({}, 95), ({"q_len": 40, "k_len": 40}, 70)):
        x = [normal(torch, s, "bfloat16", 200, 2, 64).requires_grad_() for s in (1, 2, 3)]
        d_o = normal(torch, 4, "bfloat16", 200, 2, 64)
        junk()                                                   # (what the allocator hands out next)
        o = op(*x, offsets, offsets, **limits)
        junk()
        o.backward(d_o)
        got = dict(zip(("dq", "dk", "dv"), (t.grad for t in x)), o=o.detach())
        for name, t in got.items():
            assert bool((t[end:] == 0).all()), name
        lse = op.forward(*(t.detach() for t in x), q_offsets=offsets, k_offsets=offsets, **limits)[1]
        for of in (slice(0, 30), slice(30, end)):
            part = {n: t[of] for n, t in got.items()}
            check_sequence(torch, part | {"lse": lse[:, of]}, *(t.detach()[of] for t in x), 20, 2, d_o=d_o[of])


def check_norms(torch, got, q, k, v, window, sinks, d_o):
    """The gradients of one sequence against 64 bits by their norms.  P and dS are rounded once, relative to themselves, which is u / sqrt(3) of a sum's norm at most
    where roundings are independent; D adds as much again, and the result is rounded to its type once."""
    u = oracle.UNIT[q.dtype]
    heads, kv = q.shape[1], k.shape[1]
    want = {n: 0 for n in ("dk", "dv")}
    for h in range(heads):
        one, _ = oracle.attention(q[:, h], k[:, h * kv // heads], v[:, h * kv // heads], window, sinks, None, d_o[:, h])
        want["dq"] = one["dq"]
        for name in ("dk", "dv"):
            want[name] = want[name] + one[name]
        of = {"dq": got["dq"][:, h]}
        if (h + 1) % (heads // kv) == 0:
            of.update({n: got[n][:, h * kv // heads] for n in ("dk", "dv")})
        for name, t in of.items():
            x = want[name]
            off, result = (float((y.double() - x).norm() / x.norm()) for y in (t, x.to(q.dtype)))
            assert off <= math.sqrt(result ** 2 + 2 * u * u / 3), (name, h, off, result)
            if name != "dq":
                want[name] = 0


@pytest.mark.parametrize("size", [0, -6, -10, -12])
@pytest.mark.parametrize("queries,keys,heads,kv,dim,window,sinks", [(1500, 1500, 1, 1, 64, 0, 0), (1500, 1500, 1, 1, 64, 400, 4), (1100, 1300, 6, 2, 128, 0, 0),
                                                                    (2100, 2100, 16, 16, 64, 1000, 5), (1000, 1000, 24, 8, 96, 0, 0)])
def test_small_gradients_in_float16(torch, Attention, queries, keys, heads, kv, dim, window, sinks, size):
    """Gradients of o of about 2^size over long rows: P dP is below what float16 holds in full."""
    q, d_o = (normal(torch, s, "float16", queries, heads, dim, by=b) for s, b in ((1, 1.0), (4, 2.0 ** size)))
    k, v = (normal(torch, s, "float16", keys, kv, dim) for s in (2, 3))
    got = run(torch, Attention(window, sinks), q[None], k[None], v[None], d_o[None])
    check_norms(torch, {n: t[0] for n, t in got.items()}, q, k, v, window, sinks, d_o)


def test_gradients_of_all_sizes_in_a_ragged_batch(torch, Attention):
    """Each sequence's gradients are rounded by its own size, however long the others are and wherever it begins."""
    lengths, sizes = [33, 0, 900, 1, 64, 1003, 95, 31], [-3, 0, -12, 0, -9, 0, -12, -12]
    starts = [sum(lengths[:i]) for i in range(len(lengths) + 1)]
    n = starts[-1] + 5
    q, d_o = (normal(torch, s, "float16", n, 4, 64) for s in (1, 4))
    k, v = (normal(torch, s, "float16", n, 2, 64) for s in (2, 3))
    for a, b, size in zip(starts, starts[1:], sizes):
        d_o[a:b] *= 2.0 ** size
    offsets = torch.tensor(starts, dtype=torch.int32, device="cuda")
    for window, sinks in ((0, 0), (200, 3)):
        got = run(torch, Attention(window, sinks), q, k, v, d_o, q_offsets=offsets, k_offsets=offsets, q_len=1003, k_len=1003)
        for a, b in zip(starts, starts[1:]):
            if b - a > 1:
                of = slice(a, b)
                check_norms(torch, {x: got[x][of] for x in ("dq", "dk", "dv")}, q[of], k[of], v[of], window, sinks, d_o[of])


def test_gradients_of_all_sizes_of_a_float16(torch, Attention):
    """From the smallest numbers of the type to its largest, in neighbouring rows too, within the bounds."""
    for low, high in ((-24, -24), (-24, 0), (-14, 15), (4, 15)):
        g = torch.Generator().manual_seed(8)
        size = 2.0 ** (low + (high - low) * torch.rand(1, 200, 2, 1, generator=g))
        q = normal(torch, 1, "float16", 1, 200, 2, 64)
        k, v = (normal(torch, s, "float16", 1, 200, 1, 64, by=b) for s, b in ((2, 1.0), (3, 2.0 ** -6)))
        d_o = (torch.randn(1, 200, 2, 64, generator=g).clamp(-1.9, 1.9) * size).half().cuda()
        for window, sinks in ((0, 0), (40, 2)):
            got = run(torch, Attention(window, sinks), q, k, v, d_o)
            check_sequence(torch, {n: t[0] for n, t in got.items()}, q[0], k[0], v[0], window, sinks, d_o=d_o[0])


def odd_values(torch, v, at):
    """v with elements that are not finite, {(key, column): value}."""
    for (j, d), x in at.items():
        v[j, :, d] = x
    return v


def want_odd(torch, seen, v):
    """Where (rows, columns) a result is plus infinity, minus infinity and NaN by the values that each row sees."""
    see, v = seen.to(v.device).double(), v.double()
    plus, minus, nan = ((see @ x.double()) > 0 for x in (v == math.inf, v == -math.inf, v.isnan()))
    nan = nan | (plus & minus)
    return plus & ~nan, minus & ~nan, nan


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("queries,keys,heads,dim,window,sinks", [(300, 300, 1, 64, 50, 4), (300, 300, 60, 64, 50, 4), (300, 300, 240, 128, 50, 4), (310, 300, 60, 96, 0, 0),
                                                                 (20, 5000, 2, 64, 0, 0), (40, 6000, 2, 128, 4000, 2), (2100, 2100, 2, 64, 0, 0), (2100, 2100, 16, 128, 600, 70)])
def test_values_that_are_not_finite_reach_who_sees_them(torch, Attention, dtype, queries, keys, heads, dim, window, sinks):
    """Infinities of one sign stay, of both make NaN, each in its own column; the rest is within its bounds.  (Scores are small: no weight vanishes.)"""
    q = normal(torch, 1, dtype, queries, heads, dim, by=0.3)
    k, v = (normal(torch, s, dtype, keys, 1, dim) for s in (2, 3))
    half, last = keys // 2, keys - 1
    odd_values(torch, v, {(half, 3): math.inf, (half + 1, 3): -math.inf, (half + 7, 5): math.nan, (half - 20, 7): -math.inf, (0, 9): math.inf, (last, 11): math.nan,
                          (last - 2, dim - 1): math.inf, (half, dim - 2): -math.inf})
    o, lse = Attention(window, sinks).forward(q[None], k[None], v[None])
    seen = oracle.visible(queries, keys, window, sinks, "cuda")
    odd = want_odd(torch, seen, v[:, 0])
    for h in (0, heads - 1):
        want, bound = oracle.attention(q[:, h], k[:, 0], v[:, 0], window, sinks)
        got = o[0, :, h].double()
        for name, x, where in zip(("infinity", "minus infinity", "NaN"), (got == math.inf, got == -math.inf, got.isnan()), odd):
            assert torch.equal(x, where), (name, h, int((x != where).sum()))
        finite = ~(odd[0] | odd[1] | odd[2])
        within(torch, "o", got[finite], want["o"][finite], bound["o"][finite])
        within(torch, "lse", lse[0, h], want["lse"], bound["lse"])


def time_of(torch, call):
    """The fastest of five, in microseconds."""
    best = math.inf
    for _ in range(6):
        start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        start.record()
        call()
        end.record()
        end.synchronize()
        best = min(best, start.elapsed_time(end) * 1e3)
    return best


@pytest.mark.parametrize("heads,dim,window", [(8, 64, 0), (8, 128, 0), (8, 128, 1024)])
def test_values_that_are_not_finite_cost_one_pass_more(torch, Attention, heads, dim, window):
    """A second pass of the same tiles with two products where the first has one, at half as many keys at a time: three to six times a call in all, 12 is room for clocks."""
    q, k, v = (normal(torch, s, "bfloat16", 1, 4096, heads, dim) for s in (1, 2, 3))
    op = Attention(window, 4)
    plain = time_of(torch, lambda: op.forward(q, k, v))
    v[0, 2] = math.nan                                            # all rows see it
    every = time_of(torch, lambda: op.forward(q, k, v))
    v[0, 2] = 0
    v[0, 1000, :, 5] = math.inf                                   # seen by some
    some = time_of(torch, lambda: op.forward(q, k, v))
    assert max(every, some) <= 12 * plain + 50, (plain, every, some)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,heads,kv,dim,window,sinks", [(300, 2, 1, 64, 50, 4), (300, 60, 20, 96, 0, 0), (1500, 4, 2, 128, 150, 4), (2100, 8, 2, 64, 0, 0), (1100, 16, 16, 64, 300, 3),
                                                         (900, 96, 32, 128, 256, 70)])
def test_gradients_next_to_what_is_not_finite(torch, Attention, dtype, n, heads, kv, dim, window, sinks):
    """As for 300 tokens above, at sizes at which tiles are seen whole, cut into parts, shared by four wavefronts or by none."""
    q, d_o = (normal(torch, s, dtype, n, heads, dim, by=b) for s, b in ((1, 0.5), (4, 1.0)))
    k, v = (normal(torch, s, dtype, n, kv, dim) for s in (2, 3))
    op, at, group = Attention(window, sinks), n // 2, heads // kv
    seen = oracle.visible(n, n, window, sinks, "cuda")
    want = [oracle.attention(q[:, h], k[:, -1], v[:, -1], window, sinks, d_o=d_o[:, h]) for h in range(heads - group, heads)]   # of the last key head

    bad_k, bad_v = k.clone(), v.clone()
    bad_k[at], bad_v[at + 1] = math.nan, math.inf
    got = run(torch, op, q[None], bad_k[None], bad_v[None], d_o[None])
    blind = ~seen[:, at] & ~seen[:, at + 1]
    assert int(blind.sum()) >= n // 2
    within(torch, "dq", got["dq"][0, :, -1][blind], want[-1][0]["dq"][blind], want[-1][1]["dq"][blind])
    # (rows that see the infinite value have dS = NaN and the key's gradients with them; the rows that see the NaN key are NaN throughout)
    assert bool(torch.isnan(got["dq"][0, :, -1][~blind]).all())

    bad_do = d_o.clone()
    bad_do[at, :, 3], bad_do[at + 5, :, 3], bad_do[at, :, 6], bad_do[n - 1, :, dim - 1] = math.inf, math.inf, -math.inf, math.nan
    got = run(torch, op, q[None], k[None], v[None], bad_do[None])
    total, bound = (sum(w[i]["dv"] for w in want) for i in (0, 1))
    bound = bound + oracle.UNIT[q.dtype] * total.abs()
    dv = got["dv"][0, :, -1]
    plain = [d for d in range(dim) if d not in (3, 6, dim - 1)]
    within(torch, "dv", dv[:, plain], total[:, plain], bound[:, plain])
    for d, rows in ((3, [at, at + 5]), (6, [at]), (dim - 1, [n - 1])):
        odd = seen[rows].any(0)
        assert torch.equal(torch.isfinite(dv[:, d]), ~odd), d
        within(torch, f"dv, column {d}", dv[~odd][:, d], total[~odd][:, d], bound[~odd][:, d])
    bad = seen[[at, at + 5, n - 1]].any(0)
    total, bound = (sum(w[i]["dk"] for w in want) for i in (0, 1))
    bound = bound + oracle.UNIT[q.dtype] * total.abs()
    dk = got["dk"][0, :, -1]
    within(torch, "dk", dk[~bad], total[~bad], bound[~bad])
    assert not bool(torch.isfinite(dk[bad]).any())


@pytest.mark.parametrize("queries,heads,kv,dim,window,sinks", [(200, 2, 1, 64, 0, 0), (200, 2, 1, 128, 40, 2), (300, 60, 20, 64, 0, 0), (300, 90, 30, 96, 60, 3), (40, 4, 4, 64, 0, 0)])
def test_gradients_of_scores_beyond_float16(torch, Attention, queries, heads, kv, dim, window, sinks):
    """P (dP - D) of more than 65,504, where the results are not."""
    q = normal(torch, 1, "float16", queries, heads, dim)
    k, v = (normal(torch, s, "float16", queries, kv, dim, by=b) for s, b in ((2, 0.25), (3, 12000.0)))
    v = v.clamp(-60000.0, 60000.0)
    d_o = torch.where(normal(torch, 4, "float16", queries, heads, dim) < 0, -1.9, 1.9).half()
    scale = 2.0 ** -4
    got = run(torch, Attention(window, sinks, scale), q[None], k[None], v[None], d_o[None])
    got = {n: t[0] for n, t in got.items()}
    seen, group = oracle.visible(queries, queries, window, sinks, "cuda"), heads // kv

    def largest(h):
        """|dS| of a head."""
        g = d_o[:, h].double()
        p = torch.exp(q[:, h].double() @ k[:, h // group].double().T * scale - got["lse"][h].double()[:, None]) * seen
        return float((p * (g @ v[:, h // group].double().T - (g * got["o"][:, h].double()).sum(-1, keepdim=True))).abs().max())

    most = [largest(h) for h in range(heads)]
    assert max(most) > 70000, max(most)
    for g in sorted({0, kv // 2, kv - 1, most.index(max(most)) // group}):
        of, at = slice(g * group, (g + 1) * group), slice(g, g + 1)
        part = {n: got[n][:, of] for n in ("o", "dq")} | {n: got[n][:, at] for n in ("dk", "dv")} | {"lse": got["lse"][of]}
        check_sequence(torch, part, q[:, of], k[:, at], v[:, at], window, sinks, scale, d_o[:, of])


@pytest.mark.parametrize("heads,dim,window", [(8, 64, 0), (8, 128, 1024), (32, 64, 0)])
def test_gradients_that_are_not_finite_cost_one_pass_more(torch, Attention, heads, dim, window):
    """As the forward call: three to six times a call, 12 is room for clocks."""
    q, k, v, d_o = (normal(torch, s, "float16", 1, 4096, heads, dim) for s in (1, 2, 3, 4))
    op = Attention(window, 4)
    o, lse = op.forward(q, k, v)
    plain = time_of(torch, lambda: op.backward(d_o, q, k, v, o, lse))
    d_o[0, 2000, :, 5] = math.inf                                 # what float16 training with a scaled loss meets
    one = time_of(torch, lambda: op.backward(d_o, q, k, v, o, lse))
    d_o[0, 2000, :, 5] = 0
    v[0, 2, :, 1] = math.inf
    o, lse = op.forward(q, k, v)
    value = time_of(torch, lambda: op.backward(d_o, q, k, v, o, lse))
    assert max(one, value) <= 12 * plain + 50, (plain, one, value)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [64, 96, 128])
@pytest.mark.parametrize("heads,kv", [(4, 2), (8, 4)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (200, 70), (64, 0)])
def test_long_ragged_batches(torch, Attention, dtype, dim, heads, kv, window, sinks):
    """Thousands of tokens: workgroups of 64 and of 128 queries and of 128 keys, tiles of keys cut into parts, and sequences without queries, with one, with more
    queries than keys and the other way round."""
    import ctypes
    from paper_2307_05740_amd.binding import lib
    lengths, keys = [1500, 0, 1, 777, 64, 1031], [1500, 20, 1, 900, 33, 1159]
    nq, nk = sum(lengths) + 7, sum(keys) + 3
    q, d_o = (normal(torch, s, dtype, nq, heads, dim) for s in (1, 4))
    k, v = (normal(torch, s, dtype, nk, kv, dim) for s in (2, 3))
    ragged = {n: torch.tensor([sum(x[:i]) for i in range(len(x) + 1)], dtype=torch.int32, device="cuda") for n, x in (("q_offsets", lengths), ("k_offsets", keys))}
    ragged.update(q_len=1500, k_len=1500)
    op = Attention(window, sinks)
    if sinks or (window == 0 and kv == 2):                       # (sums of parts are 128 keys of dk and dv in 32 bits)
        a = op._describe(q, k, v, **ragged)
        assert lib().arrow_attention_workspace_bytes(ctypes.byref(a)) > 8 * nq * heads + 8 * 128 * dim, "no tile of keys is cut"
    got = run(torch, op, q, k, v, d_o, **ragged)
    a = b = 0
    for n, m in zip(lengths, keys):
        one = {x: got[x][a:a + n] for x in ("o", "dq")}
        one.update({x: got[x][b:b + m] for x in ("dk", "dv")}, lse=got["lse"][:, a:a + n])
        check_sequence(torch, one, q[a:a + n], k[b:b + m], v[b:b + m], window, sinks, d_o=d_o[a:a + n])
        a, b = a + n, b + m
    assert bool(got["o"][a:].isnan().all()) and bool(got["dq"][a:].isnan().all()) and bool(got["dk"][b:].isnan().all()), "no sequence's"
    again = run(torch, op, q, k, v, d_o, **ragged)
    assert torch.equal(got["lse"][:, :a], again["lse"][:, :a])   # (what lies behind is not written)
    assert all(torch.equal(got[n].view(torch.int16), again[n].view(torch.int16)) for n in ("o", "dq", "dk", "dv"))


@pytest.mark.parametrize("queries,heads,kv,window", [(700, 2, 1, 0), (700, 24, 8, 200)])
def test_gradients_of_o_with_a_large_column(torch, Attention, queries, heads, kv, window):
    """A column of d_o that is large where the values have nothing: the others keep float16's precision."""
    q, d_o = (normal(torch, s, "float16", queries, heads, 64, by=b) for s, b in ((1, 1.0), (4, 0.3)))
    k, v = (normal(torch, s, "float16", queries, kv, 64) for s in (2, 3))
    d_o[..., 5], v[..., 5] = 30000.0, 0.0
    got = run(torch, Attention(window, 3), q[None], k[None], v[None], d_o[None])
    check_norms(torch, {n: t[0] for n, t in got.items()}, q, k, v, window, 3, d_o)
