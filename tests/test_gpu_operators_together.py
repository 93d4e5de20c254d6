"""The operators on sequences together, as a program that trains or serves calls them, on streams and in graphs."""
import importlib.util
import math
import os

import pytest

from oracle import attention_oracle, operators_oracle as oracle

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible: these tests need a real MI355X")
    return torch


def normal(torch, seed, dtype, *shape, by=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * by).to(getattr(torch, dtype)).cuda()


class Server:
    """One layer of a server: heads are rotated, tokens get places, keys and values go to a cache in 4 bits, queries are answered."""

    def __init__(self, batch, pages, page, columns, heads, kv, dim, window, sinks):
        from paper_2307_05740_amd.packed import ArrowPackedAttention
        from paper_2307_05740_amd.pages import ArrowPages
        from paper_2307_05740_amd.rotation import ArrowRotation
        self.heads, self.kv, self.dim, self.page = heads, kv, dim, page
        self.rotate, self.pages, self.attend = ArrowRotation(dim), ArrowPages(pages, page, window, sinks), ArrowPackedAttention(window, sinks)
        self.table, self.held, self.free = self.pages.state(batch, columns)
        self.pool = self.attend.pool(pages, page, kv, dim)

    def token(self, qkv, lengths):
        """qkv (batch, heads + 2 key heads, dim) of each sequence's token at lengths - 1."""
        q, k, v = qkv.split((self.heads, self.kv, self.kv), -2)
        q, k = self.rotate.forward(q, k, positions=lengths, shift=-1)
        slots = self.pages.step(self.table, self.held, self.free, lengths, 1)
        self.attend.append(k, v, self.pool, slots.flatten())
        return self.attend.decode(q, self.pool, self.table, lengths), q, k


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("window,sinks,page", [(0, 0, 16), (40, 3, 16), (64, 20, 32)])
def test_a_server(torch, dtype, window, sinks, page):
    """Tokens one by one; sequences that end and others that begin in their place; every answer is that of the keys and values that were written."""
    batch, heads, kv, dim, steps = 5, 4, 2, 64, 130
    server = Server(batch, 40 if not window else 26, page, 160 // page, heads, kv, dim, window, sinks)
    keys, values = [[] for _ in range(batch)], [[] for _ in range(batch)]
    for step in range(steps):
        for b in range(batch):
            if step % (37 + 11 * b) == 36:                        # this one ends
                keys[b], values[b] = [], []
        now = [len(x) for x in keys]
        if 0 in now and step:
            server.pages.step(server.table, server.held, server.free, torch.tensor(now, dtype=torch.int32, device="cuda"), 0)
        lengths = torch.tensor([n + 1 for n in now], dtype=torch.int32, device="cuda")
        qkv = normal(torch, step, dtype, batch, heads + 2 * kv, dim)
        o, q, k = server.token(qkv, lengths)
        turned, bound = oracle.rotation(qkv[:, heads:heads + kv], None, lengths.long() - 1, server.rotate.turns, dim)
        assert bool(((k.double() - turned["y"]).abs() <= bound["y"]).all())
        v = qkv[:, heads + kv:]
        for b in range(batch):
            keys[b].append(oracle.packed(k[b]).to(k.dtype))
            values[b].append(oracle.packed(v[b]).to(v.dtype))
        if step % 9 and step < steps - 1:
            continue
        for b in range(batch):
            kb, vb = torch.stack(keys[b]), torch.stack(values[b])
            for h in range(heads):
                want, bound = attention_oracle.attention(q[b, h][None], kb[:, h * kv // heads], vb[:, h * kv // heads], window, sinks)
                assert bool(((o[b, h].double() - want["o"][0]).abs() <= bound["o"][0]).all()), (step, b, h)
    # every page is in one place
    assert sorted(server.table[server.table >= 0].tolist() + server.free[1:1 + int(server.free[0])].tolist()) == list(range(server.pages.pages))


def test_a_server_in_a_graph(torch):
    """A whole step captured once and replayed for every token, beside another server whose steps are eager."""
    make = lambda: Server(3, 30, 16, 12, 8, 2, 128, 50, 4)   # noqa: E731
    one, other = make(), make()
    lengths, qkv = torch.zeros(3, dtype=torch.int32, device="cuda"), normal(torch, 0, "bfloat16", 3, 12, 128)
    warm = make()
    warm.token(qkv, lengths + 1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lengths += 1
        o, q, k = one.token(qkv, lengths)
    at = torch.zeros_like(lengths)
    for step in range(120):
        qkv.copy_(normal(torch, step, "bfloat16", 3, 12, 128))
        graph.replay()
        at += 1
        want = other.token(qkv, at)
        torch.cuda.synchronize()
        assert torch.equal(o, want[0]) and torch.equal(k, want[2]) and torch.equal(one.table, other.table)


def test_a_chunk_behind_a_cache(torch):
    """The second chunk of a prompt: what is cached is read back, and the attention of whole sequences goes over it and the new keys."""
    from paper_2307_05740_amd.attention import ArrowAttention
    server = Server(1, 20, 16, 20, 4, 2, 64, 0, 0)
    first, second = 100, 37
    qkv = normal(torch, 1, "bfloat16", first + second, 8, 64)
    q, k, v = qkv.split((4, 2, 2), -2)
    q, k = server.rotate.forward(q, k)
    n = torch.tensor([first], dtype=torch.int32, device="cuda")
    slots = server.pages.step(server.table, server.held, server.free, n, first).flatten()
    server.attend.append(k[:first], v[:first], server.pool, slots)
    kc, vc = server.attend.read(server.pool, slots, 64, torch.bfloat16)
    kk, vv = torch.cat([kc, k[first:]]), torch.cat([vc, v[first:]])
    o, _ = ArrowAttention().forward(q[first:][None], kk[None], vv[None])
    for h in range(4):
        want, bound = attention_oracle.attention(q[first:, h], kk[:, h // 2], vv[:, h // 2])
        assert bool(((o[0, :, h].double() - want["o"]).abs() <= bound["o"]).all())


def test_a_training_step(torch):
    """Autograd through the lookup, rotation, attention and log probabilities gives what their gradients give one after the other."""
    from paper_2307_05740_amd.attention import ArrowAttention
    from paper_2307_05740_amd.embedding import ArrowEmbedding
    from paper_2307_05740_amd.logprobs import ArrowLogProbs
    from paper_2307_05740_amd.rotation import ArrowRotation
    rows, heads, kv, dim = 97, 4, 2, 32
    embed, rotate, attend, score = ArrowEmbedding(rows), ArrowRotation(dim), ArrowAttention(20, 2), ArrowLogProbs()
    table = normal(torch, 1, "bfloat16", rows, (heads + 2 * kv) * dim).requires_grad_()
    wq, wk = (torch.nn.Parameter(1 + 0.2 * normal(torch, s, "float32", dim)) for s in (2, 3))
    ids = torch.randint(0, rows, (2, 50), generator=torch.Generator().manual_seed(4)).cuda()
    targets = torch.randint(-1, heads * dim, (2, 50), generator=torch.Generator().manual_seed(5)).cuda()
    x = embed(table, ids).unflatten(-1, (-1, dim))
    q, k, v = x.split((heads, kv, kv), -2)
    y = attend(*rotate(q, k, wq, wk), v).flatten(-2)
    logp, entropy = score(y, targets)
    loss = -(logp + 0.1 * entropy).mean()
    loss.backward()
    # by hand
    with torch.no_grad():
        x = embed.forward(table, ids).unflatten(-1, (-1, dim))
        q, k, v = x.split((heads, kv, kv), -2)
        qr, kr = rotate.forward(q, k, wq, wk)
        o, lse = attend.forward(qr, kr, v)
        r = score.forward(o.flatten(-2), targets)
        g = torch.full((2, 50), -1 / 100, device="cuda")
        dy = score.backward(g, g * 0.1, o.flatten(-2), targets, r.stats, r.entropy)
        dqr, dkr, dv = attend.backward(dy.unflatten(-1, (-1, dim)), qr, kr, v, o, lse)
        dq, dk, dwq, dwk = rotate.backward(dqr, dkr, q, k, wq, wk)
        want = embed.backward(torch.cat([dq, dk, dv], -2).flatten(-2), ids)
    assert torch.equal(logp, r.logp) and torch.equal(entropy, r.entropy)
    assert torch.equal(wq.grad, dwq) and torch.equal(wk.grad, dwk) and torch.equal(table.grad, want)


def test_on_another_stream(torch):
    """Calls on a stream that is not the default one, which waits for what they need and is waited for."""
    from paper_2307_05740_amd.logprobs import ArrowLogProbs
    stream = torch.cuda.Stream()
    server, other = (Server(4, 60, 16, 20, 8, 2, 128, 0, 0) for _ in range(2))
    qkv, lengths = normal(torch, 1, "bfloat16", 4, 12, 128), torch.tensor([1, 1, 1, 1], dtype=torch.int32, device="cuda")
    x, t = normal(torch, 2, "bfloat16", 300, 5000), torch.arange(300, device="cuda")
    score = ArrowLogProbs()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        got = server.token(qkv, lengths)
        r = score.forward(x, t, 5)
        d = score.backward(r.logp, r.entropy, x, t, r.stats, r.entropy)
    torch.cuda.current_stream().wait_stream(stream)
    want = other.token(qkv, lengths)
    s = score.forward(x, t, 5)
    assert all(torch.equal(a, b) for a, b in zip(got + tuple(r), want + tuple(s)))
    assert torch.equal(d, score.backward(s.logp, s.entropy, x, t, s.stats, s.entropy))


def test_two_streams_and_two_graphs_at_once(torch):
    """The same objects called on two streams that do not wait for each other, and captured twice: calls share no memory."""
    from paper_2307_05740_amd.logprobs import ArrowLogProbs
    from paper_2307_05740_amd.packed import ArrowPackedAttention
    from paper_2307_05740_amd.rotation import ArrowRotation
    rotate, score, attend = ArrowRotation(128), ArrowLogProbs(), ArrowPackedAttention()
    pool = attend.pool(300, 16, 2, 128)
    slots = torch.arange(300 * 16, device="cuda")
    attend.append(normal(torch, 1, "bfloat16", 4800, 2, 128), normal(torch, 2, "bfloat16", 4800, 2, 128), pool, slots)
    table, lengths = torch.arange(300, dtype=torch.int32, device="cuda").view(1, 300), torch.tensor([4800], dtype=torch.int32, device="cuda")
    weights = [1 + 0.3 * normal(torch, s, "float32", 128) for s in (3, 4)]

    def inputs(seed):
        q, k = normal(torch, seed, "bfloat16", 700, 8, 128), normal(torch, seed + 1, "bfloat16", 700, 2, 128)
        return q, k, normal(torch, seed + 2, "float32", 3, 200_000), torch.arange(3, device="cuda")

    def work(q, k, x, t):
        y = rotate.forward(q, k, *weights)
        back = rotate.backward(*y, q, k, *weights)
        r = score.forward(x, t, 20)
        return (*y, *back, *r, score.backward(r.logp, r.entropy, x, t, r.stats, r.entropy), attend.decode(q[:1], pool, table, lengths))

    ins = [inputs(10), inputs(20)]
    want = [work(*i) for i in ins]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ins]
    got = [[], []]
    for _ in range(20):
        for i, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                got[i].append(work(*ins[i]))
    torch.cuda.synchronize()
    for i in (0, 1):
        assert all(torch.equal(a, b) for run in got[i] for a, b in zip(run, want[i]))
    del got
    graphs, outs = [torch.cuda.CUDAGraph() for _ in ins], []
    for graph, i in zip(graphs, ins):
        with torch.cuda.graph(graph):
            outs.append(work(*i))
    for turn in range(6):
        for out in outs:
            for o in out:
                o.zero_()
        torch.cuda.synchronize()
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        eager = work(*ins[turn % 2])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, want[turn % 2]))
        for i in (0, 1):
            assert all(torch.equal(a, b) for a, b in zip(outs[i], want[i]))


def test_gradients_of_broadcast_operands(torch):
    """Heads and tokens that are one in memory, gradients whose elements have one address, weights that queries and keys share."""
    from paper_2307_05740_amd.logprobs import ArrowLogProbs
    from paper_2307_05740_amd.rotation import ArrowRotation
    rotate, score = ArrowRotation(64), ArrowLogProbs()
    x, w = normal(torch, 1, "float32", 1, 9, 1, 64).requires_grad_(), (1 + 0.2 * normal(torch, 2, "float32", 64)).requires_grad_()
    q, k = rotate(x.expand(3, 9, 4, 64), x.expand(3, 9, 1, 64), w, w)
    (q.sum() + (k * 2).sum()).backward()
    one = x.detach()
    gq, gk = torch.ones(3, 9, 4, 64, device="cuda"), torch.full((3, 9, 1, 64), 2.0, device="cuda")
    dq, dk, dwq, dwk = rotate.backward(gq, gk, one.expand(3, 9, 4, 64).contiguous(), one.expand(3, 9, 1, 64).contiguous(), w.detach(), w.detach())
    torch.testing.assert_close(x.grad, dq.sum((0, 2), keepdim=True) + dk.sum((0, 2), keepdim=True), rtol=2.0 ** -18, atol=2.0 ** -18)     # (fifteen numbers near one, in other orders)
    # the same 108 and 27 terms, in an order that goes by how sequences lie: each sum is off by at most its number of terms times 2^-24 of the sizes' sum, and a term is
    # a normed element times one of a pair of ones, or twos, that is turned
    n = (one.double() / (one.double().square().mean(-1, keepdim=True) + 1e-6).sqrt()).abs().sum((0, 1, 2)) * 2 ** 0.5
    assert bool(((w.grad.double() - (dwq + dwk)).abs() <= 2 * 2.0 ** -24 * (109 * 12 * n + 28 * 3 * 2 * n + 2 * (12 + 6) * n)).all())
    rows = normal(torch, 3, "bfloat16", 7, 50).requires_grad_()
    logp, entropy = score(rows, torch.arange(7, device="cuda"))
    entropy.sum().backward()
    r = score.forward(rows.detach(), torch.arange(7, device="cuda"))
    assert torch.equal(rows.grad, score.backward(None, torch.ones(7, device="cuda"), rows.detach(), torch.arange(7, device="cuda"), r.stats, r.entropy))
    with pytest.raises(RuntimeError):
        score.forward(rows.detach()[:1].expand(7, 50), torch.arange(7, device="cuda"))       # rows that lie upon each other are refused


def test_in_inference_mode(torch):
    from paper_2307_05740_amd.logprobs import ArrowLogProbs
    from paper_2307_05740_amd.rotation import ArrowRotation
    x, q = normal(torch, 1, "bfloat16", 5, 333), normal(torch, 2, "bfloat16", 6, 3, 32)
    with torch.inference_mode():
        r, y = ArrowLogProbs().forward(x, torch.arange(5, device="cuda"), 3), ArrowRotation(32).forward(q, q.clone())
        assert r.logp.is_inference() and y[0].is_inference()
        r.logp.add_(1)
    s, z = ArrowLogProbs().forward(x, torch.arange(5, device="cuda"), 3), ArrowRotation(32).forward(q, q.clone())
    assert torch.equal(r.logp, s.logp + 1) and torch.equal(r.lse, s.lse) and torch.equal(r.top_ids, s.top_ids) and torch.equal(y[0], z[0])


def test_by_the_general_way(torch):
    """Devices without a number, subclasses of tensors and strided targets go by the classes' own checks, to the same results."""
    from paper_2307_05740_amd.logprobs import ArrowLogProbs
    from paper_2307_05740_amd.packed import ArrowPackedAttention
    from paper_2307_05740_amd.pages import ArrowPages
    from paper_2307_05740_amd.rotation import ArrowRotation
    q, k, w = normal(torch, 1, "bfloat16", 2, 30, 4, 64), normal(torch, 2, "bfloat16", 2, 30, 2, 64), normal(torch, 3, "float32", 64)
    n, x = torch.tensor([20, 7], dtype=torch.int32, device="cuda"), normal(torch, 4, "float32", 20, 300)
    t = torch.arange(40, device="cuda")[::2]

    def run(dev):
        r = ArrowRotation(64, device=dev)
        out = [*r.forward(q, k, w, w), *r.backward(q, k, q, k, w, w), *r.backward(q, k, q, k)[:2]]
        p, a = ArrowPages(9, 16, 20, 2, device=dev), ArrowPackedAttention(20, 2, device=dev)
        state = p.state(2, 4)
        slots = p.step(*state, n, 20)
        offsets = torch.tensor([0, 3, 5], dtype=torch.int32, device="cuda")
        out += [slots, p.step(*state, n + 3, 5, offsets), *state]
        assert p.step(*state, n, 0) is None
        pool = a.pool(9, 16, 2, 64)
        a.append(k[0, :20], k[1, :20], pool, slots[0])
        out += [*a.read(pool, slots[0], 64, torch.bfloat16), a.decode(q[:, 0], pool, state[0], n, k=k[:, 3], v=k[:, 4]), pool]
        s = ArrowLogProbs(0.5, device=dev)
        for top in (0, 3):
            o = s.forward(x, t, top)
            out += [y for y in o if y is not None]
        return out + [s.backward(o.logp, o.entropy, x, t, o.stats, o.entropy), s.backward(o.logp, None, x, t, o.stats)]

    assert all(torch.equal(a, b) for a, b in zip(run("cuda:0"), run("cuda")))


def test_classes_refuse(torch):
    """What does not fit is refused by name before anything is started."""
    from paper_2307_05740_amd.logprobs import ArrowLogProbs
    from paper_2307_05740_amd.packed import ArrowPackedAttention
    from paper_2307_05740_amd.pages import ArrowPages
    from paper_2307_05740_amd.rotation import ArrowRotation
    q, k, w = normal(torch, 1, "bfloat16", 30, 4, 64), normal(torch, 2, "bfloat16", 30, 2, 64), normal(torch, 3, "float32", 64)
    r = ArrowRotation(64)
    for args, kw in (((q, k[:29]), {}), ((q[..., :32], k[..., :32]), {}), ((q, k.float()), {}), ((q, k, w), {}), ((q, k, w[:32], w[:32]), {}), ((q, k, w.half(), w.half()), {}),
                     ((q, k), {"positions": torch.arange(29, device="cuda")}), ((q, k), {"positions": torch.arange(30.0, device="cuda")}), ((q, k), {"q_out": q[:3]}),
                     ((q.transpose(1, 2).contiguous().transpose(1, 2), k), {}), ((q.double(), k.double()), {}), ((q.cpu(), k.cpu()), {})):
        with pytest.raises((ValueError, TypeError)):
            r.forward(*args, **kw)
    with pytest.raises(RuntimeError, match="aligned"):
        r.forward(torch.zeros(8 * 4 * 64 + 8, dtype=torch.bfloat16, device="cuda")[1:2049].view(8, 4, 64), k[:8])
    with pytest.raises((ValueError, TypeError)):
        r.backward(q[:29], k, q, k)
    p = ArrowPages(9, 16)
    table, held, free = p.state(2, 4)
    n = torch.zeros(2, dtype=torch.int32, device="cuda")
    for args, kw in (((table, held, free, n.long()), {}), ((table, held[:1], free, n), {}), ((table, held, free[1:], n), {}), ((table.T, held, free, n), {}),
                     ((table, held, free, n), {"tokens": -1}), ((table, held, free, n), {"offsets": n}), ((table, held, free, n), {"slots": torch.zeros(2, 1, device="cuda")})):
        with pytest.raises((ValueError, TypeError)):
            p.step(*args, **kw)
    a = ArrowPackedAttention()
    pool, slots = a.pool(9, 16, 2, 64), torch.zeros(30, dtype=torch.int64, device="cuda")
    for call in (lambda: a.append(k, k, pool, slots.int()), lambda: a.append(k, k[:29], pool, slots), lambda: a.append(k, k, pool.float(), slots), lambda: a.append(q, q, pool, slots),
                 lambda: a.append(k.float(), k.float(), pool, slots), lambda: a.append(k[..., :48], k[..., :48], pool, slots), lambda: a.append(k, k, pool[..., 1:], slots),
                 lambda: a.read(pool, slots, 48, torch.bfloat16), lambda: a.read(pool, slots, 64, torch.float32), lambda: a.read(pool, slots, 64, torch.bfloat16, k=k[:3]),
                 lambda: a.decode(q[:2], pool, table, n, k=k[:2]), lambda: a.decode(q[:2], pool, table.long(), n), lambda: a.decode(q[:3], pool, table, n),
                 lambda: a.decode(q[:2, :3], pool, table, n), lambda: a.decode(q[:2].float(), pool, table, n)):
        with pytest.raises((ValueError, TypeError, RuntimeError)):
            call()
    s, x, t = ArrowLogProbs(), normal(torch, 4, "float32", 20, 30), torch.arange(20, device="cuda")
    o = s.forward(x, t)
    for call in (lambda: s.forward(x, t[:19]), lambda: s.forward(x, t.float()), lambda: s.forward(x.double(), t), lambda: s.forward(x, t, 31), lambda: s.forward(x, t, -1),
                 lambda: s.forward(x.T, t), lambda: s.forward(x, t.cpu()), lambda: s.backward(o.logp[:3], None, x, t, o.stats), lambda: s.backward(o.logp, o.entropy, x, t, o.stats),
                 lambda: s.backward(o.logp, None, x, t, o.lse), lambda: s.backward(o.logp.double(), None, x, t, o.stats), lambda: s.backward(o.logp, None, x, t, o.stats, d_logits=x[:3])):
        with pytest.raises((ValueError, TypeError, RuntimeError)):
            call()
    torch.cuda.synchronize()


def test_the_example(torch):
    spec = importlib.util.spec_from_file_location("stream_model", os.path.join(ROOT, "examples", "stream_model.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    first, last, off = example.main(["--steps", "5", "--tokens", "150", "--positions", "--entropy", "0.01", "--bits", "4"])
    assert all(math.isfinite(x) for x in (first, last, off))
    # over the same tokens, and weights, a cache in 16 bits and one in 4 differ by what the latter rounds: both run, page by page
    model = example.StreamModel(positions=True)
    ids, _ = example.serve(model, 120, bits=16)
    again, _ = example.serve(model, 120, bits=4)
    assert ids.shape == again.shape == (3, 120)


def example_of():
    spec = importlib.util.spec_from_file_location("stream_model", os.path.join(ROOT, "examples", "stream_model.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    return example


def test_the_example_hands_out_pages_without_waiting(torch):
    """Nothing comes back to the host for a token."""
    example = example_of()
    caches = example.PackedCaches(example.StreamModel(positions=True), 3, columns=10, pages=20)
    caches.grow(3)
    torch.cuda.set_sync_debug_mode("error")
    try:
        for length in (40, 41, 42, 60):
            caches.grow(length)
    finally:
        torch.cuda.set_sync_debug_mode("default")
    assert caches.held.tolist() == [60] * 3 and caches.slots.shape == (3 * 18,)


def test_the_example_has_the_same_cache_in_4_bits(torch):
    """A server's two caches, the one in 16 bits of what the one in 4 keeps, page by page as they are given back and used again: attention over either is within what rounding does."""
    example = example_of()
    model = example.StreamModel()
    args = dict(batch=3, columns=12, pages=3 * (model.attend.window // 16 + 4))
    wide, narrow = example.Caches(model, **args), example.PackedCaches(model, **args)
    for caches in (wide, narrow):
        caches.grow(40)
    rounded = lambda x: oracle.packed(x).to(x.dtype)   # noqa: E731
    for layer in range(2):
        k, v = (normal(torch, 10 * layer + i, "bfloat16", 3, 40, model.kv_heads, model.dim) for i in range(2))
        wide.append(layer, rounded(k), rounded(v))
        narrow.append(layer, k, v)
    for length in range(41, 180):
        for caches in (wide, narrow):
            caches.grow(length)
        for layer in range(2):
            q, k, v = (normal(torch, 1000 * layer + 10 * length + i, "bfloat16", 3, heads, model.dim) for i, heads in enumerate((model.heads, model.kv_heads, model.kv_heads)))
            got, want = narrow.decode(layer, q, k, v), wide.decode(layer, q, rounded(k), rounded(v))
            # each is off by 2 u of sum p |v| at most, and by less than 2^-16 of it for scores and sums; no value is larger than 6
            assert bool(((got.double() - want.double()).abs() <= 6 * (4 * 2.0 ** -8 + 2.0 ** -15)).all()), (length, layer)
