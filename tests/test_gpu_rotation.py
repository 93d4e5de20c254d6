"""Head norms with the rotation by position, and their gradients, against the 64-bit oracle; the bounds are the oracle's."""
import math

import pytest

from oracle import operators_oracle as oracle

pytestmark = pytest.mark.gpu

TYPES = ("float32", "bfloat16", "float16")


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible: these tests need a real MI355X")
    return torch


@pytest.fixture(scope="module")
def Rotation(torch):
    from paper_2307_05740_amd.rotation import ArrowRotation
    return ArrowRotation


def normal(torch, seed, dtype, *shape, by=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * by).to(getattr(torch, dtype)).cuda()


def within(torch, name, got, want, bound):
    off = (got.double() - want).abs()
    assert bool((off <= bound).all()), (name, float((off / bound.clamp(min=1e-300)).max()), int((~(off <= bound)).sum()), off.numel())


def positions_of(torch, q, positions, shift):
    if positions is None:
        positions = torch.arange(q.shape[-3], device=q.device).expand(q.shape[:-2])
    return positions.long() + shift


def check(torch, op, q, k, wq, wk, positions=None, shift=0, gq=None, gk=None):
    """Both directions; outputs come into tensors of NaN."""
    p = positions_of(torch, q, positions, shift)
    turns = op.turns.cpu().cuda()
    yq, yk = op.forward(q, k, wq, wk, positions, shift, torch.full(q.shape, math.nan, dtype=q.dtype, device="cuda"), torch.full(k.shape, math.nan, dtype=q.dtype, device="cuda"))
    nan = [torch.full(t.shape, math.nan, dtype=q.dtype, device="cuda") for t in (q, k)]
    grads = op.backward(gq, gk, q, k, wq, wk, positions, shift, *nan) if gq is not None else (None,) * 4
    for name, x, w, y, dy, dx, dw in (("q", q, wq, yq, gq, grads[0], grads[2]), ("k", k, wk, yk, gk, grads[1], grads[3])):
        want, bound = oracle.rotation(x, w, p, turns, op.rotary, op.interleaved, op.eps, dy)
        within(torch, name, y, want["y"], bound["y"])
        if dy is not None:
            within(torch, "d" + name, dx, want["dx"], bound["dx"])
            if w is None:
                assert dw is None
            else:
                assert dw.dtype == w.dtype
                within(torch, "dw" + name, dw, want["dw"], bound["dw"] + oracle.UNIT[w.dtype] * want["dw"].abs())
    return yq, yk


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim,rotary", [(8, 0), (16, 16), (24, 16), (32, 32), (64, 64), (64, 32), (72, 48), (80, 80), (96, 96), (104, 16), (128, 128), (128, 64), (136, 128),
                                        (248, 240), (256, 256)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_sizes_of_heads(torch, Rotation, dtype, dim, rotary, interleaved):
    op = Rotation(dim, rotary=rotary, interleaved=interleaved)
    q, gq = (normal(torch, s, dtype, 2, 9, 3, dim) for s in (1, 2))
    k, gk = (normal(torch, s, dtype, 2, 9, 1, dim) for s in (3, 4))
    wq, wk = (1 + 0.3 * normal(torch, s, "float32", dim) for s in (5, 6))
    check(torch, op, q, k, wq, wk, gq=gq, gk=gk)
    check(torch, op, q, k, wq.to(q.dtype), wk.to(q.dtype), gq=gq, gk=gk)
    check(torch, op, q, k, None, None, gq=gq, gk=gk)


@pytest.mark.parametrize("tokens", [1, 2, 7, 8, 9, 63, 1023, 1024, 1025, 2048, 8191, 8192, 8197, 20000])
@pytest.mark.parametrize("heads,kv", [(1, 1), (5, 1), (8, 2)])
def test_numbers_of_tokens(torch, Rotation, tokens, heads, kv):
    """Around the numbers from which workgroups take more tokens at a time, and from which they go round."""
    dtype = TYPES[1 + tokens % 2]
    op = Rotation(64)
    q, gq = (normal(torch, s, dtype, tokens, heads, 64) for s in (1, 2))
    k, gk = (normal(torch, s, dtype, tokens, kv, 64) for s in (3, 4))
    wq, wk = (1 + 0.3 * normal(torch, s, "float32", 64) for s in (5, 6))
    check(torch, op, q, k, wq, wk, gq=gq, gk=gk)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("heads,kv,dim,rotary", [(1, 1, 256, 256), (2, 1, 128, 128), (3, 1, 96, 96), (6, 3, 80, 32), (16, 1, 8, 0), (70, 2, 32, 32)])
@pytest.mark.parametrize("batch,tokens", [(3, 1031), (40, 97), (2, 4000)])
def test_tokens_of_workgroups(torch, Rotation, interleaved, heads, kv, dim, rotary, batch, tokens):
    """Many tokens of a few heads and few ones of many, in sequences that follow each other or lie apart, so that they end inside what a workgroup has at a time."""
    op = Rotation(dim, rotary=rotary, interleaved=interleaved)
    for room in (0, 1):
        (q, gq), (k, gk) = ([normal(torch, s, "bfloat16", batch, tokens + room, h, dim)[:, :tokens] for s in seeds] for h, seeds in ((heads, (1, 2)), (kv, (3, 4))))
        wq, wk = (1 + 0.3 * normal(torch, s, "float32", dim) for s in (5, 6))
        check(torch, op, q, k, wq, wk, gq=gq, gk=gk)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["int32", "int64"])
def test_positions(torch, Rotation, dtype, kind):
    """Given ones, far and negative ones, and lengths that count the new token."""
    g = torch.Generator().manual_seed(1)
    most = 2**31 - 1 if kind == "int32" else 2**40
    p = torch.randint(-most, most, (5, 3), generator=g)
    p[0] = torch.tensor([0, 1, most])
    p = p.to(getattr(torch, kind)).cuda()
    q, k = normal(torch, 2, dtype, 5, 3, 4, 128), normal(torch, 3, dtype, 5, 3, 2, 128)
    gq, gk = normal(torch, 4, dtype, 5, 3, 4, 128), normal(torch, 5, dtype, 5, 3, 2, 128)
    for shift in (0, -1, 12345678901):
        check(torch, Rotation(128), q, k, None, None, p, shift, gq, gk)
    check(torch, Rotation(128, base=500000.0), q[:, 0], k[:, 0], None, None, p[:, 0].contiguous(), -1, gq[:, 0], gk[:, 0])
    # (pairs that lie side by side: a lane has the same elements with and without a rotation, and adds their squares in the same order)
    y = Rotation(128, interleaved=True).forward(q, k, positions=torch.zeros_like(p))[0]
    z = Rotation(128, rotary=0).forward(q, k)[0]
    assert torch.equal(y, z)


def test_given_frequencies(torch, Rotation):
    f = [0.5 ** i for i in range(16)]
    q, k = normal(torch, 2, "float32", 30, 4, 40), normal(torch, 3, "float32", 30, 2, 40)
    op = Rotation(40, rotary=32, frequencies=f)
    check(torch, op, q, k, None, None)
    assert torch.equal(op.forward(q, k)[0], Rotation(40, rotary=32, frequencies=torch.tensor(f, device="cuda")).forward(q, k)[0])


@pytest.mark.parametrize("dtype", TYPES)
def test_views_and_in_place(torch, Rotation, dtype):
    """q, k and v out of one projection, heads before tokens, rows far apart, and results over their operands."""
    op = Rotation(64)
    both = normal(torch, 1, dtype, 2, 33, 4 + 2 + 2, 64)
    q, k, v = both.split((4, 2, 2), -2)
    gq, gk = normal(torch, 2, dtype, 2, 33, 4, 64), normal(torch, 3, dtype, 2, 33, 2, 64)
    wq, wk = (1 + 0.3 * normal(torch, s, "float32", 64) for s in (5, 6))
    yq, yk = check(torch, op, q, k, wq, wk, gq=gq, gk=gk)
    turned = normal(torch, 1, dtype, 2, 33, 8, 64).transpose(1, 2).contiguous().transpose(1, 2)
    check(torch, op, turned[:, :, :4], turned[:, :, 4:6], wq, wk, gq=gq, gk=gk)
    want = op.backward(gq, gk, q, k, wq, wk)
    mine = [gq.clone(), gk.clone()]
    got = op.backward(*mine, q, k, wq, wk, dq=mine[0], dk=mine[1])
    assert all(torch.equal(a, b) for a, b in zip(want, got)) and got[0] is mine[0]
    keep = v.clone()
    op.forward(q, k, wq, wk, q_out=q, k_out=k)
    assert torch.equal(q, yq) and torch.equal(k, yk) and torch.equal(v, keep)


def test_values_out_of_the_ordinary(torch, Rotation):
    """Rows of zeros, of very large and very small elements; what is not finite stays in its own head."""
    op = Rotation(64, eps=1e-6)
    q = normal(torch, 1, "float32", 6, 3, 64)
    q[0, 0] = 0
    q[1, 1] *= 1e15
    q[2, 2] *= 1e-15
    k = normal(torch, 2, "float32", 6, 1, 64)
    check(torch, op, q, k, None, None, gq=normal(torch, 3, "float32", 6, 3, 64), gk=normal(torch, 4, "float32", 6, 1, 64))
    want = op.forward(q, k)[0]
    q[3, 1, 5], q[4, 0, 63] = math.nan, math.inf
    got = op.forward(q, k)[0]
    other = torch.ones(6, 3, dtype=torch.bool, device="cuda")
    other[3, 1] = other[4, 0] = False
    assert torch.equal(got[other], want[other]) and bool(got[3, 1].isnan().all()) and bool(got[4, 0].isnan().any())


def test_nothing_to_do(torch, Rotation):
    op = Rotation(64)
    for lead in ((0,), (0, 5), (3, 0)):
        q, k = normal(torch, 1, "bfloat16", *lead, 4, 64), normal(torch, 2, "bfloat16", *lead, 1, 64)
        w = torch.ones(64, device="cuda")
        assert op.forward(q, k, w, w)[0].shape == q.shape
        dq, dk, dwq, dwk = op.backward(q, k, q, k, w, w)
        assert dq.shape == q.shape and not bool(dwq.any()) and not bool(dwk.any())


def test_gradient_against_differences(torch, Rotation):
    """Along one direction, in 32 bits: (f(x + t E) - f(x - t E)) / 2 t is off by t^2 times the third derivative, here below 1e-4 of it, and 2^-22 / t by rounding."""
    op = Rotation(32)
    q, e, g = (normal(torch, s, "float32", 40, 2, 32) for s in (1, 2, 3))
    k, z = normal(torch, 4, "float32", 40, 1, 32), torch.zeros(40, 1, 32, device="cuda")
    w = 1 + 0.3 * normal(torch, 5, "float32", 32)
    t = 2.0 ** -7
    f = lambda x: float((op.forward(x, k, w, w)[0].double() * g.double()).sum())   # noqa: E731
    left = (f(q + t * e) - f(q - t * e)) / (2 * t)
    right = float((op.backward(g, z, q, k, w, w)[0].double() * e.double()).sum())
    size = float((op.backward(g, z, q, k, w, w)[0].double() * e.double()).abs().sum())
    assert abs(left - right) <= (16 * t * t + 2.0 ** -22 / t) * size, (left, right, size)


def test_autograd(torch, Rotation):
    op = Rotation(64)
    both = normal(torch, 1, "bfloat16", 2, 20, 6, 64).requires_grad_()
    wq, wk = (torch.nn.Parameter(1 + 0.3 * normal(torch, s, "float32", 64)) for s in (5, 6))
    gq, gk = normal(torch, 2, "bfloat16", 2, 20, 4, 64), normal(torch, 3, "bfloat16", 2, 20, 2, 64)
    q, k = both.split((4, 2), -2)
    yq, yk = op(q, k, wq, wk)
    torch.autograd.backward((yq, yk), (gq, gk))
    dq, dk, dwq, dwk = op.backward(gq, gk, q.detach(), k.detach(), wq.detach(), wk.detach())
    assert torch.equal(both.grad, torch.cat((dq, dk), 2)) and torch.equal(wq.grad, dwq) and torch.equal(wk.grad, dwk)
    both.grad = None
    q, k = both.split((4, 2), -2)
    op(q, k)[0].sum().backward()                                  # a gradient whose elements have one address, and none for k
    want = op.backward(torch.ones_like(gq), torch.zeros_like(gk), q.detach(), k.detach())
    assert torch.equal(both.grad[:, :, :4], want[0]) and not bool(both.grad[:, :, 4:].any())


def test_the_same_every_time_and_captured(torch, Rotation):
    op = Rotation(128)
    q, gq = (normal(torch, s, "bfloat16", 3000, 8, 128) for s in (1, 2))
    k, gk = (normal(torch, s, "bfloat16", 3000, 2, 128) for s in (3, 4))
    w = torch.ones(128, device="cuda")
    lengths = torch.arange(1, 3001, device="cuda", dtype=torch.int32)
    run = lambda: (*op.forward(q, k, w, w, lengths, -1), *op.backward(gq, gk, q, k, w, w, lengths, -1))   # noqa: E731
    first = run()
    assert all(torch.equal(a, b) for _ in range(3) for a, b in zip(first, run()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    for seed in (7, 8, 9):
        q.copy_(normal(torch, seed, "bfloat16", 3000, 8, 128))
        lengths += 1000
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, run()))


def test_offsets_beyond_32_bits(torch, Rotation):
    """Operands of 6 GB: places in bytes and elements beyond 2^32 and 2^31."""
    tokens = 370_000
    op = Rotation(256)
    q = torch.empty(tokens, 32, 256, dtype=torch.bfloat16, device="cuda").normal_()
    k = torch.empty(tokens, 1, 256, dtype=torch.bfloat16, device="cuda").normal_()
    y, _ = op.forward(q, k)
    dq = op.backward(y, k, q, k)[0]
    for part in (slice(0, 3), slice(tokens // 2, tokens // 2 + 3), slice(tokens - 3, tokens)):
        p = torch.arange(tokens, device="cuda")[part]
        want, bound = oracle.rotation(q[part], None, p, op.turns, 256, dy=y[part])
        within(torch, "y", y[part], want["y"], bound["y"])
        within(torch, "dx", dq[part], want["dx"], bound["dx"])


def test_views_of_one_tensor(torch, Rotation):
    """What is written may lie between what is read, element by element of the outer dimensions: projections with all heads, heads in turn, results in one tensor."""
    op, g = Rotation(64), torch.Generator().manual_seed(1)
    wq, wk = (torch.rand(64, generator=g).cuda() + 0.5 for _ in range(2))
    for batch, tokens in ((3, 5), (1, 7), (4, 1), (1, 1)):
        x = torch.randn(batch, tokens, 6, 64, generator=g).bfloat16().cuda()
        d = torch.randn(batch, tokens, 6, 64, generator=g).bfloat16().cuda()
        for split in (lambda t: (t[:, :, :4], t[:, :, 4:]), lambda t: (t[:, :, ::2], t[:, :, 1::2]), lambda t: (t[:, :, 1:3], t[:, :, 5:])):
            q, k = split(x)
            want = op.forward(q.contiguous(), k.contiguous(), wq, wk)
            grads = op.backward(split(d)[0].contiguous(), split(d)[1].contiguous(), q.contiguous(), k.contiguous(), wq, wk)
            out, dx = torch.zeros_like(x), torch.zeros_like(x)
            got = op.forward(q, k, wq, wk, q_out=split(out)[0], k_out=split(out)[1])
            back = op.backward(*split(d), q, k, wq, wk, dq=split(dx)[0], dk=split(dx)[1])
            assert all(torch.equal(a, b) for a, b in zip((*got, *back[:2]), (*want, *grads[:2])))
            both, again = x.clone(), d.clone()
            op.forward(*split(both), wq, wk, q_out=split(both)[0], k_out=split(both)[1])
            op.backward(*split(again), q, k, wq, wk, dq=split(again)[0], dk=split(again)[1])
            assert all(torch.equal(a, b) for a, b in zip((*split(both), *split(again)), (*want, *grads[:2])))
            rest = [h for h in range(6) if not any(torch.equal(x[:, :, h], s[:, :, i]) for s in (q, k) for i in range(s.shape[2]))]
            assert torch.equal(both[:, :, rest], x[:, :, rest]) and torch.equal(again[:, :, rest], d[:, :, rest])
            # queries and their results in the two halves of every row of one tensor
            pair = torch.cat([q, torch.zeros_like(q)], 2)
            op.forward(pair[:, :, :q.shape[2]], k, wq, wk, q_out=pair[:, :, q.shape[2]:])
            assert torch.equal(pair[:, :, q.shape[2]:], want[0]) and torch.equal(pair[:, :, :q.shape[2]], q)
