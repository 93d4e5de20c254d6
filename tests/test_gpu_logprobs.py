"""Log probabilities, entropies, most likely tokens and the gradient against the 64-bit oracle; the bounds are the oracle's."""
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
def LogProbs(torch):
    from paper_2307_05740_amd.logprobs import ArrowLogProbs
    return ArrowLogProbs


def normal(torch, seed, dtype, *shape, by=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * by).to(getattr(torch, dtype)).cuda()


def targets_of(torch, seed, rows, n):
    g = torch.Generator().manual_seed(seed)
    t = torch.randint(0, n, (rows,), generator=g)
    t[::5] = -1
    t[3::7] = n
    return t.cuda()


def within(torch, name, got, want, bound):
    got = got.double()
    ok = (got == want) | (got.isnan() & want.isnan()) | ((got - want).abs() <= bound)
    assert bool(ok.all()), (name, int((~ok).sum()), ok.numel(), got[~ok][:3], want[~ok][:3], bound.expand_as(want)[~ok][:3])


def check(torch, op, x, t, top=0, seed=9, grads=True):
    rows = x.shape[0]
    g = normal(torch, seed, "float32", rows) if grads else None
    h = normal(torch, seed + 1, "float32", rows, by=0.1) if grads else None
    want, bound = oracle.logprobs(x, t, op.scale, top, g, h)
    for of in (t, t.int()):
        r = op.forward(x, of, top)
        for name in ("logp", "entropy", "lse"):
            within(torch, name, getattr(r, name), want[name], bound[name])
        if top:
            assert torch.equal(r.top_ids, want["top_ids"]), (r.top_ids[0], want["top_ids"][0])
            within(torch, "top_logp", r.top_logp, want["top_logp"], bound["top_logp"])
        else:
            assert r.top_logp is None and r.top_ids is None
        if grads:
            d = op.backward(g, h, x, of, r.stats, r.entropy, torch.full(x.shape, math.nan, dtype=x.dtype, device="cuda"))
            within(torch, "d_logits", d, want["d_logits"], bound["d_logits"])
    return r


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 2, 3, 7, 8, 9, 15, 64, 100, 500, 2047, 2048, 2049, 4100, 8191, 8193, 16400, 32768, 32776, 50257, 70001, 128001])
def test_vocabularies(torch, LogProbs, dtype, n):
    """One token to several parts of a row, odd sizes: rows begin at any address."""
    rows = 7
    x, t = normal(torch, n, dtype, rows, n, by=3.0), targets_of(torch, 2, rows, n)
    check(torch, LogProbs(), x, t, min(n, 5))
    check(torch, LogProbs(0.7), x, t)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("top", [1, 2, 5, 20, 31, 32])
@pytest.mark.parametrize("n", [32, 33, 200, 1000, 5000, 32000, 100003])
def test_numbers_of_top_tokens(torch, LogProbs, dtype, top, n):
    """In types of few bits many logits are alike: the lower index comes first."""
    x, t = normal(torch, n, dtype, 5, n), targets_of(torch, 2, 5, n)
    check(torch, LogProbs(1.3), x, t, top, grads=False)


@pytest.mark.parametrize("rows,n", [(1, 5000), (1, 200001), (2, 32000), (3, 129), (64, 10007), (255, 1024), (600, 3000), (1500, 777), (20000, 33)])
def test_numbers_of_rows(torch, LogProbs, rows, n):
    x, t = normal(torch, n, "bfloat16", rows, n, by=2.0), targets_of(torch, 2, rows, n)
    check(torch, LogProbs(), x, t, 3)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pieces,rows", [(2, 70), (23, 9), (24, 9), (28, 33), (64, 70), (65, 70), (128, 9), (129, 70), (256, 3), (512, 5), (513, 5), (768, 4097), (769, 4097), (768, 30), (1024, 9), (1025, 9), (4096, 3), (4097, 3), (6144, 3), (6145, 3), (8192, 3), (8193, 2), (12287, 2), (12288, 2), (12289, 2), (30000, 2)])
def test_edges_of_the_kernels(torch, LogProbs, dtype, pieces, rows):
    """Rows of that many pieces of 16 bytes, less one element, and of one element more, with and without most likely tokens."""
    each = 128 // torch.finfo(getattr(torch, dtype)).bits
    for n in ((pieces - 1) * each, (pieces - 1) * each + 1):
        x, t = normal(torch, n, dtype, rows, n, by=2.0), targets_of(torch, 2, rows, n)
        for top in (0, 3, 8, 9, 16, 17, 20, 21, 32) if pieces < 200 else (0, 20) if rows < 4000 else (0, 3):
            check(torch, LogProbs(1.1), x, t, min(n, top), grads=False)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [9, 16, 31, 32, 33, 63, 64, 65, 91, 92, 93, 127, 128, 129, 183, 184, 185, 191, 192, 193, 255, 256, 257, 370, 376, 400])
def test_few_logits_and_many_tokens(torch, LogProbs, dtype, n):
    """Rows of which a lane has single logits, and of nearly as many that it has pieces of: any address, logits that are alike, masked ones."""
    x = normal(torch, n, dtype, 37, n, by=2.0)
    x[1::4] = x[1::4].round()
    x[2, n // 2:], x[3] = -math.inf, 0
    for top in (1, 8, 9, 12, 20, 32):
        check(torch, LogProbs(0.8), x, targets_of(torch, 2, 37, n), min(n, top), grads=False)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [300_000, 2_200_000])
def test_many_parts(torch, LogProbs, dtype, n):
    """More keys than the workgroup that joins parts holds; all logits alike; the largest ones in one part, and as one lane's keys."""
    x = torch.zeros(4, n, device="cuda")
    x[0] = torch.randn(n, generator=torch.Generator().manual_seed(n)).cuda()
    x[1, n // 2:n // 2 + 40] = 1.0
    x[2, ::n // 31] = 2.0
    x[3] = x[0].abs().round()
    x = x.to(getattr(torch, dtype))
    for top in (1, 20, 32):
        check(torch, LogProbs(), x, targets_of(torch, 2, 4, n), top, grads=False)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [40, 3000, 40000])
def test_order_of_logits_that_are_alike(torch, LogProbs, dtype, n):
    """All alike; few different ones; in falling and rising order; all large ones where one lane of a workgroup has them."""
    rows = []
    g = torch.Generator().manual_seed(1)
    rows.append(torch.zeros(n))
    rows.append(torch.where(torch.arange(n) % 2 == 0, 0.0, -0.0))
    rows.append(torch.randint(0, 3, (n,), generator=g).float())
    rows.append(-torch.arange(n).float() / 64)
    rows.append(torch.arange(n).float() / 64)
    rows.append(torch.where(torch.arange(n) % 2048 < 8, 1.0, 0.0) + torch.rand(n, generator=g) / 4)
    rows.append(torch.where(torch.arange(n) % 256 == 3, 5.0, -5.0))
    x = torch.stack(rows).to(getattr(torch, dtype)).cuda()
    for top in (1, 8, 32):
        check(torch, LogProbs(), x, targets_of(torch, 2, len(rows), n), top, grads=False)


@pytest.mark.parametrize("n", [40, 40000])
def test_more_keys_than_a_list_has_room_for(torch, LogProbs, n):
    """A wavefront's first lanes have one large logit each, and one lane of the others all of the largest: thousands lie beyond the border."""
    x = torch.zeros(3, n)
    i = torch.arange(n)
    x[:, i % 2048 >= 2040] = 1.0 + torch.rand(3, int((i % 2048 >= 2040).sum()), generator=torch.Generator().manual_seed(1))
    x[1] = torch.where(i // 8 % 256 == 255, 2.0, x[1])
    x[2] = torch.where(i // 8 % 256 < 8, 2.0, 0.0)
    for dtype in TYPES:
        y = x.to(getattr(torch, dtype)).cuda()
        for top in (8, 32):
            check(torch, LogProbs(), y, targets_of(torch, 2, 3, n), top, grads=False)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [300, 500, 1000, 1800, 4000, 10000, 40000])
@pytest.mark.parametrize("rows", [2, 600])
def test_large_logits_in_few_lanes(torch, LogProbs, dtype, n, rows):
    """One lane less than there are tokens on top has all the large logits, of 16, 64 or 256: far more than there is room for reach the border."""
    each = 128 // torch.finfo(getattr(torch, dtype)).bits
    piece = torch.arange(n) // each
    for top in (2, 8, 32):
        x = torch.rand(rows, n, generator=torch.Generator().manual_seed(top))
        for row, lanes in enumerate((16, 64, 256)):
            x[row::3, piece % lanes < top - 1] += 2.0
        y = x.to(getattr(torch, dtype)).cuda()
        check(torch, LogProbs(), y, targets_of(torch, 2, rows, n), top, grads=False)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [1, 3, 4, 5, 15, 16, 17, 511, 512, 513])
@pytest.mark.parametrize("n", [5, 248, 256, 263, 400, 505, 511, 520, 1030, 2040, 4080, 4090])
def test_short_rows(torch, LogProbs, dtype, rows, n):
    """Several rows to a wavefront, or one; numbers of rows that leave places empty; a row does not depend on its neighbours."""
    x, t = normal(torch, n, dtype, rows, n, by=2.0), targets_of(torch, 2, rows, n)
    x[rows // 2, n // 2:] = -math.inf
    r = check(torch, LogProbs(0.9), x, t, 4)
    y = normal(torch, n + 1, dtype, rows, n)
    y[rows - 1], y[::3, n // 3], y[::3, 0] = x[rows - 1], -math.inf, x[::3, 0]
    y[rows - 1] = x[rows - 1]
    again = LogProbs(0.9).forward(y, t, 4)
    assert all(torch.equal(a[rows - 1], b[rows - 1]) for a, b in zip(again, r))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [50, 33000])
def test_masked_and_odd_logits(torch, LogProbs, dtype, n):
    """-infinity and the type's lowest value as masks, of a few tokens, all but a few, and all; infinities and NaN; targets among them."""
    low = torch.finfo(getattr(torch, dtype)).min
    x = normal(torch, 1, dtype, 12, n, by=3.0)
    x[0, ::3] = -math.inf
    x[1, 5:] = -math.inf
    x[2] = -math.inf
    x[3, ::3] = low
    x[4, 5:] = low
    x[5] = low
    x[6, n // 2] = math.nan
    x[7, n // 3] = math.inf
    x[8] = math.nan
    x[9, 1:] = -math.inf
    x[10, :] = -math.inf
    x[10, n - 1] = low
    x[11] = 0
    t = torch.tensor([0, 4, 7, 3, n - 1, 9, 1, n // 3, 2, 0, n - 1, -1], device="cuda")
    for top in (0, 7, 32):
        check(torch, LogProbs(), x, t, top)
    check(torch, LogProbs(), x[:, :49], t.clamp(max=48), 32)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [30, 100, 700, 3001, 40000])
def test_order_of_the_smallest_numbers(torch, LogProbs, dtype, n):
    """Logits below the type's normal numbers, of either sign, among zeros: none of them is taken for a zero."""
    least = torch.finfo(getattr(torch, dtype)).smallest_normal * torch.finfo(getattr(torch, dtype)).eps
    steps = torch.randint(-60, 61, (4, n), generator=torch.Generator().manual_seed(n)).double()
    steps[1] = steps[1].clamp(max=0)
    steps[2, 3:] = 0
    x = (steps * least).to(getattr(torch, dtype)).cuda()
    assert bool((x.double().cpu() == steps * least).all())
    for top in (3, 9, 30):
        check(torch, LogProbs(), x, targets_of(torch, 2, 4, n), top, grads=False)


def test_large_logits(torch, LogProbs):
    """Differences count, whatever the size of the logits."""
    x = normal(torch, 1, "float32", 6, 3000) + torch.tensor([0.0, 1e3, -1e3, 1e5, 1e30, -3e38], device="cuda")[:, None]
    check(torch, LogProbs(), x, targets_of(torch, 2, 6, 3000), 9)


@pytest.mark.parametrize("dtype", TYPES)
def test_strides_shapes_and_in_place(torch, LogProbs, dtype):
    op = LogProbs()
    big = normal(torch, 1, dtype, 24, 1000)
    x = big[:, 3:504]                                             # rows at odd addresses, of odd length
    t = targets_of(torch, 2, 24, 501)
    r = check(torch, op, x, t, 4)
    shaped = x.contiguous().view(2, 3, 4, 501)
    s = op.forward(shaped, t.view(2, 3, 4), 4)
    assert s.logp.shape == (2, 3, 4) and s.top_ids.shape == (2, 3, 4, 4) and torch.equal(s.top_ids.view(24, 4), r.top_ids)
    g = normal(torch, 3, "float32", 24)
    want = op.backward(g, None, x, t, r.stats)
    keep = big.clone()
    got = op.backward(g, None, x, t, r.stats, d_logits=x)
    assert torch.equal(got, want) and torch.equal(big[:, :3], keep[:, :3]) and torch.equal(big[:, 504:], keep[:, 504:])
    other = torch.zeros(24, 600, dtype=x.dtype, device="cuda")
    x = keep[:, 3:504]
    op.backward(g, None, x, t, r.stats, d_logits=other[:, 5:506])  # rows that lie otherwise than the logits'
    assert torch.equal(other[:, 5:506], want) and not bool(other[:, :5].any()) and not bool(other[:, 506:].any())
    one = op.forward(x[0], t[0])
    assert one.logp.shape == () and torch.equal(one.lse, r.lse[0])


def test_gradients_of_one_output(torch, LogProbs):
    op, x, t = LogProbs(), normal(torch, 1, "float32", 9, 300), targets_of(torch, 2, 9, 300)
    r = op.forward(x, t)
    g = normal(torch, 3, "float32", 9)
    for a, b in ((g, None), (None, g), (None, None)):
        want, bound = oracle.logprobs(x, t, 1.0, 0, a if a is not None else torch.zeros_like(g), b if b is not None else torch.zeros_like(g))
        within(torch, "d_logits", op.backward(a, b, x, t, r.stats, r.entropy if b is not None else None), want["d_logits"], bound["d_logits"])


def test_gradient_against_differences(torch, LogProbs):
    """Along one direction: off by t^2 times third derivatives, which are below 6 |E|^3 here, and by rounding of 2^-21 / t."""
    op, x, e, t = LogProbs(0.8), normal(torch, 1, "float32", 20, 50), normal(torch, 2, "float32", 20, 50), targets_of(torch, 2, 20, 50)
    g, h = normal(torch, 3, "float32", 20), normal(torch, 4, "float32", 20)

    def f(y):
        r = op.forward(y, t)
        return float((r.logp.double() * g + r.entropy.double() * h).sum())

    step = 2.0 ** -6
    r = op.forward(x, t)
    left = (f(x + step * e) - f(x - step * e)) / (2 * step)
    right = float((op.backward(g, h, x, t, r.stats, r.entropy).double() * e.double()).sum())
    room = float((g.abs() + h.abs()).sum()) * (6 * step * step * float(e.abs().max()) ** 3 + 2.0 ** -21 / step)
    assert abs(left - right) <= room, (left, right, room)


def test_autograd_and_nothing_to_do(torch, LogProbs):
    op, t = LogProbs(), targets_of(torch, 2, 8, 77)
    x = normal(torch, 1, "bfloat16", 8, 77).requires_grad_()
    logp, entropy = op(x, t)
    (-logp.sum() - 0.1 * entropy.sum()).backward()
    r = op.forward(x.detach(), t)
    want = op.backward(torch.full_like(logp, -1.0), torch.full_like(logp, -0.1), x.detach(), t, r.stats, r.entropy)
    assert torch.equal(x.grad, want)
    x.grad = None
    op(x, t)[0].mean().backward()                                 # a gradient whose elements have one address
    assert torch.equal(x.grad, op.backward(torch.full_like(logp, 1 / 8), None, x.detach(), t, r.stats))
    empty = op.forward(torch.zeros(0, 9, device="cuda"), torch.zeros(0, dtype=torch.int64, device="cuda"), 3)
    assert empty.logp.shape == (0,) and empty.top_ids.shape == (0, 3)


def test_the_same_every_time_and_captured(torch, LogProbs):
    op = LogProbs()
    x, t = normal(torch, 1, "bfloat16", 40, 50257, by=2.0), targets_of(torch, 2, 40, 50257)
    g = normal(torch, 3, "float32", 40)

    def run():
        r = op.forward(x, t, 20)
        return (*r, op.backward(g, g, x, t, r.stats, r.entropy))

    first = run()
    assert all(torch.equal(a, b) for _ in range(3) for a, b in zip(first, run()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    for seed in (5, 6, 7):
        x.copy_(normal(torch, seed, "bfloat16", 40, 50257))
        t.copy_(targets_of(torch, seed, 40, 50257))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, run()))


def test_offsets_beyond_32_bits(torch, LogProbs):
    """Logits of 9 GB: places in bytes and elements beyond 2^32 and 2^31."""
    rows, n = 130_001, 33_001
    x = torch.empty(rows, n, dtype=torch.bfloat16, device="cuda").normal_()
    t = torch.randint(0, n, (rows,), device="cuda")
    op = LogProbs()
    r = op.forward(x, t, 2)
    g = torch.ones(rows, device="cuda")
    at = torch.tensor([0, 1, rows // 2, rows - 2, rows - 1], device="cuda")
    want, bound = oracle.logprobs(x[at], t[at], 1.0, 2, g[at], None)
    within(torch, "logp", r.logp[at], want["logp"], bound["logp"])
    assert torch.equal(r.top_ids[at], want["top_ids"])
    d = op.backward(g, None, x, t, r.stats, d_logits=x)
    within(torch, "d_logits", d[at], want["d_logits"], bound["d_logits"])


@pytest.mark.parametrize("dtype,n,low", [("bfloat16", 1 << 20, -16.75), ("float16", 1 << 20, -16.75), ("float32", 1 << 19, -16.7), ("float16", 200_003, -16.75)])
def test_long_sums_of_small_terms(torch, LogProbs, dtype, n, low):
    """Many rows of many logits that are each less than half a step of a sum of 32 bits which begins with 1: one after the other they would all be lost."""
    op, rows = LogProbs(), 512
    x = torch.full((rows, n), low, dtype=getattr(torch, dtype), device="cuda")
    each = 16 // x.element_size()
    x[:, :256 * each:each] = 0.0
    x += torch.arange(rows, device="cuda", dtype=x.dtype)[:, None] % 4
    t = torch.arange(rows, device="cuda") % n
    for part, masked in ((slice(0, None), False), (slice(0, 3), False), (slice(0, None), True)):
        if masked:                          # (a token of every lane that cannot be, for which it adds up everything again)
            x[:, 256 * each + 1:512 * each + 1:each] = -math.inf
        r = op.forward(x[part], t[part])
        some = torch.arange(x[part].shape[0], device="cuda")[::200]
        want, bound = oracle.logprobs(x[some], t[some])
        for name in ("logp", "entropy", "lse"):
            within(torch, name, getattr(r, name)[some], want[name], bound[name])


@pytest.mark.parametrize("dtype", TYPES)
def test_many_rows_of_200000(torch, LogProbs, dtype):
    op = LogProbs()
    x, t = normal(torch, 1, dtype, 520, 200_000, by=3.0), targets_of(torch, 2, 520, 200_000)
    r = op.forward(x, t)
    d = op.backward(torch.ones_like(r.logp), None, x, t, r.stats)
    for some in (slice(0, 8), slice(512, 520)):
        want, bound = oracle.logprobs(x[some], t[some], 1.0, 0, torch.ones(8, device="cuda"), None)
        for name, got in (("logp", r.logp), ("entropy", r.entropy), ("lse", r.lse), ("d_logits", d)):
            within(torch, name, got[some], want[name], bound[name])


@pytest.mark.parametrize("n,top,border,rows", [(17, 9, 67_108_860, 67_108_911), (5, 0, 268_435_440, 268_435_471)])
def test_more_rows_than_a_launch_has(torch, LogProbs, n, top, border, rows):
    """67,108,860 rows of a wavefront each are the most that a launch has, or 268,435,440 of 16 lanes."""
    op, g = LogProbs(), torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((rows, n), generator=g, device="cuda", dtype=torch.float16)
    t = (torch.arange(rows, device="cuda", dtype=torch.int32) * 7) % (n + 1)
    r = op.forward(x, t, top)
    d = op.backward(r.logp, r.entropy, x, t, r.stats, r.entropy)
    for at in (slice(0, 9), slice(border - 7, border + 9), slice(rows - 9, rows)):
        want = op.forward(x[at], t[at], top)
        assert all(torch.equal(a[at], b) for a, b in zip(r, want) if a is not None), at
        assert torch.equal(d[at], op.backward(r.logp[at], r.entropy[at], x[at], t[at], r.stats[at], r.entropy[at])), at


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("n,top", [(9, 0), (9, 5), (40, 20), (700, 3), (5000, 0), (9000, 4), (70_000, 0), (140_000, 2)])
def test_the_largest_scales(torch, LogProbs, dtype, n, top):
    """A temperature of next to nothing: whatever is on top has all of the probability."""
    for scale in (2.0e38, 3.0e38):
        op = LogProbs(scale)
        x = -torch.randint(0, 2, (6, n), generator=torch.Generator().manual_seed(n)).to(getattr(torch, dtype)).cuda()
        x[:, n // 2] = 0
        x[0, :] = -1
        x[0, 1] = 0
        t = torch.tensor([1, 0, n // 2, 3, n - 1, 2], device="cuda")
        want, bound = oracle.logprobs(x, t, op.scale, top, torch.ones(6, device="cuda"), None)
        r = op.forward(x, t, top)
        for name in ("logp", "entropy", "lse"):
            within(torch, name, getattr(r, name), want[name], bound[name])
        if top:
            assert torch.equal(r.top_ids, want["top_ids"])
            within(torch, "top_logp", r.top_logp, want["top_logp"], bound["top_logp"])
        within(torch, "d_logits", op.backward(torch.ones(6, device="cuda"), None, x, t, r.stats), want["d_logits"], bound["d_logits"])
