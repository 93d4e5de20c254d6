"""Embedding lookup and its gradient against the 64-bit oracle; the bounds are the oracle's."""
import math

import pytest

from oracle import attention_oracle as oracle

pytestmark = pytest.mark.gpu

TYPES = ("float32", "bfloat16", "float16")


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible: these tests need a real MI355X")
    return torch


@pytest.fixture(scope="module")
def Embedding(torch):
    from paper_2307_05740_amd.embedding import ArrowEmbedding
    return ArrowEmbedding


def normal(torch, seed, dtype, *shape):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(*shape, generator=g).to(getattr(torch, dtype)).cuda()


def tokens(torch, seed, n, rows, kind):
    g = torch.Generator().manual_seed(seed)
    if kind == "one":
        ids = torch.full((n,), rows // 2)
    elif kind == "text":                                          # the m-th most frequent about 1 / m of the time, and padding
        ids = (torch.exp(torch.rand(n, generator=g, dtype=torch.float64) * math.log(rows + 1.0)) - 1).long().clamp(0, rows - 1)
        ids[::17] = -1
        ids[5::31] = rows
    else:
        ids = torch.randint(0, rows, (n,), generator=g)
    return ids.cuda()


def check_grad(torch, got, dY, ids, rows, scale):
    want, bound = oracle.embedding_grad(dY, ids, rows, scale, got.dtype)
    off = (got.double() - want).abs()
    assert bool((off <= bound).all()), (float((off / bound.clamp(min=1e-300)).max()), int((off > bound).sum()))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("columns", [1, 3, 4, 7, 8, 9, 15, 64, 100, 513, 2048, 5000])
def test_lookup_and_gradient(torch, Embedding, dtype, columns):
    rows, n, scale = 301, 333, 1.7
    W, dY, ids = normal(torch, 1, dtype, rows, columns), normal(torch, 2, dtype, n, columns), tokens(torch, 3, n, rows, "text")
    op = Embedding(rows, scale)
    u = oracle.UNIT[W.dtype]
    for of in (ids, ids.int()):
        Y = op.forward(W, of, torch.full_like(dY, math.nan))
        want = oracle.embedding(W, ids, float(torch.tensor(scale, dtype=torch.float32)))
        assert bool(((Y.double() - want).abs() <= (u + 2.0 ** -24) * want.abs() + 2 * oracle.TINY[W.dtype]).all())
        check_grad(torch, op.backward(dY, of, torch.full_like(W, math.nan)), dY, ids, rows, scale)
    check_grad(torch, op.backward(dY, ids, dtype=torch.float32), dY, ids, rows, scale)


@pytest.mark.parametrize("n", [0, 1, 63, 64, 65, 255, 256, 257, 1000, 4097, 40000])
@pytest.mark.parametrize("rows", [1, 2, 255, 511, 512, 70000])
@pytest.mark.parametrize("kind", ["one", "text", "even"])
def test_numbers_of_tokens_and_rows(torch, Embedding, n, rows, kind):
    dY, ids = normal(torch, 2, "float32", n, 12), tokens(torch, 3, n, rows, kind)
    check_grad(torch, Embedding(rows).backward(dY, ids, torch.full((rows, 12), math.nan, device="cuda")), dY, ids, rows, 1.0)


def test_rows_beyond_two_to_the_twentieth(torch, Embedding):
    rows, n = 3_000_017, 5000
    dY, ids = normal(torch, 2, "bfloat16", n, 8), tokens(torch, 3, n, rows, "even")
    got = Embedding(rows, 0.5).backward(dY, ids)
    check_grad(torch, got, dY, ids, rows, 0.5)


def test_offsets_beyond_32_bits(torch, Embedding):
    """A table of 5 GB: rows whose places in bytes and elements pass 2^32 and 2^31."""
    rows, columns = 640_000, 4096
    W = torch.zeros(rows, columns, dtype=torch.bfloat16, device="cuda")
    ids = torch.tensor([0, rows - 1, 600_001, 1, rows - 1], device="cuda")
    W[ids] = normal(torch, 1, "bfloat16", 5, columns)
    op = Embedding(rows)
    assert torch.equal(op.forward(W, ids), W[ids])
    dY = normal(torch, 2, "bfloat16", 5, columns)
    dW = op.backward(dY, ids, W)
    assert torch.equal(dW[600_001], dY[2]) and torch.equal(dW[rows - 1], (dY[1].float() + dY[4].float()).bfloat16())
    used = torch.zeros(rows, dtype=torch.bool, device="cuda")
    used[ids] = True
    for part in range(0, rows, 64_000):
        assert not bool(dW[part:part + 64_000][~used[part:part + 64_000]].any())


def test_garbage_in_the_workspace(torch, Embedding):
    """Rows without tokens are zero whatever an earlier call left: of rows that had tokens then, and of all kinds of words."""
    op, rows, n = Embedding(5000), 5000, 3000
    for word in (0, 0xFF, 0x01, 0x7F):
        for seed in (1, 2):
            junk = torch.full((1 << 22,), word, dtype=torch.uint8, device="cuda")
            del junk
            dY, ids = normal(torch, seed, "float32", n, 16), tokens(torch, seed, n, rows, "even")
            check_grad(torch, op.backward(dY, ids), dY, ids, rows, 1.0)


def test_strides_and_shapes(torch, Embedding):
    rows, columns = 50, 36
    big = normal(torch, 1, "bfloat16", rows, 2 * columns + 1)
    W = big[:, 1:columns + 1]                                     # rows at odd addresses
    ids = tokens(torch, 3, 24, rows, "even").view(2, 3, 4)
    op = Embedding(rows)
    assert torch.equal(op.forward(W, ids), W[ids])
    dY = normal(torch, 2, "bfloat16", 24, 2 * columns + 1)[:, 1:columns + 1]
    out = torch.full_like(big, 7.0)
    op.backward(dY, ids.view(-1), out[:, 1:columns + 1])
    check_grad(torch, out[:, 1:columns + 1], dY, ids, rows, 1.0)
    assert bool((out[:, 0] == 7).all()) and bool((out[:, columns + 1:] == 7).all())
    check_grad(torch, op.backward(dY.reshape(2, 3, 4, columns), ids), dY, ids, rows, 1.0)


def test_the_same_every_time_and_captured(torch, Embedding):
    rows, n, columns = 1000, 8192, 256
    op = Embedding(rows)
    dY, ids = normal(torch, 2, "bfloat16", n, columns), tokens(torch, 3, n, rows, "text")
    first = op.backward(dY, ids)
    assert all(torch.equal(first, op.backward(dY, ids)) for _ in range(3))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dW = op.backward(dY, ids)
    for seed in (5, 6, 7):
        ids.copy_(tokens(torch, seed, n, rows, "text"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(dW, op.backward(dY, ids))


def test_gradient_against_differences(torch, Embedding):
    """The lookup is linear: <forward(W + E) - forward(W), dY> = <E, dW>, up to what rounding the two does."""
    rows, columns, n = 40, 64, 200
    ids, dY = tokens(torch, 3, n, rows, "text"), normal(torch, 2, "float32", n, columns)
    W, E = normal(torch, 1, "float32", rows, columns), normal(torch, 4, "float32", rows, columns)
    op = Embedding(rows, 3.0)
    diff = op.forward(W + E, ids).double() - op.forward(W, ids).double()
    left = float((diff * dY.double()).sum())
    right = float((op.backward(dY, ids).double() * E.double()).sum())
    room = 2.0 ** -22 * 3.0 * float((dY.double().abs().sum()) * (W.abs().max() + E.abs().max())) + 2.0 ** -20 * abs(right)
    assert abs(left - right) <= room, (left, right, room)


@pytest.mark.parametrize("n", [17, 511, 2047, 2048, 2049])
@pytest.mark.parametrize("rows,columns", [(1, 130), (64, 1), (65, 1100), (1025, 5), (20_001, 260)])
@pytest.mark.parametrize("kind", ["one", "text", "even"])
def test_few_tokens_and_slices_of_columns(torch, Embedding, n, rows, columns, kind):
    """Around the number of tokens that a gradient takes in one launch; rows that reach over several of its groups of lanes."""
    dY, ids = normal(torch, 2, "bfloat16", n, columns), tokens(torch, 3, n, rows, kind)
    op = Embedding(rows, 1.5)
    check_grad(torch, op.backward(dY, ids, torch.full((rows, columns), math.nan, dtype=torch.bfloat16, device="cuda")), dY, ids, rows, 1.5)
    again = op.backward(dY, ids.int(), dtype=torch.float32)
    check_grad(torch, again, dY, ids, rows, 1.5)
    assert torch.equal(again, op.backward(dY, ids, dtype=torch.float32))


@pytest.mark.parametrize("columns", [3, 127, 128, 200])
def test_few_tokens_of_a_large_table(torch, Embedding, columns):
    """Rows shorter and longer than a slice, of more rows than one launch takes of the former, and of some fewer."""
    for rows in (262_144, 262_145, 300_001):
        dY, ids = normal(torch, 2, "bfloat16", 500, columns), tokens(torch, 3, 500, rows, "text")
        check_grad(torch, Embedding(rows).backward(dY, ids, torch.full((rows, columns), math.nan, dtype=torch.bfloat16, device="cuda")), dY, ids, rows, 1.0)


@pytest.mark.parametrize("dtype", TYPES)
def test_one_id_without_dimensions(torch, Embedding, dtype):
    W, dY = normal(torch, 1, dtype, 20, 40), normal(torch, 2, dtype, 40)
    op, ids = Embedding(20, 2.0), torch.tensor(7, device="cuda")
    W.requires_grad_()
    Y = op(W, ids)
    assert Y.shape == (40,) and torch.equal(Y, 2 * W[7])
    Y.backward(dY)
    want = torch.zeros_like(W)
    want[7] = 2 * dY
    assert torch.equal(W.grad, want)
    assert torch.equal(op.backward(dY, ids, dtype=torch.float32), want.float())
    with pytest.raises(ValueError, match="dY"):
        op.backward(dY[0], ids)


@pytest.mark.parametrize("n", [65_535, 65_536, 65_537, 200_000, 600_001])
@pytest.mark.parametrize("rows", [300, 32_000, 70_000, 300_000])
@pytest.mark.parametrize("kind", ["one", "text", "even"])
def test_many_tokens(torch, Embedding, n, rows, kind):
    """Around the number of tokens from which a digit is sorted by three kernels, with ids of one to three digits, and so many that chunks of the sums are longer."""
    dY, ids = normal(torch, 2, "float32", n, 12), tokens(torch, 3, n, rows, kind)
    op = Embedding(rows)
    got = op.backward(dY, ids, torch.full((rows, 12), math.nan, device="cuda"))
    check_grad(torch, got.cpu(), dY.cpu(), ids.cpu(), rows, 1.0)     # (there: additions of 64 bits to one row contend on a GPU)
    assert torch.equal(got, op.backward(dY, ids.int()))


@pytest.mark.parametrize("dtype", TYPES)
def test_many_tokens_of_wide_rows(torch, Embedding, dtype):
    rows, n, columns = 5003, 70_001, 1030
    dY, ids = normal(torch, 2, dtype, n, columns), tokens(torch, 3, n, rows, "text")
    check_grad(torch, Embedding(rows, 0.5).backward(dY, ids).cpu(), dY.cpu(), ids.cpu(), rows, 0.5)


def test_many_tokens_captured(torch, Embedding):
    rows, n, columns = 40_000, 100_000, 64
    op = Embedding(rows)
    dY, ids = normal(torch, 2, "bfloat16", n, columns), tokens(torch, 3, n, rows, "text")
    op.backward(dY, ids)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dW = op.backward(dY, ids)
    for seed in (5, 6, 7):
        ids.copy_(tokens(torch, seed, n, rows, "text"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(dW, op.backward(dY, ids))
