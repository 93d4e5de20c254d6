"""The example that trains and serves a small model with the operators on sequences together, and their gradients under torch's autograd."""
import importlib.util
import math
import os

import pytest

from oracle import attention_oracle as oracle

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible: these tests need a real MI355X")
    return torch


@pytest.fixture(scope="module")
def example(torch):
    spec = importlib.util.spec_from_file_location("stream_model", os.path.join(ROOT, "examples", "stream_model.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_the_model_learns_and_serves_what_it_learned(example):
    """From knowing nothing (ln 128) to more than halfway to knowing a sequence's eight tokens (ln 8); logits of single tokens differ from the whole
    sequence's by roundings to 16 bits of x, o and the projections, some tens of 2^-9 of the logits' deviation in two layers."""
    first, last, off = example.main(["--steps", "200", "--tokens", "200"])
    assert first > 0.9 * math.log(128) and last < 0.5 * (math.log(128) + math.log(8)), (first, last)
    assert off < 0.25, off


def test_autograd_gives_the_operators_gradients(torch):
    from paper_2307_05740_amd.attention import ArrowAttention
    from paper_2307_05740_amd.embedding import ArrowEmbedding
    g = torch.Generator().manual_seed(1)
    both = torch.randn(2, 70, 3, 4, 32, generator=g).bfloat16().cuda().requires_grad_()
    d_o = torch.randn(2, 70, 4, 32, generator=g).bfloat16().cuda()
    op = ArrowAttention(20, 2)
    q, k, v = both.unbind(2)
    op(q, k, v).backward(d_o)
    for b in range(2):
        for h in range(4):
            want, bound = oracle.attention(q[b, :, h].detach(), k[b, :, h].detach(), v[b, :, h].detach(), 20, 2, d_o=d_o[b, :, h])
            for i, n in enumerate(("dq", "dk", "dv")):
                assert bool(((both.grad[b, :, i, h].double() - want[n]).abs() <= bound[n]).all()), n
    W = torch.randn(50, 24, generator=g).cuda().requires_grad_()
    ids = torch.randint(-1, 50, (3, 40), generator=g).cuda()
    dY = torch.randn(3, 40, 24, generator=g).cuda()
    ArrowEmbedding(50, 2.0)(W, ids).backward(dY)
    want, bound = oracle.embedding_grad(dY, ids, 50, 2.0, torch.float32)
    assert bool(((W.grad.double() - want).abs() <= bound).all())
