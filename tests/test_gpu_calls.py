"""What calls on tensors have to do with torch beside the tensors: who watches allocations sees theirs, and what torch fills it fills for them; what they return stands by itself."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible: these tests need a real MI355X")
    return torch


def calls(torch):
    """Every call of the operators on sequences that returns what it has made: name -> (function, tensors that it makes for its caller)."""
    from paper_2307_05740_amd.attention import ArrowAttention
    from paper_2307_05740_amd.embedding import ArrowEmbedding
    from paper_2307_05740_amd.logprobs import ArrowLogProbs
    from paper_2307_05740_amd.packed import ArrowPackedAttention
    from paper_2307_05740_amd.pages import ArrowPages
    from paper_2307_05740_amd.rotation import ArrowRotation
    g = torch.Generator().manual_seed(1)
    x = lambda *shape: torch.randn(*shape, generator=g).bfloat16().cuda()   # noqa: E731
    q, k, v, w = x(2, 40, 4, 64), x(2, 40, 2, 64), x(2, 40, 2, 64), torch.rand(64, generator=g).cuda() + 0.5
    attend, embed, rotate, packed, score = ArrowAttention(), ArrowEmbedding(50), ArrowRotation(64), ArrowPackedAttention(), ArrowLogProbs()
    pages = ArrowPages(8, 16)
    table, held, free = pages.state(2, 3)
    length = torch.full((2,), 40, dtype=torch.int32, device="cuda")
    slots = pages.step(table, held, free, length, 40)
    pool = packed.pool(8, 16, 2, 64)
    packed.append(k.flatten(0, 1), v.flatten(0, 1), pool, slots.flatten())
    o, lse = attend.forward(q, k, v)
    ids, table_of = torch.randint(0, 50, (30,), generator=g).cuda(), x(50, 64)
    logits, targets = x(20, 300), torch.randint(0, 300, (20,), generator=g).cuda()
    r = score.forward(logits, targets)
    ones = torch.ones(20, device="cuda")
    return {
        "attention": (lambda: attend.forward(q, k, v), 2),
        "attention gradient": (lambda: attend.backward(q, q, k, v, o, lse), 3),
        "embedding": (lambda: embed.forward(table_of, ids), 1),
        "embedding gradient": (lambda: embed.backward(x(30, 64), ids), 1),
        "rotation": (lambda: rotate.forward(q, k, w, w), 2),
        "rotation gradient": (lambda: rotate.backward(q, k, q, k, w, w), 4),
        "pages": (lambda: pages.step(table, held, free, length, 2), 1),
        "read": (lambda: packed.read(pool, slots.flatten(), 64, torch.bfloat16), 2),
        "decode": (lambda: packed.decode(q[:, 0], pool, table, length), 1),
        "log probabilities": (lambda: score.forward(logits, targets, 3), 6),
        "log probabilities' gradient": (lambda: score.backward(ones, ones, logits, targets, r.stats, r.entropy), 1),
    }


def test_results_stand_by_themselves(torch):
    """Each has memory of its own, of its size: keeping one keeps no other, and one that is made larger reaches into none."""
    for name, (call, made) in calls(torch).items():
        out = call()
        out = list(out) if isinstance(out, tuple) else [out]
        out = [t for t in out if t is not None]
        assert len(out) == made, name
        assert len({t.untyped_storage().data_ptr() for t in out}) == made, name
        assert all(t.storage_offset() == 0 and t.untyped_storage().nbytes() == t.numel() * t.element_size() for t in out), name


def test_who_watches_allocations_sees_them(torch):
    """Dispatch modes and profilers, for every call."""
    from torch.utils._python_dispatch import TorchDispatchMode

    class Seen(TorchDispatchMode):
        def __init__(self):
            super().__init__()
            self.empties = 0

        def __torch_dispatch__(self, func, types, args=(), kwargs=None):
            self.empties += func is torch.ops.aten.empty.memory_format
            return func(*args, **(kwargs or {}))

    for name, (call, made) in calls(torch).items():
        call()
        with Seen() as seen:
            call()
        assert seen.empties >= made, (name, seen.empties)
        with torch.profiler.profile(activities=[torch.profiler.ProfilerActivity.CPU]) as prof:
            call()
        assert sum(e.count for e in prof.key_averages() if e.key == "aten::empty") >= made, name


def test_deterministic_algorithms_fill_what_is_not_written(torch):
    """Results of tokens that no sequence has are left as they are: NaN where torch fills new memory."""
    from paper_2307_05740_amd.attention import ArrowAttention
    op, x = ArrowAttention(), torch.ones(64, 2, 64, dtype=torch.bfloat16, device="cuda")
    offsets = torch.tensor([0, 16, 40], dtype=torch.int32, device="cuda")
    want, _ = op.forward(x, x, x, q_offsets=offsets, k_offsets=offsets)
    for _ in range(4):
        torch.full_like(x, 5.0)                    # (memory that the next results have is not NaN by itself)
        torch.full((2, 64), 5.0, device="cuda")
    before = torch.are_deterministic_algorithms_enabled()
    torch.use_deterministic_algorithms(True)
    try:
        o, lse = op.forward(x, x, x, q_offsets=offsets, k_offsets=offsets)
        grads = op.backward(x, x, x, x, o.nan_to_num(), lse.nan_to_num(), q_offsets=offsets, k_offsets=offsets)
    finally:
        torch.use_deterministic_algorithms(before)
    assert torch.equal(o[:40], want[:40]) and bool(o[40:].isnan().all()) and bool(lse[:, 40:].isnan().all())
    assert all(bool(g[:40].isfinite().all()) and bool(g[40:].isnan().all()) for g in grads)
