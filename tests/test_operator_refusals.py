"""What the entries of arrow_rotation.h, arrow_pages.h, arrow_packed.h and arrow_logprobs.h refuse, and what they accept without work, without a GPU: no argument below
reaches a kernel."""
import ctypes
import math

import pytest

from paper_2307_05740_amd import binding

SOME = 1 << 24                     # an address that nothing reads


@pytest.fixture()
def L():
    return binding.lib()


def refused(rc, word):
    assert rc == binding.ARROW_EINVAL, rc
    assert word in binding.arrow_last_error(), binding.arrow_last_error()


# ---- rotation ----
def rotation(**change):
    a = binding.arrow_rotation_t(dtype=binding.ARROW_BF16, weight_dtype=binding.ARROW_F32, batch=2, tokens=8, q_heads=4, kv_heads=2, dim=64, rotary=64, eps=1e-6,
                                 turns=SOME)
    for name in ("q", "q_out", "dq"):
        setattr(a, name, binding.arrow_strides_t(8 * 256, 256, 64))
    for name in ("k", "k_out", "dk"):
        setattr(a, name, binding.arrow_strides_t(8 * 128, 128, 64))
    for name, value in change.items():
        setattr(a, name, value)
    return a


ROTATION = [
    ({"dtype": 7}, "dtype"), ({"weight_dtype": binding.ARROW_F16}, "weight_dtype"), ({"batch": -1}, "batch"), ({"tokens": -1}, "tokens"),
    ({"batch": 1 << 20, "tokens": 1 << 20}, "tokens"), ({"q_heads": 0}, "q_heads"), ({"kv_heads": 0}, "kv_heads"), ({"dim": 4}, "dim"), ({"dim": 264}, "dim"),
    ({"dim": 60}, "dim"), ({"rotary": 8}, "rotary"), ({"rotary": 80}, "rotary"), ({"rotary": -16}, "rotary"), ({"interleaved": 2}, "interleaved"), ({"eps": -1.0}, "eps"),
    ({"eps": math.nan}, "eps"), ({"eps": math.inf}, "eps"), ({"positions": SOME, "position_bytes": 2}, "position_bytes"),
    ({"positions": SOME + 4, "position_bytes": 8}, "positions"), ({"shift": 1 << 53}, "shift"), ({"turns": 0}, "turns"), ({"turns": SOME + 4}, "turns"),
    ({"q": binding.arrow_strides_t(2048, 256, 60)}, "multiples of 8"), ({"k": binding.arrow_strides_t(-8, 128, 64)}, "not negative"),
]


@pytest.mark.parametrize("change,word", ROTATION + [({"q_out": binding.arrow_strides_t(2048, 0, 64)}, "overlap"), ({"k_out": binding.arrow_strides_t(0, 128, 64)}, "overlap")])
def test_rotation_refuses(L, change, word):
    refused(L.arrow_rotation_forward(ctypes.byref(rotation(**change)), SOME, 2 * SOME, 0, 0, 3 * SOME, 4 * SOME, 0), word)


@pytest.mark.parametrize("change,word", ROTATION + [({"dq": binding.arrow_strides_t(2048, 256, 0)}, "overlap")])
def test_rotation_gradients_refuse(L, change, word):
    p = [i * SOME for i in range(1, 5)]
    refused(L.arrow_rotation_backward(ctypes.byref(rotation(**change)), *p, 5 * SOME, 6 * SOME, 7 * SOME, 8 * SOME, 0, 0, 0, 0, 0), word)


def test_rotation_refuses_pointers(L):
    a = rotation()
    call = lambda q, k, wq, wk, qo, ko, a=a: L.arrow_rotation_forward(ctypes.byref(a), q, k, wq, wk, qo, ko, 0)   # noqa: E731
    for at, word in (((0, 2 * SOME, 0, 0, 3 * SOME, 4 * SOME), "q is NULL"), ((SOME, 0, 0, 0, 3 * SOME, 4 * SOME), "k is NULL"), ((SOME, 2 * SOME, 0, 0, 0, 4 * SOME), "q_out"),
                     ((SOME, 2 * SOME, 0, 0, 3 * SOME, 0), "k_out"), ((SOME + 8, 2 * SOME, 0, 0, 3 * SOME, 4 * SOME), "aligned"),
                     ((SOME, 2 * SOME, 5 * SOME, 0, 3 * SOME, 4 * SOME), "both or neither"), ((SOME, 2 * SOME, 5 * SOME + 2, 6 * SOME, 3 * SOME, 4 * SOME), "aligned"),
                     ((SOME, 2 * SOME, 0, 0, 2 * SOME, 4 * SOME), "q_out is k"), ((SOME, 2 * SOME, 0, 0, 3 * SOME, 3 * SOME), "q_out is k")):
        refused(call(*at), word)
    refused(call(SOME, 2 * SOME, 0, 0, SOME, 4 * SOME, rotation(q_out=binding.arrow_strides_t(8 * 512, 512, 64))), "in place")
    refused(L.arrow_rotation_forward(None, SOME, SOME, 0, 0, SOME, SOME, 0), "NULL")
    for nothing in (rotation(batch=0), rotation(tokens=0)):
        assert call(0, 0, 0, 0, 0, 0, nothing) == binding.ARROW_OK
        assert L.arrow_rotation_backward(ctypes.byref(nothing), *[0] * 11, 0, 0) == binding.ARROW_OK


def test_rotation_gradients_refuse_pointers(L):
    a = rotation()
    need = L.arrow_rotation_workspace_bytes(ctypes.byref(a))
    assert need >= 2 * 64 * 4 and L.arrow_rotation_workspace_bytes(None) == 0
    good = dict(gq=SOME, gk=2 * SOME, q=3 * SOME, k=4 * SOME, wq=5 * SOME, wk=6 * SOME, dq=7 * SOME, dk=8 * SOME, dwq=9 * SOME, dwk=10 * SOME, ws=16 * SOME, n=need)
    call = lambda **change: L.arrow_rotation_backward(ctypes.byref(a), *dict(good, **change).values(), 0)   # noqa: E731
    for change, word in (({"gq": 0}, "d_q_out"), ({"gk": 0}, "d_k_out"), ({"q": 0}, "q is NULL"), ({"dq": 0}, "dq"), ({"dk": 7 * SOME}, "dq or dk"), ({"dq": 3 * SOME}, "dq or dk"),
                         ({"dwk": 0}, "both or neither"), ({"dwk": 9 * SOME}, "the same"), ({"ws": 0}, "workspace"), ({"ws": 16 * SOME + 16}, "workspace")):
        refused(call(**change), word)
    assert call(n=need - 1) == binding.ARROW_ETOOSMALL


@pytest.mark.parametrize("tokens", [1, 7, 1024, 100_000, 1 << 24])
@pytest.mark.parametrize("heads,kv", [(1, 1), (32, 8), (1, 64), (64, 1)])
def test_the_workspace_of_rotation_gradients_is_bounded(L, tokens, heads, kv):
    a = rotation(batch=1, tokens=tokens, q_heads=heads, kv_heads=kv, q=binding.arrow_strides_t(0, 64 * heads, 64), q_out=binding.arrow_strides_t(0, 64 * heads, 64),
                 dq=binding.arrow_strides_t(0, 64 * heads, 64), k=binding.arrow_strides_t(0, 64 * kv, 64), k_out=binding.arrow_strides_t(0, 64 * kv, 64),
                 dk=binding.arrow_strides_t(0, 64 * kv, 64))
    need = L.arrow_rotation_workspace_bytes(ctypes.byref(a))
    assert 2 * 64 * 4 <= need <= 1024 * 64 * 4


# ---- pages ----
def pages(**change):
    a = binding.arrow_pages_t(batch=3, columns=4, page=16, window=0, sinks=0, tokens=1, pages=10)
    for name, value in change.items():
        setattr(a, name, value)
    return a


@pytest.mark.parametrize("change,word", [
    ({"batch": -1}, "batch"), ({"batch": (1 << 24) + 1}, "batch"), ({"page": 0}, "page"), ({"page": 24}, "page"), ({"page": 1 << 21}, "page"), ({"columns": -1}, "columns"),
    ({"columns": 1 << 23}, "columns"), ({"batch": 1 << 20, "columns": 1 << 12}, "entries"), ({"window": -1}, "window"), ({"sinks": -1}, "sinks"), ({"pages": -1}, "pages"),
    ({"pages": (1 << 30) + 1}, "pages"), ({"tokens": -1}, "tokens"), ({"tokens": 1 << 30}, "tokens"), ({"offsets": SOME, "rows": -1}, "rows"),
    ({"offsets": SOME, "rows": 1 << 31}, "rows"),
])
def test_pages_refuse(L, change, word):
    refused(L.arrow_pages_step(ctypes.byref(pages(**change)), SOME, 2 * SOME, 3 * SOME, 4 * SOME, 5 * SOME, 0, 0, 0), word)
    assert L.arrow_pages_workspace_bytes(ctypes.byref(pages(**change))) == 0


def test_pages_refuse_pointers(L):
    good = [SOME, 2 * SOME, 3 * SOME, 4 * SOME, 5 * SOME]
    call = lambda at, a=pages(), ws=0, n=0: L.arrow_pages_step(ctypes.byref(a), *at, ws, n, 0)   # noqa: E731
    for i, name in enumerate(("lengths", "held", "table", "list", "slots")):
        refused(call(good[:i] + [0] + good[i + 1:]), f"{name} is NULL")
        refused(call(good[:i] + [good[i] + 2] + good[i + 1:]), f"{name} is not")
    refused(call([SOME, SOME + 4, 3 * SOME, 4 * SOME, 5 * SOME]), "overlap")
    refused(call([SOME, 2 * SOME, 3 * SOME, 3 * SOME + 44, 5 * SOME]), "overlap")
    refused(call(good, pages(offsets=SOME + 2, rows=1)), "offsets")
    refused(L.arrow_pages_step(None, *good, 0, 0, 0), "NULL")
    large = pages(batch=2000, columns=4, pages=100)
    need = L.arrow_pages_workspace_bytes(ctypes.byref(large))
    assert need >= 3 * 2000 * 4
    refused(call(good, large, 0, need), "workspace")
    assert call(good, large, 16 * SOME, need - 1) == binding.ARROW_ETOOSMALL
    assert call([0, 0, 0, 4 * SOME, 0], pages(batch=0)) == binding.ARROW_OK
    assert L.arrow_pages_workspace_bytes(ctypes.byref(pages())) == 0 and L.arrow_pages_workspace_bytes(None) == 0


# ---- the cache in 4 bits ----
def packed(**change):
    block = 16 * (64 + 4)
    c = binding.arrow_packed_t(dtype=binding.ARROW_BF16, batch=2, q_heads=4, kv_heads=2, dim=64, scale=1.0, page=16, columns=4, pages=4, max_len=64, page_step=2 * block,
                               head_step=block, table=SOME, lengths=SOME)
    for name, value in change.items():
        setattr(c, name, value)
    return c


ROWS = binding.arrow_strides_t(128, 128, 64)
POOL = [
    ({"dtype": binding.ARROW_F32}, "dtype"), ({"dtype": 9}, "dtype"), ({"kv_heads": 0}, "kv_heads"), ({"dim": 16}, "dim"), ({"dim": 96}, "dim"), ({"dim": 256}, "dim"),
    ({"page": 8}, "page"), ({"page": 48}, "page"), ({"page": 1 << 21}, "page"), ({"pages": -1}, "pages"), ({"page_step": 24}, "pool"), ({"page_step": 1024}, "pool"),
    ({"head_step": 0}, "pool"), ({"head_step": -1088}, "pool"),
]


@pytest.mark.parametrize("change,word", POOL)
def test_packed_rows_refuse(L, change, word):
    c = packed(**change)
    refused(L.arrow_packed_append(ctypes.byref(c), 3, SOME, 2 * SOME, ROWS, ROWS, 3 * SOME, 4 * SOME, 0), word)
    refused(L.arrow_packed_read(ctypes.byref(c), 3, 3 * SOME, 4 * SOME, SOME, 2 * SOME, ROWS, ROWS, 0), word)


def test_packed_rows_refuse_pointers(L):
    c = packed()
    append = lambda k, v, slots, pool, ks=ROWS, vs=ROWS, n=3, c=c: L.arrow_packed_append(ctypes.byref(c), n, k, v, ks, vs, slots, pool, 0)   # noqa: E731
    read = lambda k, v, slots, pool, ks=ROWS, vs=ROWS, n=3, c=c: L.arrow_packed_read(ctypes.byref(c), n, slots, pool, k, v, ks, vs, 0)   # noqa: E731
    for call in (append, read):
        for at, word in (((0, 2 * SOME, 3 * SOME, 4 * SOME), "k is NULL"), ((SOME, 0, 3 * SOME, 4 * SOME), "v is NULL"), ((SOME, 2 * SOME, 0, 4 * SOME), "slots is NULL"),
                         ((SOME, 2 * SOME, 3 * SOME + 4, 4 * SOME), "slots"), ((SOME, 2 * SOME, 3 * SOME, 0), "pool is NULL"), ((SOME, 2 * SOME, 3 * SOME, 4 * SOME + 8), "pool"),
                         ((SOME + 8, 2 * SOME, 3 * SOME, 4 * SOME), "aligned"), ((4 * SOME, 2 * SOME, 3 * SOME, 4 * SOME), "pool")):
            refused(call(*at), word)
        refused(call(SOME, 2 * SOME, 3 * SOME, 4 * SOME, binding.arrow_strides_t(0, 100, 64)), "multiples of 8")
        refused(call(SOME, 2 * SOME, 3 * SOME, 4 * SOME, n=-1), "tokens")
        refused(call(SOME, 2 * SOME, 3 * SOME, 4 * SOME, n=1 << 31), "tokens")
        assert call(0, 0, 0, 4 * SOME, n=0) == binding.ARROW_OK
    refused(read(SOME, SOME, 3 * SOME, 4 * SOME), "the other")
    refused(read(SOME, 2 * SOME, 3 * SOME, 4 * SOME, binding.arrow_strides_t(0, 32, 64)), "overlap")
    assert append(SOME, 2 * SOME, 3 * SOME, 0, c=packed(pages=0)) == binding.ARROW_OK
    refused(L.arrow_packed_append(None, 3, SOME, SOME, ROWS, ROWS, SOME, SOME, 0), "NULL")


@pytest.mark.parametrize("change,word", POOL + [
    ({"batch": -1}, "batch"), ({"q_heads": 3}, "q_heads"), ({"window": -1}, "window"), ({"sinks": -1}, "sinks"), ({"scale": 0.0}, "scale"), ({"scale": math.nan}, "scale"),
    ({"columns": -1}, "columns"), ({"columns": 1 << 23}, "columns"), ({"max_len": -1}, "max_len"), ({"table": 0}, "table"), ({"lengths": 0}, "lengths"), ({"lengths": SOME + 2}, "aligned"),
])
def test_packed_decode_refuses(L, change, word):
    st = binding.arrow_strides_t(256, 0, 64)
    refused(L.arrow_packed_decode(ctypes.byref(packed(**change)), SOME, st, 0, 0, ROWS, ROWS, 4 * SOME, 5 * SOME, st, 16 * SOME, 1 << 30, 0), word)


def test_packed_decode_refuses_pointers(L):
    st, c = binding.arrow_strides_t(256, 0, 64), packed()
    call = lambda q, k, v, pool, o, ws=16 * SOME, n=1 << 30, c=c: L.arrow_packed_decode(ctypes.byref(c), q, st, k, v, ROWS, ROWS, pool, o, st, ws, n, 0)   # noqa: E731
    for at, word in (((0, 0, 0, 4 * SOME, 5 * SOME), "q is NULL"), ((SOME, 0, 0, 4 * SOME, 0), "o is NULL"), ((SOME, 2 * SOME, 0, 4 * SOME, 5 * SOME), "both or neither"),
                     ((SOME, 2 * SOME + 8, 3 * SOME, 4 * SOME, 5 * SOME), "aligned"), ((SOME, 0, 0, 4 * SOME, SOME), "o is one"), ((SOME, 0, 0, 4 * SOME, 4 * SOME), "o is one")):
        refused(call(*at), word)
    long = packed(columns=4000, max_len=64000, pages=8000)
    need = L.arrow_packed_decode_workspace_bytes(ctypes.byref(long))
    assert need >= 2 * 2 * 4 * 66 * 4
    refused(call(SOME, 0, 0, 4 * SOME, 5 * SOME, 0, need, long), "workspace")
    assert call(SOME, 0, 0, 4 * SOME, 5 * SOME, 16 * SOME, need - 1, long) == binding.ARROW_ETOOSMALL
    assert call(0, 0, 0, 4 * SOME, 0, 0, 0, packed(batch=0)) == binding.ARROW_OK
    assert L.arrow_packed_decode_workspace_bytes(None) == 0


# ---- log probabilities ----
def logprobs(**change):
    a = binding.arrow_logprobs_t(dtype=binding.ARROW_BF16, target_bytes=8, top=2, vocabulary=100, rows=5, stride=100, d_stride=100, scale=1.0)
    for name, value in change.items():
        setattr(a, name, value)
    return a


@pytest.mark.parametrize("change,word", [
    ({"dtype": 3}, "dtype"), ({"target_bytes": 2}, "target_bytes"), ({"top": -1}, "top"), ({"top": 33}, "top"), ({"top": 5, "vocabulary": 4}, "top"), ({"vocabulary": 0}, "vocabulary"),
    ({"vocabulary": (1 << 30) + 1}, "vocabulary"), ({"rows": -1}, "rows"), ({"rows": 1 << 31}, "rows"), ({"stride": 99}, "apart"), ({"scale": 0.0}, "scale"),
    ({"scale": math.inf}, "scale"), ({"scale": math.nan}, "scale"),
])
def test_logprobs_refuse(L, change, word):
    a = logprobs(**change)
    refused(L.arrow_logprobs_forward(ctypes.byref(a), *[i * SOME for i in range(1, 9)], 0, 0, 0), word)
    refused(L.arrow_logprobs_backward(ctypes.byref(a), *[i * SOME for i in range(1, 8)], 0), word)
    assert L.arrow_logprobs_workspace_bytes(ctypes.byref(a)) == 0


def test_logprobs_refuse_pointers(L):
    names = ("logits", "targets", "logp", "entropy", "lse", "stats", "top_logp", "top_ids")
    good = [i * SOME for i in range(1, 9)]
    call = lambda at, a=logprobs(), ws=0, n=0: L.arrow_logprobs_forward(ctypes.byref(a), *at, ws, n, 0)   # noqa: E731
    for i, name in enumerate(names):
        refused(call(good[:i] + [0] + good[i + 1:]), f"{name} is NULL")
        refused(call(good[:i] + [good[i] + 1] + good[i + 1:]), f"{name} is not")
    refused(call(good[:5] + [6 * SOME + 4] + good[6:]), "stats is not")
    refused(call(good[:2] + [SOME + 400] + good[3:]), "overlaps an input")
    refused(call(good[:3] + [3 * SOME + 8] + good[4:]), "overlap")
    refused(L.arrow_logprobs_forward(None, *good, 0, 0, 0), "NULL")
    large = logprobs(vocabulary=200_000, stride=200_000)
    need = L.arrow_logprobs_workspace_bytes(ctypes.byref(large))
    assert need >= 5 * 7 * (16 + 16)
    refused(call([i * 64 * SOME for i in range(1, 9)], large, 0, need), "workspace")
    assert call([i * 64 * SOME for i in range(1, 9)], large, 1024 * SOME, need - 1) == binding.ARROW_ETOOSMALL
    assert call([0] * 8, logprobs(rows=0)) == binding.ARROW_OK


def test_logprobs_gradients_refuse_pointers(L):
    good = dict(d_logp=SOME, d_entropy=2 * SOME, logits=3 * SOME, targets=4 * SOME, stats=5 * SOME, entropy=6 * SOME, d_logits=7 * SOME)
    call = lambda a=logprobs(), **change: L.arrow_logprobs_backward(ctypes.byref(a), *dict(good, **change).values(), 0)   # noqa: E731
    for change, word in (({"logits": 0}, "logits is NULL"), ({"targets": 0}, "targets"), ({"stats": 0}, "stats"), ({"entropy": 0}, "entropy"), ({"d_logits": 0}, "d_logits is NULL"),
                         ({"d_logp": SOME + 2}, "aligned"), ({"d_logits": 3 * SOME + 8}, "overlaps"), ({"d_logits": SOME}, "overlaps"), ({"d_logits": 7 * SOME + 1}, "d_logits is not")):
        refused(call(**change), word)
    refused(call(logprobs(d_stride=101), d_logits=3 * SOME), "overlaps")
    refused(call(logprobs(d_stride=99)), "apart")
    assert call(logprobs(rows=0), **{n: 0 for n in good}) == binding.ARROW_OK


def test_classes_refuse_before_any_call():
    """What the Python classes refuse of themselves."""
    from paper_2307_05740_amd.logprobs import ArrowLogProbs
    from paper_2307_05740_amd.packed import ArrowPackedAttention
    from paper_2307_05740_amd.pages import ArrowPages
    from paper_2307_05740_amd.rotation import ArrowRotation
    import torch
    for kw in ({"rotary": 8}, {"rotary": 80}, {"rotary": -16}, {"frequencies": [1.0]}):
        with pytest.raises(ValueError):
            ArrowRotation(64, device="cpu", **kw)
    for args in ((-1, 16), (4, 0), (4, 24), (4, 16, -1), (4, 16, 0, -1)):
        with pytest.raises(ValueError):
            ArrowPages(*args, device="cpu")
    for args in ((-1,), (0, -1)):
        with pytest.raises(ValueError):
            ArrowPackedAttention(*args, device="cpu")
    for scale in (0.0, -1.0, math.inf, math.nan):
        with pytest.raises(ValueError):
            ArrowLogProbs(scale, device="cpu")
    # tensors that are not on a GPU
    x, t = torch.zeros(2, 8), torch.zeros(2, dtype=torch.int64)
    with pytest.raises(ValueError, match="cpu"):
        ArrowLogProbs(device="cpu").forward(x, t)
    with pytest.raises(ValueError, match="cpu"):
        ArrowRotation(16, device="cpu").forward(torch.zeros(2, 1, 16), torch.zeros(2, 1, 16))
    p = ArrowPages(4, 16, device="cpu")
    table, held, free = p.state(2, 3)
    assert free.tolist() == [4, 3, 2, 1, 0]
    with pytest.raises(ValueError, match="cpu"):
        p.step(table, held, free, held)
    a = ArrowPackedAttention(device="cpu")
    with pytest.raises(ValueError, match="cpu"):
        a.read(a.pool(2, 16, 1, 64), t, 64, torch.bfloat16)


# ---- what is written lies apart from all else ----
def steps(*s):
    return binding.arrow_strides_t(*s)


@pytest.mark.parametrize("change,at", [
    ({"q_out": steps(2048, 64, 64)}, {}),                                     # (token t, head h + 1) is (token t + 1, head h)
    ({"k_out": steps(64, 64, 512)}, {}), ({"q_out": steps(256, 256, 64)}, {}), ({"q_out": steps(2048, 128, 64)}, {}),
    ({}, {"qo": SOME + 512}), ({}, {"qo": 2 * SOME + 256}), ({}, {"ko": SOME + 1024}), ({}, {"ko": 2 * SOME - 256}), ({}, {"ko": 3 * SOME + 128}), ({}, {"qo": 4 * SOME - 128}),
    ({}, {"qo": 5 * SOME - 1024}), ({"positions": 8 * SOME, "position_bytes": 8}, {"qo": 8 * SOME}), ({"turns": 8 * SOME}, {"ko": 8 * SOME + 128}),
    # views of one tensor: queries from head 0 on, keys from 4 on; a head too early
    ({name: steps(8 * 512, 512, 64) for name in ("q", "k", "q_out", "k_out")}, {"q": SOME, "qo": SOME, "k": SOME + 3 * 128, "ko": SOME + 3 * 128}),
    ({name: steps(8 * 512, 512, 64) for name in ("q", "k", "q_out", "k_out")}, {"q": SOME, "qo": SOME, "k": SOME + 4 * 128 + 512, "ko": SOME + 7 * 128}),
])
def test_rotation_refuses_what_overlaps(L, change, at):
    p = dict(dict(q=SOME, k=2 * SOME, wq=5 * SOME, wk=6 * SOME, qo=3 * SOME, ko=4 * SOME), **at)
    refused(L.arrow_rotation_forward(ctypes.byref(rotation(**change)), *p.values(), 0), "overlap")


@pytest.mark.parametrize("change,at", [
    ({"dq": steps(2048, 64, 64)}, {}), ({"dk": steps(64, 64, 512)}, {}), ({}, {"dq": SOME + 512}), ({}, {"dq": 2 * SOME - 16}), ({}, {"dk": 2 * SOME + 256}), ({}, {"dq": 3 * SOME + 256}),
    ({}, {"dk": 4 * SOME + 256}), ({}, {"dk": 7 * SOME + 256}), ({}, {"dwq": 7 * SOME + 64}), ({}, {"dwk": 5 * SOME + 64}), ({}, {"dwq": 10 * SOME + 128}), ({}, {"dwk": SOME}),
    ({}, {"ws": 4 * SOME}), ({}, {"dwq": 16 * SOME + 256}), ({"positions": 8 * SOME, "position_bytes": 4}, {}),
])
def test_rotation_gradients_refuse_what_overlaps(L, change, at):
    a = rotation(**change)
    p = dict(dict(gq=SOME, gk=2 * SOME, q=3 * SOME, k=4 * SOME, wq=5 * SOME, wk=6 * SOME, dq=7 * SOME, dk=8 * SOME, dwq=9 * SOME, dwk=10 * SOME, ws=16 * SOME), **at)
    refused(L.arrow_rotation_backward(ctypes.byref(a), *p.values(), L.arrow_rotation_workspace_bytes(ctypes.byref(a)), 0), "overlap")


TALL = steps(256, 256, 64)           # rows of four heads


@pytest.mark.parametrize("change,at", [
    ({"page_step": 1088, "head_step": 1088}, {}), ({"page_step": 1088, "head_step": 2176}, {}), ({}, {"ks": steps(0, 64, 64)}), ({}, {"vs": steps(0, 64, 128)}),
    ({}, {"k": 2 * SOME + 128}), ({}, {"k": 4 * SOME + 1088}), ({}, {"v": 4 * SOME - 128}), ({}, {"slots": SOME + 8}), ({}, {"ks": TALL, "vs": TALL, "v": SOME + 128}),
    ({"head_step": 4096, "page_step": 8192}, {"k": 4 * SOME + 4096 + 1024}),
])
def test_packed_read_refuses_what_overlaps(L, change, at):
    p = dict(dict(slots=3 * SOME, pool=4 * SOME, k=SOME, v=2 * SOME, ks=ROWS, vs=ROWS), **at)
    refused(L.arrow_packed_read(ctypes.byref(packed(**change)), 3, *p.values(), 0), "pool: blocks" if "pool" not in at and change.get("page_step") == 1088 else "overlap")


@pytest.mark.parametrize("change,at", [({}, {"k": 4 * SOME + 1088}), ({}, {"v": 4 * SOME - 128}), ({}, {"slots": 4 * SOME + 16}), ({}, {"slots": 4 * SOME - 16})])
def test_packed_append_refuses_what_overlaps(L, change, at):
    p = dict(dict(k=SOME, v=2 * SOME, ks=ROWS, vs=ROWS, slots=3 * SOME, pool=4 * SOME), **at)
    refused(L.arrow_packed_append(ctypes.byref(packed(**change)), 3, *p.values(), 0), "overlap")


@pytest.mark.parametrize("change,at", [
    ({}, {"os": steps(64, 0, 64)}), ({}, {"os": steps(128, 0, 64)}), ({}, {"o": SOME + 512}), ({}, {"o": SOME - 512}), ({}, {"o": 2 * SOME + 256}), ({}, {"o": 3 * SOME - 256}),
    ({}, {"o": 4 * SOME + 1088}), ({}, {"k": 4 * SOME + 1088}), ({}, {"v": 4 * SOME + 16}), ({"table": 5 * SOME + 4}, {}), ({"lengths": 4 * SOME + 4}, {}),
    ({"columns": 100, "max_len": 1600, "batch": 1}, {"ws": 4 * SOME}), ({"columns": 100, "max_len": 1600, "batch": 1}, {"ws": SOME}),
])
def test_packed_decode_refuses_what_overlaps(L, change, at):
    c = packed(**dict({"table": 6 * SOME, "lengths": 7 * SOME}, **change))
    st = steps(256, 0, 64)
    p = dict(dict(q=SOME, qs=st, k=2 * SOME, v=3 * SOME, ks=ROWS, vs=ROWS, pool=4 * SOME, o=5 * SOME, os=st, ws=16 * SOME), **at)
    assert "ws" not in at or L.arrow_packed_decode_workspace_bytes(ctypes.byref(c)) > 0
    refused(L.arrow_packed_decode(ctypes.byref(c), *p.values(), 1 << 30, 0), "overlap")


@pytest.mark.parametrize("change", [{"batch": 1 << 22}, {"batch": 1 << 30}, {"batch": 1, "q_heads": 1 << 24}])
def test_packed_decode_refuses_more_rows_than_a_launch_has(L, change):
    """By name, before the new token's key and value are written."""
    c, st = packed(**dict({"table": 1 << 44, "lengths": 1 << 45}, **change)), steps(0, 0, 64)
    os = steps(64 * c.q_heads, 0, 64)
    refused(L.arrow_packed_decode(ctypes.byref(c), SOME, st, 2 * SOME, 3 * SOME, steps(0, 0, 64), steps(0, 0, 64), 4 * SOME, 1 << 46, os, 1 << 47, 1 << 40, 0), "2^24 - 1 rows")


def test_packed_decode_cuts_no_more_stretches_than_a_launch_has(L):
    c = packed(batch=(1 << 18) - 1, q_heads=64, kv_heads=1, columns=1 << 22, max_len=1 << 26)
    need = L.arrow_packed_decode_workspace_bytes(ctypes.byref(c))
    rows = c.batch * 4                                            # (of sixteen heads)
    assert need // (c.batch * 64 * 66 * 4) * rows * 256 < 1 << 32


@pytest.mark.parametrize("kind", [binding.arrow_attention_t, binding.arrow_cache_t, binding.arrow_embedding_t, binding.arrow_rotation_t, binding.arrow_pages_t, binding.arrow_packed_t,
                                  binding.arrow_logprobs_t])
def test_numbers_that_a_field_has_no_room_for(kind):
    """A table of 2^32 + 4 columns is none of four."""
    a = kind()
    for name, of in kind._fields_:
        if of in (ctypes.c_int32, ctypes.c_int64):
            most = 1 << (8 * ctypes.sizeof(of) - 1)
            for value in (most, 2 * most + 4, -most - 1):
                with pytest.raises(ValueError, match=name):
                    setattr(a, name, value)
                with pytest.raises(ValueError, match=name):
                    kind(**{name: value})
            for value in (most - 1, -most, 4):
                setattr(a, name, value)
                assert getattr(a, name) == value
