"""What the entries on sequences refuse, and what they accept without work, without a GPU: no argument below reaches a kernel."""
import ctypes
import math

import pytest

from paper_2307_05740_amd import binding

SOME = 1 << 20                     # an address that nothing reads


@pytest.fixture()
def L():
    return binding.lib()


def attention(**change):
    a = binding.arrow_attention_t(dtype=binding.ARROW_BF16, batch=1, q_heads=4, kv_heads=2, dim=64, q_len=8, k_len=8, window=0, sinks=0, scale=1.0)
    for name in ("q", "o", "d_o", "dq"):
        setattr(a, name, binding.arrow_strides_t(8 * 256, 256, 64))
    for name in ("k", "v", "dk", "dv"):
        setattr(a, name, binding.arrow_strides_t(8 * 128, 128, 64))
    for name, value in change.items():
        setattr(a, name, value)
    return a


def cache(**change):
    c = binding.arrow_cache_t(dtype=binding.ARROW_BF16, batch=1, q_heads=4, kv_heads=2, dim=64, scale=1.0, page=16, columns=4, pages=4, max_len=64,
                              k_page=16 * 128, k_token=128, k_head=64, v_page=16 * 128, v_token=128, v_head=64, table=SOME, lengths=SOME)
    for name, value in change.items():
        setattr(c, name, value)
    return c


def embedding(**change):
    e = binding.arrow_embedding_t(dtype=binding.ARROW_BF16, grad_dtype=binding.ARROW_BF16, id_bytes=8, columns=64, rows=100, tokens=10, w_stride=64,
                                  y_stride=64, scale=1.0)
    for name, value in change.items():
        setattr(e, name, value)
    return e


def refused(rc, word):
    assert rc == binding.ARROW_EINVAL, rc
    assert word in binding.arrow_last_error(), binding.arrow_last_error()


@pytest.mark.parametrize("change,word", [
    ({"dtype": binding.ARROW_F32}, "dtype"), ({"dtype": 7}, "dtype"), ({"batch": -1}, "batch"), ({"q_heads": 3}, "q_heads"), ({"kv_heads": 0}, "kv_heads"),
    ({"dim": 4}, "dim"), ({"dim": 136}, "dim"), ({"dim": 65}, "dim"), ({"q_len": -1}, "q_len"), ({"k_len": 1 << 27}, "k_len"), ({"window": -1}, "window"),
    ({"sinks": -2}, "sinks"), ({"scale": 0.0}, "scale"), ({"scale": -1.0}, "scale"), ({"scale": math.nan}, "scale"), ({"scale": math.inf}, "scale"),
    ({"q_offsets": SOME}, "offsets"), ({"k_offsets": SOME}, "offsets"), ({"q_offsets": SOME, "k_offsets": SOME, "q_tokens": -1}, "q_tokens"),
    ({"q": binding.arrow_strides_t(0, 260, 64)}, "multiples of 8"), ({"k": binding.arrow_strides_t(0, 1 << 25, 64)}, "between tokens"),
    ({"v": binding.arrow_strides_t(0, -128, 64)}, "between tokens"), ({"o": binding.arrow_strides_t(0, 0, 64)}, "overlap"),
    ({"o": binding.arrow_strides_t(0, 256, 0)}, "overlap"), ({"batch": 2, "o": binding.arrow_strides_t(0, 256, 64)}, "overlap"),
])
def test_forward_refuses(L, change, word):
    a = attention(**change)
    refused(L.arrow_attention_forward(ctypes.byref(a), SOME, 2 * SOME, 3 * SOME, 4 * SOME, 5 * SOME, 0), word)


def test_forward_refuses_pointers(L):
    a = attention()
    for at, word in (((0, SOME, SOME, 2 * SOME), "q is NULL"), ((SOME, 0, SOME, 2 * SOME), "k is NULL"), ((SOME, SOME, 0, 2 * SOME), "v is NULL"),
                     ((SOME, SOME, SOME, 0), "o is NULL"), ((SOME + 2, SOME, SOME, 2 * SOME), "aligned"), ((SOME, SOME, SOME, SOME), "o is one of")):
        refused(L.arrow_attention_forward(ctypes.byref(a), *at, 0, 0), word)
    refused(L.arrow_attention_forward(None, SOME, SOME, SOME, SOME, 0, 0), "NULL")
    refused(L.arrow_attention_forward(ctypes.byref(a), SOME, SOME, SOME, 2 * SOME, SOME + 2, 0), "lse")
    for nothing in (attention(batch=0), attention(q_len=0)):
        assert L.arrow_attention_forward(ctypes.byref(nothing), 0, 0, 0, 0, 0, 0) == binding.ARROW_OK


def test_backward_refuses(L):
    a = attention()
    need = L.arrow_attention_workspace_bytes(ctypes.byref(a))
    assert need >= 4 * 8 * 4
    p = [i * SOME for i in range(1, 6)]                          # q k v o lse
    out = [i * SOME for i in range(7, 10)]
    call = lambda a, p, d_o, out, ws, n: L.arrow_attention_backward(ctypes.byref(a), *p, d_o, *out, ws, n, 0)   # noqa: E731
    refused(call(a, p, 0, out, 16 * SOME, need), "d_o is NULL")
    refused(call(a, p, 6 * SOME, [7 * SOME, 7 * SOME, 9 * SOME], 16 * SOME, need), "are the same")
    refused(call(a, p, 6 * SOME, [SOME, 8 * SOME, 9 * SOME], 16 * SOME, need), "are the same")
    refused(call(a, p[:4] + [0], 6 * SOME, out, 16 * SOME, need), "lse")
    refused(call(a, p, 6 * SOME, out, 0, need), "workspace")
    refused(call(a, p, 6 * SOME, out, 16 * SOME + 16, need), "workspace")
    assert call(a, p, 6 * SOME, out, 16 * SOME, need - 1) == binding.ARROW_ETOOSMALL
    for change, word in (({"dq": binding.arrow_strides_t(0, 0, 64)}, "dq"), ({"dk": binding.arrow_strides_t(0, 128, 4)}, "dk"),
                         ({"dv": binding.arrow_strides_t(0, 128, 0)}, "dv"), ({"dim": 0}, "dim")):
        refused(call(attention(**change), p, 6 * SOME, out, 16 * SOME, need), word)
    assert L.arrow_attention_workspace_bytes(None) == 0
    assert call(attention(batch=0), [0] * 5, 0, [0] * 3, 0, 0) == binding.ARROW_OK


def test_the_workspace_has_room_for_every_part(L):
    """Sums of parts: as many as there are for any length, window and number of first keys; 128 keys, dk and dv of 32 bits each."""
    for n in (1, 127, 128, 129, 1000, 5000):
        for window in (0, 1, 100, 2000):
            for sinks in (0, 1, 129, 6000):
                a = attention(q_len=n, k_len=n, window=window, sinks=sinks)
                need = L.arrow_attention_workspace_bytes(ctypes.byref(a))
                assert need >= 4 * n * 4 and need < 4 * n * 4 + 256 + (-(-n // 128)) * 64 * 2 * 2 * 128 * 64 * 4


@pytest.mark.parametrize("change,word", [
    ({"dtype": binding.ARROW_F32}, "dtype"), ({"dim": 12}, "dim"), ({"q_heads": 5}, "q_heads"), ({"page": 0}, "page"), ({"page": 24}, "page"),
    ({"page": 1 << 21}, "page"), ({"columns": -1}, "columns"), ({"columns": 1 << 23}, "columns"), ({"pages": -1}, "pages"), ({"max_len": -1}, "max_len"),
    ({"table": 0}, "table"), ({"lengths": 0}, "lengths"), ({"k_token": 100}, "k_pool"), ({"v_head": 8}, "v_pool"), ({"k_page": 0}, "k_pool"), ({"scale": 0.0}, "scale"),
    ({"window": -1}, "window"),
])
def test_cache_entries_refuse(L, change, word):
    c, st = cache(**change), binding.arrow_strides_t(256, 0, 64)
    kv = binding.arrow_strides_t(128, 128, 64)
    refused(L.arrow_attention_decode(ctypes.byref(c), SOME, st, 0, 0, kv, kv, 2 * SOME, 3 * SOME, 4 * SOME, st, 16 * SOME, 1 << 30, 0), word)
    refused(L.arrow_cache_append(ctypes.byref(c), 1, SOME, 5 * SOME, kv, kv, 2 * SOME, 3 * SOME, 0), word)


def test_cache_entries_refuse_pointers(L):
    c, st, kv = cache(), binding.arrow_strides_t(256, 0, 64), binding.arrow_strides_t(128, 128, 64)
    call = lambda q, k, v, kp, vp, o, ws=16 * SOME, n=1 << 30: L.arrow_attention_decode(ctypes.byref(c), q, st, k, v, kv, kv, kp, vp, o, st, ws, n, 0)   # noqa: E731
    refused(call(0, 0, 0, 2 * SOME, 3 * SOME, 4 * SOME), "q is NULL")
    refused(call(SOME, 0, 0, 0, 3 * SOME, 4 * SOME), "k_pool is NULL")
    refused(call(SOME, 0, 0, 2 * SOME, 2 * SOME, 4 * SOME), "the same")
    refused(call(SOME, SOME, 0, 2 * SOME, 3 * SOME, 4 * SOME), "both or neither")
    refused(call(SOME, 5 * SOME, 6 * SOME + 8, 2 * SOME, 3 * SOME, 4 * SOME), "v is not")
    refused(call(SOME, 0, 0, 2 * SOME, 3 * SOME, SOME), "o is one of")
    refused(call(SOME, 0, 0, 2 * SOME, 3 * SOME, 0), "o is NULL")
    big = cache(max_len=100_000, columns=8192)
    need = L.arrow_attention_decode_workspace_bytes(ctypes.byref(big))
    assert need > 0
    rc = L.arrow_attention_decode(ctypes.byref(big), SOME, st, 0, 0, kv, kv, 2 * SOME, 3 * SOME, 4 * SOME, st, 16 * SOME, need - 1, 0)
    assert rc == binding.ARROW_ETOOSMALL
    refused(L.arrow_cache_append(ctypes.byref(c), -1, SOME, 5 * SOME, kv, kv, 2 * SOME, 3 * SOME, 0), "tokens")
    refused(L.arrow_cache_append(ctypes.byref(c), 1, 0, 5 * SOME, kv, kv, 2 * SOME, 3 * SOME, 0), "k is NULL")
    assert L.arrow_cache_append(ctypes.byref(c), 0, 0, 0, kv, kv, 2 * SOME, 3 * SOME, 0) == binding.ARROW_OK
    empty = cache(batch=0)
    assert L.arrow_attention_decode(ctypes.byref(empty), 0, st, 0, 0, kv, kv, 0, 0, 0, st, 0, 0, 0) == binding.ARROW_OK
    assert L.arrow_attention_decode_workspace_bytes(None) == 0


@pytest.mark.parametrize("change,word", [
    ({"dtype": 9}, "dtype"), ({"id_bytes": 2}, "id_bytes"), ({"columns": 0}, "columns"), ({"rows": 0}, "rows"), ({"rows": 1 << 31}, "rows"),
    ({"tokens": -1}, "tokens"), ({"tokens": 1 << 31}, "tokens"), ({"w_stride": 63}, "apart"), ({"y_stride": 1}, "apart"), ({"scale": math.nan}, "scale"),
])
def test_embedding_refuses(L, change, word):
    e = embedding(**change)
    refused(L.arrow_embedding_forward(ctypes.byref(e), SOME, 2 * SOME, 3 * SOME, 0), word)
    refused(L.arrow_embedding_backward(ctypes.byref(e), SOME, 2 * SOME, 3 * SOME, 16 * SOME, 1 << 30, 0), word)
    assert L.arrow_embedding_workspace_bytes(ctypes.byref(e)) == 0


def test_embedding_refuses_pointers(L):
    e = embedding()
    forward = lambda *p: L.arrow_embedding_forward(ctypes.byref(e), *p, 0)   # noqa: E731
    refused(forward(0, 2 * SOME, 3 * SOME), "W is NULL")
    refused(forward(SOME, 0, 3 * SOME), "ids is NULL")
    refused(forward(SOME, 2 * SOME, 0), "Y is NULL")
    refused(forward(SOME + 1, 2 * SOME, 3 * SOME), "aligned")
    refused(forward(SOME, 2 * SOME + 4, 3 * SOME), "aligned")
    refused(forward(SOME, 2 * SOME, SOME + 100 * 128 - 2), "overlaps")
    refused(forward(SOME, 2 * SOME, 2 * SOME + 64), "overlaps")
    need = L.arrow_embedding_workspace_bytes(ctypes.byref(e))
    back = lambda dY, ids, dW, ws, n: L.arrow_embedding_backward(ctypes.byref(e), dY, ids, dW, ws, n, 0)   # noqa: E731
    refused(back(SOME, 2 * SOME, 0, 16 * SOME, need), "dW is NULL")
    refused(back(SOME, 2 * SOME, 3 * SOME, 0, need), "workspace")
    refused(back(SOME, 2 * SOME, 3 * SOME, 16 * SOME + 8, need), "workspace")
    assert back(SOME, 2 * SOME, 3 * SOME, 16 * SOME, need - 1) == binding.ARROW_ETOOSMALL
    refused(back(SOME, 2 * SOME, SOME, 16 * SOME, need), "overlaps")
    refused(back(SOME, 2 * SOME, 16 * SOME, 16 * SOME, need), "overlaps")
    refused(back(0, 2 * SOME, 3 * SOME, 16 * SOME, need), "dY is NULL")
    e.grad_dtype = binding.ARROW_F16
    refused(back(SOME, 2 * SOME, 3 * SOME, 16 * SOME, need), "grad_dtype")
    nothing = embedding(tokens=0)
    assert L.arrow_embedding_forward(ctypes.byref(nothing), 0, 0, 0, 0) == binding.ARROW_OK


def test_classes_refuse_tensors():
    import torch

    from paper_2307_05740_amd.attention import ArrowAttention
    from paper_2307_05740_amd.embedding import ArrowEmbedding
    with pytest.raises(ValueError):
        ArrowAttention(window=-1)
    q = torch.zeros(1, 4, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="is on cpu"):
        ArrowAttention().forward(q, q, q)
    with pytest.raises(ValueError, match="expected"):
        ArrowAttention().forward(q[0], q, q)
    with pytest.raises(ValueError, match="both or neither"):
        ArrowAttention().forward(q[0], q[0], q[0], q_offsets=torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError, match="on cpu"):
        ArrowAttention().decode(q[0], q, q, torch.zeros(1, 1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32))
    with pytest.raises(ValueError):
        ArrowEmbedding(0)
    with pytest.raises(ValueError, match="on cpu"):
        ArrowEmbedding(4).forward(torch.zeros(4, 8), torch.zeros(3, dtype=torch.int64))
    with pytest.raises(ValueError, match="ids"):
        ArrowEmbedding(4).forward(torch.zeros(4, 8), torch.zeros(3, dtype=torch.int16))
    with pytest.raises(TypeError):
        ArrowEmbedding(4).forward(torch.zeros(4, 8, dtype=torch.float64), torch.zeros(3, dtype=torch.int64))


def test_workspaces_of_any_number_of_tokens(L):
    """None, one, and those around the sizes at which the sort or the chunks of the sums change."""
    for tokens in (0, 1, 7, 8, 9, 4096, 4097, 65535, 65536, 1_000_000, 1 << 30):
        for rows in (1, 2, 32767, 32768, 2**31 - 2):
            e = embedding(tokens=tokens, rows=rows)
            assert L.arrow_embedding_workspace_bytes(ctypes.byref(e)) >= 4 * (rows + 4 * tokens)


def test_forward_in_a_workspace(L):
    """Refusals of the forward call that cuts keys, and what it needs."""
    few = attention(q_len=16, k_len=9000)
    need = L.arrow_attention_forward_split_bytes(ctypes.byref(few))
    assert need > 0 and need % 256 == 0
    at = (1 * SOME, 2 * SOME, 3 * SOME, 4 * SOME, 5 * SOME)
    refused(L.arrow_attention_forward_split(ctypes.byref(few), *at, 0, need, 0), "workspace")
    refused(L.arrow_attention_forward_split(ctypes.byref(few), *at, 6 * SOME + 16, need, 0), "workspace")
    assert L.arrow_attention_forward_split(ctypes.byref(few), *at, 6 * SOME, need - 1, 0) == binding.ARROW_ETOOSMALL
    refused(L.arrow_attention_forward_split(None, *at, 0, 0, 0), "NULL")
    for whole in (attention(q_len=16, k_len=100), attention(q_len=0, k_len=9000), attention(q_len=4000, k_len=4000, window=100)):
        assert L.arrow_attention_forward_split_bytes(ctypes.byref(whole)) == 0
    assert L.arrow_attention_forward_split_bytes(None) == 0
