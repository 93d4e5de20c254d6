"""Attention under an arrow-shaped mask (``include/arrow_attention.h``) on torch tensors.

Key j is visible to query i, at position p = i + keys - queries of its sequence, where j <= p and (no window, or
j > p - window, or j < sinks): a band and a first block column.  :class:`ArrowAttention` holds the mask and marshals arguments; every
step runs in the library's HIP kernels, on the current stream of the tensors' device.  Tensors that another stream has written or
will free are the caller's to order, as with torch's own operators.  Workspaces are torch's, taken for the time of a call.
"""
from __future__ import annotations

import ctypes
import math

from . import binding
from .binding import arrow_attention_t, arrow_cache_t, arrow_strides_t, lib


def _dtype_of(torch, dtype) -> int:
    if dtype == torch.bfloat16:
        return binding.ARROW_BF16
    if dtype == torch.float16:
        return binding.ARROW_F16
    raise TypeError(f"attention takes bfloat16 and float16 tensors, not {dtype}")


def _address(t) -> int:
    return t.data_ptr() if t is not None else 0


def _results(done):
    """What a native call gave: results, or the library's error code."""
    if type(done) is int:
        binding._check(done)
    return done


class ArrowAttention:
    """A mask (``window`` keys back, 0 = all earlier ones, and the first ``sinks`` keys) and a scale of the scores, by
    default 1 / sqrt(size of a head)."""

    def __init__(self, window: int = 0, sinks: int = 0, scale: float | None = None, device="cuda:0"):
        import torch
        self._torch = torch
        self.device = torch.device(device)
        self.window, self.sinks, self.scale = int(window), int(sinks), scale
        if self.window < 0 or self.sinks < 0:
            raise ValueError("window and sinks are not negative")
        # The plain case, tensors that are what they have to be, is looked over and started in native code (csrc/tensor_call.cpp); it
        # says None to anything else, which then goes the way below and is reported there.
        self._call = binding._tensor_call(self.device)
        mask = (self.device.index, min(self.window, 2**31 - 1), min(self.sinks, 2**31 - 1), -1.0 if scale is None else max(0.0, float(scale)))
        address = lambda name: binding._address(getattr(lib(), name))   # noqa: E731
        if self._call is not None:
            self._forward = (address("arrow_attention_forward_split"), address("arrow_attention_forward_split_bytes"), *mask)
            self._backward = (address("arrow_attention_backward"), address("arrow_attention_workspace_bytes"), *mask)
            self._decode = (address("arrow_attention_decode"), address("arrow_attention_decode_workspace_bytes"), *mask)

    def _stream(self) -> int:
        return binding._current_stream(self._torch, self.device)

    def _on_device(self):
        return self._torch.cuda.device(self.device)

    def _check(self, like, **tensors) -> None:
        """Device, type and innermost step of what is not None."""
        for name, t in tensors.items():
            if t is None:
                continue
            if t.device != like.device or t.dtype != like.dtype:
                raise ValueError(f"{name}: {t.dtype} on {t.device}, {like.dtype} on {like.device} expected")
            if t.shape[-1] > 1 and t.stride(-1) != 1 and t.numel():
                raise ValueError(f"{name}: the elements of a head do not lie next to each other")

    # ---- whole sequences --------------------------------------------------------------------------------------------
    def _describe(self, q, k, v, q_offsets, k_offsets, q_len, k_len) -> arrow_attention_t:
        torch = self._torch
        ragged = q_offsets is not None
        if (k_offsets is None) == ragged:
            raise ValueError("offsets of queries and keys: both or neither")
        if q.dim() != (3 if ragged else 4) or k.dim() != q.dim() or v.shape != k.shape or k.shape[-1] != q.shape[-1]:
            raise ValueError(f"q {tuple(q.shape)}, k {tuple(k.shape)}, v {tuple(v.shape)}: "
                             + ("(tokens, heads, dim) expected" if ragged else "(batch, tokens, heads, dim) expected"))
        if q.device.type != "cuda" or (self.device.index is not None and q.device != self.device):
            raise ValueError(f"q is on {q.device}, this mask on {self.device}")
        self._check(q, q=q, k=k, v=v)
        a = arrow_attention_t()
        a.dtype = _dtype_of(torch, q.dtype)
        a.q_heads, a.kv_heads, a.dim = q.shape[-2], k.shape[-2], q.shape[-1]
        a.window, a.sinks = min(self.window, 2**31 - 1), min(self.sinks, 2**31 - 1)
        a.scale = self.scale if self.scale is not None else 1.0 / math.sqrt(max(1, a.dim))
        if ragged:
            for name, t in (("q_offsets", q_offsets), ("k_offsets", k_offsets)):
                if t.dtype != torch.int32 or t.device != q.device or t.dim() != 1 or not t.is_contiguous() or t.shape != q_offsets.shape or not t.numel():
                    raise ValueError(f"{name}: one int32 more than there are sequences, on {q.device}")
            a.batch = q_offsets.shape[0] - 1
            a.q_tokens, a.k_tokens = q.shape[0], k.shape[0]
            a.q_len = min(q.shape[0], int(q_len)) if q_len is not None else q.shape[0]
            a.k_len = min(k.shape[0], int(k_len)) if k_len is not None else k.shape[0]
            a.q_offsets, a.k_offsets = q_offsets.data_ptr(), k_offsets.data_ptr()
        else:
            if q_len is not None or k_len is not None:
                raise ValueError("q_len and k_len go with offsets")
            if q.shape[0] != k.shape[0]:
                raise ValueError(f"{q.shape[0]} sequences of queries, {k.shape[0]} of keys")
            a.batch, a.q_len, a.k_len = q.shape[0], q.shape[1], k.shape[1]
        for name, t in (("q", q), ("k", k), ("v", v)):
            self._steps(a, name, t)
        return a

    @staticmethod
    def _steps(a, name: str, t) -> None:
        """Steps of an operand; one that is never taken counts as none."""
        s, n = t.stride(), t.shape
        st = getattr(a, name)
        st.sequence = s[0] if t.dim() == 4 and n[0] > 1 else 0
        st.token = s[-3] if n[-3] > 1 else 0
        st.head = s[-2] if n[-2] > 1 else 0

    def _lse_shape(self, a, q):
        return (a.q_heads, q.shape[0]) if q.dim() == 3 else (a.batch, a.q_heads, a.q_len)

    def forward(self, q, k, v, o=None, lse=None, q_offsets=None, k_offsets=None, q_len=None, k_len=None):
        """``(o, lse)``.  q: (batch, tokens, heads, dim), k and v: (batch, keys, key heads, dim); or, with int32 offsets of
        batch + 1 values each, (tokens of all sequences, heads, dim), of which no sequence has more than q_len (k_len); without these the work, and the
        gradients' workspace, are laid out as if each sequence might have all tokens.
        lse: float32, (batch, heads, tokens), or (heads, tokens of all sequences).  Results of tokens that no sequence has are not written."""
        if self._call is not None:
            done = self._call.attention_forward(*self._forward, q, k, v, o, lse, q_offsets, k_offsets, q_len, k_len)
            if done is not None:
                return _results(done)
        torch = self._torch
        a = self._describe(q, k, v, q_offsets, k_offsets, q_len, k_len)
        if o is None:
            o = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        if lse is None:
            lse = torch.empty(self._lse_shape(a, q), dtype=torch.float32, device=q.device)
        if o.shape != q.shape or lse.shape != self._lse_shape(a, q) or lse.dtype != torch.float32 or lse.device != q.device or not lse.is_contiguous():
            raise ValueError(f"o {tuple(o.shape)} or lse {tuple(lse.shape)} of {lse.dtype}: {tuple(q.shape)} and contiguous float32 "
                             f"{self._lse_shape(a, q)} expected")
        self._check(q, o=o)
        self._steps(a, "o", o)
        with self._on_device():
            ws = torch.empty(lib().arrow_attention_forward_split_bytes(ctypes.byref(a)), dtype=torch.uint8, device=q.device)
            binding._check(lib().arrow_attention_forward_split(ctypes.byref(a), _address(q), _address(k), _address(v), _address(o), _address(lse), _address(ws),
                                                               ws.numel(), self._stream()))
        return o, lse

    def backward(self, d_o, q, k, v, o, lse, dq=None, dk=None, dv=None, q_offsets=None, k_offsets=None, q_len=None, k_len=None):
        """``(dq, dk, dv)`` for the gradient d_o of the o that ``forward`` gave for these arguments together with lse.  Those of tokens that no
        sequence has are not written."""
        if self._call is not None:
            done = self._call.attention_backward(*self._backward, d_o, q, k, v, o, lse, dq, dk, dv, q_offsets, k_offsets, q_len, k_len)
            if done is not None:
                return _results(done)
        torch = self._torch
        a = self._describe(q, k, v, q_offsets, k_offsets, q_len, k_len)
        dq = torch.empty(q.shape, dtype=q.dtype, device=q.device) if dq is None else dq
        dk = torch.empty(k.shape, dtype=k.dtype, device=k.device) if dk is None else dk
        dv = torch.empty(v.shape, dtype=v.dtype, device=v.device) if dv is None else dv
        for name, t, like in (("d_o", d_o, q), ("o", o, q), ("dq", dq, q), ("dk", dk, k), ("dv", dv, v)):
            if t.shape != like.shape:
                raise ValueError(f"{name} {tuple(t.shape)}: {tuple(like.shape)} expected")
            self._check(q, **{name: t})
            self._steps(a, name, t)
        if lse.shape != self._lse_shape(a, q) or lse.dtype != torch.float32 or lse.device != q.device or not lse.is_contiguous():
            raise ValueError(f"lse {tuple(lse.shape)} of {lse.dtype}: contiguous float32 {self._lse_shape(a, q)} expected")
        with self._on_device():
            ws = torch.empty(lib().arrow_attention_workspace_bytes(ctypes.byref(a)), dtype=torch.uint8, device=q.device)
            binding._check(lib().arrow_attention_backward(
                ctypes.byref(a), _address(q), _address(k), _address(v), _address(o), _address(lse), _address(d_o), _address(dq), _address(dk),
                _address(dv), _address(ws), ws.numel(), self._stream()))
        return dq, dk, dv

    def __call__(self, q, k, v, q_offsets=None, k_offsets=None, q_len=None, k_len=None):
        """o as ``forward`` gives it, with its gradient for torch's autograd.  Tokens that no sequence has get zeros in both."""
        return _attention_function().apply(self, q, k, v, q_offsets, k_offsets, q_len, k_len)

    # ---- a cache in pages ---------------------------------------------------------------------------------------------
    def _cache(self, k_cache, v_cache, table, lengths, q_heads: int, max_len) -> arrow_cache_t:
        torch = self._torch
        if k_cache.dim() != 4 or v_cache.shape != k_cache.shape:
            raise ValueError(f"pools {tuple(k_cache.shape)} and {tuple(v_cache.shape)}: (pages, tokens of a page, heads, dim) expected")
        if k_cache.device.type != "cuda" or (self.device.index is not None and k_cache.device != self.device):
            raise ValueError(f"the cache is on {k_cache.device}, this mask on {self.device}")
        self._check(k_cache, k_cache=k_cache, v_cache=v_cache)
        for name, t, dims in (("table", table, 2), ("lengths", lengths, 1)):
            if t.dtype != torch.int32 or t.device != k_cache.device or t.dim() != dims or not t.is_contiguous():
                raise ValueError(f"{name}: contiguous int32 of {dims} dimension(s) on {k_cache.device} expected")
        if table.shape[0] != lengths.shape[0]:
            raise ValueError(f"a table of {table.shape[0]} sequences, {lengths.shape[0]} lengths")
        c = arrow_cache_t()
        c.dtype = _dtype_of(torch, k_cache.dtype)
        c.batch, c.columns = table.shape
        c.pages, c.page, c.kv_heads, c.dim = k_cache.shape
        c.q_heads = q_heads
        c.window, c.sinks = min(self.window, 2**31 - 1), min(self.sinks, 2**31 - 1)
        c.scale = self.scale if self.scale is not None else 1.0 / math.sqrt(max(1, c.dim))
        c.max_len = c.columns * c.page if max_len is None else int(max_len)
        for m, t in (("k", k_cache), ("v", v_cache)):
            for i, step in enumerate(("page", "token", "head")):
                setattr(c, f"{m}_{step}", t.stride(i) if t.shape[i] > 1 else 0)
        c.table, c.lengths = table.data_ptr(), lengths.data_ptr()
        return c

    def append(self, k, v, k_cache, v_cache, table, lengths) -> None:
        """Write k and v, (batch, tokens, key heads, dim), to the last places of the sequences: lengths, int32, count them.
        Pools: (pages, tokens of a page, key heads, dim); token t of sequence b is in page table[b, t // size], int32."""
        c = self._cache(k_cache, v_cache, table, lengths, k_cache.shape[-2], None)
        if k.dim() != 4 or v.shape != k.shape or k.shape[0] != c.batch or tuple(k.shape[2:]) != tuple(k_cache.shape[2:]):
            raise ValueError(f"k {tuple(k.shape)}, v {tuple(v.shape)}: ({c.batch}, tokens, {c.kv_heads}, {c.dim}) expected")
        self._check(k_cache, k=k, v=v)
        steps = arrow_attention_t()
        self._steps(steps, "k", k)
        self._steps(steps, "v", v)
        with self._on_device():
            binding._check(lib().arrow_cache_append(ctypes.byref(c), k.shape[1], _address(k), _address(v), steps.k, steps.v, _address(k_cache),
                                                    _address(v_cache), self._stream()))

    def decode(self, q, k_cache, v_cache, table, lengths, max_len=None, k=None, v=None, o=None):
        """o of one query per sequence, q: (batch, heads, dim), at the last of its lengths[b] positions (0: an idle sequence).  k and v,
        (batch, key heads, dim): the new token's, written to their place first (of a sequence longer than its row of the table, left out); without them they are there already.
        max_len: the longest length; only how the work is split goes by it."""
        if self._call is not None:
            done = self._call.attention_decode(*self._decode, q, k_cache, v_cache, table, lengths, max_len, k, v, o)
            if done is not None:
                return _results(done)
        torch = self._torch
        if q.dim() != 3:
            raise ValueError(f"q {tuple(q.shape)}: (batch, heads, dim) expected")
        c = self._cache(k_cache, v_cache, table, lengths, q.shape[1], max_len)
        o = torch.empty(q.shape, dtype=q.dtype, device=q.device) if o is None else o
        if q.shape[0] != c.batch or q.shape[2] != c.dim or o.shape != q.shape:
            raise ValueError(f"q {tuple(q.shape)}, o {tuple(o.shape)}: ({c.batch}, heads, {c.dim}) expected")
        if (k is None) != (v is None):
            raise ValueError("k and v of the new token: both or neither")
        for name, t in (("k", k), ("v", v)):
            if t is not None and tuple(t.shape) != (c.batch, c.kv_heads, c.dim):
                raise ValueError(f"{name} {tuple(t.shape)}: ({c.batch}, {c.kv_heads}, {c.dim}) expected")
        self._check(k_cache, q=q, k=k, v=v, o=o)
        steps = [arrow_strides_t(t.stride(0) if t.shape[0] > 1 else 0, 0, t.stride(1) if t.shape[1] > 1 else 0) if t is not None else arrow_strides_t()
                 for t in (q, k, v, o)]
        with self._on_device():
            ws = torch.empty(lib().arrow_attention_decode_workspace_bytes(ctypes.byref(c)), dtype=torch.uint8, device=q.device)
            binding._check(lib().arrow_attention_decode(ctypes.byref(c), _address(q), steps[0], _address(k), _address(v), steps[1], steps[2],
                                                        _address(k_cache), _address(v_cache), _address(o), steps[3], _address(ws), ws.numel(),
                                                        self._stream()))
        return o


_function = None


def _attention_function():
    """The call as a node of torch's autograd."""
    global _function
    if _function is None:
        import torch

        def blank(t, q_offsets):
            """Zeros for the tokens that no sequence of a ragged batch has: what is there goes into products with other gradients."""
            return torch.zeros(t.shape, dtype=t.dtype, device=t.device) if q_offsets is not None else None

        class Attention(torch.autograd.Function):
            @staticmethod
            def forward(ctx, op, q, k, v, *lengths):
                o, lse = op.forward(q, k, v, blank(q, lengths[0]), None, *lengths)
                ctx.save_for_backward(q, k, v, o, lse, *lengths[:2])
                ctx.op, ctx.limits = op, lengths[2:]
                return o

            @staticmethod
            @torch.autograd.function.once_differentiable
            def backward(ctx, d_o):
                q, k, v, o, lse, *offsets = ctx.saved_tensors
                if d_o.stride(-1) != 1 or d_o.data_ptr() % 16 or any(s % 8 for s in d_o.stride()[:-1]):
                    d_o = d_o.clone(memory_format=torch.contiguous_format)
                grads = (blank(t, offsets[0]) for t in (q, k, v))
                return None, *ctx.op.backward(d_o, q, k, v, o, lse, *grads, *offsets, *ctx.limits), None, None, None, None

        _function = Attention
    return _function
