"""A cache of keys and values in 4 bits and the attention of single tokens over it (``include/arrow_packed.h``), on torch tensors.

The mask is :class:`ArrowAttention`'s.  A pool is one uint8 tensor, (pages, key heads, bytes of a page); tokens go to it and come from it by slots, page * tokens of a page +
token, as :class:`ArrowPages` gives them.  :class:`ArrowPackedAttention` marshals arguments; every step runs in the library's HIP kernels, on the
current stream of the tensors' device.  Workspaces are torch's, taken for the time of a call.
"""
from __future__ import annotations

import ctypes
import math

from . import binding
from .attention import _address, _dtype_of, _results
from .binding import arrow_packed_t, arrow_strides_t, lib


class ArrowPackedAttention:
    """A mask (``window`` keys back, 0 = all earlier ones, and the first ``sinks`` keys) and a scale of the scores, by default 1 / sqrt(size of a head)."""

    def __init__(self, window: int = 0, sinks: int = 0, scale: float | None = None, device="cuda:0"):
        import torch
        self._torch = torch
        self.device = torch.device(device)
        self.window, self.sinks, self.scale = int(window), int(sinks), scale
        if self.window < 0 or self.sinks < 0:
            raise ValueError("window and sinks are not negative")
        # the plain case goes by native code, as in attention.py
        self._call = binding._tensor_call(self.device)
        if self._call is not None:
            address = lambda name: binding._address(getattr(lib(), name))   # noqa: E731
            self._append = (address("arrow_packed_append"), self.device.index)
            self._read = (address("arrow_packed_read"), self.device.index)
            self._decode = (address("arrow_packed_decode"), address("arrow_packed_decode_workspace_bytes"), self.device.index, min(self.window, 2**31 - 1),
                            min(self.sinks, 2**31 - 1), -1.0 if scale is None else max(0.0, float(scale)))

    def _stream(self) -> int:
        return binding._current_stream(self._torch, self.device)

    def pool(self, pages: int, page: int, kv_heads: int, dim: int):
        """Room for ``pages`` pages of ``page`` tokens (a power of two, 16 or more), of heads of 32, 64 or 128 elements."""
        return self._torch.zeros((pages, kv_heads, page * (dim + dim // 16)), dtype=self._torch.uint8, device=self.device)

    def _describe(self, pool, dim: int, dtype) -> arrow_packed_t:
        torch = self._torch
        if dim not in (32, 64, 128):
            raise ValueError(f"heads of {dim}: 32, 64 or 128 expected")
        size = dim + dim // 16
        if pool.dtype != torch.uint8 or pool.dim() != 3 or pool.shape[2] % size or (pool.shape[2] > 1 and pool.stride(2) != 1 and pool.numel()):
            raise ValueError(f"pool {tuple(pool.shape)} of {pool.dtype}: uint8 (pages, key heads, {size} x tokens of a page) expected")
        if pool.device.type != "cuda" or (self.device.index is not None and pool.device != self.device):
            raise ValueError(f"the pool is on {pool.device}, this mask on {self.device}")
        c = arrow_packed_t()
        c.dtype = _dtype_of(torch, dtype)
        c.pages, c.kv_heads, c.page, c.dim = pool.shape[0], pool.shape[1], pool.shape[2] // size, dim
        c.page_step, c.head_step = (pool.stride(i) if pool.shape[i] > 1 else 0 for i in (0, 1))
        return c

    def _rows(self, name, t, shape, dtype, device) -> arrow_strides_t:
        """Steps of (rows, heads, dim); one that is never taken counts as none."""
        if t.dtype != dtype or t.device != device or tuple(t.shape) != tuple(shape):
            raise ValueError(f"{name} {tuple(t.shape)} of {t.dtype} on {t.device}: {tuple(shape)} of {dtype} on {device} expected")
        if t.stride(-1) != 1 and t.numel():
            raise ValueError(f"{name}: the elements of a head do not lie next to each other")
        row, head = (t.stride(i) if t.shape[i] > 1 else 0 for i in (0, 1))
        return arrow_strides_t(row, row, head)

    def _places(self, slots, pool):
        torch = self._torch
        if slots.dtype != torch.int64 or slots.device != pool.device or slots.dim() != 1 or not slots.is_contiguous():
            raise ValueError(f"slots {tuple(slots.shape)} of {slots.dtype} on {slots.device}: contiguous int64 of one dimension on {pool.device} expected")

    def append(self, k, v, pool, slots) -> None:
        """Write k and v, (tokens, key heads, dim), to slots, int64 (tokens); tokens whose slot is not in the pool (-1) are left out.  No slot comes twice."""
        if self._call is not None:
            done = self._call.packed_append(*self._append, k, v, pool, slots)
            if done is not None:
                _results(done)
                return
        torch = self._torch
        if k.dim() != 3:
            raise ValueError(f"k {tuple(k.shape)}: (tokens, key heads, dim) expected")
        c = self._describe(pool, k.shape[-1], k.dtype)
        self._places(slots, pool)
        shape = (slots.shape[0], c.kv_heads, c.dim)
        ks, vs = (self._rows(n, t, shape, k.dtype, pool.device) for n, t in (("k", k), ("v", v)))
        with torch.cuda.device(pool.device):
            binding._check(lib().arrow_packed_append(ctypes.byref(c), slots.shape[0], _address(k), _address(v), ks, vs, _address(slots), _address(pool),
                                                     self._stream()))

    def read(self, pool, slots, dim: int, dtype, k=None, v=None):
        """``(k, v)``, (tokens, key heads, dim) of ``dtype``, from slots; zeros where a slot is not in the pool."""
        if self._call is not None:
            done = self._call.packed_read(*self._read, pool, slots, dim, dtype, k, v)
            if done is not None:
                return _results(done)
        torch = self._torch
        c = self._describe(pool, dim, dtype)
        self._places(slots, pool)
        shape = (slots.shape[0], c.kv_heads, dim)
        k = torch.empty(shape, dtype=dtype, device=pool.device) if k is None else k
        v = torch.empty(shape, dtype=dtype, device=pool.device) if v is None else v
        ks, vs = (self._rows(n, t, shape, dtype, pool.device) for n, t in (("k", k), ("v", v)))
        with torch.cuda.device(pool.device):
            binding._check(lib().arrow_packed_read(ctypes.byref(c), slots.shape[0], _address(slots), _address(pool), _address(k), _address(v), ks, vs,
                                                   self._stream()))
        return k, v

    def decode(self, q, pool, table, lengths, max_len=None, k=None, v=None, o=None):
        """o of one query per sequence, q: (batch, heads, dim), at the last of its lengths[b] positions (0: an idle sequence).  k and v, (batch, key heads, dim): the new
        token's, written to their place first (of a sequence longer than its row of the table, left out); without them they are there already.
        max_len: the longest length; only how the work is split goes by it."""
        if self._call is not None:
            done = self._call.packed_decode(*self._decode, q, pool, table, lengths, max_len, k, v, o)
            if done is not None:
                return _results(done)
        torch = self._torch
        if q.dim() != 3:
            raise ValueError(f"q {tuple(q.shape)}: (batch, heads, dim) expected")
        c = self._describe(pool, q.shape[-1], q.dtype)
        for name, t, dims in (("table", table, 2), ("lengths", lengths, 1)):
            if t.dtype != torch.int32 or t.device != pool.device or t.dim() != dims or not t.is_contiguous() or t.shape[0] != q.shape[0]:
                raise ValueError(f"{name} {tuple(t.shape)}: contiguous int32 of {dims} dimension(s) for {q.shape[0]} sequences on {pool.device} expected")
        c.batch, c.columns = table.shape
        c.q_heads = q.shape[1]
        c.window, c.sinks = min(self.window, 2**31 - 1), min(self.sinks, 2**31 - 1)
        c.scale = self.scale if self.scale is not None else 1.0 / math.sqrt(c.dim)
        c.max_len = c.columns * c.page if max_len is None else int(max_len)
        c.table, c.lengths = table.data_ptr(), lengths.data_ptr()
        if (k is None) != (v is None):
            raise ValueError("k and v of the new token: both or neither")
        o = torch.empty(q.shape, dtype=q.dtype, device=q.device) if o is None else o
        own = (c.batch, c.kv_heads, c.dim)
        steps = [self._rows(n, t, shape, q.dtype, pool.device) if t is not None else arrow_strides_t()
                 for n, t, shape in (("q", q, q.shape), ("k", k, own), ("v", v, own), ("o", o, q.shape))]
        with torch.cuda.device(pool.device):
            ws = torch.empty(lib().arrow_packed_decode_workspace_bytes(ctypes.byref(c)), dtype=torch.uint8, device=pool.device)
            binding._check(lib().arrow_packed_decode(ctypes.byref(c), _address(q), steps[0], _address(k), _address(v), steps[1], steps[2], _address(pool),
                                                     _address(o), steps[3], _address(ws), ws.numel(), self._stream()))
        return o
