"""Page tables and slot maps of a cache in pages, kept on the GPU from the lengths of its sequences (``include/arrow_pages.h``), on torch tensors.

:class:`ArrowPages` knows the pool and the mask, and marshals arguments; a step runs in the library's HIP kernels, on the current stream of the tensors'
device, and the host sees none of it.  The table is the one that :class:`ArrowAttention` and :class:`ArrowPackedAttention` read, the slots are where
:class:`ArrowPackedAttention` writes.  Workspaces are torch's, taken for the time of a call.
"""
from __future__ import annotations

import ctypes

from . import binding
from .attention import _address, _results
from .binding import arrow_pages_t, lib


class ArrowPages:
    """A pool of ``pages`` pages of ``page`` tokens, for sequences of which a ``window`` (0: all) and the first ``sinks`` tokens stay visible."""

    def __init__(self, pages: int, page: int, window: int = 0, sinks: int = 0, device="cuda:0"):
        import torch
        self._torch = torch
        self.device = torch.device(device)
        self.pages, self.page, self.window, self.sinks = int(pages), int(page), int(window), int(sinks)
        if self.pages < 0 or self.page < 1 or self.page & (self.page - 1):
            raise ValueError(f"{pages} pages of {page} tokens: a power of two expected")
        if self.window < 0 or self.sinks < 0:
            raise ValueError("window and sinks are not negative")
        # the plain case goes by native code, as in attention.py
        self._call = binding._tensor_call(self.device)
        if self._call is not None:
            address = lambda name: binding._address(getattr(lib(), name))   # noqa: E731
            self._step = (address("arrow_pages_step"), address("arrow_pages_workspace_bytes"), self.device.index, self.pages, self.page,
                          min(self.window, 2**31 - 1), min(self.sinks, 2**31 - 1))

    def _stream(self) -> int:
        return binding._current_stream(self._torch, self.device)

    def state(self, batch: int, columns: int):
        """``(table, held, free)`` of ``batch`` empty sequences with room for ``columns`` pages each: all pages are free."""
        torch = self._torch
        table = torch.full((batch, columns), -1, dtype=torch.int32, device=self.device)
        held = torch.zeros(batch, dtype=torch.int32, device=self.device)
        free = torch.arange(self.pages, -1, -1, dtype=torch.int32, device=self.device)      # (how many, then they: the last one, page 0, is taken first)
        return table, held, free

    def step(self, table, held, free, lengths, tokens: int = 1, offsets=None, slots=None):
        """Take table, held and free to the new ``lengths``, int32 (batch), and return the places of the new tokens, int64: (batch, tokens), the last ``tokens`` of each
        sequence; or, with int32 offsets of batch + 1 values, (tokens) of all sequences together.  None where tokens is 0."""
        if self._call is not None:
            done = self._call.pages_step(*self._step, table, held, free, lengths, tokens, offsets, slots)
            if done is not None:
                done = _results(done)
                return done if tokens else None
        torch = self._torch
        if table.dim() != 2 or table.device.type != "cuda" or (self.device.index is not None and table.device != self.device):
            raise ValueError(f"table {tuple(table.shape)} on {table.device}: (sequences, columns) on {self.device} expected")
        batch, tokens = table.shape[0], int(tokens)
        if tokens < 0:
            raise ValueError(f"tokens = {tokens}")
        shapes = (("table", table, table.shape), ("held", held, (batch,)), ("free", free, (1 + self.pages,)), ("lengths", lengths, (batch,)),
                  ("offsets", offsets, (batch + 1,)))
        for name, t, shape in shapes:
            if t is not None and (t.dtype != torch.int32 or t.device != table.device or tuple(t.shape) != tuple(shape) or not t.is_contiguous()):
                raise ValueError(f"{name} {tuple(t.shape)} of {t.dtype} on {t.device}: contiguous int32 {tuple(shape)} on {table.device} expected")
        shape = (tokens,) if offsets is not None else (batch, tokens)
        if slots is None:
            slots = torch.empty(shape, dtype=torch.int64, device=table.device)
        elif slots.dtype != torch.int64 or slots.device != table.device or tuple(slots.shape) != shape or not slots.is_contiguous():
            raise ValueError(f"slots {tuple(slots.shape)} of {slots.dtype}: contiguous int64 {shape} on {table.device} expected")
        a = arrow_pages_t()
        a.batch, a.columns, a.page, a.pages = batch, table.shape[1], self.page, self.pages
        a.window, a.sinks = min(self.window, 2**31 - 1), min(self.sinks, 2**31 - 1)
        if offsets is not None:
            a.offsets, a.rows = offsets.data_ptr(), tokens
        else:
            a.tokens = tokens
        with torch.cuda.device(table.device):
            ws = torch.empty(lib().arrow_pages_workspace_bytes(ctypes.byref(a)), dtype=torch.uint8, device=table.device)
            binding._check(lib().arrow_pages_step(ctypes.byref(a), _address(lengths), _address(held), _address(table), _address(free), _address(slots), _address(ws),
                                                  ws.numel(), self._stream()))
        return slots if tokens else None
