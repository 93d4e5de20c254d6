"""Embedding lookup with scaling, and its gradient by sorted tokens (``include/arrow_embedding.h``), on torch tensors.

``Y[t] = scale W[ids[t]]`` and ``dW[v] = scale sum of dY[t] over ids[t] = v``; ids outside the table are padding: zero rows, added
to nothing.  :class:`ArrowEmbedding` marshals arguments; every step runs in the library's HIP kernels, on the current stream of the
tensors' device.  Workspaces are torch's, taken for the time of a call.
"""
from __future__ import annotations

import ctypes
import math

from . import binding
from .attention import _results
from .binding import arrow_embedding_t, lib


class ArrowEmbedding:
    """A table of ``rows`` rows and a scale of what is looked up in it."""

    def __init__(self, rows: int, scale: float = 1.0, device="cuda:0"):
        import torch
        self._torch = torch
        self.device = torch.device(device)
        self.rows, self.scale = int(rows), float(scale)
        if self.rows < 1:
            raise ValueError("a table has rows")
        # the plain case goes by native code, as in attention.py
        self._call = binding._tensor_call(self.device)
        if self._call is not None:
            address = lambda name: binding._address(getattr(lib(), name))   # noqa: E731
            self._forward = (address("arrow_embedding_forward"), self.device.index, self.rows, self.scale)
            self._backward = (address("arrow_embedding_backward"), address("arrow_embedding_workspace_bytes"), self.device.index, self.rows, self.scale)
        self._dtypes = {torch.float32: binding.ARROW_F32, torch.bfloat16: binding.ARROW_BF16, torch.float16: binding.ARROW_F16}

    def _stream(self) -> int:
        return binding._current_stream(self._torch, self.device)

    def _describe(self, ids, table, rows, grad_dtype=None) -> arrow_embedding_t:
        """`table`: W or dW, `rows`: Y or dY as (tokens, columns)."""
        torch = self._torch
        if ids.dtype not in (torch.int32, torch.int64):
            raise ValueError(f"ids are int32 or int64, not {ids.dtype}")
        if rows.dtype not in self._dtypes:
            raise TypeError(f"embedding takes float32, bfloat16 and float16 tensors, not {rows.dtype}")
        if table.dim() != 2 or table.shape[0] != self.rows or rows.shape != (ids.numel(), table.shape[1]) or table.shape[1] < 1:
            raise ValueError(f"table {tuple(table.shape)}, {tuple(rows.shape)} of {ids.numel()} tokens: {self.rows} rows of one length expected")
        for t in (ids, table, rows):
            if t.device.type != "cuda" or t.device != rows.device or (self.device.index is not None and t.device != self.device):
                raise ValueError(f"a tensor is on {t.device}, this table on {self.device}")
        columns = table.shape[1]
        for t in (table, rows):
            if (columns > 1 and t.stride(1) != 1 and t.numel()) or (t.shape[0] > 1 and t.stride(0) < columns):
                raise ValueError("the elements of a row do not lie next to each other, or rows overlap")
        e = arrow_embedding_t()
        e.dtype = self._dtypes[rows.dtype]
        e.grad_dtype = self._dtypes[grad_dtype if grad_dtype is not None else rows.dtype]
        e.id_bytes = ids.element_size()
        e.columns, e.rows, e.tokens, e.scale = columns, self.rows, ids.numel(), self.scale
        e.w_stride = table.stride(0) if table.shape[0] > 1 else columns
        e.y_stride = rows.stride(0) if rows.shape[0] > 1 else columns
        return e

    def forward(self, W, ids, Y=None):
        """Y, (shape of ids, columns), of W (rows, columns)."""
        if self._call is not None:
            done = self._call.embedding_forward(*self._forward, W, ids, Y)
            if done is not None:
                return _results(done)
        torch = self._torch
        ids = ids.contiguous()
        shape = (*ids.shape, W.shape[-1])
        Y = torch.empty(shape, dtype=W.dtype, device=W.device) if Y is None else Y
        if Y.dtype != W.dtype or tuple(Y.shape) != shape:
            raise ValueError(f"Y {tuple(Y.shape)} of {Y.dtype}: {shape} of {W.dtype} expected")
        flat = Y if Y.dim() == 2 else Y.view(math.prod(ids.shape), W.shape[-1])
        e = self._describe(ids, W, flat)
        with torch.cuda.device(W.device):
            binding._check(lib().arrow_embedding_forward(ctypes.byref(e), W.data_ptr(), ids.data_ptr(), Y.data_ptr(), self._stream()))
        return Y

    def __call__(self, W, ids):
        """Y as ``forward`` gives it, with its gradient for torch's autograd."""
        return _embedding_function().apply(self, W, ids)

    def backward(self, dY, ids, dW=None, dtype=None):
        """dW, (rows, columns), of dY (shape of ids, columns): every row is written.  dtype: dY's (the default) or float32."""
        if self._call is not None and dtype is None:
            done = self._call.embedding_backward(*self._backward, dY, ids, dW)
            if done is not None:
                return _results(done)
        torch = self._torch
        ids = ids.contiguous()
        if dY.dim() < 1 or tuple(dY.shape[:-1]) != tuple(ids.shape):
            raise ValueError(f"dY {tuple(dY.shape)} of ids {tuple(ids.shape)}")
        flat = dY if dY.dim() == 2 else dY.reshape(math.prod(ids.shape), dY.shape[-1])
        if dW is None:
            dW = torch.empty((self.rows, dY.shape[-1]), dtype=dtype or dY.dtype, device=dY.device)
        if dW.dtype not in (dY.dtype, torch.float32) or (dtype is not None and dW.dtype != dtype):
            raise ValueError(f"dW of {dW.dtype}: {dY.dtype} or float32 expected")
        e = self._describe(ids, dW, flat, dW.dtype)
        with torch.cuda.device(dY.device):
            ws = torch.empty(lib().arrow_embedding_workspace_bytes(ctypes.byref(e)), dtype=torch.uint8, device=dY.device)
            binding._check(lib().arrow_embedding_backward(ctypes.byref(e), flat.data_ptr(), ids.data_ptr(), dW.data_ptr(), ws.data_ptr(), ws.numel(),
                                                          self._stream()))
        return dW


_function = None


def _embedding_function():
    """The call as a node of torch's autograd."""
    global _function
    if _function is None:
        import torch

        class Embedding(torch.autograd.Function):
            @staticmethod
            def forward(ctx, op, W, ids):
                ctx.save_for_backward(ids)
                ctx.op = op
                return op.forward(W, ids)

            @staticmethod
            @torch.autograd.function.once_differentiable
            def backward(ctx, dY):
                return None, ctx.op.backward(dY.contiguous(), ctx.saved_tensors[0]), None

        _function = Embedding
    return _function
