"""Norms of queries and keys for each head with the rotation by position (``include/arrow_rotation.h``), on torch tensors.

``u = w x / sqrt(mean x^2 + eps)`` for each head ``x``, and pairs of ``u``'s first ``rotary`` elements turned by ``position * frequency``.
:class:`ArrowRotation` marshals arguments; every step runs in the library's HIP kernels, on the current stream of the tensors' device.  Workspaces
are torch's, taken for the time of a call.
"""
from __future__ import annotations

import ctypes
import math

from . import binding
from .attention import _address, _results
from .binding import arrow_rotation_t, arrow_strides_t, lib


class ArrowRotation:
    """Heads of ``dim`` elements, of which the first ``rotary`` (default: all) are rotated: pair i by ``base ** (-2 i / rotary)`` for each position, or by
    ``frequencies[i]`` (a sequence or tensor of rotary / 2 values).  Pair i are elements i and i + rotary / 2, or, interleaved, 2 i and 2 i + 1."""

    def __init__(self, dim: int, base: float = 10000.0, rotary: int | None = None, interleaved: bool = False, eps: float = 1e-6, frequencies=None,
                 device="cuda:0"):
        import torch
        self._torch = torch
        self.device = torch.device(device)
        self.dim, self.rotary = int(dim), int(dim if rotary is None else rotary)
        self.interleaved, self.eps = bool(interleaved), float(eps)
        if self.rotary < 0 or self.rotary > self.dim or self.rotary % 16:
            raise ValueError(f"rotary = {self.rotary} is none of 0, 16, 32, ... up to dim = {self.dim}")
        if frequencies is None:
            frequencies = [float(base) ** (-2.0 * i / self.rotary) for i in range(self.rotary // 2)]
        f = torch.as_tensor(frequencies, dtype=torch.float64)
        if f.shape != (self.rotary // 2,):
            raise ValueError(f"frequencies {tuple(f.shape)}: ({self.rotary // 2},) expected")
        self.turns = (f / (2.0 * math.pi)).to(self.device)
        self._dtypes = {torch.float32: binding.ARROW_F32, torch.bfloat16: binding.ARROW_BF16, torch.float16: binding.ARROW_F16}
        # the plain case goes by native code, as in attention.py
        self._call = binding._tensor_call(self.device)
        if self._call is not None:
            address = lambda name: binding._address(getattr(lib(), name))   # noqa: E731
            same = (self.device.index, self.dim, self.rotary, int(self.interleaved), self.turns.data_ptr(), self.eps)
            self._forward = (address("arrow_rotation_forward"), *same)
            self._backward = (address("arrow_rotation_backward"), address("arrow_rotation_workspace_bytes"), *same)

    def _stream(self) -> int:
        return binding._current_stream(self._torch, self.device)

    @staticmethod
    def _steps(t) -> arrow_strides_t:
        """Steps of a tensor; one that is never taken counts as none."""
        step = lambda d: t.stride(d) if t.shape[d] > 1 else 0   # noqa: E731
        return arrow_strides_t(step(0) if t.dim() == 4 else 0, step(t.dim() - 3), step(t.dim() - 2))

    def _check(self, name, t, shape, dtype, device) -> None:
        if t.device != device or t.dtype != dtype:
            raise ValueError(f"{name}: {t.dtype} on {t.device}, {dtype} on {device} expected")
        if tuple(t.shape) != tuple(shape):
            raise ValueError(f"{name} {tuple(t.shape)}: {tuple(shape)} expected")
        if t.dim() and t.shape[-1] > 1 and t.stride(-1) != 1 and t.numel():
            raise ValueError(f"{name}: the elements of a head do not lie next to each other")

    def _describe(self, q, k, q_weight, k_weight, positions, shift) -> arrow_rotation_t:
        torch = self._torch
        if q.dtype not in self._dtypes:
            raise TypeError(f"rotation takes float32, bfloat16 and float16 tensors, not {q.dtype}")
        if q.dim() not in (3, 4) or k.dim() != q.dim() or k.shape[:-2] != q.shape[:-2] or k.shape[-1] != q.shape[-1] or q.shape[-1] != self.dim:
            raise ValueError(f"q {tuple(q.shape)}, k {tuple(k.shape)}: (batch, tokens, heads, {self.dim}) or (tokens, heads, {self.dim}) expected")
        if q.device.type != "cuda" or q.device != self.turns.device:
            raise ValueError(f"q is on {q.device}, this rotation on {self.turns.device}")
        for name, t in (("q", q), ("k", k)):
            self._check(name, t, t.shape, q.dtype, q.device)
        a = arrow_rotation_t()
        a.dtype = a.weight_dtype = self._dtypes[q.dtype]
        if (q_weight is None) != (k_weight is None):
            raise ValueError("weights of queries and of keys: both or neither")
        if q_weight is not None:
            if q_weight.dtype not in (q.dtype, torch.float32):
                raise TypeError(f"weights are {q.dtype} or float32, not {q_weight.dtype}")
            for name, t in (("q_weight", q_weight), ("k_weight", k_weight)):
                self._check(name, t, (self.dim,), q_weight.dtype, q.device)
            a.weight_dtype = self._dtypes[q_weight.dtype]
        a.batch, a.tokens = (q.shape[0] if q.dim() == 4 else 1), q.shape[-3]
        a.q_heads, a.kv_heads, a.dim, a.rotary = q.shape[-2], k.shape[-2], self.dim, self.rotary
        a.interleaved, a.eps, a.shift = int(self.interleaved), self.eps, int(shift)
        if positions is not None:
            if positions.dtype not in (torch.int32, torch.int64) or positions.device != q.device or positions.shape != q.shape[:-2] or not positions.is_contiguous():
                raise ValueError(f"positions: contiguous int32 or int64 {tuple(q.shape[:-2])} on {q.device} expected")
            a.positions, a.position_bytes = positions.data_ptr(), positions.element_size()
        a.turns = self.turns.data_ptr() if self.rotary else 0
        a.q, a.k = self._steps(q), self._steps(k)
        return a

    def forward(self, q, k, q_weight=None, k_weight=None, positions=None, shift: int = 0, q_out=None, k_out=None):
        """``(q_out, k_out)`` of q (batch, tokens, heads, dim) or (tokens, heads, dim), k likewise, with weights of (dim), float32 or q's type.  positions: int32 or
        int64, of q's shape without heads and dim; by default a token's place in its sequence.  ``shift`` is added to each: -1 turns lengths that
        count the new token into its position.  q_out may be q, k_out k."""
        if self._call is not None:
            done = self._call.rotation_forward(*self._forward, q, k, q_weight, k_weight, positions, shift, q_out, k_out)
            if done is not None:
                return _results(done)
        torch = self._torch
        a = self._describe(q, k, q_weight, k_weight, positions, shift)
        q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device) if q_out is None else q_out
        k_out = torch.empty(k.shape, dtype=k.dtype, device=k.device) if k_out is None else k_out
        for name, t, like in (("q_out", q_out, q), ("k_out", k_out, k)):
            self._check(name, t, like.shape, q.dtype, q.device)
            setattr(a, name, self._steps(t))
        with torch.cuda.device(q.device):
            binding._check(lib().arrow_rotation_forward(ctypes.byref(a), _address(q), _address(k), _address(q_weight), _address(k_weight), _address(q_out),
                                                        _address(k_out), self._stream()))
        return q_out, k_out

    def backward(self, d_q, d_k, q, k, q_weight=None, k_weight=None, positions=None, shift: int = 0, dq=None, dk=None):
        """``(dq, dk, dq_weight, dk_weight)`` for the gradients d_q and d_k of what ``forward`` gave for these arguments; the weights' are None where there
        are no weights.  dq may be d_q, dk d_k."""
        if self._call is not None:
            done = self._call.rotation_backward(*self._backward, d_q, d_k, q, k, q_weight, k_weight, positions, shift, dq, dk)
            if done is not None:
                done = _results(done)
                return done if len(done) == 4 else (*done, None, None)
        torch = self._torch
        a = self._describe(q, k, q_weight, k_weight, positions, shift)
        dq = torch.empty(q.shape, dtype=q.dtype, device=q.device) if dq is None else dq
        dk = torch.empty(k.shape, dtype=k.dtype, device=k.device) if dk is None else dk
        for name, to, t, like in (("d_q", "q_out", d_q, q), ("d_k", "k_out", d_k, k), ("dq", "dq", dq, q), ("dk", "dk", dk, k)):
            self._check(name, t, like.shape, q.dtype, q.device)
            setattr(a, to, self._steps(t))
        dwq = dwk = ws = None
        with torch.cuda.device(q.device):
            if q_weight is not None:
                dwq, dwk = torch.empty_like(q_weight), torch.empty_like(k_weight)
                ws = torch.empty(lib().arrow_rotation_workspace_bytes(ctypes.byref(a)), dtype=torch.uint8, device=q.device)
            binding._check(lib().arrow_rotation_backward(
                ctypes.byref(a), _address(d_q), _address(d_k), _address(q), _address(k), _address(q_weight), _address(k_weight), _address(dq), _address(dk),
                _address(dwq), _address(dwk), _address(ws), ws.numel() if ws is not None else 0, self._stream()))
        return dq, dk, dwq, dwk

    def __call__(self, q, k, q_weight=None, k_weight=None, positions=None, shift: int = 0):
        """``(q_out, k_out)`` as ``forward`` gives them, with their gradients for torch's autograd."""
        return _rotation_function().apply(self, q, k, q_weight, k_weight, positions, shift)


_function = None


def _rotation_function():
    """The call as a node of torch's autograd."""
    global _function
    if _function is None:
        import torch

        def heads(g, like):
            """A gradient as the kernels take it: any address and steps, of one type."""
            if g is None:
                return torch.zeros(like.shape, dtype=like.dtype, device=like.device)
            step = 16 // g.element_size()
            if g.stride(-1) != 1 or g.data_ptr() % 16 or any(s % step for s in g.stride()[:-1]):
                return g.clone(memory_format=torch.contiguous_format)
            return g

        class Rotation(torch.autograd.Function):
            @staticmethod
            def forward(ctx, op, q, k, q_weight, k_weight, positions, shift):
                ctx.save_for_backward(q, k, q_weight, k_weight, positions)
                ctx.op, ctx.shift = op, shift
                return op.forward(q, k, q_weight, k_weight, positions, shift)

            @staticmethod
            @torch.autograd.function.once_differentiable
            def backward(ctx, d_q, d_k):
                q, k, q_weight, k_weight, positions = ctx.saved_tensors
                return None, *ctx.op.backward(heads(d_q, q), heads(d_k, k), q, k, q_weight, k_weight, positions, ctx.shift), None, None

        _function = Rotation
    return _function
