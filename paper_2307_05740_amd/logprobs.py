"""Log probabilities of given tokens, entropies and the most likely tokens of rows of logits (``include/arrow_logprobs.h``), on torch tensors.

``lse = log sum exp(scale x)``, ``logp = scale x[target] - lse``, ``H = lse - sum p scale x``; the loss of a model is minus the sum of logp, and what a
server answers with are the tokens on top.  :class:`ArrowLogProbs` marshals arguments; every step runs in the library's HIP kernels, on the current stream
of the tensors' device.  Workspaces are torch's, taken for the time of a call.
"""
from __future__ import annotations

import collections
import ctypes
import math

from . import binding
from .attention import _address, _results
from .binding import arrow_logprobs_t, lib

LogProbs = collections.namedtuple("LogProbs", ("logp", "entropy", "lse", "stats", "top_logp", "top_ids"))


class ArrowLogProbs:
    """Probabilities of logits times ``scale`` (one over a temperature)."""

    def __init__(self, scale: float = 1.0, device="cuda:0"):
        import torch
        self._torch = torch
        self.device = torch.device(device)
        self.scale = float(scale)
        if not self.scale > 0.0 or math.isinf(self.scale):
            raise ValueError(f"scale = {scale} is not positive and finite")
        self._dtypes = {torch.float32: binding.ARROW_F32, torch.bfloat16: binding.ARROW_BF16, torch.float16: binding.ARROW_F16}
        # the plain case goes by native code, as in attention.py
        self._call = binding._tensor_call(self.device)
        if self._call is not None:
            address = lambda name: binding._address(getattr(lib(), name))   # noqa: E731
            self._forward = (address("arrow_logprobs_forward"), address("arrow_logprobs_workspace_bytes"), self.device.index, self.scale)
            self._backward = (address("arrow_logprobs_backward"), self.device.index, self.scale)

    def _stream(self) -> int:
        return binding._current_stream(self._torch, self.device)

    def _describe(self, logits, targets, top):
        """The arguments, and the targets as the kernels take them."""
        torch = self._torch
        if logits.dtype not in self._dtypes:
            raise TypeError(f"logits are float32, bfloat16 or float16, not {logits.dtype}")
        if targets.dtype not in (torch.int32, torch.int64):
            raise TypeError(f"targets are int32 or int64, not {targets.dtype}")
        if logits.device.type != "cuda" or (self.device.index is not None and logits.device != self.device) or targets.device != logits.device:
            raise ValueError(f"logits are on {logits.device}, targets on {targets.device}, these probabilities on {self.device}")
        if logits.dim() < 1 or targets.shape != logits.shape[:-1] or logits.shape[-1] < 1:
            raise ValueError(f"logits {tuple(logits.shape)}, targets {tuple(targets.shape)}: (..., vocabulary) and (...) expected")
        if not 0 <= top <= min(32, logits.shape[-1]):
            raise ValueError(f"top = {top}: 0 .. 32, at most {logits.shape[-1]}")
        a = arrow_logprobs_t()
        a.dtype, a.target_bytes, a.top, a.vocabulary = self._dtypes[logits.dtype], targets.element_size(), top, logits.shape[-1]
        a.rows, a.scale = targets.numel(), self.scale
        return a, targets.contiguous()

    @staticmethod
    def _rows(name, t, a) -> int:
        """Elements from row to row of (..., vocabulary)."""
        if t.shape[-1] > 1 and t.stride(-1) != 1 and t.numel():
            raise ValueError(f"{name}: the elements of a row do not lie next to each other")
        if a.rows <= 1:
            return a.vocabulary
        flat = t if t.dim() == 2 else t.view(a.rows, a.vocabulary)   # (a view that there is not says so)
        return flat.stride(0)

    def forward(self, logits, targets, top: int = 0) -> LogProbs:
        """``LogProbs(logp, entropy, lse, stats, top_logp, top_ids)`` of logits (..., vocabulary) and targets (...), int32 or int64; of ``top`` tokens, (..., top) each in
        falling order (None where top is 0).  Targets outside the vocabulary are padding: their logp is 0.  stats, (..., 2), is for ``backward``."""
        if self._call is not None:
            done = self._call.logprobs_forward(*self._forward, logits, targets, top)
            if done is not None:
                done = _results(done)
                return LogProbs(*done) if top else LogProbs(*done, None, None)
        torch = self._torch
        a, targets = self._describe(logits, targets, top)
        a.stride = self._rows("logits", logits, a)
        shape, dev = targets.shape, logits.device
        logp, entropy, lse = (torch.empty(shape, dtype=torch.float32, device=dev) for _ in range(3))
        stats = torch.empty((*shape, 2), dtype=torch.float32, device=dev)
        top_logp = torch.empty((*shape, top), dtype=torch.float32, device=dev) if top else None
        top_ids = torch.empty((*shape, top), dtype=torch.int64, device=dev) if top else None
        with torch.cuda.device(dev):
            ws = torch.empty(lib().arrow_logprobs_workspace_bytes(ctypes.byref(a)), dtype=torch.uint8, device=dev)
            binding._check(lib().arrow_logprobs_forward(ctypes.byref(a), _address(logits), _address(targets), _address(logp), _address(entropy), _address(lse),
                                                        _address(stats), _address(top_logp), _address(top_ids), _address(ws), ws.numel(), self._stream()))
        return LogProbs(logp, entropy, lse, stats, top_logp, top_ids)

    def backward(self, d_logp, d_entropy, logits, targets, stats, entropy=None, d_logits=None):
        """d_logits for the gradients of logp and entropy (float32, either may be None), with the stats and entropy that ``forward`` gave.  d_logits may be logits."""
        if self._call is not None:
            done = self._call.logprobs_backward(*self._backward, d_logp, d_entropy, logits, targets, stats, entropy, d_logits)
            if done is not None:
                return _results(done)
        torch = self._torch
        a, targets = self._describe(logits, targets, 0)
        a.stride = self._rows("logits", logits, a)
        if d_entropy is not None and entropy is None:
            raise ValueError("a gradient of the entropy takes the entropy")
        for name, t in (("d_logp", d_logp), ("d_entropy", d_entropy), ("stats", stats), ("entropy", entropy)):
            shape = (*targets.shape, 2) if name == "stats" else tuple(targets.shape)
            if t is not None and (t.dtype != torch.float32 or t.device != logits.device or tuple(t.shape) != shape or not t.is_contiguous()):
                raise ValueError(f"{name}: contiguous float32 {shape} on {logits.device} expected")
        if stats is None:
            raise ValueError("stats: those of the forward call expected")
        d_logits = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device) if d_logits is None else d_logits
        if d_logits.shape != logits.shape or d_logits.dtype != logits.dtype or d_logits.device != logits.device:
            raise ValueError(f"d_logits {tuple(d_logits.shape)} of {d_logits.dtype}: {tuple(logits.shape)} of {logits.dtype} expected")
        a.d_stride = self._rows("d_logits", d_logits, a)
        with torch.cuda.device(logits.device):
            binding._check(lib().arrow_logprobs_backward(ctypes.byref(a), _address(d_logp), _address(d_entropy), _address(logits), _address(targets),
                                                         _address(stats), _address(entropy), _address(d_logits), self._stream()))
        return d_logits

    def __call__(self, logits, targets):
        """``(logp, entropy)`` as ``forward`` gives them, with their gradients for torch's autograd."""
        return _logprobs_function().apply(self, logits, targets)


_function = None


def _logprobs_function():
    """The call as a node of torch's autograd."""
    global _function
    if _function is None:
        import torch

        class LogProbsFunction(torch.autograd.Function):
            @staticmethod
            def forward(ctx, op, logits, targets):
                r = op.forward(logits, targets)
                ctx.save_for_backward(logits, targets, r.stats, r.entropy)
                ctx.op = op
                ctx.set_materialize_grads(False)
                return r.logp, r.entropy

            @staticmethod
            @torch.autograd.function.once_differentiable
            def backward(ctx, d_logp, d_entropy):
                logits, targets, stats, entropy = ctx.saved_tensors
                d_logp, d_entropy = (g.float().contiguous() if g is not None else None for g in (d_logp, d_entropy))
                return None, ctx.op.backward(d_logp, d_entropy, logits, targets, stats, entropy), None

        _function = LogProbsFunction
    return _function
