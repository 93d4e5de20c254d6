"""Head norms with the rotation, the cache in 4 bits, page tables and log probabilities from their definitions, in 64 bits (pages: on lists), with elementwise bounds of what
rounding may do to a result in a type of unit roundoff u that holds everything else in 32 bits (e = 2^-24).

Rotation.  The mean of `dim` squares and its root are off by less than h = (dim + 12) e, relative; an angle by a = 2 pi (2^-25 + 2^-51 |turns|) + 8 e, from the
product in 64 bits, its rounding to 32 and the functions of it.  A rotated pair is off by (|x| + |y|) (h + a).
Log probabilities.  With d = scale (x - max): exp d is off by (4 |d| + 8) e, relative, and sums, which a lane adds up in at most 256 steps and their sums in 128,
and some 60 more join, by 512 e more.
"""
from __future__ import annotations

import math

import torch

from .attention_oracle import TINY, UNIT

E = 2.0 ** -24
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ---- rotation ----
def _turned(x, p, turns, rotary, interleaved, back=False):
    """Pairs of x (..., tokens, heads, dim) by the angles of p (..., tokens), and |x| + |y| of each element's pair (0 where it has none)."""
    r = rotary
    a = 2.0 * math.pi * torch.remainder(p[..., None].double() * turns, 1.0)[..., None, :]
    cos, sin = torch.cos(a), torch.sin(a) * (-1.0 if back else 1.0)
    first = torch.arange(0, r, 2) if interleaved else torch.arange(r // 2)
    second = first + 1 if interleaved else first + r // 2
    y, size = x.clone(), torch.zeros_like(x)
    u, v = x[..., first], x[..., second]
    y[..., first], y[..., second] = u * cos - v * sin, v * cos + u * sin
    size[..., first] = size[..., second] = u.abs() + v.abs()
    return y, size


def rotation(x, w, p, turns, rotary, interleaved=False, eps=1e-6, dy=None):
    """x (..., tokens, heads, dim), w (dim) or None, p (..., tokens): dicts of y and, with dy, dx and dw (32 bits), and their bounds."""
    t, dim = x.dtype, x.shape[-1]
    u, tiny = UNIT[t], TINY[t]
    x = x.double()
    w = torch.ones(dim, dtype=torch.float64, device=x.device) if w is None else w.double()
    turns = turns.double().to(x.device)
    h = (dim + 12) * E
    a = 8 * E + 2 * math.pi * (2.0 ** -25 + 2.0 ** -51 * (p.double().abs()[..., None] * turns).amax(-1) if rotary else torch.zeros_like(p, dtype=torch.float64))
    a = a[..., None, None]
    r = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    y, size = _turned(x * r * w, p, turns, rotary, interleaved)
    got, bound = {"y": y}, {"y": (size + y.abs()) * (h + a) + u * y.abs() + 2 * tiny}
    if dy is not None:
        g, g_size = _turned(dy.double(), p, turns, rotary, interleaved, back=True)
        e_g = (g_size + g.abs()) * (a + 4 * E)
        n = x * r
        mean = (w * g * n).mean(-1, keepdim=True)
        e_mean = (w.abs() * n.abs() * (e_g + 2 * h * g.abs())).mean(-1, keepdim=True)
        dx = r * (w * g - n * mean)
        got["dx"] = dx
        bound["dx"] = r * (w.abs() * e_g + n.abs() * e_mean + 2 * h * ((w * g).abs() + n.abs() * mean.abs())) + u * dx.abs() + 2 * tiny
        terms = g * n
        count = terms.numel() // dim
        got["dw"] = terms.flatten(0, -2).sum(0)
        bound["dw"] = (n.abs() * e_g + terms.abs() * (h + (count + 64) * E)).flatten(0, -2).sum(0)
    return got, bound


# ---- the cache in 4 bits ----
def packed(x):
    """What (..., dim) elements are in 4 bits, as values in 64 bits: the nearest of each block's levels."""
    most = 2.0 ** (13 if x.dtype == torch.float16 else 125)
    x = x.double().unflatten(-1, (-1, 32))
    size = x.abs().amax(-1, keepdim=True)
    bad = ~torch.isfinite(size)
    part, e = torch.frexp(torch.where(bad, 0.0, size))            # size = part 2^e, 1/2 <= part < 1: the smallest power of two that it is at most seven times of
    step = torch.exp2((e - torch.where(part <= 0.875, 3, 2)).double()).clamp(2.0 ** -126, most)
    y = x.abs() / step
    best, gap = torch.zeros_like(y), torch.full_like(y, math.inf)
    for i in (0, 2, 4, 6, 1, 3, 5, 7):                            # (even codes first: of two at one distance they are taken)
        off = (y - LEVELS[i]).abs()
        best, gap = torch.where(off < gap, LEVELS[i], best), torch.minimum(gap, off)
    return torch.where(bad, math.nan, best * step * torch.sign(x)).flatten(-2)


# ---- pages ----
class Pages:
    """State and step of include/arrow_pages.h on Python's lists."""

    def __init__(self, pages, page, window, sinks, batch, columns):
        self.pages, self.page, self.window, self.sinks, self.columns = pages, page, window, sinks, columns
        self.table = [[-1] * columns for _ in range(batch)]
        self.held = [0] * batch
        self.stack = list(range(pages - 1, -1, -1))

    def needed(self, length):
        length = max(0, min(length, self.columns * self.page))
        return [c for c in range(self.columns) if c * self.page < length and
                (not self.window or (c + 1) * self.page > length - self.window or c * self.page < self.sinks)]

    def step(self, lengths, fresh):
        """fresh: new tokens of each sequence; the slots of each."""
        given, slots = [], []
        for b, n in enumerate(lengths):
            now = set(self.needed(n))
            for c in self.needed(self.held[b]):
                if c not in now:
                    if 0 <= self.table[b][c] < self.pages:
                        given.append(self.table[b][c])
                    self.table[b][c] = -1
        self.stack += reversed(given)
        for b, n in enumerate(lengths):
            before = set(self.needed(self.held[b]))
            for c in self.needed(n):
                if c not in before and c * self.page >= n - fresh[b]:
                    self.table[b][c] = self.stack.pop() if self.stack else -1
            own = []
            for t in range(n - fresh[b], n):
                c = t // self.page
                p = self.table[b][c] if 0 <= t and c < self.columns else -1
                own.append(p * self.page + t % self.page if 0 <= p < self.pages else -1)
            slots.append(own)
        self.held = list(lengths)
        return slots


# ---- log probabilities ----
def logprobs(x, targets, scale=1.0, top=0, d_logp=None, d_entropy=None):
    """x (rows, vocabulary), targets (rows): dicts of logp, entropy, lse, and top_ids, top_logp, d_logits where asked for, and the bounds of the floats."""
    t, (rows, n) = x.dtype, x.shape
    u, tiny = UNIT[t], TINY[t]
    x = x.double()
    m = x.amax(-1, keepdim=True)
    empty, bad = m[:, 0] == -math.inf, ~(m[:, 0] < math.inf)
    d = torch.where(x == m, 0.0, scale * (x - m))
    p = torch.exp(d)
    s = p.sum(-1, keepdim=True)
    p = p / s
    log = torch.log(s)
    seen = torch.where(p > 0, d, 0.0)
    mean = (p * seen).sum(-1)
    known = (targets >= 0) & (targets < n)
    at = targets.clamp(0, n - 1)[:, None].long()
    d_t = d.gather(1, at)[:, 0]
    r = (p * (4 * seen.abs() + 8)).sum(-1) * E + 512 * E          # of the sum, relative
    of_log = r + 4 * E * (1 + log[:, 0].abs())
    lse = scale * m[:, 0] + log[:, 0]
    got = {"lse": lse, "logp": torch.where(known, d_t - log[:, 0], 0.0), "entropy": log[:, 0] - mean}
    bound = {"lse": of_log + 4 * E * (lse.abs() + (scale * m[:, 0]).abs()),
             "logp": torch.where(known, of_log + 4 * E * torch.nan_to_num(d_t.abs(), posinf=0.0), 0.0),
             "entropy": of_log + (p * seen.abs() * (4 * seen.abs() + 16)).sum(-1) * E + (r + 512 * E) * mean.abs() + 4 * E * mean.abs()}
    for name, of in (("lse", m[:, 0] * scale), ("logp", torch.where(known, -math.inf, 0.0)), ("entropy", torch.zeros_like(lse))):
        got[name] = torch.where(empty, of, got[name])
        got[name] = torch.where(bad & (known if name == "logp" else True), math.nan, got[name])
    if top:
        key = torch.where(torch.isnan(x), math.inf, x)
        order = torch.argsort(torch.isnan(x).double(), dim=-1, descending=True, stable=True)
        by = torch.argsort(key.gather(1, order), dim=-1, descending=True, stable=True)
        ids = order.gather(1, by)[:, :top]
        value = d.gather(1, ids) - log
        got["top_ids"], got["top_logp"] = ids, torch.where(empty[:, None], -math.inf, torch.where(bad[:, None], math.nan, value))
        bound["top_logp"] = of_log[:, None] + 4 * E * torch.nan_to_num(d.gather(1, ids).abs(), posinf=0.0)
    if d_logp is not None or d_entropy is not None:
        zero = torch.zeros(rows, dtype=torch.float64, device=x.device)
        g = torch.where(known, (d_logp if d_logp is not None else zero).double(), 0.0)[:, None] * scale
        h = (d_entropy if d_entropy is not None else zero).double()[:, None] * scale
        inner = torch.where(p > 0, d - log, 0.0) + got["entropy"][:, None]
        one = torch.zeros_like(x).scatter_(1, at, 1.0) * known[:, None]
        grad = g * one - p * (g + h * inner)
        of_p = (4 * seen.abs() + 16) * E + of_log[:, None]
        off = p * ((g.abs() + (h * inner).abs()) * of_p + h.abs() * (of_log[:, None] + bound["entropy"][:, None] + 8 * E * (seen.abs() + log.abs() + 1))) + 4 * E * grad.abs()
        got["d_logits"] = torch.where(empty[:, None], 0.0, torch.where(bad[:, None], math.nan, grad))
        bound["d_logits"] = off + 4 * E * (g * one).abs() + u * grad.abs() + 2 * tiny
    return got, bound
