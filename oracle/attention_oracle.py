"""The operators on sequences in 64 bits, from their definitions, with elementwise bounds of what rounding may do to a
result in a type of unit roundoff u (bfloat16 2^-8, float16 2^-11) that holds scores and sums in 32 bits.

Bounds.  A score in 32 bits is off by at most e_s = (dim + 16) 2^-24 scale sum_d |q_d k_d|, and so is a probability, relative to itself, before
it is rounded; sums of n terms are off by n 2^-24 of the terms' magnitudes.  With h = max e_s + (n + 64) 2^-24:
  o:   (P |V|) (2 u + h): once for P, once for o; where P is off by `p_unit` of itself instead, (P |V|) (p_unit + h) (1 + u) + u |o|;
  dv:  (P^T |dO|) (2 u + h);
  dS = P (dP - D) is rounded once; D = <dO, o> takes the rounded o, off by E_o (the bound above):
       E_S = P (|dP - D| (u + h) + <|dO|, E_o> + h (|dO| |V|^T + <|dO|, |o|>)),
  dq:  scale E_S |K| + u |dq| + h scale |dS| |K|, and dk likewise.
float16 has steps of 2^-24 near zero: half of one per rounded P or dS more (`tiny`), one for each result.
"""
from __future__ import annotations

import math

import torch

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25, torch.float32: 0.0}


def visible(queries: int, keys: int, window: int, sinks: int, device="cpu"):
    """(queries, keys) truth values."""
    p = torch.arange(queries, device=device)[:, None] + keys - queries
    j = torch.arange(keys, device=device)[None, :]
    return (j <= p) & ((j > p - window) | (j < sinks)) if window else j <= p


def _clean(x):
    return torch.where(torch.isfinite(x), x, 0.0)


def attention(q, k, v, window=0, sinks=0, scale=None, d_o=None, seen=None, p_unit=None):
    """One head: q (n, d), k and v (m, d), all of one type.  Results and bounds: dicts of o, lse and, with d_o, dq, dk, dv.
    What is not seen does not count, whatever it holds."""
    n, m, d = q.shape[0], k.shape[0], q.shape[1]
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    u, tiny = UNIT[q.dtype], TINY[q.dtype]
    seen = visible(n, m, window, sinks, q.device) if seen is None else seen
    q, k, v = q.double(), _clean(k.double()), _clean(v.double())
    s = torch.where(seen, q @ k.T * scale, -math.inf)
    top = s.amax(-1, keepdim=True) if m else torch.full((n, 1), -math.inf, dtype=torch.float64, device=q.device)
    top = torch.where(torch.isfinite(top), top, 0.0)
    e = torch.exp(s - top)
    total = e.sum(-1, keepdim=True)
    lse = (top + torch.log(total))[:, 0]
    p = e / torch.where(total == 0, 1.0, total)
    o = p @ v
    e_s = (d + 16) * 2.0 ** -24 * scale * torch.where(seen, q.abs() @ k.abs().T, 0.0)
    e_s = e_s.amax(-1, keepdim=True) if m else torch.zeros((n, 1), dtype=torch.float64, device=q.device)
    h = e_s + (m + 64) * 2.0 ** -24
    see = seen.double()
    # (a running maximum may be up to 2^8 below the final one; its terms are never below 1 at their largest)
    b_o = (p @ v.abs()) * (2 * u + h) if p_unit is None else (p @ v.abs()) * (p_unit + h) * (1 + u) + u * o.abs()
    b_o = b_o + tiny * (see @ v.abs()) + 2 * tiny
    got = {"o": o, "lse": lse}
    bound = {"o": b_o, "lse": e_s[:, 0] + 2.0 ** -20 * (1 + torch.where(torch.isfinite(lse), lse.abs(), 0.0))}
    if d_o is not None:
        g = d_o.double()
        dp, delta = g @ v.T, (g * o).sum(-1, keepdim=True)
        ds = p * (dp - delta)
        e_ds = p * ((dp - delta).abs() * (u + h) + (g.abs() * b_o).sum(-1, keepdim=True) + h * (g.abs() @ v.abs().T + (g.abs() * o.abs()).sum(-1, keepdim=True)))
        e_ds = e_ds + tiny * see
        hq = (n + 64) * 2.0 ** -24
        got.update(dq=scale * ds @ k, dk=scale * ds.T @ q, dv=p.T @ g)
        bound.update(dq=scale * (e_ds + h * ds.abs()) @ k.abs(), dk=scale * (e_ds + hq * ds.abs()).T @ q.abs(),
                     dv=(p * (u + h) + hq * p + tiny * see).T @ g.abs())
        for name in ("dq", "dk", "dv"):
            bound[name] = bound[name] + u * got[name].abs() + 2 * tiny
    return got, bound


def embedding(W, ids, scale):
    """Y of W (rows, columns) and ids of any shape; those outside the table give zero rows."""
    known = (ids >= 0) & (ids < W.shape[0])
    return torch.where(known[..., None], W.double()[torch.where(known, ids, 0).long()] * scale, 0.0)


def embedding_grad(dY, ids, rows, scale, dtype):
    """dW and its bound: sums in 32 bits, rounded to `dtype` once."""
    dY, ids = dY.reshape(-1, dY.shape[-1]).double(), ids.reshape(-1).long()
    known = (ids >= 0) & (ids < rows)
    dY, ids = dY[known], ids[known]
    dW = torch.zeros(rows, dY.shape[1], dtype=torch.float64, device=dY.device)
    size = torch.zeros_like(dW)
    dW.index_add_(0, ids, dY * scale)
    size.index_add_(0, ids, (dY * scale).abs())
    n = torch.bincount(ids, minlength=rows).double()[:, None]
    return dW, size * (n + 4) * 2.0 ** -24 + UNIT[dtype] * dW.abs() + 2 * TINY[dtype]
