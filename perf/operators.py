"""The operators on sequences, as cases that can be timed: attention under an arrow-shaped mask (forward, training
step, single new tokens over a paged cache) and the embedding lookup with its gradient.

With ``own`` true a pass calls the public classes ``ArrowAttention`` and ``ArrowEmbedding``; otherwise it computes the same
with elementary torch operations in 32 bits, rounded once at the end.  ``exact`` is the definition in 64 bits.

Key j is visible to query i of a sequence (at position p = i + keys - queries) where j <= p and (no window, or j > p - window, or
j < sinks).  A row without visible keys gives o = 0 and lse = -inf.
"""
from __future__ import annotations

import math
import random

import torch

own = False
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
INF = float("inf")


# ------------------------------------------------------------------------------------------------
# the cases
# ------------------------------------------------------------------------------------------------
def _attention(op, batch, length, q_heads, kv_heads, dim, window, sinks, dtype, past=0, ragged=False):
    """`length` queries per sequence (ragged: of all sequences together), `past` keys before them."""
    return {"op": op, "batch": batch, "length": length, "past": past, "ragged": ragged, "q_heads": q_heads, "kv_heads": kv_heads,
            "dim": dim, "window": window, "sinks": sinks, "dtype": dtype}


def _decode(batch, length, q_heads, kv_heads, dim, window, sinks, page, dtype):
    """Sequences of lengths from a quarter of `length` to `length`."""
    return {"op": "decode", "batch": batch, "length": length, "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim,
            "window": window, "sinks": sinks, "page": page, "dtype": dtype}


def _embedding(op, tokens, rows, columns, dtype):
    return {"op": op, "tokens": tokens, "rows": rows, "columns": columns, "dtype": dtype}


def listed():
    c = []

    def add(name, case):
        c.append(dict(case, name=name))

    # a short prompt of odd length in a small model: the call itself counts
    add("prefill 1000 h8 d64", _attention("prefill", 1, 1000, 8, 8, 64, 256, 4, "bf16"))
    # the long prompt of a model with few key heads
    add("prefill 16k h16/2 d128", _attention("prefill", 1, 16384, 16, 2, 128, 4096, 16, "bf16"))
    # requests of all lengths packed into one batch, one of them empty, behind a common number of cached keys
    add("prefill ragged 8k h32/8", _attention("prefill", 9, 8192, 32, 8, 128, 1024, 4, "f16", past=200, ragged=True))
    # a training step of a small model, as many key heads as query heads
    add("train 4x2048 h16 d64", _attention("train", 4, 2048, 16, 16, 64, 512, 4, "bf16"))
    # a training step over a long context with shared key heads
    add("train 8k h32/8 d128", _attention("train", 1, 8192, 32, 8, 128, 2048, 16, "bf16"))
    # a training step without a window, of odd length and a head size that is no power of two
    add("train 2x1531 h12/2 d96", _attention("train", 2, 1531, 12, 2, 96, 0, 0, "f16"))
    # one user's next token, short context
    add("decode 1x1000 h8/2", _decode(1, 1000, 8, 2, 128, 0, 0, 16, "bf16"))
    # a serving batch over full contexts: the cache's bytes count
    add("decode 32x16k h32/8", _decode(32, 16000, 32, 8, 128, 0, 0, 64, "bf16"))
    # long streams of which a window and the first tokens are kept
    add("decode 64x60k window", _decode(64, 60001, 16, 4, 64, 4096, 4, 32, "f16"))
    # the lookup of a training batch
    add("embedding 16k of 32000x4096", _embedding("embedding", 16384, 32000, 4096, "bf16"))
    # its gradient: hot tokens, and most rows of the table without any
    add("embedding grad 16k of 32000x4096", _embedding("embedding grad", 16384, 32000, 4096, "bf16"))
    # both in one step of a small model in 32 bits, with odd sizes
    add("embedding step 777 of 5003x500", _embedding("embedding step", 777, 5003, 500, "f32"))
    return c


def draw(rng):
    def logint(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    def heads(most):
        kv = rng.choice((1, 2, 4, 8))
        return min(most, kv * rng.choice((1, 1, 2, 3, 4, 8))) // kv * kv, kv

    op = rng.choice(("prefill", "prefill", "train", "train", "decode", "decode", "embedding", "embedding grad", "embedding step"))
    dtype = rng.choice(("bf16", "bf16", "f16"))
    if op in ("prefill", "train"):
        q_heads, kv_heads = heads(32)
        batch = rng.choice((1, 1, 2, 3, 5, 8))
        ragged = rng.random() < 0.3 and batch > 1
        most = (1.2e9 if op == "train" else 2.4e9) / q_heads          # pairs of a head's queries and keys
        length = logint(1, int(math.sqrt(most if ragged else most / batch)))
        window = 0 if rng.random() < 0.25 else logint(8, max(9, length))
        sinks = rng.choice((0, 4, logint(1, 200)))
        past = rng.choice((0, 0, logint(1, 500))) if op == "prefill" else 0
        return _attention(op, batch, length, q_heads, kv_heads, rng.choice((64, 64, 80, 96, 128, 128)), window, sinks, dtype, past, ragged)
    if op == "decode":
        q_heads, kv_heads = heads(32)
        batch = logint(1, 64)
        length = logint(1, max(2, min(60000, int(3.5e6 / (batch * kv_heads)))))
        window = 0 if rng.random() < 0.5 else logint(8, max(9, length))
        return _decode(batch, length, q_heads, kv_heads, rng.choice((64, 80, 128, 128)), window, rng.choice((0, 4, logint(1, 200))),
                       rng.choice((1, 16, 16, 32, 64, 256)), dtype)
    columns = logint(8, 4096) if rng.random() < 0.5 else rng.choice((64, 128, 512, 1024, 2048, 4096))
    return _embedding(op, logint(1, 16384), logint(16, 32000), columns, rng.choice(("bf16", "f16", "f32")))


def _lengths(case):
    """Queries of each sequence: a part of them each, the second one empty, the third one of one token."""
    if not case["ragged"]:
        return [case["length"]] * case["batch"]
    rng, n = random.Random(case["length"] * 31 + case["batch"]), case["batch"]
    share = [0.0 if i == 1 else rng.uniform(0.2, 1.8) for i in range(n)]
    got = [0 if i == 1 else max(1, int(case["length"] * s / sum(share))) for i, s in enumerate(share)]
    if n > 2:
        got[2] = 1
    return got


def _visible(queries, keys, window, sinks):
    """Pairs of queries and keys that see each other."""
    first, last = keys - queries + 1, keys              # visible keys of the first and the last query without a window
    full = lambda n: n * (n + 1) // 2 if n > 0 else 0    # noqa: E731
    rows = lambda cap: (full(min(last, cap)) - full(min(first - 1, cap))) + cap * max(0, last - max(first - 1, cap))   # noqa: E731
    if not window:
        return rows(last)
    # those in the window, and those of the first keys that have left it: row with n keys has min(max(n - window, 0), sinks)
    left = lambda n: full(min(n, sinks)) + sinks * max(0, n - sinks) if n > 0 else 0   # noqa: E731
    return rows(window) + left(last - window) - left(first - 1 - window)


def work(case):
    size = TYPES[case["dtype"]].itemsize
    if case["op"] in ("prefill", "train"):
        dim, q_heads, kv_heads = case["dim"], case["q_heads"], case["kv_heads"]
        lengths = _lengths(case)
        pairs = sum(_visible(n, n + case["past"] if n else 0, case["window"], case["sinks"]) for n in lengths) * q_heads
        q = sum(lengths) * q_heads * dim * size
        k = sum(n + case["past"] if n else 0 for n in lengths) * kv_heads * dim * size
        lse = 4 * sum(lengths) * q_heads
        if case["op"] == "prefill":
            return {"bytes": 2 * q + 2 * k + lse, "flops": 4 * dim * pairs}
        return {"bytes": 4 * q + 4 * k + lse, "flops": 14 * dim * pairs}
    if case["op"] == "decode":
        seen = sum(_keys_of_a_token(n, case["window"], case["sinks"]) for n in _cached(case))
        row = case["dim"] * size
        return {"bytes": 2 * row * case["kv_heads"] * seen + 2 * row * case["batch"] * (case["q_heads"] + 2 * case["kv_heads"]) + 4 * (seen // case["page"]),
                "flops": 4 * case["dim"] * case["q_heads"] * seen}
    tokens, rows, row = case["tokens"], case["rows"], case["columns"] * size
    ids = _ids(case, 0, "cpu")
    distinct = int(torch.unique(ids[ids >= 0]).numel())
    lookup, grad = distinct * row + tokens * (row + 8), tokens * (row + 8) + rows * row
    return {"bytes": (lookup if case["op"] != "embedding grad" else 0) + (grad if case["op"] != "embedding" else 0), "flops": tokens * case["columns"]}


def _keys_of_a_token(length, window, sinks):
    first = max(0, length - window) if window else 0
    return min(sinks, first) + length - first


def _cached(case):
    """Tokens of each sequence, the new one among them."""
    rng = random.Random(case["length"] * 17 + case["batch"])
    return [case["length"]] + [rng.randint(max(1, case["length"] // 4), case["length"]) for _ in range(case["batch"] - 1)]


# ------------------------------------------------------------------------------------------------
# the inputs
# ------------------------------------------------------------------------------------------------
def _ids(case, seed, device):
    """Tokens as a text has them, the n-th most frequent one about 1 / n of the time; one in a hundred is padding (-1)."""
    g = torch.Generator(device=device).manual_seed(seed * 7 + 3)
    u = torch.rand(case["tokens"], device=device, generator=g, dtype=torch.float64)
    ids = (torch.exp(u * math.log(case["rows"] + 1.0)) - 1.0).long().clamp_(0, case["rows"] - 1)
    pad = torch.rand(case["tokens"], device=device, generator=g) < 0.01
    return torch.where(pad, -1, ids)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    dtype = TYPES[case["dtype"]]

    def normal(*shape, by=1.0):
        return torch.randn(*shape, device=DEV, generator=g, dtype=dtype).mul_(by)

    s = {"case": dict(case)}
    if case["op"] in ("prefill", "train"):
        lengths, dim, past = _lengths(case), case["dim"], case["past"]
        keys = [n + past if n else 0 for n in lengths]
        if case["ragged"]:
            lead_q, lead_k = (sum(lengths),), (sum(keys),)
            s["q_len"], s["k_len"] = max(lengths), max(keys)
            for name, of in (("q_offsets", lengths), ("k_offsets", keys)):
                s[name] = torch.tensor([sum(of[:i]) for i in range(len(of) + 1)], dtype=torch.int32, device=DEV)
        else:
            lead_q, lead_k = (case["batch"], case["length"]), (case["batch"], case["length"] + past)
        # scores of deviation 2: some keys stand out
        s["q"], s["k"] = normal(*lead_q, case["q_heads"], dim, by=2.0), normal(*lead_k, case["kv_heads"], dim)
        s["v"] = normal(*lead_k, case["kv_heads"], dim)
        if case["op"] == "train":
            s["do"] = normal(*lead_q, case["q_heads"], dim)
        return s
    if case["op"] == "decode":
        lengths, page, window = _cached(case), case["page"], case["window"]
        shape = (case["kv_heads"], case["dim"])
        at = torch.tensor(lengths, device=DEV)
        columns = -(-max(lengths) // page)
        # pages that nobody sees any more are given back: their entries are -1
        first = (torch.arange(columns, device=DEV) * page)[None, :]
        kept = first < at[:, None]
        if window:
            kept &= (first + page > at[:, None] - window) | (first < case["sinks"])
        pages = int(kept.sum())
        table = torch.full((case["batch"], columns), -1, dtype=torch.int32, device=DEV)
        table[kept] = torch.randperm(pages, device=DEV, generator=g).int()
        s.update(table=table, lengths=at.int(), max_len=max(lengths), k_cache=normal(pages, page, *shape), v_cache=normal(pages, page, *shape),
                 q=normal(case["batch"], case["q_heads"], case["dim"], by=2.0), k=normal(case["batch"], *shape), v=normal(case["batch"], *shape))
        return s
    s["ids"] = _ids(case, seed, DEV)
    s["scale"] = math.sqrt(case["columns"])
    if case["op"] != "embedding grad":
        s["W"] = normal(case["rows"], case["columns"], by=0.02)
    if case["op"] != "embedding":
        s["dY"] = normal(case["tokens"], case["columns"])
    return s


# ------------------------------------------------------------------------------------------------
# a pass
# ------------------------------------------------------------------------------------------------
def run(s):
    return _kernels(s) if own else _plain(s)


def _kernels(s):
    from paper_2307_05740_amd.attention import ArrowAttention
    from paper_2307_05740_amd.embedding import ArrowEmbedding
    c = s["case"]
    if "op" not in s:                      # what a program keeps for as long as it runs: the mask, and room to work in
        s["op"] = (ArrowEmbedding(c["rows"], scale=s["scale"], device=DEV) if "rows" in c else
                   ArrowAttention(window=c["window"], sinks=c["sinks"], device=DEV))
    op = s["op"]
    if c["op"] == "decode":
        o = op.decode(s["q"], s["k_cache"], s["v_cache"], s["table"], s["lengths"], s["max_len"], k=s["k"], v=s["v"])
        return {"o": o, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    if c["op"] in ("prefill", "train"):
        ragged = {n: s[n] for n in ("q_offsets", "k_offsets", "q_len", "k_len")} if c["ragged"] else {}
        o, lse = op.forward(s["q"], s["k"], s["v"], **ragged)
        if c["op"] == "prefill":
            return {"o": o, "lse": lse}
        dq, dk, dv = op.backward(s["do"], s["q"], s["k"], s["v"], o, lse, **ragged)
        return {"o": o, "lse": lse, "dq": dq, "dk": dk, "dv": dv}
    out = {}
    if c["op"] != "embedding grad":
        out["Y"] = op.forward(s["W"], s["ids"])
    if c["op"] != "embedding":
        out["dW"] = op.backward(s["dY"], s["ids"])
    return out


def _plain(s):
    c = s["case"]
    if c["op"] == "decode":
        return _plain_decode(s)
    if c["op"] in ("prefill", "train"):
        return _plain_attention(s)
    out = {}
    ids, known = s["ids"].clamp(min=0), (s["ids"] >= 0)[:, None]
    if "W" in s:
        out["Y"] = torch.where(known, s["W"][ids].float() * s["scale"], 0.0).to(s["W"].dtype)
    if "dY" in s:
        dW = torch.zeros(c["rows"], c["columns"], dtype=torch.float32, device=DEV)
        dW.index_add_(0, ids, torch.where(known, s["dY"].float() * s["scale"], 0.0))
        out["dW"] = dW.to(s["dY"].dtype)
    return out


def _plain_mask(s):
    """(queries, keys) truth values; of a ragged batch: of all its tokens."""
    c = s["case"]
    if c["ragged"]:
        seq = []
        for name, t in (("q_offsets", s["q"]), ("k_offsets", s["k"])):
            seq.append(torch.searchsorted(s[name][1:].contiguous(), torch.arange(t.shape[0], device=DEV, dtype=torch.int32), right=True))
        qo, ko = s["q_offsets"], s["k_offsets"]
        p = (torch.arange(s["q"].shape[0], device=DEV) - qo[seq[0]] + (ko[seq[0] + 1] - ko[seq[0]]) - (qo[seq[0] + 1] - qo[seq[0]]))[:, None]
        j = (torch.arange(s["k"].shape[0], device=DEV) - ko[seq[1]])[None, :]
        same = seq[0][:, None] == seq[1][None, :]
    else:
        p = (torch.arange(c["length"], device=DEV) + c["past"])[:, None]
        j = torch.arange(c["length"] + c["past"], device=DEV)[None, :]
        same = True
    seen = (j <= p) & same
    if c["window"]:
        seen &= (j > p - c["window"]) | (j < c["sinks"])
    return seen


def _plain_attention(s):
    c, dtype = s["case"], s["q"].dtype
    kv, group, dim = c["kv_heads"], c["q_heads"] // c["kv_heads"], c["dim"]
    scale = 1.0 / math.sqrt(dim)
    batch = 1 if c["ragged"] else c["batch"]

    def split(t):                                  # (batch, key head, query heads of it x tokens, dim) in 32 bits
        t = t.reshape(batch, -1, kv, t.shape[-2] // kv, dim)
        return t.permute(0, 2, 3, 1, 4).float()

    q, k, v = split(s["q"]), split(s["k"])[:, :, 0].contiguous(), split(s["v"])[:, :, 0].contiguous()
    n, m = q.shape[3], k.shape[2]
    q = q.reshape(batch, kv, group * n, dim)
    seen = _plain_mask(s)
    x = (torch.matmul(q, k.transpose(2, 3).contiguous()) * scale).reshape(batch, kv, group, n, m).masked_fill_(~seen, -INF)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -INF, 0.0, top)
    p = x.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    lse = (top + total.log()).squeeze(-1)
    p = p.div_(torch.where(total == 0, 1.0, total)).reshape(batch, kv, group * n, m)
    o = torch.matmul(p, v)

    def join(t, tokens):                           # back to (batch, tokens, heads, dim)
        t = t.reshape(batch, -1, tokens, dim).transpose(1, 2).to(dtype).contiguous()
        return t[0] if c["ragged"] else t

    lse = lse.reshape(batch, kv * group, n)
    out = {"o": join(o, n), "lse": lse[0] if c["ragged"] else lse}
    if c["op"] == "train":
        do = split(s["do"]).reshape(batch, kv, group * n, dim)
        ds = torch.matmul(do, v.transpose(2, 3).contiguous()).sub_((do * o).sum(-1, keepdim=True)).mul_(p).mul_(scale)
        dv = torch.matmul(p.transpose(2, 3).contiguous(), do)
        out.update(dq=join(torch.matmul(ds, k), n), dk=join(torch.matmul(ds.transpose(2, 3).contiguous(), q), m), dv=join(dv, m))
    return out


def _plain_decode(s):
    c = s["case"]
    kv, group, dim, page = c["kv_heads"], c["q_heads"] // c["kv_heads"], c["dim"], c["page"]
    rows, length = torch.arange(c["batch"], device=DEV), s["lengths"].long()
    # the new token's place
    at = s["table"][rows, (length - 1) // page].long() * page + (length - 1) % page
    s["k_cache"].view(-1, kv, dim)[at] = s["k"]
    s["v_cache"].view(-1, kv, dim)[at] = s["v"]
    # the visible keys: the first ones that have left the window, then the window
    first = (length - c["window"]).clamp(min=0) if c["window"] else torch.zeros_like(length)
    sinks = first.clamp(max=c["sinks"])
    most = _keys_of_a_token(s["max_len"], c["window"], c["sinks"])
    i = torch.arange(most, device=DEV)[None, :]
    j = torch.where(i < sinks[:, None], i, i - sinks[:, None] + first[:, None])
    seen = j < length[:, None]
    j = torch.where(seen, j, length[:, None] - 1)
    at = torch.gather(s["table"].long(), 1, j // page) * page + j % page
    k = s["k_cache"].view(-1, kv, dim)[at].float().permute(0, 2, 3, 1).contiguous()
    v = s["v_cache"].view(-1, kv, dim)[at].float().permute(0, 2, 1, 3).contiguous()
    x = torch.matmul(s["q"].reshape(c["batch"], kv, group, dim).float(), k) * (1.0 / math.sqrt(dim))
    x = x.masked_fill_(~seen[:, None, None, :], -INF)
    p = torch.exp(x - x.amax(-1, keepdim=True))
    o = torch.matmul(p / p.sum(-1, keepdim=True), v)
    return {"o": o.reshape(c["batch"], kv * group, dim).to(s["q"].dtype), "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


# ------------------------------------------------------------------------------------------------
# the definition in 64 bits, one sequence and head after the other
# ------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "decode":
        return _exact_decode(s)
    if case["op"] in ("prefill", "train"):
        return _exact_attention(s)
    ids, scale = s["ids"], s["scale"]
    out = {}
    if "W" in s:
        padded = torch.cat([s["W"].double(), torch.zeros(1, case["columns"], dtype=torch.float64, device=DEV)])
        out["Y"] = padded[ids] * scale           # (-1 is the last row)
    if "dY" in s:
        dW = torch.zeros(case["rows"] + 1, case["columns"], dtype=torch.float64, device=DEV)
        order = torch.argsort(ids, stable=True)
        for part in order.split(1024):
            dW.index_put_((ids[part],), s["dY"][part].double() * scale, accumulate=True)
        out["dW"] = dW[:-1]
    return out


def _exact_attention(s):
    c = s["case"]
    dim, group = c["dim"], c["q_heads"] // c["kv_heads"]
    train = c["op"] == "train"
    grads = {"dq": "q", "dk": "k", "dv": "v"} if train else {}
    flat = {n: s[n].reshape(-1, *s[n].shape[-2:]) for n in ("q", "k", "v", "do") if n in s}
    out = {"o": torch.zeros(flat["q"].shape, dtype=torch.float64, device=DEV),
           "lse": torch.full((c["q_heads"], flat["q"].shape[0]), -INF, dtype=torch.float64, device=DEV)}
    for n, of in grads.items():
        out[n] = torch.zeros(flat[of].shape, dtype=torch.float64, device=DEV)
    q0 = k0 = 0
    for n in _lengths(c):
        m = n + c["past"] if n else 0
        if n == 0:
            continue
        ago = torch.arange(m - n, m, device=DEV)[:, None] - torch.arange(m, device=DEV)[None, :]
        hidden = ago < 0
        if c["window"]:
            hidden |= (ago >= c["window"]) & (torch.arange(m, device=DEV) >= c["sinks"])[None, :]
        for h in range(c["q_heads"]):
            q = flat["q"][q0:q0 + n, h].double()
            k, v = (flat[t][k0:k0 + m, h // group].double() for t in ("k", "v"))
            x = (q @ k.T / math.sqrt(dim)).masked_fill_(hidden, -INF)
            lse = torch.logsumexp(x, -1)
            p = x.sub_(lse[:, None]).exp_()
            o = p @ v
            out["o"][q0:q0 + n, h], out["lse"][h, q0:q0 + n] = o, lse
            if train:
                do = flat["do"][q0:q0 + n, h].double()
                out["dv"][k0:k0 + m, h // group] += p.T @ do
                ds = p.mul_((do @ v.T) - (do * o).sum(-1)[:, None]) / math.sqrt(dim)
                out["dq"][q0:q0 + n, h] = ds @ k
                out["dk"][k0:k0 + m, h // group] += ds.T @ q
        q0, k0 = q0 + n, k0 + m
    if not c["ragged"]:
        out["lse"] = out["lse"].reshape(c["q_heads"], c["batch"], -1).transpose(0, 1).contiguous()
        for n, of in dict(o="q", **grads).items():
            out[n] = out[n].reshape(s[of].shape)
    return out


def _exact_decode(s):
    c = s["case"]
    dim, group, page = c["dim"], c["q_heads"] // c["kv_heads"], c["page"]
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    for b, n in enumerate(s["lengths"].tolist()):
        pos = torch.arange(n, device=DEV)
        if c["window"]:
            pos = pos[(pos >= n - c["window"]) | (pos < c["sinks"])]
        where = s["table"][b].long()[pos // page]
        slot = pos % page
        new = (pos == n - 1)[:, None, None]
        k = torch.where(new, s["k"][b].double(), s["k_cache"][where, slot].double())
        v = torch.where(new, s["v"][b].double(), s["v_cache"][where, slot].double())
        for h in range(c["q_heads"]):
            x = k[:, h // group] @ s["q"][b, h].double() / math.sqrt(dim)
            o[b, h] = torch.softmax(x, 0) @ v[:, h // group]
    return {"o": o, "k_cache": None, "v_cache": None}
