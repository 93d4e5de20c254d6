#!/usr/bin/env python3
"""A small language model over a stream, from training to serving, with the operators on sequences run together.

Training: embedding lookup -> layers of attention with a window and first tokens that stay visible -> logits by the tied table, and the
gradients of all of it (the table's from the lookup by sorted tokens).  Serving: the prompt goes through the same forward call and into a
cache in pages, then tokens come one by one over that cache; pages that have left the window are given back and used
again.  The text is synthetic: each sequence keeps to eight tokens of its own, which the model has to pick up from what it sees.

    python examples/stream_model.py [--steps 200] [--tokens 200] [--positions] [--entropy 0.01] [--bits 4]

Prints the loss at both ends, and how far the logits of single tokens are from those of the whole sequence.  --positions: queries and keys are normed for each head
and rotated by their position.  --entropy: the loss is that of log probabilities from their own operator, less so much of the entropy.  --bits 4: served over a cache
in 4 bits, whose pages are handed out on the GPU; logits then differ by what the cache rounds, too.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2307_05740_amd.attention import ArrowAttention      # noqa: E402
from paper_2307_05740_amd.embedding import ArrowEmbedding      # noqa: E402
from paper_2307_05740_amd.logprobs import ArrowLogProbs        # noqa: E402
from paper_2307_05740_amd.packed import ArrowPackedAttention   # noqa: E402
from paper_2307_05740_amd.pages import ArrowPages              # noqa: E402
from paper_2307_05740_amd.rotation import ArrowRotation        # noqa: E402

DEV = "cuda:0"


class StreamModel(torch.nn.Module):
    def __init__(self, vocabulary=128, width=256, layers=2, heads=8, kv_heads=2, window=48, sinks=4, positions=False):
        super().__init__()
        self.heads, self.kv_heads, self.dim, self.vocabulary = heads, kv_heads, width // heads, vocabulary
        g = torch.Generator().manual_seed(1)
        weight = lambda *s: torch.nn.Parameter((torch.randn(*s, generator=g) * s[0] ** -0.5).to(DEV))   # noqa: E731
        self.table = torch.nn.Parameter((torch.randn(vocabulary, width, generator=g) * width ** -0.5).to(DEV))
        self.qkv = torch.nn.ParameterList(weight(width, (heads + 2 * kv_heads) * self.dim) for _ in range(layers))
        self.out = torch.nn.ParameterList(weight(width, width) for _ in range(layers))
        self.embed = ArrowEmbedding(vocabulary, scale=width ** 0.5, device=DEV)
        self.attend = ArrowAttention(window, sinks, device=DEV)
        self.rotate = ArrowRotation(self.dim, device=DEV) if positions else None
        self.norms = torch.nn.ParameterList(torch.nn.Parameter(torch.ones(self.dim, device=DEV)) for _ in range(2 * layers if positions else 0))

    def split(self, x, layer, lengths=None):
        """Queries, keys and values, (..., heads, dim): views of one tensor, of which the first two may be normed and rotated.  lengths: of sequences whose last token x is."""
        x = torch.nn.functional.rms_norm(x, x.shape[-1:]) @ self.qkv[layer].bfloat16()
        q, k, v = x.unflatten(-1, (-1, self.dim)).split((self.heads, self.kv_heads, self.kv_heads), -2)
        if self.rotate is not None:
            at = {} if lengths is None else {"positions": lengths, "shift": -1}
            q, k = self.rotate(q, k, self.norms[2 * layer], self.norms[2 * layer + 1], **at)
        return q, k, v

    def logits(self, x):
        return torch.nn.functional.rms_norm(x, x.shape[-1:]).float() @ self.table.T

    def forward(self, ids, caches=None):
        """Logits of (batch, tokens); with caches, the keys and values of each layer go to them."""
        x = self.embed(self.table.bfloat16(), ids)
        for layer in range(len(self.qkv)):
            q, k, v = self.split(x, layer)
            if caches is not None:
                caches.append(layer, k, v)
            x = x + self.attend(q, k, v).flatten(-2) @ self.out[layer].bfloat16()
        return self.logits(x)

    def step(self, ids, caches):
        """Logits of one new token per sequence, (batch)."""
        x = self.embed(self.table.bfloat16(), ids)
        for layer in range(len(self.qkv)):
            q, k, v = self.split(x, layer, caches.lengths)
            o = caches.decode(layer, q, k, v)
            x = x + o.flatten(-2) @ self.out[layer].bfloat16()
        return self.logits(x)


class Caches:
    """Pages of all layers, and who has which.  A sequence keeps the pages that its window and the first tokens lie in."""

    def __init__(self, model, batch, columns, pages, page=16):
        shape = (pages, page, model.kv_heads, model.dim)
        self.page, self.window, self.sinks, self.attend = page, model.attend.window, model.attend.sinks, model.attend
        self.pools = [[torch.empty(shape, dtype=torch.bfloat16, device=DEV) for _ in range(2)] for _ in model.qkv]
        self.free = list(range(pages))
        self.of = [dict() for _ in range(batch)]                  # column -> page
        self.host = torch.full((batch, columns), -1, dtype=torch.int32)
        self.table = self.host.to(DEV)
        self.lengths = torch.zeros(batch, dtype=torch.int32, device=DEV)

    def append(self, layer, k, v):
        self.attend.append(k, v, *self.pools[layer], self.table, self.lengths)

    def decode(self, layer, q, k, v):
        return self.attend.decode(q, *self.pools[layer], self.table, self.lengths, k=k, v=v)

    def grow(self, length):
        """Room for all sequences to have `length` tokens; what nobody sees any more is given back."""
        self.lengths.fill_(length)
        changed = False
        for row, own in zip(self.host, self.of):
            for c in [c for c in own if (c + 1) * self.page <= length - self.window and c * self.page >= self.sinks]:
                self.free.append(own.pop(c))
                row[c] = -1
                changed = True
            for c in range((length + self.page - 1) // self.page):
                seen = (c + 1) * self.page > length - self.window or c * self.page < self.sinks
                if seen and c not in own:
                    own[c] = self.free.pop(0)
                    row[c] = own[c]
                    changed = True
        if changed:
            self.table.copy_(self.host)


class PackedCaches:
    """The same in 4 bits; who has which page is known on the GPU only."""

    def __init__(self, model, batch, columns, pages, page=16):
        window, sinks = model.attend.window, model.attend.sinks
        self.pages, self.attend = ArrowPages(pages, page, window, sinks, device=DEV), ArrowPackedAttention(window, sinks, device=DEV)
        self.pools = [self.attend.pool(pages, page, model.kv_heads, model.dim) for _ in model.qkv]
        self.table, self.held, self.free = self.pages.state(batch, columns)
        self.lengths, self.length, self.slots = torch.zeros(batch, dtype=torch.int32, device=DEV), 0, None

    def append(self, layer, k, v):
        self.attend.append(k.flatten(0, 1), v.flatten(0, 1), self.pools[layer], self.slots)

    def decode(self, layer, q, k, v):
        return self.attend.decode(q, self.pools[layer], self.table, self.lengths, k=k, v=v)

    def grow(self, length):
        more, self.length = length - self.length, length
        self.lengths.fill_(length)
        self.slots = self.pages.step(self.table, self.held, self.free, self.lengths, more).flatten()


def text(batch, tokens, vocabulary, seed):
    """Sequences of eight tokens each: who knows which ones has a loss of ln 8."""
    g = torch.Generator().manual_seed(seed)
    own = torch.randint(0, vocabulary, (batch, 8), generator=g)
    return own.gather(1, torch.randint(0, 8, (batch, tokens), generator=g)).to(DEV)


def loss_of(logits, targets, entropy):
    """Cross entropy; with `entropy`, from log probabilities, less so much of the entropy."""
    if entropy is None:
        return torch.nn.functional.cross_entropy(logits.flatten(0, 1), targets.flatten())
    logp, h = ArrowLogProbs(device=DEV)(logits, targets)
    return -(logp + entropy * h).mean()


def train(model, steps, batch=32, tokens=128, entropy=None):
    optimizer = torch.optim.Adam(model.parameters(), lr=2e-3)
    losses = []
    for i in range(steps):
        ids = text(batch, tokens + 1, model.vocabulary, seed=i)
        loss = loss_of(model(ids[:, :-1]), ids[:, 1:], entropy)
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        losses.append(loss.detach())
    return float(losses[0]), float(losses[-1])


@torch.no_grad()
def serve(model, tokens, batch=3, prompt=40, bits=16):
    """Greedy tokens after a prompt; the largest difference of a step's logits from those of the whole sequence, over the latter's deviation."""
    page = 16
    kind = PackedCaches if bits == 4 else Caches
    caches = kind(model, batch, columns=(tokens + page - 1) // page, pages=batch * (model.attend.window // page + 4), page=page)
    ids = text(batch, prompt, model.vocabulary, seed=99)
    # (a prompt may be longer than what stays visible; its last tokens are all that a page is kept for)
    caches.grow(prompt)
    steps = [model(ids, caches)[:, -1]]
    for length in range(prompt + 1, tokens + 1):
        ids = torch.cat([ids, steps[-1].argmax(-1, keepdim=True)], 1)
        caches.grow(length)
        steps.append(model.step(ids[:, -1], caches))
    whole = model(ids)[:, prompt - 1:]
    return ids, float((torch.stack(steps, 1) - whole).abs().max() / whole.std())


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--tokens", type=int, default=200)
    ap.add_argument("--positions", action="store_true")
    ap.add_argument("--entropy", type=float)
    ap.add_argument("--bits", type=int, choices=(4, 16), default=16)
    a = ap.parse_args(argv)
    torch.manual_seed(0)
    model = StreamModel(positions=a.positions)
    first, last = train(model, a.steps, entropy=a.entropy)
    ids, off = serve(model, a.tokens, bits=a.bits)
    print(f"loss {first:.3f} -> {last:.3f} in {a.steps} steps; {ids.shape[1]} tokens served, logits within {off:.3f} deviations of the whole sequence's")
    return first, last, off


if __name__ == "__main__":
    main()
