"""Rounds of a federated transformer on one GPU: the local step of all clients, and their updates bounded before the ring.

Every round, for all clients at once:

1. the clients' tokens are looked up (``Embedding.lookup``), normalised (``LayerNorm.forward``), attend to one another in a
   sliding window with a few first tokens (``WindowAttention.forward``), and are normalised again; the output projection is
   tied to the table;
2. backward, the same way round (``LayerNorm.grad``, ``WindowAttention.grad``, ``Embedding.grad``): every gradient is written
   into its piece of the client's row of the update matrix;
3. the Byzantine clients alter their rows (``Brace.inject_attack``), every row is clipped to the same norm
   (``GradientClip.clip``), so that no client moves the sum by more than that, the ring adds the rows up (``Brace.aggregate``,
   plain-sum rule) and the clients' weights move (``Brace.apply_update``).

The text is synthetic: the next token is a fixed permutation of the one before the present.  Run: ``python
examples/transformer_round.py``.
"""

from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2501_17392_b200 import brace as B  # noqa: E402


class Transformer:
    """One block of `clients` clients: each client's parameters are a row of `weights`, their gradients a row of `updates`.
    `dtype` is the type of queries, keys, values and of what the attention makes of them."""

    def __init__(self, clients=8, vocab=300, dim=64, heads=4, tokens=128, window=32, sinks=2, dtype=torch.float32, seed=0):
        self.n, self.vocab, self.dim, self.heads, self.tokens, self.dtype = clients, vocab, dim, heads, tokens, dtype
        shapes = {"table": (vocab, dim), "scale1": (dim,), "shift1": (dim,), "qkv": (dim, 3 * dim), "mix": (dim, dim),
                  "scale2": (dim,), "shift2": (dim,)}
        self.d = sum(math.prod(s) for s in shapes.values())
        ld = (self.d + 127) // 128 * 128
        self.weights, self.updates = (torch.zeros(clients, ld, device="cuda") for _ in range(2))
        self.w, self.g, at = {}, {}, 0
        for name, s in shapes.items():
            size = math.prod(s)
            for rows, to in ((self.weights, self.w), (self.updates, self.g)):
                piece = rows[:, at:at + size]
                to[name] = piece.unflatten(1, s) if len(s) > 1 else piece
            at += size
        gen = torch.Generator(device="cuda").manual_seed(seed)
        for name in ("table", "qkv", "mix"):
            start = torch.randn(shapes[name], device="cuda", generator=gen) * (0.02 if name == "table" else dim ** -0.5)
            self.w[name].copy_(start)
        for name in ("scale1", "scale2"):
            self.w[name].fill_(1.0)
        self.embedding = B.Embedding(vocab, dim, tokens, clients=clients)
        self.norm = B.LayerNorm(dim, tokens, clients=clients)
        self.attention = B.WindowAttention(heads, dim // heads, tokens, batch=clients, window=window, sinks=sinks)
        t = (clients, tokens)
        self.h, self.x1, self.x2, self.dx, self.dr = (torch.empty(*t, dim, device="cuda") for _ in range(5))
        self.stats = [torch.empty(t, device="cuda") for _ in range(4)]
        self.out, self.dqkv = torch.empty(*t, heads, dim // heads, device="cuda", dtype=dtype), torch.empty(*t, 3 * dim, device="cuda", dtype=dtype)
        self.lse = torch.empty(clients, heads, tokens, device="cuda")

    def _split(self, x):
        """Queries, keys and values as views of their projection's result."""
        x = x.unflatten(2, (3 * self.heads, -1))
        return x[:, :, :self.heads], x[:, :, self.heads:2 * self.heads], x[:, :, 2 * self.heads:]

    def step(self, ids, target):
        """Mean loss of the clients' local batches; leaves every client's gradients in its row of `updates`."""
        w, g, scale = self.w, self.g, math.sqrt(self.dim)
        mean1, rstd1, mean2, rstd2 = self.stats
        self.embedding.lookup(w["table"], ids, self.h, scale=scale)
        self.norm.forward(self.h, self.x1, weight=w["scale1"], bias=w["shift1"], mean=mean1, rstd=rstd1)
        q, k, v = self._split((self.x1 @ w["qkv"]).to(self.dtype))
        self.attention.forward(q, k, v, self.out, lse=self.lse)
        mixed = self.out.flatten(2).float()
        r = self.h + mixed @ w["mix"]
        self.norm.forward(r, self.x2, weight=w["scale2"], bias=w["shift2"], mean=mean2, rstd=rstd2)
        logp = (self.x2 @ w["table"].mT).log_softmax(-1)
        loss = -logp.gather(-1, target[..., None]).mean()
        dlogits = logp.exp_().scatter_add_(-1, target[..., None], -torch.ones_like(target, dtype=torch.float32)[..., None]) / self.tokens
        g["table"].copy_(dlogits.mT @ self.x2)
        self.norm.grad(dlogits @ w["table"], r, mean2, rstd2, self.dr, weight=w["scale2"], dweight=g["scale2"], dbias=g["shift2"])
        g["mix"].copy_(mixed.mT @ self.dr)
        dout = (self.dr @ w["mix"].mT).to(self.dtype).unflatten(2, (self.heads, -1))
        self.attention.grad(dout, q, k, v, self.out, self.lse, *self._split(self.dqkv))
        dqkv = self.dqkv.float()
        g["qkv"].copy_(self.x1.mT @ dqkv)
        self.norm.grad(dqkv @ w["qkv"].mT, self.h, mean1, rstd1, self.dx, weight=w["scale1"], dweight=g["scale1"], dbias=g["shift1"])
        self.embedding.grad(self.dx.add_(self.dr), ids, g["table"], scale=scale, accumulate=True)
        return loss


def train(rounds=40, clients=8, byzantine=2, eta=0.3, max_norm=1.0, seed=0, log=None, **sizes):
    """Mean loss over the clients, and the clients' norms before clipping, at each round."""
    model = Transformer(clients, seed=seed, **sizes)
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    follows = torch.randperm(model.vocab, device="cuda", generator=gen)
    ring = B.Brace(clients, byzantine, model.d, B.default_params(rule=B.RULE_SUM, mean=1))
    attack = B.make_attack(B.ATTACK_SCALE_OWN, scale=-10.0)
    clip = B.GradientClip([model.updates[:, :model.d]])
    out, norms, losses = ring.new_output(), torch.empty(clients, device="cuda"), []
    for _ in range(rounds):
        text = torch.randint(0, model.vocab, (clients, model.tokens), device="cuda", generator=gen)
        target = follows[text.roll(1, 1)]      # of the token before: it has to be attended to
        losses.append(model.step(text, target))
        ring.inject_attack(attack, model.updates, model.updates)
        clip.clip(max_norm, norms=norms, nonfinite=B.CLIP_ZERO)
        ring.aggregate(model.updates, out)
        ring.apply_update(out, model.weights, eta)
        if log:
            log(f"round {len(losses)}: loss {float(losses[-1]):.4f}, norms {float(norms.min()):.2f} to {float(norms.max()):.2f}")
    assert bool((model.weights == model.weights[0]).all()), "the clients' weights differ"
    return [float(x) for x in losses], norms


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--rounds", type=int, default=40)
    ap.add_argument("--clients", type=int, default=8)
    ap.add_argument("--byzantine", type=int, default=2)
    a = ap.parse_args()
    train(a.rounds, a.clients, a.byzantine, log=print)
