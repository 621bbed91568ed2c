"""Rounds of a federated language model on one GPU, from tokens to weights.

Every round, for all clients at once:

1. the clients look their tokens up in their embedding tables (``Embedding.lookup``);
2. a small model -- one matrix, output projection tied to the table -- gives the loss and its gradients, which are
   written into the clients' rows of the update matrix; the table's gradient has two parts, the output projection's
   product and, added to it, the sums over the sorted tokens (``Embedding.grad`` with ``accumulate``);
3. the Byzantine clients alter their rows, the ring aggregates the signs (``Brace.inject_attack``, ``aggregate``);
4. the clients' tables move by the aggregate (``Brace.apply_update``), their matrix by its orthogonalised momentum,
   read straight from the packed consensus bits (``Orthogonalizer.muon_step`` with all clients as replicas).

The text is synthetic: the next token is a fixed permutation of the present one.  Run: ``python
examples/language_model_round.py``.
"""

from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2501_17392_b200 import brace as B  # noqa: E402


def train(rounds=40, clients=10, byzantine=2, vocab=300, dim=64, tokens=256, eta=8e-3, lr=0.05, seed=0, log=None):
    """Mean loss over the clients at each round."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n, square, table = clients, dim * dim, vocab * dim
    d = table + square
    ld = (d + 127) // 128 * 128
    start = torch.zeros(ld, device="cuda")
    start[:table] = torch.randn(table, device="cuda", generator=gen) * 0.02
    start[table:d] = torch.eye(dim, device="cuda").flatten() * 0.5
    weights = start.repeat(n, 1)                    # client c's parameters are row c
    updates = torch.zeros(n, ld, device="cuda")
    tables, grads = (x.as_strided((n, vocab, dim), (ld, dim, 1)) for x in (weights, updates))
    matrix, dmatrix = (x.as_strided((n, dim, dim), (ld, dim, 1), table) for x in (weights, updates))
    momentum = torch.zeros(dim, dim, device="cuda")
    follows = torch.randperm(vocab, device="cuda", generator=gen)
    scale = math.sqrt(dim)

    embedding = B.Embedding(vocab, dim, tokens, clients=n)
    square_step = B.Orthogonalizer(dim, dim)
    ring = B.Brace(n, byzantine, d, B.default_params(lam=0.0))
    ring_table = B.Brace(n, 0, table, B.default_params(lam=0.0))    # the same rows, up to the end of the table
    attack = B.make_attack(B.ATTACK_SCALE_OWN, scale=-10.0)
    out = ring.new_output()
    h = torch.empty(n, tokens, dim, device="cuda")
    losses = []
    for _ in range(rounds):
        ids = torch.randint(0, vocab, (n, tokens), device="cuda", generator=gen)
        embedding.lookup(tables, ids, h, scale=scale)
        z = h @ matrix
        logits = z @ tables.mT
        target = follows[ids][..., None]
        logp = logits.log_softmax(-1)
        losses.append(-logp.gather(-1, target).mean())
        dlogits = logp.exp().scatter_add(-1, target, -torch.ones_like(target, dtype=torch.float32)) / tokens
        dz = dlogits @ tables
        grads.copy_(dlogits.mT @ z)
        dmatrix.copy_(h.mT @ dz)
        embedding.grad(dz @ matrix.mT, ids, grads, scale=scale, accumulate=True)
        ring.inject_attack(attack, updates, updates)
        ring.aggregate(updates, out)
        ring_table.apply_update(out, weights, eta)
        square_step.muon_step(out[0], momentum, matrix[:, None], lr, bit_offset=table)
        if log:
            log(f"round {len(losses)}: loss {float(losses[-1]):.4f}")
    square_step.check()
    assert bool((weights == weights[0]).all()), "the clients' weights differ"
    return [float(x) for x in losses]


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--rounds", type=int, default=40)
    ap.add_argument("--clients", type=int, default=10)
    ap.add_argument("--byzantine", type=int, default=2)
    a = ap.parse_args()
    train(a.rounds, a.clients, a.byzantine, log=print)
