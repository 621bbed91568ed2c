"""The operators of a client's local step together, as a round of a federated transformer uses them.

Gradients against automatic differentiation in 64 bits, relative to the 2-norm of a parameter's gradient: in float32 a value
passes through some 12 products and sums of up to 400 terms, each within sqrt(400) 2^-24 of itself in the root mean square:
12 * 20 * 2^-24 = 1.5e-5, taken times 10 for what the softmax and the norm amplify; in bfloat16 the attention's six tensors are
rounded once each, and p and ds inside: 8 * 2^-8."""

import importlib.util
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("transformer_round", os.path.join(ROOT, "examples", "transformer_round.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def loss64(w, ids, target, heads, window, sinks):
    """One client's loss."""
    dim, n = w["table"].shape[1], len(ids)
    h = w["table"][ids] * math.sqrt(dim)
    norm = lambda x, a, b: torch.nn.functional.layer_norm(x, (dim,), a, b, 1e-5)  # noqa: E731
    q, k, v = (norm(h, w["scale1"], w["shift1"]) @ w["qkv"]).view(n, 3, heads, -1).permute(1, 2, 0, 3)
    i = torch.arange(n, device="cuda")
    back = i[:, None] - i
    sees = (back >= 0) & ((back < window) | (i < sinks))
    p = ((q @ k.mT) / math.sqrt(dim // heads)).masked_fill(~sees, -math.inf).softmax(-1)
    r = h + (p @ v).transpose(0, 1).reshape(n, dim) @ w["mix"]
    return torch.nn.functional.cross_entropy(norm(r, w["scale2"], w["shift2"]) @ w["table"].mT, target)


@pytest.mark.parametrize("dtype,tolerance", [(torch.float32, 1.5e-4), (torch.bfloat16, 8 * 2.0 ** -8)])
def test_gradients_of_the_local_step(example, dtype, tolerance):
    sizes = dict(vocab=157, dim=64, heads=2, tokens=301, window=50, sinks=3)
    model = example.Transformer(3, dtype=dtype, seed=1, **sizes)
    gen = torch.Generator(device="cuda").manual_seed(2)
    model.weights += 0.05 * torch.randn(model.weights.shape, device="cuda", generator=gen)      # every client its own
    ids, target = (torch.randint(0, 157, (3, 301), device="cuda", generator=gen) for _ in range(2))
    loss = model.step(ids, target)
    total = 0.0
    for c in range(3):
        w = {k: x[c].double().requires_grad_() for k, x in model.w.items()}
        one = loss64(w, ids[c], target[c], 2, 50, 3)
        total += float(one.detach()) / 3
        for (name, _), want in zip(w.items(), torch.autograd.grad(one, list(w.values()))):
            got = model.g[name][c].double()
            assert float((got - want).norm() / want.norm()) <= tolerance, (c, name)
    assert abs(float(loss) - total) <= tolerance * total


def test_rounds_run_and_clipping_bounds_every_client(example):
    losses, norms = example.train(rounds=4, clients=5, byzantine=1, max_norm=0.25, vocab=50, dim=32, tokens=40, window=10)
    assert all(math.isfinite(x) for x in losses) and bool(norms.isfinite().all())
