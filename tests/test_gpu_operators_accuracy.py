"""Accuracy of the orthogonalised update over spectra, against 64 bits.

Where the singular values fall off, a rounding error outside the matrix's range grows by a = 3.4445 a step while the matrix
itself grows to about 1.  The bound follows the norms of the iteration: in step k the operands X, S and P are rounded and
their products summed, each off by u of its size at random, u = 2^-22 where an operand is two float16 planes; what that
makes of the step's X is off by u |X_k| for each of the four, and grows by at most a^(steps - k) to the end.  The four of
each step are independent:  u sqrt(4 sum_k (|X_k| a^(steps - k))^2) of the result's norm."""

import pytest
import torch

from paper_2501_17392_b200 import brace as B

pytestmark = pytest.mark.gpu

A0, B0, C0, STEPS = 3.4445, -4.7750, 2.0315, 5


def update(rows, cols, spectrum, seed):
    """Noise of full rank, singular values 1 / i^2, or a product of that rank."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    k = min(rows, cols)
    if spectrum == "full":
        return torch.randn(rows, cols, device="cuda", generator=g)
    if spectrum == "decay":
        u, v = (torch.linalg.qr(torch.randn(n, k, device="cuda", generator=g))[0] for n in (rows, cols))
        return (u / torch.arange(1, k + 1, device="cuda").float() ** 2) @ v.mT
    return torch.randn(rows, spectrum, device="cuda", generator=g) @ torch.randn(spectrum, cols, device="cuda", generator=g)


def iteration(x, dtype=torch.float64):
    """The result, and the Frobenius norms of X_0 .. X_(steps - 1)."""
    a, b, c, eps = (float(torch.tensor(v)) for v in (A0, B0, C0, 1e-7))
    x = x.to(dtype)
    x = x / (x.square().sum().sqrt() + eps)
    turn = x.shape[0] > x.shape[1]
    x, norms = x.mT if turn else x, []
    for _ in range(STEPS):
        norms.append(float(x.norm()))
        s = x @ x.mT
        x = a * x + (b * s + c * (s @ s)) @ x
    return x.mT if turn else x, norms


def rel(got, want):
    return float((got.double() - want).norm() / want.norm())


def limit(want, norms, u=2.0 ** -22):
    grown = sum(4 * (n * A0 ** (STEPS - k)) ** 2 for k, n in enumerate(norms)) ** 0.5
    return u * grown / float(want.norm())


# one launch by one CTA and by several, tiles by one CTA, shared contractions, and tiles by pairs of CTAs
SHAPES = [(64, 64), (100, 90), (120, 600), (600, 120), (128, 1500), (200, 333), (333, 200), (600, 600), (300, 2400),
          (1500, 1500), (1990, 2000), (2100, 1800)]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("spectrum", ["full", "decay", 1, 4, 33])
def test_bfloat16_results_lose_their_own_rounding_only(shape, spectrum):
    g = update(*shape, spectrum, seed=shape[0])
    want, norms = iteration(g)
    out = torch.empty(shape, device="cuda", dtype=torch.bfloat16)
    B.Orthogonalizer(*shape).orthogonalize(g, out)
    # rounding the 64-bit result loses the same up to the elements' luck: a twentieth of it for 4096 elements and more
    assert rel(out, want) <= 1.05 * rel(want.bfloat16(), want) + limit(want, norms)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("spectrum", ["decay", 1, 4, 33])
def test_other_results_on_low_ranks(shape, dtype, spectrum):
    g = update(*shape, spectrum, seed=shape[0] + 1)
    want, norms = iteration(g)
    out = torch.empty(shape, device="cuda", dtype=dtype)
    B.Orthogonalizer(*shape).orthogonalize(g, out)
    own = 1.05 * rel(want.half(), want) if dtype == torch.float16 else 2.0 ** -24
    assert rel(out, want) <= own + limit(want, norms)


@pytest.mark.parametrize("spectrum", ["full", 1, 33])
def test_weights_in_bfloat16_take_the_whole_step(spectrum):
    # weights of zero: what is stored is the step itself
    shape = (300, 500)
    g = update(*shape, spectrum, seed=7)
    want, norms = iteration(g)
    m, w = torch.zeros(shape, device="cuda"), torch.zeros(shape, device="cuda", dtype=torch.bfloat16)
    B.Orthogonalizer(*shape).muon_step(g, m, w, lr=1.0, nesterov=False)
    assert rel(-w, want) <= 1.05 * rel(want.bfloat16(), want) + limit(want, norms)


@pytest.mark.parametrize("shape", [(64, 64), (600, 600), (1500, 1500)])
@pytest.mark.parametrize("spectrum", ["full", 1, 33])
def test_half_precision_is_what_it_says(shape, spectrum):
    # asked for by name: one float16 plane an operand, with what low ranks make of it
    g = update(*shape, spectrum, seed=3)
    want, norms = iteration(g)
    out = torch.empty(shape, device="cuda")
    B.Orthogonalizer(*shape, params=B.ortho_params(precision=B.ORTHO_HALF)).orthogonalize(g, out)
    assert rel(out, want) <= limit(want, norms, u=2.0 ** -11)


@pytest.mark.parametrize("shape", [(512, 512), (768, 768), (700, 1400), (1300, 800), (1024, 1024), (1400, 1400)])
@pytest.mark.parametrize("spectrum", ["full", "decay", 1, 4, 33])
def test_float32_results_are_no_worse_than_float32_products(shape, spectrum):
    # the claim itself, on the same input: from a short side of 512 on the error is not above plain float32's
    g = update(*shape, spectrum, seed=shape[1])
    want, _ = iteration(g)
    out = torch.empty(shape, device="cuda")
    B.Orthogonalizer(*shape).orthogonalize(g, out)
    assert rel(out, want) <= rel(iteration(g, torch.float32)[0], want)
