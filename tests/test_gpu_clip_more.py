"""Clipping of values near the largest ones that float32 holds, as a Byzantine client may send them.

Bound: a norm within 10 roundings of 2^-24, the factor and two products (the second by a power of two) another 4, and half of the
smallest number where a result is below 2^-126."""

import pytest
import torch

from paper_2501_17392_b200 import brace as B

pytestmark = pytest.mark.gpu

u = 2.0 ** -24


@pytest.mark.parametrize("n", [300, 50001, 3_000_001])
@pytest.mark.parametrize("size,max_norm", [(1e37, 1.0), (1e37, 1e-6), (1e37, 1e-30), (3e38, 1e-3), (1e20, 1e-20), (1e37, 1e30),
                                           (1e37, 0.0), (3e38, 1e-45)])
@pytest.mark.parametrize("dtype,half", [(torch.float32, 2.0 ** -24), (torch.bfloat16, 2.0 ** -8)])
def test_clip_of_the_largest_values(n, size, max_norm, dtype, half):
    g = torch.Generator(device="cuda").manual_seed(n)
    x = (torch.rand(2, n, device="cuda", generator=g) * 2 - 1).mul_(size).to(dtype)
    x[1, ::7] = 0
    y = torch.empty(2, n, device="cuda", dtype=dtype)
    B.GradientClip([x], [y]).clip(max_norm, eps=0.0)
    norm = x.double().norm(dim=1, keepdim=True)
    want = x.double() * (float(torch.tensor(max_norm)) / norm).clamp(max=1.0)
    bound = 14 * u * want.abs() + half * want.abs() * (1 + half) + 2.0 ** (-150 if dtype is torch.float32 else -134) * 2
    assert bool(((y.double() - want).abs() <= bound).all())
    assert max_norm == 0.0 or max_norm < 1e-38 or abs(float(y[0].double().norm()) / min(max_norm, float(norm[0])) - 1) < 2 * half
