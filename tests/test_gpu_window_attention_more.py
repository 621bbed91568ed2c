"""Windowed attention where float16 and long sums lose most: weights below what float16 holds beside a large one.  Values,
bounds and their derivation are test_gpu_window_attention.py's; what is tighter here is said at each test."""

import math

import pytest
import torch

from paper_2501_17392_b200 import brace as B
from test_gpu_window_attention import BF16, F16, F32, Plain, randn, sees, within

pytestmark = pytest.mark.gpu

TYPES = [F32, BF16, F16]


def one_large_weight(n, dtype, size):
    """q, k, v, do of a text whose first key has a score 25 times log 2 above the others', and values of 0; the other
    values, and do, are of size `size`."""
    q, k, v, do = (randn(1, n, 2, 64, seed=s) for s in range(4))
    q[..., 0], k[..., 0] = 4.0, 0.0
    k[:, 0] *= 0.25
    k[:, 0, :, 0] = 25.2 * math.log(2) * 8 / 4
    v[:, 0] = 0.0
    return [t.to(dtype) for t in (q, k, v * size, do * size)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [40, 300, 1500])
def test_small_weights_beside_a_large_one(n, dtype):
    """P is held times 2^7 in float16, against a largest weight of 1: half a step of its smallest numbers is 2^-32."""
    q, k, v, _ = one_large_weight(n, dtype, 1000.0)
    plan = B.WindowAttention(2, 64, n, window=n, grad=False)
    out, lse = torch.empty_like(q), torch.empty(1, 2, n, device="cuda")
    plan.forward(q, k, v, out, lse=lse)
    w = Plain(q[0], k[0], v[0], n, 0, plan.scale)
    bound = w.out_bound
    if dtype == F16:
        bound = bound - (2.0 ** -24 - 2.0 ** -32) * (sees(n, n, 0).double() @ w.v.abs())
    within(out[0], w.out.transpose(0, 1), bound.transpose(0, 1), "out")
    within(lse[0], w.lse, w.lse_bound, "lse")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [40, 300, 1500])
def test_small_weights_in_the_gradient_of_values(n, dtype):
    """As under loss scaling: large do.  p, at most 1, is held times 2^15 in float16: half a step of its smallest numbers is
    2^-40."""
    q, k, v, do = one_large_weight(n, dtype, 1.0)
    do *= 100.0
    plan = B.WindowAttention(2, 64, n, window=n)
    out, lse = torch.empty_like(q), torch.empty(1, 2, n, device="cuda")
    plan.forward(q, k, v, out, lse=lse)
    dq, dk, dv = (torch.empty_like(q) for _ in range(3))
    plan.grad(do, q, k, v, out, lse, dq, dk, dv)
    w = Plain(q[0], k[0], v[0], n, 0, plan.scale, do[0])
    bound = w.dv_bound
    if dtype == F16:
        bound = bound - (2.0 ** -24 - 2.0 ** -40) * (sees(n, n, 0).double().mT @ do[0].transpose(0, 1).double().abs())
    within(dv[0], w.dv.transpose(0, 1), bound.transpose(0, 1), "dv")
    within(dq[0], w.dq.transpose(0, 1), w.dq_bound.transpose(0, 1), "dq")
    within(dk[0], w.dk.transpose(0, 1), w.dk_bound.transpose(0, 1), "dk")
