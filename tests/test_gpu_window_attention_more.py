"""Windowed attention where float16 and long sums lose most: weights below what float16 holds beside a large one.  Values,
bounds and their derivation are test_gpu_window_attention.py's; what is tighter here is said at each test."""

import math

import pytest
import torch

from paper_2501_17392_b200 import brace as B
from test_gpu_window_attention import BF16, F16, F32, U, Plain, randn, sees, u, within

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
    """P is held times 2^9 in float16, against a largest weight of 1: half a step of its smallest numbers is 2^-34."""
    q, k, v, _ = one_large_weight(n, dtype, 1000.0)
    plan = B.WindowAttention(2, 64, n, window=n, grad=False)
    out, lse = torch.empty_like(q), torch.empty(1, 2, n, device="cuda")
    plan.forward(q, k, v, out, lse=lse)
    w = Plain(q[0], k[0], v[0], n, 0, plan.scale)
    bound = w.out_bound
    if dtype == F16:
        bound = bound - (2.0 ** -24 - 2.0 ** -34) * (sees(n, n, 0).double() @ w.v.abs())
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


def banded(q, k, v, do, window, sinks, scale):
    """dq, dk and dv of one sequence with one key head in 64 bits, some queries of a head at a time."""
    n, heads, _ = q.shape
    k, v = k[:, 0].double(), v[:, 0].double()
    dq, dk, dv = torch.zeros(q.shape, dtype=torch.float64, device="cuda"), torch.zeros_like(k), torch.zeros_like(v)
    for a in range(0, n, 2048):
        i = torch.arange(a, min(n, a + 2048), device="cuda")
        lo = max(0, a - window + 1)
        keys = torch.cat([torch.arange(min(sinks, lo), device="cuda"), torch.arange(lo, int(i[-1]) + 1, device="cuda")])
        back = i[:, None] - keys
        hidden = (back < 0) | ((back >= window) & (keys >= sinks))
        for h in range(heads):
            p = (q[i, h].double() @ k[keys].T * scale).masked_fill(hidden, -math.inf).softmax(-1)
            dp = do[i, h].double() @ v[keys].T
            ds = p * (dp - (p * dp).sum(-1, keepdim=True)) * scale
            dq[i, h] = ds @ k[keys]
            dk.index_add_(0, keys, ds.T @ q[i, h].double())
            dv.index_add_(0, keys, p.T @ do[i, h].double())
    return dq, dk, dv


def worse(got, want):
    """The error of `got`, as a multiple of that of the exact value's rounding alone."""
    return float((got.double() - want).norm() / (want.to(got.dtype).double() - want).norm())


@pytest.mark.parametrize("dtype,dim,sinks", [(F16, 64, 4), (F16, 128, 0), (BF16, 64, 4)])
def test_sums_of_one_sign_over_many_queries(dtype, dim, sinks):
    """A key is read by up to 262,144 queries whose do are of one sign; with first tokens, whose tiles are shared out, the tiles
    behind them are not.  Steps of 16 queries cut a sum off by 1e-7 of the whole each on average (what is measured without
    taking sums out: 1.6e-3 after 17,000 of them, 7 times float16's rounding, and 4.4e-4 in dk); after 256 blocks of 64 that is
    1.0e-4, next to a rounding of 2.0e-4 (root mean square) a factor of 1.12.  P's rounding averages out over the queries.

    The workspace has exactly the size that is asked for, and its neighbours stay as they are."""
    n, heads, window = 17000, 64, 4096
    q, do = randn(1, n, heads, dim, seed=1).to(dtype), (randn(1, n, heads, dim, seed=2).abs() * 1e-2).to(dtype)
    k, v = randn(1, n, 1, dim, seed=3).to(dtype), randn(1, n, 1, dim, seed=4).to(dtype)
    need = int(B.lib().brace_window_attention_window_workspace_bytes(1, n, heads, 1, dim, window, sinks))
    whole = torch.full((need + 1024,), 255, dtype=torch.uint8, device="cuda")
    at = -whole.data_ptr() % 256 + 256
    plan = B.WindowAttention(heads, dim, n, kv_heads=1, window=window, sinks=sinks, workspace=whole[at:at + need])
    out, lse = torch.empty_like(q), torch.empty(1, heads, n, device="cuda")
    plan.forward(q, k, v, out, lse=lse)
    dq, dk, dv = (torch.empty_like(t) for t in (q, k, v))
    plan.grad(do, q, k, v, out, lse, dq, dk, dv)
    before = dk.clone(), dv.clone()
    whole[at:at + need] = 1
    plan.grad(do, q, k, v, out, lse, dq, dk, dv)
    assert torch.equal(before[0], dk) and torch.equal(before[1], dv)
    assert bool((whole[:at] == 255).all()) and bool((whole[at + need:] == 255).all())
    _, wk, wv = banded(q[0], k[0], v[0], do[0], window, sinks, plan.scale)
    assert worse(dk[0, :, 0], wk) < 1.5 and worse(dv[0, :, 0], wv) < 1.5
    # a shorter text and a shorter window in the same workspace
    m = 9001
    few = B.WindowAttention(heads, dim, n, kv_heads=1, window=3000, sinks=sinks, workspace=plan.workspace)
    a = [t[:, :m] for t in (do, q, k, v, out)]
    lse = lse[:, :, :m].contiguous()
    few.forward(*a[1:], lse=lse)
    few.grad(*a, lse, dq[:, :m], dk[:, :m], dv[:, :m])
    _, wk, wv = banded(q[0, :m], k[0, :m], v[0, :m], do[0, :m], 3000, sinks, plan.scale)
    assert worse(dk[0, :m, 0], wk) < 1.5 and worse(dv[0, :m, 0], wv) < 1.5
    assert torch.equal(dk[:, m:], before[0][:, m:]) and torch.equal(dv[:, m:], before[1][:, m:])
    assert bool((whole[:at] == 255).all()) and bool((whole[at + need:] == 255).all())


def dq_of_long_text(k, v, do, seed=0):
    """dq of a text with one head, all of which is seen, in a workspace of exactly the size that is asked for (it holds dq's sums
    and, later, those of dk and dv); a function that gives some rows' exact values and the sums of absolute values."""
    n, dim = k.shape[1], k.shape[3]
    q = randn(1, n, 1, dim, seed=seed).to(k.dtype)
    need = int(B.lib().brace_window_attention_window_workspace_bytes(1, n, 1, 1, dim, n, 0))
    whole = torch.full((need + 1024,), 255, dtype=torch.uint8, device="cuda")
    at = -whole.data_ptr() % 256 + 256
    plan = B.WindowAttention(1, dim, n, window=n, workspace=whole[at:at + need])
    out, lse = torch.empty_like(q), torch.empty(1, 1, n, device="cuda")
    plan.forward(q, k, v, out, lse=lse)
    dq, dk, dv = (torch.empty_like(t) for t in (q, k, v))
    plan.grad(do, q, k, v, out, lse, dq, dk, dv)
    assert bool((whole[:at] == 255).all()) and bool((whole[at + need:] == 255).all())

    def exact(i):
        p = (q[0, i, 0].double() @ k[0, :, 0].double().T * plan.scale).masked_fill(torch.arange(n, device="cuda") > i[:, None], -math.inf).softmax(-1)
        # delta as the formula has it, from the rounded output
        ds = p * (do[0, i, 0].double() @ v[0, :, 0].double().T - (do[0, i, 0].double() * out[0, i, 0].double()).sum(-1, keepdim=True))
        return ds @ k[0, :, 0].double() * plan.scale, ds.abs() @ k[0, :, 0].double().abs() * plan.scale

    return dq[0, :, 0], exact


@pytest.mark.parametrize("dtype,n,dim", [(F16, 140001, 64), (F16, 131072, 128), (F16, 600000, 64), (BF16, 600000, 64)])
def test_sums_of_one_sign_over_many_keys_in_the_gradient(dtype, n, dim):
    """Keys that are the values: a query's dq grows evenly along the text, as its do.  What the steps of 16 keys cut off is at most
    1e-7 of the whole each, twice in float16's two planes; without taking sums out 600,000 keys leave 1.1e-3, 5.6 times
    float16's rounding.  Taken out every 16,384 keys it is at most 2 * 1.0e-4, as much as the rounding: a factor below sqrt(2)."""
    v, do = randn(1, n, 1, dim, seed=1).to(dtype), randn(1, n, 1, dim, seed=2, scale=1e-2).to(dtype)
    dq, exact = dq_of_long_text(v, v, do)
    i = torch.arange(n - 200, n, device="cuda")
    assert worse(dq[i], exact(i)[0]) < 1.5


@pytest.mark.parametrize("dtype,n,dim", [(F16, 140001, 64), (F16, 131072, 128), (BF16, 140001, 64)])
def test_sums_over_many_keys_that_nearly_cancel(dtype, n, dim):
    """dq of values that rise along the text and keys of one sign: what is left is some 240 times smaller than the sums of
    absolute values.  A step cuts off 2e-7 of what is summed so far, which is at most the absolute sum of its 16,384 keys
    (of the first 65,536 where there are fewer: 4096 steps, twice as many in float16, of a sum that is half of it on average):
    2048 * 2e-7 = 4.1e-4, or 8192 * 2e-7 / 2 = 8.2e-4, of the absolute sums and the rounding of the result (another 2^-8 at
    most, and of ds to bfloat16 on the way)."""
    k, v, do = (randn(1, n, 1, dim, seed=s) for s in (1, 2, 3))
    v += torch.linspace(-1, 1, n, device="cuda")[:, None, None]
    dq, exact = dq_of_long_text(k.abs().to(dtype), v.to(dtype), (do.abs() * 1e-2).to(dtype))
    for a in (60000, n - 200):
        i = torch.arange(a, a + 200, device="cuda")
        want, size = exact(i)
        within(dq[i], want, (4.1e-4 if a > 65536 else 8.2e-4) * size + U[dtype] * want.abs())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 130, 699])
def test_fewer_tokens_than_the_plan_is_for(n, dtype):
    q, k, v = (randn(2, n, h, 64, seed=s).to(dtype) for s, h in enumerate((4, 2, 2)))
    do = randn(2, n, 4, 64, seed=9, scale=0.1).to(dtype)
    plan = B.WindowAttention(4, 64, 700, batch=2, kv_heads=2, window=90, sinks=3)
    out, lse = torch.empty_like(q), torch.empty(2, 4, n, device="cuda")
    plan.forward(q, k, v, out)
    first = out.clone()
    plan.forward(q, k, v, out.zero_(), lse=lse)
    assert torch.equal(first, out)        # with lse or without
    grads = [torch.empty_like(t) for t in (q, k, v)]
    plan.workspace.fill_(255)
    plan.grad(do, q, k, v, out, lse, *grads)
    for i in range(2):
        w = Plain(q[i], k[i], v[i], 90, 3, plan.scale, do[i])
        for got, name in zip((out, *grads), ("out", "dq", "dk", "dv")):
            within(got[i], getattr(w, name).transpose(0, 1), getattr(w, name + "_bound").transpose(0, 1), name)


@pytest.mark.parametrize("dtype,n,dim,ramp", [(F16, 262144, 64, False), (F16, 262144, 128, True), (F16, 200001, 64, True),
                                              (BF16, 600000, 128, False), (BF16, 540001, 64, True),
                                              (BF16, 70001, 64, False)])
def test_sums_of_one_sign_over_many_keys(dtype, n, dim, ramp):
    """As over many queries: 262,144 keys with values of one sign came out 1.7e-3 too small, 9 times float16's rounding.
    `ramp`: later keys have larger scores, so that results are scaled again under way."""
    q, k, v = (randn(1, n, 1, dim, seed=s) for s in range(3))
    if ramp:
        k *= torch.linspace(0.2, 2.5, n, device="cuda")[:, None, None]
    q, k, v = q.to(dtype), k.to(dtype), v.abs().to(dtype)
    out, lse = torch.empty_like(q), torch.empty(1, 1, n, device="cuda")
    plan = B.WindowAttention(1, dim, n, window=n, sinks=5, grad=False)
    plan.forward(q, k, v, out, lse=lse)
    for a in (0, 5000, 16300, n // 2, n - 300):
        i = torch.arange(a, a + 200, device="cuda")
        s = (q[0, i, 0].double() @ k[0, :, 0].double().T * plan.scale).masked_fill(torch.arange(n, device="cuda") > i[:, None], -math.inf)
        assert worse(out[0, i, 0], s.softmax(-1) @ v[0, :, 0].double()) < (1.5 if a else 2)
        # a score is off by (dim + 2) 2^-23 of its products' absolute sum, below 8 dim in all
        assert float((lse[0, 0, i] - s.logsumexp(-1)).abs().max()) < plan.scale * (dim + 2) * 2.0 ** -23 * 8 * dim + 2.0 ** -19 + 20 * u


@pytest.mark.parametrize("batch,heads", [(5, 32), (19, 16)])
def test_long_sums_of_many_tiles(batch, heads):
    """320 tiles of keys that 262,144 queries read, each shared out over four CTAs, and 1216 that 131,072 read, each a CTA's own:
    it takes its sums out on the way.  The last sequence is shorter.  do has both signs: what up to 4096 steps cut off is less than
    float16's rounding."""
    n, dim, short = 8192, 64, 5001
    q, do = (randn(batch, n, heads, dim, seed=s).to(F16) for s in (1, 2))
    do *= 1e-2
    k, v = (randn(batch, n, 1, dim, seed=s).to(F16) for s in (3, 4))
    lengths = torch.tensor([n] * (batch - 1) + [short], dtype=torch.int32, device="cuda")
    plan = B.WindowAttention(heads, dim, n, batch=batch, kv_heads=1, window=n)
    out, lse = torch.empty_like(q), torch.empty(batch, heads, n, device="cuda")
    plan.forward(q, k, v, out, lse=lse, lengths=lengths)
    dq, dk, dv = (torch.empty_like(t) for t in (q, k, v))
    plan.workspace.fill_(255)
    plan.grad(do, q, k, v, out, lse, dq, dk, dv, lengths=lengths)
    for b, m in ((0, n), (batch - 1, short)):
        wq, wk, wv = banded(q[b, :m], k[b, :m], v[b, :m], do[b, :m], n, 0, plan.scale)
        assert worse(dk[b, :m, 0], wk) < 1.5 and worse(dv[b, :m, 0], wv) < 1.5 and worse(dq[b, :m], wq) < 2
        assert bool((dk[b, m:] == 0).all()) and bool((dv[b, m:] == 0).all()) and bool((dq[b, m:] == 0).all())


@pytest.mark.parametrize("dtype,dim", [(F16, 64), (F16, 128), (BF16, 64)])
def test_long_windows_behind_first_tokens(dtype, dim):
    """A window of more than 65,536 keys and a few first tokens before it, whose block is cut short; one text ends early.  do has
    both signs."""
    n, heads, window, sinks, lengths = 100001, 2, 70000, 5, [100001, 80000]
    q, do = (randn(2, n, heads, dim, seed=s).to(dtype) for s in (1, 2))
    do *= 1e-2
    k, v = (randn(2, n, 1, dim, seed=s).to(dtype) for s in (3, 4))
    ln = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    plan = B.WindowAttention(heads, dim, n, batch=2, kv_heads=1, window=window, sinks=sinks)
    out, lse = torch.empty_like(q), torch.empty(2, heads, n, device="cuda")
    plan.forward(q, k, v.abs(), out, lse=lse, lengths=ln)
    for b, m in enumerate(lengths):
        for a in (100, 65600, 75000, m - 200):
            i = torch.arange(a, a + 200, device="cuda")
            j = torch.arange(m, device="cuda")
            back = i[:, None] - j
            hidden = (back < 0) | ((back >= window) & (j >= sinks))
            for h in range(heads):
                s = (q[b, i, h].double() @ k[b, :m, 0].double().T * plan.scale).masked_fill(hidden, -math.inf)
                assert worse(out[b, i, h], s.softmax(-1) @ v[b, :m, 0].double().abs()) < (2 if a < 1000 or a == 65600 or dtype == F16 else 1.5)
    plan.forward(q, k, v, out, lse=lse, lengths=ln)
    dq, dk, dv = (torch.empty_like(t) for t in (q, k, v))
    plan.grad(do, q, k, v, out, lse, dq, dk, dv, lengths=ln)
    for b, m in enumerate(lengths):
        wq, wk, wv = banded(q[b, :m], k[b, :m], v[b, :m], do[b, :m], window, sinks, plan.scale)
        # bfloat16: p and ds are rounded for the sums, each as much as the result is
        most = 2.5 if dtype == BF16 else 2
        assert worse(dq[b, :m], wq) < most and worse(dk[b, :m, 0], wk) < most and worse(dv[b, :m, 0], wv) < most
        assert not any(bool(t[b, m:].any()) for t in (out, dq, dk, dv))
