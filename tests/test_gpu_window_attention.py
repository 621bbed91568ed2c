"""Attention with a sliding window and first tokens that stay visible, and its gradients, on a GPU against a plain 64-bit
implementation.

Tolerances, from the formulas (u = 2^-24; U = half a step of the inputs' type, 2^-8 bfloat16, 2^-11 float16, u float32;
D = the head's dimension, N = the keys of a row).  All are against sums of absolute values:
* a score is a float32 sum of D products, cut off at worst: within E_s = scale (D + 2) 2^-23 sum|q k|; with the
  exponential's own error of a few ulp and of its argument's size, a probability is within e = 2 max E_s + 2^-19 of itself;
* out: sum p |v| (e + U + N 2^-23), U for the rounding of p to the inputs' type (none in float32), and its own rounding;
* lse: E_s + 2^-19 + u |lse|;
* dp: (D + 2) 2^-23 sum|do v|; delta is made from the rounded out: U sum|do out| more, u in float32;
* ds = p (dp - delta): ds is rounded to the inputs' type, U |ds|; so dq = scale sum ds k is within
  scale sum (|ds| (e + U) + p (err dp + err delta)) |k|, and N 2^-23 of the absolute sum; dk the same, over queries;
* dv: sum p |do| (e + U + N 2^-23)."""

import math

import pytest
import torch

from paper_2501_17392_b200 import brace as B

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
u = 2.0 ** -24
U = {F32: 2.0 ** -24, F16: 2.0 ** -11, BF16: 2.0 ** -8}
TINY = {F32: 2.0 ** -126, F16: 2.0 ** -24, BF16: 2.0 ** -126}


def gen(seed=0):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(*shape, seed=0, scale=1.0):
    return torch.randn(*shape, device="cuda", generator=gen(seed)) * scale


def within(got, want, bound, what=""):
    t = got.dtype
    bound = bound + U[t] * (want.abs() + bound) + TINY[t]
    off = (got.double() - want).abs()
    assert bool((off <= bound).all()), f"{what} off by {float((off / bound.clamp_min(1e-300)).nan_to_num(math.inf).max())} times the bound"


def sees(n, window, sinks, device="cuda"):
    i = torch.arange(n, device=device)
    back = i[:, None] - i
    return (back >= 0) & ((back < window) | (i < sinks))


class Plain:
    """Values and bounds of one sequence (tokens first), 64 bits."""

    def __init__(self, q, k, v, window, sinks, scale, dout=None):
        self.t, self.u = q.dtype, U[q.dtype]
        n, h, d = q.shape
        share = h // k.shape[1]
        self.q, self.k, self.v = (x.double().transpose(0, 1) for x in (q, k.repeat_interleave(share, 1), v.repeat_interleave(share, 1)))
        self.share, self.scale, n23 = share, scale, n * 2.0 ** -23
        hidden = ~sees(n, window, sinks, q.device)
        s = self.q @ self.k.mT * scale
        es = abs(scale) * (d + 2) * 2.0 ** -23 * (self.q.abs() @ self.k.abs().mT)
        s = s.masked_fill(hidden, -math.inf)
        es = es.masked_fill(hidden, 0).amax(-1, keepdim=True)
        spread = (s.amax(-1, keepdim=True) - s.masked_fill(hidden, math.inf).amin(-1, keepdim=True)) * 2.0 ** -22
        e = 2 * es + 2.0 ** -19 + spread
        self.lse = torch.logsumexp(s, -1)
        self.lse_bound = es[..., 0] + 2.0 ** -19 + u * self.lse.abs()
        p = (s - self.lse[..., None]).exp()
        up = 0.0 if self.t == F32 else self.u
        # a probability below what the type holds next to the row's largest one
        small = 0.0 if self.t != F16 else 2.0 ** -24
        e2 = e + up + n23
        self.out = p @ self.v
        seen = (~hidden).double()
        self.out_bound = (p * e2 + small * seen) @ self.v.abs()
        if dout is None:
            return
        do = dout.double().transpose(0, 1)
        dp = do @ self.v.mT
        edp = (d + 2) * 2.0 ** -23 * (do.abs() @ self.v.abs().mT)
        delta = (do * self.out).sum(-1, keepdim=True)
        edelta = ((self.u + (d + 2) * 2.0 ** -23) * (do * self.out).abs().sum(-1, keepdim=True)
                  + (do.abs() * self.out_bound).sum(-1, keepdim=True))
        ds = p * (dp - delta)
        eds = ds.abs() * (e2 + 2 * u) + p * (edp + edelta)
        if self.t == F16:     # ds is held against the largest product there can be, 2^-38 of it is lost
            eds = eds + 2.0 ** -38 * d * do.abs().amax() * self.v.abs().amax() * seen
        self.dq = scale * ds @ self.k
        self.dq_bound = abs(scale) * (eds + n23 * ds.abs()) @ self.k.abs()
        total = n23 * self.share
        fold = lambda x: x.unflatten(0, (-1, share)).sum(1)  # noqa: E731
        self.dk, self.dk_bound = fold(scale * ds.mT @ self.q), fold(abs(scale) * (eds + total * ds.abs()).mT @ self.q.abs())
        self.dv, self.dv_bound = fold(p.mT @ do), fold((p * (e2 + total) + small * seen).mT @ do.abs())


def views(b, n, heads, dim, dtype, seed, layout="packed", scale=1.0):
    """q, k, v (and as many of a second set) as views of one projection, as separate tensors, heads first, or with odd
    strides."""
    h, g = heads
    if layout == "packed":
        x = randn(b, n, h + 2 * g, dim, seed=seed, scale=scale).to(dtype)
        return x[:, :, :h], x[:, :, h:h + g], x[:, :, h + g:]
    if layout == "heads":     # [batch, heads, tokens, dim]
        return tuple(randn(b, m, n, dim, seed=seed + i, scale=scale).to(dtype).transpose(1, 2) for i, m in enumerate((h, g, g)))
    pad = 8 if layout == "wide" else 1
    return tuple(randn(b, n + 1, m, dim + pad, seed=seed + i, scale=scale).to(dtype)[:, 1:, :, :dim] for i, m in enumerate((h, g, g)))


def check(b, n, heads, dim, window, sinks, dtype=F32, lengths=None, layout="packed", seed=1, grad=True, scale=None, size=1.0,
          dsize=1e-2):
    h, g = heads
    q, k, v = views(b, n, heads, dim, dtype, seed, layout, size)
    plan = B.WindowAttention(h, dim, n, batch=b, kv_heads=g, window=window, sinks=sinks, scale=scale)
    scale = plan.scale if scale is None else scale
    scale = float(torch.tensor(scale, dtype=F32))
    out, _, _ = views(b, n, heads, dim, dtype, seed + 10, layout)
    out.fill_(math.nan)
    lse = torch.full((b, h, n), math.nan, device="cuda")
    ln = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    plan.forward(q, k, v, out, lse=lse, lengths=ln)
    dout = views(b, n, heads, dim, dtype, seed + 20, layout, dsize)[0]
    dq, dk, dv = views(b, n, heads, dim, dtype, seed + 30, layout)
    if grad:
        for t in (dq, dk, dv):
            t.fill_(math.nan)
        plan.workspace.fill_(255)
        plan.grad(dout, q, k, v, out, lse, dq, dk, dv, lengths=ln)
    for i in range(b):
        m = n if lengths is None else min(max(lengths[i], 0), n)
        if m:
            w = Plain(q[i, :m], k[i, :m], v[i, :m], window, sinks, scale, dout[i, :m] if grad else None)
            within(out[i, :m], w.out.transpose(0, 1), w.out_bound.transpose(0, 1), "out")
            within(lse[i, :, :m], w.lse, w.lse_bound, "lse")
            if grad:
                within(dv[i, :m], w.dv.transpose(0, 1), w.dv_bound.transpose(0, 1), "dv")
                within(dq[i, :m], w.dq.transpose(0, 1), w.dq_bound.transpose(0, 1), "dq")
                within(dk[i, :m], w.dk.transpose(0, 1), w.dk_bound.transpose(0, 1), "dk")
        for t in (out, dq, dk, dv) if grad else (out,):
            assert bool((t[i, m:] == 0).all())
        assert bool((lse[i, :, m:] == -math.inf).all())
    if grad:     # the same bits
        before = [t.clone() for t in (dq, dk, dv)]
        plan.workspace.fill_(1)
        plan.grad(dout, q, k, v, out, lse, dq, dk, dv, lengths=ln)
        assert all(torch.equal(x, y) for x, y in zip(before, (dq, dk, dv)))
    return plan


TYPES = [F32, BF16, F16]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 2, 3, 31, 64, 65, 127, 128, 129, 200, 255, 257, 400, 641])
def test_lengths(n, dtype):
    check(1, n, (2, 2), 64, 100, 4, dtype)
    check(2, n, (2, 1), 128, 1000, 0, dtype, seed=5)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (2, 0), (7, 3), (63, 0), (64, 64), (65, 1), (127, 5), (128, 0),
                                          (128, 16), (129, 17), (130, 128), (200, 129), (150, 300), (300, 0), (1000, 500),
                                          (2 ** 31 - 1, 2 ** 31 - 1), (1, 600)])
def test_windows_and_sinks(window, sinks, dtype):
    check(1, 517, (2, 2), 64, window, sinks, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [1, 3, 8, 15, 16, 24, 32, 40, 64, 72, 80, 96, 100, 120, 128, 136, 192, 255, 256])
def test_head_dimensions(dim, dtype):
    check(1, 301, (2, 1), dim, 90, 5, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads", [(1, 1), (3, 3), (3, 1), (8, 2), (7, 7), (12, 4)])
@pytest.mark.parametrize("layout", ["packed", "heads", "wide", "odd"])
def test_heads_and_layouts(heads, layout, dtype):
    check(2, 150, heads, 64, 70, 3, dtype, layout=layout)


@pytest.mark.parametrize("dtype", TYPES)
def test_padded_batches(dtype):
    check(6, 300, (4, 2), 64, 80, 4, dtype, lengths=[300, 0, 1, 128, 129, 299])
    check(3, 150, (2, 2), 128, 1000, 0, dtype, lengths=[-5, 1000, 77])


@pytest.mark.parametrize("dtype", TYPES)
def test_long_sequences(dtype):
    check(1, 3000, (2, 1), 64, 500, 4, dtype)
    check(1, 2500, (1, 1), 128, 2500, 0, dtype)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_long_sums(dtype):
    """More than 65,536 queries read a key, and there are tiles for all SMs: each tile's sums are made of two pieces."""
    check(9, 1100, (64, 1), 40, 1100, 3, dtype, lengths=[1100] * 7 + [777, 1099])


@pytest.mark.parametrize("dtype", TYPES)
def test_scales(dtype):
    check(1, 200, (2, 2), 64, 90, 2, dtype, scale=0.0)
    check(1, 200, (2, 2), 64, 90, 2, dtype, scale=-0.2)
    check(1, 200, (2, 2), 64, 90, 2, dtype, scale=1.0)                       # scores of tens: nearly one key a row
    check(1, 200, (2, 2), 64, 90, 2, dtype, scale=0.02, size=4.0)
    check(1, 200, (2, 2), 64, 90, 2, dtype, dsize=1e-4 if dtype == F16 else 1e-12)
    check(1, 200, (2, 2), 64, 90, 2, dtype, dsize=30.0)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_small_scales_of_large_values(dtype):
    check(1, 200, (2, 2), 64, 90, 2, dtype, scale=2.0 ** -113, size=2.0 ** 55)     # scores as of a scale of 1/8 at size 1
    check(1, 200, (2, 2), 64, 90, 2, dtype, scale=0.0, size=2.0 ** 50)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_what_is_hidden_has_no_effect(dtype, bad):
    """A key that is not finite spoils the queries that see it, a query that is not finite what it sees; no other row."""
    n, w, sinks, at = 400, 60, 3, 170
    plan = B.WindowAttention(2, 64, n, kv_heads=1, window=w, sinks=sinks)
    q, k, v = views(1, n, (2, 1), 64, dtype, 3)
    dout = randn(1, n, 2, 64, seed=9, scale=0.1).to(dtype)

    def run():
        out, lse = torch.empty(1, n, 2, 64, device="cuda", dtype=dtype), torch.empty(1, 2, n, device="cuda")
        plan.forward(q, k, v, out, lse=lse)
        grads = [torch.empty_like(t) for t in (q, k, v)]
        plan.grad(dout, q, k, v, out, lse, *grads)
        return [out, lse.transpose(1, 2)[..., None], *grads]

    # A row that a hidden place spoils is computed again in another order: both ways are within the bounds that are derived
    # above, of the exact value, and so is what is compared here (not the two ways with one another).
    fine = Plain(q[0], k[0], v[0], w, sinks, float(torch.tensor(plan.scale, dtype=F32)), dout[0])
    fine = [(fine.out, fine.out_bound), (fine.lse[..., None], fine.lse_bound[..., None]), (fine.dq, fine.dq_bound),
            (fine.dk, fine.dk_bound), (fine.dv, fine.dv_bound)]
    fine = [[t.transpose(0, 1) for t in pair] for pair in fine]
    sees_it = sees(n, w, sinks)[:, at]
    # rows of k and v that a query reads that also reads `at`
    meets = (sees(n, w, sinks)[sees_it].any(0))
    for t, others in ((v, None), (k, None)):
        keep = t[0, at, 0, 5].clone()
        t[0, at, 0, 5] = bad
        got = run()
        t[0, at, 0, 5] = keep
        rows = [~sees_it, ~sees_it, ~sees_it, ~meets, ~meets]
        for (x, bound), y, r in zip(fine, got, rows):
            within(y[0, r], x[r], bound[r])
        assert not bool(got[0][0, sees_it][..., 5].isfinite().any()) if t is v else True
    keep = dout[0, at, 1, 7].clone()
    dout[0, at, 1, 7] = bad
    got = run()
    dout[0, at, 1, 7] = keep
    mine = sees(n, w, sinks)[at]
    this = torch.arange(n, device="cuda") == at
    for (x, bound), y, r in zip(fine, got, [this | True, this | True, ~this, ~mine, ~mine]):
        within(y[0, r], x[r], bound[r])
    assert not bool(got[4][0, mine][..., 7].isfinite().any())


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_behind_a_sequence_may_hold_anything(dtype):
    n, lengths = 300, [170, 300, 0, 40]
    plan = B.WindowAttention(4, 64, n, batch=4, kv_heads=2, window=90, sinks=2)
    q, k, v = views(4, n, (4, 2), 64, dtype, 3)
    dout = randn(4, n, 4, 64, seed=9, scale=0.1).to(dtype)
    ln = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    results = []
    for fill in (0.0, math.nan, math.inf):
        for i, m in enumerate(lengths):
            for t in (q, k, v, dout):
                t[i, m:] = fill
        out, lse = torch.empty(4, n, 4, 64, device="cuda", dtype=dtype), torch.empty(4, 4, n, device="cuda")
        plan.forward(q, k, v, out, lse=lse, lengths=ln)
        grads = [torch.empty_like(t) for t in (q, k, v)]
        plan.grad(dout, q, k, v, out, lse, *grads, lengths=ln)
        results.append([out, lse.nan_to_num(7.0), *grads])
    for got in results[1:]:
        for x, y in zip(results[0], got):
            within(y, x.double(), 4 * U[dtype] * x.double().abs().amax())


def test_gradient_against_differences():
    n, w, sinks = 40, 9, 2
    q, k, v = views(1, n, (2, 1), 12, F32, 4)
    dout = randn(1, n, 2, 12, seed=8)
    plan = B.WindowAttention(2, 12, n, kv_heads=1, window=w, sinks=sinks)
    out, lse = torch.empty(1, n, 2, 12, device="cuda"), torch.empty(1, 2, n, device="cuda")
    plan.forward(q, k, v, out, lse=lse)
    grads = [torch.empty_like(t) for t in (q, k, v)]
    plan.grad(dout, q, k, v, out, lse, *grads)
    f = lambda a: float((Plain(*(t[0] for t in a), w, sinks, plan.scale).out.transpose(0, 1) * dout[0].double()).sum())  # noqa: E731
    for at, grad in enumerate(grads):
        for i in (0, 1, 5, 39):
            args = [t.double() for t in (q, k, v)]
            args[at][0, i, 0, 3] += 1e-5
            up = f_64(f, args)
            args[at][0, i, 0, 3] -= 2e-5
            down = f_64(f, args)
            assert abs((up - down) / 2e-5 - float(grad[0, i, 0, 3])) < 1e-4 * max(1.0, abs(float(grad[0, i, 0, 3])))


def f_64(f, args):
    U.setdefault(torch.float64, 2.0 ** -53)
    return f(args)


@pytest.mark.parametrize("dtype", TYPES)
def test_broadcast_inputs(dtype):
    n = 140
    q, k, v = (randn(1, n, 1, 64, seed=s).to(dtype).expand(3, n, m, 64) for s, m in ((1, 4), (2, 2), (3, 2)))
    plan = B.WindowAttention(4, 64, n, batch=3, kv_heads=2, window=50, sinks=1)
    out, lse = torch.empty(3, n, 4, 64, device="cuda", dtype=dtype), torch.empty(3, 4, n, device="cuda")
    plan.forward(q, k, v, out, lse=lse)
    dout = randn(1, 1, 1, 64, seed=4, scale=0.1).to(dtype).expand(3, n, 4, 64)
    dq, dk, dv = torch.empty_like(out), torch.empty(3, n, 2, 64, device="cuda", dtype=dtype), torch.empty(3, n, 2, 64, device="cuda", dtype=dtype)
    plan.grad(dout, q, k, v, out, lse, dq, dk, dv)
    for i in range(3):
        w = Plain(q[i], k[i], v[i], 50, 1, plan.scale, dout[i])
        for got, name in ((out, "out"), (dq, "dq"), (dk, "dk"), (dv, "dv")):
            within(got[i], getattr(w, name).transpose(0, 1), getattr(w, name + "_bound").transpose(0, 1), name)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("odd", ["q", "k", "v", "out", "dout", "dq", "dk", "dv"])
def test_one_tensor_on_no_boundary(odd, dtype):
    """All tensors on 16-byte boundaries but one."""
    n, heads = 200, {"k": 2, "v": 2, "dk": 2, "dv": 2}
    t = {}
    for i, name in enumerate(("q", "k", "v", "out", "dout", "dq", "dk", "dv")):
        h = heads.get(name, 4)
        x = randn(2, n, h, 64, seed=i, scale=0.1 if name == "dout" else 1.0).to(dtype)
        if name == odd:
            flat = torch.empty(x.numel() + 1, device="cuda", dtype=dtype)[1:]
            x = flat.copy_(x.flatten()).view(x.shape)
        t[name] = x
    plan = B.WindowAttention(4, 64, n, batch=2, kv_heads=2, window=90, sinks=3)
    lse = torch.empty(2, 4, n, device="cuda")
    plan.forward(t["q"], t["k"], t["v"], t["out"], lse=lse)
    plan.grad(t["dout"], t["q"], t["k"], t["v"], t["out"], lse, t["dq"], t["dk"], t["dv"])
    for i in range(2):
        w = Plain(t["q"][i], t["k"][i], t["v"][i], 90, 3, plan.scale, t["dout"][i])
        for name in ("out", "dq", "dk", "dv"):
            within(t[name][i], getattr(w, name).transpose(0, 1), getattr(w, name + "_bound").transpose(0, 1), name)


@pytest.mark.parametrize("dtype", TYPES)
def test_on_another_stream_and_in_a_graph(dtype):
    b, n = 2, 333
    q, k, v = views(b, n, (4, 2), 64, dtype, 3)
    dout = randn(b, n, 4, 64, seed=9, scale=0.1).to(dtype)
    out, lse = torch.empty(b, n, 4, 64, device="cuda", dtype=dtype), torch.empty(b, 4, n, device="cuda")
    grads = [torch.empty_like(t) for t in (q, k, v)]
    ln = torch.tensor([333, 200], dtype=torch.int32, device="cuda")
    plan = B.WindowAttention(4, 64, n, batch=b, kv_heads=2, window=70, sinks=5)

    def step(stream=None):
        plan.forward(q, k, v, out, lse=lse, lengths=ln, stream=stream)
        plan.grad(dout, q, k, v, out, lse, *grads, lengths=ln, stream=stream)

    step()
    torch.cuda.synchronize()
    results = (out, lse, *grads)
    want = [t.clone() for t in results]
    side = torch.cuda.Stream()
    for t in results:
        t.zero_()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want, results))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for lengths in ([333, 200], [150, 333]):      # they are read when the graph runs
        ln.copy_(torch.tensor(lengths, dtype=torch.int32))
        step()
        want = [t.clone() for t in results]
        for t in results:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(want, results))


@pytest.mark.parametrize("dtype", TYPES)
def test_workspace_of_exactly_the_size_and_guards(dtype):
    for b, n, heads, dim, w, sinks in [(2, 700, (4, 2), 64, 100, 4), (1, 300, (2, 1), 128, 50, 40), (1, 130, (3, 3), 50, 20, 2)]:
        h, g = heads
        need = int(B.lib().brace_window_attention_workspace_bytes(b, n, h, g, dim, sinks))
        whole = torch.full((need + 1024,), 255, dtype=torch.uint8, device="cuda")
        at = -whole.data_ptr() % 256 + 256
        q, k, v = views(b, n, heads, dim, dtype, 3)
        dout = randn(b, n, h, dim, seed=9, scale=0.1).to(dtype)
        out, lse = torch.empty(b, n, h, dim, device="cuda", dtype=dtype), torch.empty(b, h, n, device="cuda")
        plan = B.WindowAttention(h, dim, n, batch=b, kv_heads=g, window=w, sinks=sinks, workspace=whole[at:at + need])
        plan.forward(q, k, v, out, lse=lse)
        rows = torch.full((b, n + 2, h + 2 * g, dim + 8), 3.0, device="cuda", dtype=dtype)
        inner = rows[:, 1:-1, :, :dim]
        plan.grad(dout, q, k, v, out, lse, inner[:, :, :h], inner[:, :, h:h + g], inner[:, :, h + g:])
        torch.cuda.synchronize()
        assert bool((whole[:at] == 255).all()) and bool((whole[at + need:] == 255).all())
        inner.fill_(3.0)
        assert bool((rows == 3.0).all())


def test_no_rows():
    plan = B.WindowAttention(2, 64, 10, batch=2)
    x, lse = torch.empty(2, 0, 2, 64, device="cuda"), torch.empty(2, 2, 0, device="cuda")
    plan.forward(x, x, x, x, lse=lse)
    plan.grad(x, x, x, x, x, lse, x, x, x)
