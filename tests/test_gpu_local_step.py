"""Layer norm and clipping by the global norm on a GPU against plain 64-bit implementations.

Tolerances, from the formulas (u = 2^-24; U is half a step of the result's type, TINY half of its smallest number):
* a row's sum is held by up to 256 threads with up to 32 values each, then joined pairwise and by warps: no value passes
  through more than K = 32 + 5 + 8 additions (rows above 8192: dim / 256 + 13), so a sum is within K u sum|x|;
* mean: K u mean|x|; var is summed from differences, a shift of the mean enters squared: rstd within (K / 2 + 4) u;
* y = (x - mean) rstd w + b: |w| rstd (K u mean|x| + u |x - mean|) + (K / 2 + 6) u |xh w| + 2 u |y|, and its rounding;
* dx, of the given mean and rstd: xh is within 3 u |xh|, the row's sums within (K + 6) u of the sums of absolute values;
* the weights' gradients: n terms in any order, each within 4 u: (n + 5) u sum|dy xh|;
* norms: 16 squares at a time in float32, the rest in float64: (16 / 2 + 2) u; a clipped value another 4 u."""

import math

import pytest
import torch

from paper_2501_17392_b200 import brace as B

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
u = 2.0 ** -24
U = {F32: 2.0 ** -24, F16: 2.0 ** -11, BF16: 2.0 ** -8}
TINY = {F32: 2.0 ** -150, F16: 2.0 ** -25, BF16: 2.0 ** -134}


def gen(seed=0):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(*shape, seed=0, scale=1.0):
    return torch.randn(*shape, device="cuda", generator=gen(seed)) * scale


def within(got, want, bound):
    """|got - want| <= bound, the bound without the rounding of the result itself."""
    bound = bound + U[got.dtype] * want.abs() * (1 + U[got.dtype]) + TINY[got.dtype]
    off = (got.double() - want).abs()
    assert bool((off <= bound).all()), f"off by {float((off / bound.clamp_min(1e-300)).max())} times the bound"


def depth(dim):
    return 45 if dim <= 8192 else dim / 256 + 13


def norm64(x, w, b, eps):
    """y, mean, rstd and the bounds of their errors."""
    x, k = x.double(), depth(x.shape[-1])
    w, b = (torch.as_tensor(t, dtype=torch.float64, device="cuda") for t in (w, b))
    w, b = (t[:, None] if t.dim() == 2 else t for t in (w, b))
    mean = x.mean(-1, keepdim=True)
    rstd = ((x - mean).square().mean(-1, keepdim=True) + eps).rsqrt()
    xh = (x - mean) * rstd
    size = x.abs().mean(-1, keepdim=True)
    y = xh * w + b
    by = w.abs() * rstd * (k * u * size + u * (x - mean).abs()) + (k / 2 + 6) * u * (xh * w).abs() + 2 * u * (y.abs() + b.abs())
    # a shift of the mean by s adds s^2 to the variance
    bound_rstd = rstd * ((k / 2 + 4) * u + 0.5 * (k * u * size * rstd) ** 2)
    return (y, by + (bound_rstd / rstd) * (xh * w).abs()), (mean[..., 0], (k * u * size)[..., 0]), (rstd[..., 0], bound_rstd[..., 0])


def norm_grad64(dy, x, mean, rstd, w):
    dy, x, mean, rstd = dy.double(), x.double(), mean.double()[..., None], rstd.double()[..., None]
    w = torch.as_tensor(w, dtype=torch.float64, device="cuda")
    w = w[:, None] if w.dim() == 2 else w
    d, n, k = x.shape[-1], x.shape[-2], depth(x.shape[-1])
    xh, g = (x - mean) * rstd, dy * w
    m1, m2 = g.mean(-1, keepdim=True), (g * xh).mean(-1, keepdim=True)
    a1, a2 = g.abs().mean(-1, keepdim=True), (g * xh).abs().mean(-1, keepdim=True)
    dx = rstd * (g - m1 - xh * m2)
    bound = rstd * u * ((k + 6) * a1 + (k + 12) * xh.abs() * a2 + 6 * (g.abs() + m1.abs() + (xh * m2).abs()))
    sums = [(t.sum(-2), (n + 5) * u * t.abs().sum(-2)) for t in (dy * xh, dy)]
    return (dx, bound), *sums


def rows(*shape, dtype=F32, seed=0, scale=1.0, pad=0, at=0):
    """A tensor of random values, its rows `pad` elements further apart than they are long, `at` elements into its
    storage; what is not the tensor's is NaN."""
    *lead, d = shape
    n = math.prod(lead)
    whole = torch.full((at + n * (d + pad) + 8,), math.nan, device="cuda", dtype=dtype)
    st, size = [], d + pad
    for k in reversed(lead):
        st.insert(0, size)
        size *= k
    t = whole.as_strided(shape, (*st, 1), at)
    t.copy_(randn(*shape, seed=seed, scale=scale))
    return t


def guarded(t):
    """Values of t's storage that are not t's."""
    flat = torch.as_strided(t, (t.untyped_storage().nbytes() // t.element_size(),), (1,), 0)
    own = torch.zeros_like(flat, dtype=torch.bool)
    own.as_strided(t.shape, t.stride(), t.storage_offset()).fill_(True)
    return flat[~own]


DIMS = [1, 2, 7, 8, 31, 33, 64, 100, 128, 255, 264, 333, 768, 1000, 1024, 1025, 1032, 2048, 4096, 5000, 8192]


def check_norm(c, n, d, tx=F32, ty=F32, tw=F32, pad=0, at=0, seed=1, offset=0.5, **given):
    x = rows(c, n, d, dtype=tx, seed=seed, pad=pad, at=at)
    x += offset
    y = rows(c, n, d, dtype=ty, seed=seed + 1, pad=pad, at=at)
    w, b = rows(c, d, dtype=tw, seed=seed + 2, pad=5, at=3), rows(c, d, dtype=tw, seed=seed + 3, pad=9, at=1)
    mean, rstd = torch.empty(c, n, device="cuda"), torch.empty(c, n, device="cuda")
    plan = B.LayerNorm(d, n, clients=c)
    plan.forward(x, y, weight=w, bias=b, mean=mean, rstd=rstd)
    for got, (want, bound) in zip((y, mean, rstd), norm64(x, w, b, 1e-5)):
        within(got, want, bound)
    assert bool(guarded(y).isnan().all())
    dy = rows(c, n, d, dtype=ty, seed=seed + 4, pad=pad, at=at)
    dx = rows(c, n, d, dtype=tx, seed=seed + 5, pad=pad, at=at)
    dw, db = rows(c, d, seed=seed + 6, pad=3, at=5), rows(c, d, seed=seed + 7, pad=2, at=7)
    plan.workspace.fill_(255)
    plan.grad(dy, x, mean, rstd, dx, weight=w, dweight=dw, dbias=db)
    want = norm_grad64(dy, x, mean, rstd, w)
    for got, (value, bound) in zip((dx, dw, db), want):
        within(got, value, bound)
    for t in (dx, dw, db):
        assert bool(guarded(t).isnan().all())
    before = dw.clone(), db.clone(), dx.clone()
    plan.grad(dy, x, mean, rstd, dx, weight=w, dweight=dw, dbias=db)
    assert all(torch.equal(p, q) for p, q in zip(before, (dw, db, dx)))       # the same bits
    plan.grad(dy, x, mean, rstd, dx, weight=w, dweight=dw, dbias=db, accumulate=True)
    for got, first, (value, bound) in zip((dw, db), before, want[1:]):
        within(got, 2 * first.double(), 0 * value)
    return plan


@pytest.mark.parametrize("d", DIMS)
def test_norm_lengths(d):
    check_norm(2, 37, d)
    check_norm(1, 3, d, pad=1, at=1, seed=20)


@pytest.mark.parametrize("d", [8193, 8200, 10007, 16384, 70001, 70008])
def test_norm_long_rows(d):
    check_norm(2, 70, d)


@pytest.mark.parametrize("n", [1, 2, 31, 129, 1000, 5001])
@pytest.mark.parametrize("c", [1, 3])
def test_norm_rows(n, c):
    check_norm(c, n, 96)
    check_norm(c, n, 45, seed=9)


def test_norm_many_clients():
    check_norm(700, 3, 40)


@pytest.mark.parametrize("tx", [F32, BF16, F16])
@pytest.mark.parametrize("ty", [F32, BF16, F16])
@pytest.mark.parametrize("d,pad", [(264, 0), (264, 8), (264, 3), (77, 0), (9000, 0)])
def test_norm_types_and_strides(tx, ty, d, pad):
    check_norm(2, 45, d, tx, ty, pad=pad)


@pytest.mark.parametrize("tw", [BF16, F16])
def test_norm_weight_types(tw):
    check_norm(2, 45, 264, BF16, BF16, tw)


def test_norm_gradient_types():
    x, dy, dx = randn(2, 50, 64), randn(2, 50, 64, seed=1), torch.empty(2, 50, 64, device="cuda")
    mean, rstd = x.mean(-1), x.var(-1).rsqrt()
    for t in (BF16, F16):
        dw, db = torch.empty(2, 64, device="cuda", dtype=t), torch.empty(2, 64, device="cuda", dtype=t)
        B.LayerNorm(64, 50, clients=2).grad(dy, x, mean, rstd, dx, dweight=dw, dbias=db)
        want = norm_grad64(dy, x, mean, rstd, 1.0)
        within(dw, *want[1])
        within(db, *want[2])


def test_norm_offset_far_from_the_spread():
    check_norm(1, 40, 512, offset=3000.0)
    check_norm(1, 40, 333, offset=-3000.0)


def test_norm_rows_of_one_value():
    x = torch.full((1, 5, 100), 3.0, device="cuda")
    y, rstd = torch.empty_like(x), torch.empty(1, 5, device="cuda")
    B.LayerNorm(100, 5).forward(x, y, rstd=rstd)
    assert float(y.abs().max()) <= 45 * u * 3 / math.sqrt(1e-5)
    within(rstd, torch.full((1, 5), 1e-5, dtype=torch.float64, device="cuda").rsqrt(), 1e-4 * rstd.double())


@pytest.mark.parametrize("d", [40, 333, 2048, 9000])
def test_norm_what_is_not_finite_stays_in_its_row(d):
    x, dy = randn(2, 30, d), randn(2, 30, d, seed=1)
    x[1, 7, 3], x[0, 2, d - 1] = math.nan, math.inf
    y, mean, rstd = torch.empty_like(x), torch.empty(2, 30, device="cuda"), torch.empty(2, 30, device="cuda")
    plan = B.LayerNorm(d, 30, clients=2)
    plan.forward(x, y, mean=mean, rstd=rstd)
    bad = torch.zeros(2, 30, dtype=torch.bool, device="cuda")
    bad[1, 7] = bad[0, 2] = True
    assert bool(y[bad].isnan().all()) and bool(y[~bad].isfinite().all())
    dx = torch.empty_like(x)
    plan.grad(dy, x, mean, rstd, dx)
    assert bool(dx[bad].isnan().all()) and bool(dx[~bad].isfinite().all())


def test_norm_one_weight_for_all_and_none():
    x, w, b = randn(3, 20, 72), randn(72, seed=1), randn(72, seed=2)
    y = torch.empty_like(x)
    plan = B.LayerNorm(72, 20, clients=3, eps=0.1)
    for kw, bw in (((w, b), (w, b)), ((w, None), (w, 0.0)), ((None, b), (1.0, b)), ((None, None), (1.0, 0.0))):
        plan.forward(x, y, weight=kw[0], bias=kw[1])
        within(y, *norm64(x, *bw, float(torch.tensor(0.1)))[0])


def test_norm_gradients_of_some_only():
    x, dy, w = randn(2, 300, 72), randn(2, 300, 72, seed=3), randn(2, 72, seed=1)
    mean, rstd, dx = x.mean(-1), x.var(-1).rsqrt(), torch.empty_like(x)
    plan = B.LayerNorm(72, 300, clients=2)
    want = norm_grad64(dy, x, mean, rstd, w)
    for k in ("dweight", "dbias"):
        got = torch.empty(2, 72, device="cuda")
        plan.grad(dy, x, mean, rstd, dx, weight=w, **{k: got})
        within(got, *want[1 if k == "dweight" else 2])
        within(dx, *want[0])


def test_norm_of_broadcast_inputs():
    x = randn(1, 1, 80).expand(2, 25, 80)
    dy = randn(80, seed=4).expand(2, 25, 80)
    y, mean, rstd = torch.empty(2, 25, 80, device="cuda"), torch.empty(2, 25, device="cuda"), torch.empty(2, 25, device="cuda")
    plan = B.LayerNorm(80, 25, clients=2)
    plan.forward(x, y, mean=mean, rstd=rstd)
    within(y, *norm64(x, 1.0, 0.0, 1e-5)[0])
    dx, dw = torch.empty_like(y), torch.empty(2, 80, device="cuda")
    plan.grad(dy, x, mean, rstd, dx, dweight=dw)
    want = norm_grad64(dy, x, mean, rstd, 1.0)
    within(dx, *want[0])
    within(dw, *want[1])


def test_norm_without_rows():
    plan = B.LayerNorm(16, 8, clients=2)
    x = torch.empty(2, 0, 16, device="cuda")
    stats = torch.empty(2, 0, device="cuda")
    plan.forward(x, x.clone(), mean=stats, rstd=stats)
    dw, db = torch.ones(2, 16, device="cuda"), torch.ones(2, 16, device="cuda")
    plan.grad(x, x, stats, stats, x, dweight=dw, dbias=db, accumulate=True)
    assert bool((dw == 1).all())
    plan.grad(x, x, stats, stats, x, dweight=dw, dbias=db)
    assert bool((dw == 0).all()) and bool((db == 0).all())


def test_norm_gradient_against_differences():
    x, w, dy = randn(1, 4, 50).double(), randn(1, 50, seed=1).double() + 1, randn(1, 4, 50, seed=2).double()
    f = lambda t, v: float((norm64(t, v, 0.0, 1e-5)[0][0] * dy).sum())  # noqa: E731
    mean, rstd = x.mean(-1).float(), (x.var(-1, correction=0) + 1e-5).rsqrt().float()
    dx, dw, db = torch.empty(1, 4, 50, device="cuda"), torch.empty(1, 50, device="cuda"), torch.empty(1, 50, device="cuda")
    B.LayerNorm(50, 4).grad(dy.float(), x.float(), mean, rstd, dx, weight=w.float(), dweight=dw, dbias=db)
    h = 1e-4
    for e in (0, 17, 49):
        step = torch.zeros_like(x)
        step[0, 2, e] = h
        assert abs((f(x + step, w) - f(x - step, w)) / (2 * h) - float(dx[0, 2, e])) < 1e-4
        step = torch.zeros_like(w)
        step[0, e] = h
        assert abs((f(x, w + step) - f(x, w - step)) / (2 * h) - float(dw[0, e])) < 1e-4


# ---- clipping ------------------------------------------------------------------------------------------------------

def clip64(tensors, max_norm, eps):
    norm = sum(x.double().square().flatten(1).sum(1) for x in tensors).sqrt()
    factor = (max_norm / (norm + eps)).clamp(max=1.0)
    return norm, factor


def check_clip(tensors, outs, max_norm, eps=1e-6):
    norm, factor = clip64(tensors, max_norm, eps)
    plan = B.GradientClip(tensors, outs)
    plan.workspace.fill_(255)
    norms = torch.empty(len(norm), device="cuda")
    plan.norms(norms)
    within(norms, norm, 10 * u * norm)
    again = torch.empty_like(norms)
    sources = [x.clone() for x in tensors]
    plan.workspace.fill_(255)
    plan.clip(max_norm, norms=again, eps=eps)
    assert bool(((again - norms).abs() <= 2 * u * norms).all())    # the CTAs' shares may differ, in float64
    for x, y in zip(sources, outs if outs is not None else tensors):
        want = x.double() * factor.view(-1, *[1] * (x.dim() - 1))
        within(y, want, 14 * u * want.abs())
    return plan


def pieces(c, shapes, dtype, seed=0, at=0, scale=1e-3):
    """Tensors [c, ...] that lie one after the other in c rows."""
    ld = at + sum(math.prod(s) for s in shapes) + 3
    row = randn(c, ld, seed=seed, scale=scale).to(dtype)
    got = []
    for s in shapes:
        flat = row[:, at:at + math.prod(s)]
        got.append(flat.unflatten(1, s) if len(s) > 1 else flat)
        at += math.prod(s)
    return row, got


SHAPES = [[(1,)], [(5,), (3, 4)], [(256, 64), (64,), (64, 64)], [(1001,), (17, 33), (1,), (2048,), (4097,)],
          [(3000, 70)], [(300000,), (9,)]]


@pytest.mark.parametrize("shapes", SHAPES)
@pytest.mark.parametrize("c", [1, 3])
def test_clip_shapes(shapes, c):
    for at in (0, 1, 4):
        _, x = pieces(c, shapes, F32, seed=at, at=at)
        total = math.sqrt(sum(math.prod(s) for s in shapes)) * 1e-3
        for share in (0.5, 10.0):
            row, y = pieces(c, shapes, F32, seed=7, at=at)
            edge = row[:, :at].clone(), row[:, -3:].clone()
            check_clip(x, y, share * total)
            assert torch.equal(edge[0], row[:, :at]) and torch.equal(edge[1], row[:, -3:])
        check_clip(x, None, 0.3 * total)      # in place


@pytest.mark.parametrize("tin", [F32, BF16, F16])
@pytest.mark.parametrize("tout", [F32, BF16, F16])
@pytest.mark.parametrize("at", [(0, 0), (1, 0), (3, 3), (8, 4)])
def test_clip_types(tin, tout, at):
    shapes = [(4000,), (33, 65), (7,)]
    _, x = pieces(2, shapes, tin, seed=3, at=at[0], scale=1.0)
    _, y = pieces(2, shapes, tout, seed=4, at=at[1])
    check_clip(x, y, 20.0)


@pytest.mark.parametrize("cols,pad", [(3, 1), (64, 64), (1000, 7), (1024, 8), (5000, 3), (4096, 16)])
def test_clip_strided_rows(cols, pad):
    x, y = rows(2, 40, cols, pad=pad, at=4), rows(2, 40, cols, pad=pad + 1, at=1, dtype=BF16)
    check_clip([x, x[:, :3]], [y, rows(2, 3, cols)], 5.0)
    assert bool(guarded(y).isnan().all())
    check_clip([x], None, 5.0)
    assert bool(guarded(x).isnan().all())


@pytest.mark.parametrize("count", [8, 9, 40, 41, 340, 341, 700])
def test_clip_many_tensors(count):
    shapes = [(1 + (i * 37) % 300,) if i % 5 else (0,) for i in range(count)]
    _, x = pieces(3, shapes, F32, seed=1)
    _, y = pieces(3, shapes, F32, seed=2)
    check_clip(x, y, 0.01)


@pytest.mark.parametrize("c,d", [(5, 3_000_000), (3, 12_000_001), (40, 500_001)])
def test_clip_by_groups_of_clients(c, d):
    x = randn(c, d, seed=5)
    x *= torch.linspace(0.1, 3, c, device="cuda")[:, None]
    check_clip([x], [torch.empty_like(x)], math.sqrt(d))
    check_clip([x], None, math.sqrt(d))


@pytest.mark.parametrize("scale", [1e-37, 1e-30, 1e-19, 1e-11, 1e18, 1e30, 1e36])
def test_clip_sizes_that_leave_float32_squares(scale):
    x = randn(2, 5000, seed=8) * scale
    norms = torch.empty(2, device="cuda")
    B.GradientClip([x]).norms(norms)
    want = x.double().norm(dim=1)
    within(norms, want, 10 * u * want)
    y = torch.empty_like(x)
    plan = B.GradientClip([x], [y])
    plan.clip(1.0, eps=0.0)
    factor = (1.0 / want).clamp(max=1.0)[:, None]
    within(y, x.double() * factor, 14 * u * (x.double() * factor).abs() + 2.0 ** -126 * x.double().abs())


def test_clip_of_mixed_sizes_and_zeros():
    x = randn(3, 70000, seed=9)
    x[:, ::2] *= 1e-25
    x[:, 1000:40000] = 0
    x[2] = 0
    check_clip([x], [torch.empty_like(x)], 1.0)
    y = torch.full((1, 100), 7.0, device="cuda")
    B.GradientClip([torch.zeros(1, 100, device="cuda")], [y]).clip(0.0, eps=0.0)
    assert bool((y == 0).all())


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_clip_of_a_client_that_is_not_finite(bad):
    x = randn(3, 9000, seed=2)
    x[1, 4321] = bad
    y, norms = torch.empty_like(x), torch.empty(3, device="cuda")
    plan = B.GradientClip([x], [y])
    plan.clip(1.0, norms=norms)
    fine = torch.tensor([0, 2], device="cuda")
    want = clip64([x[fine]], 1.0, 1e-6)
    within(y[fine], x[fine].double() * want[1][:, None], 14 * u * x[fine].double().abs())
    assert bool(norms[1].isnan()) == math.isnan(bad) and not bool(norms[1].isfinite())
    plain = x[1] * (1.0 / (x[1].norm() + 1e-6))
    assert torch.equal(y[1].isnan(), plain.isnan()) and (math.isnan(bad) or float(y[1, 0]) == 0)
    plan.clip(1.0, nonfinite=B.CLIP_ZERO)
    assert bool((y[1] == 0).all()) and bool((y[0] != 0).any())


def test_clip_of_a_broadcast_input():
    x = randn(1, 5000, seed=2).expand(4, 5000)
    check_clip([x], [torch.empty(4, 5000, device="cuda")], 3.0)


# ---- streams, graphs, small workspaces -----------------------------------------------------------------------------

def test_layers_on_another_stream_and_in_a_graph():
    x, dy, w = randn(2, 200, 96), randn(2, 200, 96, seed=1), randn(2, 96, seed=2)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = torch.empty(2, 200, device="cuda"), torch.empty(2, 200, device="cuda")
    grads = torch.zeros(2, 3 * 96, device="cuda")
    dw, db = grads[:, :96], grads[:, 96:192]
    clipped, norms = torch.empty(2, 192, device="cuda"), torch.empty(2, device="cuda")
    norm, clip = B.LayerNorm(96, 200, clients=2), B.GradientClip([dw, db], [clipped[:, :96], clipped[:, 96:]])

    def step(stream=None):
        norm.forward(x, y, weight=w, mean=mean, rstd=rstd, stream=stream)
        norm.grad(dy, x, mean, rstd, dx, weight=w, dweight=dw, dbias=db, stream=stream)
        clip.clip(1.0, norms=norms, stream=stream)

    step()
    torch.cuda.synchronize()
    outputs = (y, dx, clipped, norms)
    want = [t.clone() for t in outputs]
    side = torch.cuda.Stream()
    for t in outputs:
        t.zero_()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(want, outputs))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for t in outputs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(want, outputs))
    x.copy_(randn(2, 200, 96, seed=5))       # new inputs at the same places
    graph.replay()
    torch.cuda.synchronize()
    within(y, *norm64(x, w, torch.zeros_like(w), 1e-5)[0])
    within(norms, *(t if i else t for i, t in enumerate((clip64([dw, db], 1.0, 1e-6)[0], 10 * u * norms.double()))))


def test_workspaces_of_exactly_the_size():
    for d, n, c in [(96, 2000, 3), (77, 5000, 1), (9000, 300, 2)]:
        need = int(B.lib().brace_layer_norm_workspace_bytes(c, n, d))
        whole = torch.full((need + 512,), 255, dtype=torch.uint8, device="cuda")
        at = -whole.data_ptr() % 256
        x, dy = randn(c, n, d), randn(c, n, d, seed=1)
        dx, dw = torch.empty_like(x), torch.empty(c, d, device="cuda")
        mean, rstd = x.mean(-1), x.var(-1).rsqrt()
        for k in (n, n // 2, 3):     # it serves fewer rows
            whole.fill_(255)
            plan = B.LayerNorm(d, n, clients=c, workspace=whole[at:at + need])
            a = [t[:, :k].contiguous() for t in (dy, x, mean, rstd)]
            plan.grad(*a, dx[:, :k], dweight=dw)
            within(dw, *norm_grad64(*a, 1.0)[1])
            assert bool((whole[:at] == 255).all()) and bool((whole[at + need:] == 255).all())
    x = randn(3, 100001)
    need = B.GradientClip([x]).workspace.numel()
    whole = torch.full((need + 512,), 255, dtype=torch.uint8, device="cuda")
    at = -whole.data_ptr() % 256
    norms = torch.empty(3, device="cuda")
    plan = B.GradientClip([x], workspace=whole[at:at + need])
    plan.norms(norms)
    plan.clip(1.0)
    torch.cuda.synchronize()
    assert bool((whole[:at] == 255).all()) and bool((whole[at + need:] == 255).all())


@pytest.mark.parametrize("c,shapes,tin,tout", [(3000, [(4001,)], F32, F32), (2500, [(33, 65), (7,), (2048,)], F32, BF16),
                                               (150, [(100003,), (5,), (300, 301)], BF16, F32),
                                               (12, [(1000, 1000), (999999,), (1,)], F32, F16),
                                               (1, [(7000, 1001), (12_000_001,), (3,)], F32, F32),
                                               (7, [(11, 13)] * 39 + [(1_500_000,)], F32, F32)])
def test_clip_of_large_calls(c, shapes, tin, tout):
    for at in (0, 1):
        _, x = pieces(c, shapes, tin, seed=3, at=at, scale=1.0)
        _, y = pieces(c, shapes, tout, seed=4, at=at)
        total = math.sqrt(sum(math.prod(s) for s in shapes))
        x[0] *= torch.linspace(0.2, 2, c, device="cuda").to(tin).view(-1, *[1] * (x[0].dim() - 1))
        check_clip(x, y, total)
    if tin == tout:
        check_clip(x, None, total)


def test_clip_of_a_large_call_in_a_graph():
    x = randn(9, 2_000_003, seed=5)
    y, norms = torch.empty_like(x), torch.empty(9, device="cuda")
    plan = B.GradientClip([x], [y])
    plan.clip(1000.0, norms=norms)
    torch.cuda.synchronize()
    want = y.clone(), norms.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.clip(1000.0, norms=norms)
    for _ in range(3):
        y.zero_()
        norms.zero_()
        plan.workspace[256:].fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[0]) and torch.equal(norms, want[1])
    x[4, 77] = math.nan
    graph.replay()
    torch.cuda.synchronize()
    assert bool(y[4].isnan().all()) and torch.equal(y[3], want[0][3]) and bool(norms[4].isnan())
