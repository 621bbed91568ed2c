"""The language-model operators on a GPU against plain 64-bit implementations.

Tolerances, from the formulas:
* a sum of n float32 terms in any order is within (n + 2) 2^-24 sum|x| of the exact one; the result's own rounding
  adds u |result|, u = 2^-24 (float32), 2^-11 (float16), 2^-8 (bfloat16), and in float16 at least 2^-25, half of the
  distance of its subnormal numbers.
* orthogonalisation, relative to the result's 2-norm: a step rounds three operands (X, S, P); a rounding to float16
  is off by 2^-11 / sqrt(3) of a value's size in the root mean square, the 15 roundings of five steps by 15 times that
  where the map neither damps nor amplifies them: 4.3e-3 (HALF).  With two planes the operands' 22 bits give 2.1e-6 and
  the float32 sums of up to K terms, K 2^-24 sqrt(K) / K a product, some 1e-6 more, growing with K: 1e-5 (SINGLE)."""

import math

import pytest
import torch

from paper_2501_17392_b200 import brace as B

pytestmark = pytest.mark.gpu

U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 0.0, torch.float16: 2.0 ** -25, torch.bfloat16: 0.0}
TOL = {B.ORTHO_HALF: 15 * 2.0 ** -11 / math.sqrt(3), B.ORTHO_SINGLE: 1e-5}
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
AUTO = {F32: B.ORTHO_SINGLE, F16: B.ORTHO_SINGLE, BF16: B.ORTHO_HALF}   # by the result's type


def gen(seed=0):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(*shape, seed=0, scale=1.0):
    return torch.randn(*shape, device="cuda", generator=gen(seed)) * scale


def direction64(x, steps=5, a=3.4445, b=-4.7750, c=2.0315, eps=1e-7):
    a, b, c, eps = (float(torch.tensor(v, dtype=F32)) for v in (a, b, c, eps))
    x = x.double()
    x = x / (x.square().sum((-2, -1), keepdim=True).sqrt() + eps)
    turn = x.shape[-2] > x.shape[-1]
    x = x.mT if turn else x
    for _ in range(steps):
        s = x @ x.mT
        x = a * x + (b * s + c * s @ s) @ x
    return x.mT if turn else x


def rel(got, want):
    return float((got.double() - want).norm() / want.norm())


def bound(precision, dtype):
    return TOL[precision] + U[dtype]


def signs(words, offset, shape):
    bits = (words.long()[:, None] >> torch.arange(32, device=words.device)) & 1
    return (2 * bits.flatten()[offset:offset + math.prod(shape)] - 1).view(shape)


# ---- orthogonalisation --------------------------------------------------------------------------------------------

SHAPES = [(1, 1, 1), (1, 1, 7), (2, 7, 1), (1, 16, 16), (3, 17, 5), (1, 33, 1000), (2, 64, 64), (1, 127, 129),
          (1, 128, 128), (2, 129, 127), (1, 130, 300), (1, 256, 64), (1, 255, 257), (5, 96, 200), (1, 384, 384),
          (1, 100, 5000), (1, 5000, 100), (2, 513, 700), (1, 700, 513), (1, 640, 2048), (1, 1100, 1030)]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("precision", [B.ORTHO_HALF, B.ORTHO_SINGLE])
def test_orthogonalize_shapes(shape, precision):
    b, r, c = shape
    g = randn(b, r, c, seed=r * 7 + c, scale=1e-3)
    out = torch.full((b, r, c), 7.0, device="cuda")
    plan = B.Orthogonalizer(r, c, batch=b, params=B.ortho_params(precision=precision))
    plan.orthogonalize(g, out)
    plan.check()
    want = direction64(g)
    for e in range(b):
        assert rel(out[e], want[e]) <= bound(precision, F32)


# sizes that take the products' other tile shapes and the shared contractions, wide and tall
@pytest.mark.parametrize("shape", [(1, 300, 2400), (1, 2400, 300), (1, 600, 600), (2, 700, 1100), (1, 1500, 1500),
                                   (1, 1800, 2100), (1, 2100, 1800), (3, 1990, 2000), (1, 2900, 3300), (1, 3300, 2900)])
@pytest.mark.parametrize("precision", [B.ORTHO_HALF, B.ORTHO_SINGLE])
def test_orthogonalize_large(shape, precision):
    b, r, c = shape
    g = randn(b, r, c, seed=r + c, scale=10.0)
    out = torch.full((b, r, c), 7.0, device="cuda")
    plan = B.Orthogonalizer(r, c, batch=b, params=B.ortho_params(precision=precision))
    plan.orthogonalize(g, out)
    plan.check()
    again = torch.empty_like(out)
    plan.orthogonalize(g, again)
    assert torch.equal(out, again)
    want = direction64(g)
    for e in range(b):
        assert rel(out[e], want[e]) <= bound(precision, F32)


@pytest.mark.parametrize("tin", [F32, BF16, F16])
@pytest.mark.parametrize("tout", [F32, BF16, F16])
def test_orthogonalize_types(tin, tout):
    g = randn(2, 70, 190, seed=3).to(tin)
    out = torch.empty(2, 70, 190, device="cuda", dtype=tout)
    B.Orthogonalizer(70, 190, batch=2).orthogonalize(g, out)
    assert rel(out, direction64(g)) <= bound(AUTO[tout], tout)


@pytest.mark.parametrize("steps", [1, 2, 3, 8])
@pytest.mark.parametrize("shape", [(60, 200), (200, 60), (300, 300)])
def test_orthogonalize_steps_and_coefficients(steps, shape):
    g = randn(1, *shape, seed=steps)
    out = torch.empty_like(g)
    B.Orthogonalizer(*shape, params=B.ortho_params(steps=steps, a=1.875, b=-1.25, c=0.375)).orthogonalize(g, out)
    assert rel(out, direction64(g, steps, 1.875, -1.25, 0.375)) <= bound(B.ORTHO_SINGLE, F32)


@pytest.mark.parametrize("shape", [(3, 40, 96), (1, 200, 333), (1, 333, 200)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_orthogonalize_strides_and_guard_bands(shape, dtype):
    b, r, c = shape
    # rows and matrices further apart, starting at an odd element; what lies between is not touched
    ld, st = c + 3, (c + 3) * (r + 2) + 1
    flat = randn(b * st + 11, seed=5).to(dtype)
    g = flat.as_strided((b, r, c), (st, ld, 1), 5)
    store = torch.full((b * st + 11,), 9.0, device="cuda", dtype=dtype)
    out = store.as_strided((b, r, c), (st, ld, 1), 7)
    B.Orthogonalizer(r, c, batch=b).orthogonalize(g, out)
    assert rel(out, direction64(g)) <= bound(AUTO[dtype], dtype)
    out.fill_(9.0)
    assert bool((store == 9.0).all())


@pytest.mark.parametrize("offset", [0, 1, 31, 77])
def test_orthogonalize_packed_bits(offset):
    words = torch.randint(-2 ** 31, 2 ** 31, ((offset + 3 * 50 * 61 + 31) // 32,), device="cuda", generator=gen(offset)).int()
    out = torch.empty(3, 50, 61, device="cuda")
    B.Orthogonalizer(50, 61, batch=3).orthogonalize(words, out, bit_offset=offset)
    assert rel(out, direction64(signs(words, offset, (3, 50, 61)))) <= bound(B.ORTHO_SINGLE, F32)


@pytest.mark.parametrize("precision", [B.ORTHO_HALF, B.ORTHO_SINGLE])
@pytest.mark.parametrize("shape", [(40, 90), (300, 260)])
def test_orthogonalize_zero_and_non_finite_matrices(precision, shape):
    g = randn(5, *shape, seed=1)
    g[1] = 0
    g[2, 3, 5] = float("nan")
    g[3, 0, 0] = float("-inf")
    out = torch.empty_like(g)
    B.Orthogonalizer(*shape, batch=5, params=B.ortho_params(precision=precision)).orthogonalize(g, out)
    want = direction64(g)
    assert rel(out[0], want[0]) <= bound(precision, F32) and rel(out[4], want[4]) <= bound(precision, F32)
    assert bool((out[1] == 0).all())
    assert bool(out[2].isnan().all()) and bool(out[3].isnan().all())


@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1e15, 1e35])
def test_orthogonalize_extreme_sizes(scale):
    # the squares of these leave float32's range; the norm does not
    g = randn(1, 80, 70, seed=2) * scale
    out = torch.empty_like(g)
    B.Orthogonalizer(80, 70, params=B.ortho_params(eps=1e-30)).orthogonalize(g, out)
    assert rel(out, direction64(g, eps=1e-30)) <= bound(B.ORTHO_SINGLE, F32)


def test_orthogonalize_low_rank():
    # a rounding error e of X_0 outside the matrix's range grows by a^5 = 485 while the matrix itself grows to about
    # 1: with 22 bits, 485 * 2^-22 * sqrt(240 / 4) = 9e-4
    g = randn(1, 240, 4, seed=8) @ randn(1, 4, 310, seed=9)
    out = torch.empty_like(g)
    B.Orthogonalizer(240, 310).orthogonalize(g, out)
    assert rel(out, direction64(g)) <= 9e-4


def test_orthogonalize_repeats_and_streams():
    g = randn(4, 200, 310, seed=4)
    plan = B.Orthogonalizer(200, 310, batch=4)
    a, b = torch.empty_like(g), torch.empty_like(g)
    plan.orthogonalize(g, a)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        x = g * 1.0
        plan.orthogonalize(x, b)       # on the current stream of the context manager
    side.synchronize()
    assert torch.equal(a, b)
    c = torch.empty_like(g)
    plan.orthogonalize(g, c, stream=side)
    side.synchronize()
    assert torch.equal(a, c)


def test_orthogonalize_in_a_graph():
    g = randn(1, 300, 200, seed=6)
    out = torch.empty_like(g)
    plan = B.Orthogonalizer(300, 200)
    plan.orthogonalize(g, out)
    want = out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.orthogonalize(g, out)
    g.copy_(randn(1, 300, 200, seed=66))
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert rel(out, direction64(g)) <= bound(B.ORTHO_SINGLE, F32) and not torch.equal(out, want)


def test_empty_matrices_do_nothing():
    for b, r, c in [(0, 4, 4), (1, 0, 4), (1, 4, 0)]:
        t = torch.empty(b, r, c, device="cuda")
        B.Orthogonalizer(r, c, batch=b).orthogonalize(t, t)
    torch.cuda.synchronize()


# ---- momentum step ------------------------------------------------------------------------------------------------

def muon64(g, m, w, lr, beta, nesterov, decay, scale):
    f = lambda v: float(torch.tensor(v, dtype=F32))  # noqa: E731
    lr, beta, decay, scale = f(lr), f(beta), f(decay), f(scale)
    m = beta * m.double() + g.double()
    o = direction64(g.double() + beta * m if nesterov else m)
    return m, (1 - lr * decay) * w.double() - lr * scale * o, lr * scale * o


@pytest.mark.parametrize("shape", [(2, 50, 61), (1, 260, 130), (3, 130, 256), (1, 64, 64)])
@pytest.mark.parametrize("tg", [F32, BF16, F16, torch.int32])
@pytest.mark.parametrize("tw", [F32, BF16, F16])
@pytest.mark.parametrize("nesterov", [True, False])
def test_muon_step(shape, tg, tw, nesterov):
    b, r, c = shape
    n, offset = b * r * c, 45 if tg == torch.int32 else 0
    if tg == torch.int32:
        g = torch.randint(-2 ** 31, 2 ** 31, ((offset + n + 31) // 32,), device="cuda", generator=gen(1)).int()
        gf = signs(g, offset, shape)
    else:
        g = gf = randn(b, r, c, seed=1).to(tg)
    m, w = randn(b, r, c, seed=2, scale=3.0), randn(b, r, c, seed=3, scale=0.05).to(tw)
    args = (0.03, 0.9, nesterov, 0.1, 1.5)
    want_m, want_w, step = muon64(gf, m, w, *args)
    plan = B.Orthogonalizer(r, c, batch=b)
    m_out, w_out = torch.empty_like(m), torch.empty_like(w)
    kw = dict(beta=args[1], nesterov=nesterov, weight_decay=args[3], scale=args[4], bit_offset=offset)
    plan.muon_step(g, m, w, args[0], momentum_out=m_out, weights_out=w_out, **kw)
    plan.check()
    size = (args[1] * m.double()).abs() + gf.double().abs()
    assert bool(((m_out.double() - want_m).abs() <= 2 ** -23 * size).all())
    precision = AUTO[tw]
    # float32 arithmetic on w and o: four roundings of values up to |w| + |step|; then the type's own
    off = (w_out.double() - want_w).norm()
    limit = TOL[precision] * step.norm() + (4 * U[F32] + U[tw]) * (w.double().norm() + step.norm())
    assert float(off) <= float(limit)
    # in place: the same bits
    plan.muon_step(g, m, w, args[0], **kw)
    assert torch.equal(m, m_out) and torch.equal(w, w_out)


@pytest.mark.parametrize("shape", [(1, 400, 1500), (1, 1600, 1600), (2, 2000, 1300)])
@pytest.mark.parametrize("tw", [F32, BF16])
def test_muon_step_large(shape, tw):
    g, m, w = randn(*shape, seed=1).to(BF16), randn(*shape, seed=2), randn(*shape, seed=3, scale=0.05).to(tw)
    want_m, want_w, step = muon64(g, m, w, 0.03, 0.9, True, 0.1, 1.5)
    plan = B.Orthogonalizer(shape[1], shape[2], batch=shape[0])
    plan.muon_step(g, m, w, 0.03, beta=0.9, weight_decay=0.1, scale=1.5)
    plan.check()
    limit = TOL[AUTO[tw]] * step.norm() + (4 * U[F32] + U[tw]) * (want_w.norm() + step.norm())
    assert float((w.double() - want_w).norm()) <= float(limit)


@pytest.mark.parametrize("tw", [F32, BF16])
def test_muon_step_for_replicas(tw):
    # the weights are rows of clients' parameter vectors; all take the step, nothing between them is touched
    n, r, c, at, ld = 3, 70, 90, 13, 70 * 90 + 77
    rows = randn(n, ld, seed=11).to(tw)
    before = rows.clone()
    w = rows.as_strided((n, 1, r, c), (ld, r * c, c, 1), at)
    m, g = randn(1, r, c, seed=12), randn(1, r, c, seed=13)
    one, m1 = w[1].clone(), m.clone()
    plan = B.Orthogonalizer(r, c)
    plan.muon_step(g, m1, one, 0.02, scale=0.3)
    plan.muon_step(g, m, w, 0.02, scale=0.3)
    assert torch.equal(w[1], one) and torch.equal(m, m1)
    _, want, step = muon64(g, torch.zeros_like(g) + randn(1, r, c, seed=12), before.as_strided(w.shape, w.stride(), at),
                           0.02, 0.95, True, 0.0, 0.3)
    limit = TOL[AUTO[tw]] * step.norm() * n ** 0.5 + (4 * U[F32] + U[tw]) * want.norm()
    assert float((w.double() - want).norm()) <= float(limit)
    rows.as_strided(w.shape, w.stride(), at).zero_()
    before.as_strided(w.shape, w.stride(), at).zero_()
    assert torch.equal(rows, before)


# ---- embedding ----------------------------------------------------------------------------------------------------

def ids_of(clients, tokens, vocab, seed=0, dtype=torch.int64, pad=0.1):
    u = torch.rand(clients, tokens, device="cuda", generator=gen(seed), dtype=torch.float64)
    ids = ((vocab + 1.0) ** u).long() - 1
    bad = torch.rand(clients, tokens, device="cuda", generator=gen(seed + 1)) < pad
    return torch.where(bad, torch.where(ids % 2 == 0, -1, vocab), ids.clamp(max=vocab - 1)).to(dtype)


@pytest.mark.parametrize("tt", [F32, BF16, F16])
@pytest.mark.parametrize("ta", [F32, BF16, F16])
@pytest.mark.parametrize("clients,tokens,vocab,dim", [(1, 1, 1, 1), (1, 1, 50, 64), (2, 37, 100, 33), (3, 1030, 77, 48),
                                                      (1, 5000, 3000, 130)])
def test_lookup(tt, ta, clients, tokens, vocab, dim):
    table = randn(clients, vocab, dim, seed=dim).to(tt)
    ids = ids_of(clients, tokens, vocab, dtype=torch.int32 if dim % 2 else torch.int64)
    out = torch.full((clients, tokens, dim), 3.0, device="cuda", dtype=ta)
    B.Embedding(vocab, dim, tokens, clients=clients, grad=False).lookup(table, ids, out, scale=1.7)
    valid = (ids >= 0) & (ids < vocab)
    scale = torch.tensor(1.7, dtype=F32)
    rows = table[torch.arange(clients, device="cuda")[:, None], torch.where(valid, ids, 0).long()].float() * scale.cuda()
    want = torch.where(valid[..., None], rows, 0.0).to(ta)   # one float32 product, rounded once: the same bits
    assert torch.equal(out, want)


@pytest.mark.parametrize("at,gap", [(0, 0), (1, 0), (8, 8), (2, 6), (0, 3)])
def test_lookup_layouts(at, gap):
    clients, tokens, vocab, dim = 2, 300, 90, 40
    flat = randn(clients * (vocab * (dim + gap) + 16) + 64, seed=1)
    table = flat.as_strided((clients, vocab, dim), (vocab * (dim + gap) + 16, dim + gap, 1), at)
    store = torch.full((tokens * clients * (dim + gap) + 64,), 5.0, device="cuda")
    # tokens outside, clients inside
    out = store.as_strided((clients, tokens, dim), (dim + gap, clients * (dim + gap), 1), at)
    ids = ids_of(clients, tokens, vocab)
    plan = B.Embedding(vocab, dim, tokens, clients=clients)
    plan.lookup(table, ids, out, scale=0.5)
    valid = (ids >= 0) & (ids < vocab)
    want = table[torch.arange(clients, device="cuda")[:, None], torch.where(valid, ids, 0)] * 0.5 * valid[..., None]
    assert torch.equal(out, want)
    out.fill_(5.0)
    assert bool((store == 5.0).all())
    # one table for all clients, and fewer tokens than the plan was made for
    few = torch.empty(clients, 9, dim, device="cuda")
    plan.lookup(table[0], ids[:, :9], few, scale=0.5)
    assert torch.equal(few, table[0][torch.where(valid, ids, 0)[:, :9]] * 0.5 * valid[:, :9, None])


def grad64(dy, ids, vocab, scale):
    """(sum, sum of absolute values, terms) per row of each client's table."""
    c, n, d = dy.shape
    scale = float(torch.tensor(scale, dtype=F32))
    valid = (ids >= 0) & (ids < vocab)
    key = torch.where(valid, ids.long() + vocab * torch.arange(c, device="cuda")[:, None], c * vocab).flatten()
    x = torch.where(valid[..., None], dy.double(), 0.0).reshape(-1, d) * scale
    total = torch.zeros(c * vocab + 1, d, device="cuda", dtype=torch.float64)
    size, count = total.clone(), torch.zeros(c * vocab + 1, device="cuda", dtype=torch.float64)
    total.index_add_(0, key, x)
    size.index_add_(0, key, x.abs())
    count.index_add_(0, key, torch.ones_like(key, dtype=torch.float64))
    return total[:-1].view(c, vocab, d), size[:-1].view(c, vocab, d), count[:-1].view(c, vocab, 1)


GRAD_SIZES = [(1, 1, 1, 1), (1, 1, 300, 8), (1, 33, 7, 16), (2, 64, 64, 24), (3, 1000, 63, 5), (2, 1024, 4000, 10),
              (1, 1025, 4095, 32), (2, 5001, 900, 33), (1, 8192, 64, 16), (2, 8193, 70, 8), (1, 20000, 6000, 40),
              (1, 140000, 500, 6), (1, 70000, 3, 8), (4, 100, 20000, 264), (1, 50, 100, 3000)]


@pytest.mark.parametrize("clients,tokens,vocab,dim", GRAD_SIZES)
@pytest.mark.parametrize("tt", [F32, BF16])
def test_grad(clients, tokens, vocab, dim, tt):
    dy = randn(clients, tokens, dim, seed=tokens).to(F16 if vocab % 2 else F32)
    ids = ids_of(clients, tokens, vocab, dtype=torch.int32 if dim % 3 else torch.int64)
    plan = B.Embedding(vocab, dim, tokens, clients=clients)
    out = torch.full((clients, vocab, dim), 3.0, device="cuda", dtype=tt)
    plan.grad(dy, ids, out, scale=0.7)
    total, size, count = grad64(dy, ids, vocab, 0.7)
    assert bool(((out.double() - total).abs() <= (count + 3) * 2 ** -24 * size + U[tt] * total.abs()).all())
    again = torch.empty_like(out)
    plan.grad(dy, ids, again, scale=0.7)
    assert torch.equal(out, again)
    # added to what is there: one more rounding of the sum; untouched rows keep their bits
    base = randn(clients, vocab, dim, seed=9).to(tt)
    added = base.clone()
    plan.grad(dy, ids, added, scale=0.7, accumulate=True)
    want = base.double() + total
    limit = (count + 3) * 2 ** -24 * size + (U[tt] + 2 ** -24) * (want.abs() + base.double().abs())
    assert bool(((added.double() - want).abs() <= limit).all())
    assert torch.equal(added[(count == 0).squeeze(-1)], base[(count == 0).squeeze(-1)])


@pytest.mark.parametrize("tin", [F32, BF16, F16])
@pytest.mark.parametrize("tout", [F32, BF16, F16])
@pytest.mark.parametrize("dim", [64, 66, 61])
def test_grad_types_and_layouts(tin, tout, dim):
    clients, tokens, vocab = 3, 700, 120
    ld = dim + (8 if dim == 64 else 3)
    dy = randn(tokens, clients, dim, seed=2).to(tin).transpose(0, 1)        # tokens outside, clients inside
    ids = ids_of(clients, tokens, vocab)
    st = vocab * ld + 40
    store = torch.full((clients * st + 64,), 5.0, device="cuda", dtype=tout)
    out = store.as_strided((clients, vocab, dim), (st, ld, 1), 16 if dim == 64 else 3)
    B.Embedding(vocab, dim, tokens, clients=clients).grad(dy, ids, out, scale=2.0)
    total, size, count = grad64(dy, ids, vocab, 2.0)
    assert bool(((out.double() - total).abs() <= (count + 3) * 2 ** -24 * size + U[tout] * total.abs() + TINY[tout]).all())
    out.fill_(5.0)
    assert bool((store == 5.0).all())


def test_grad_of_broadcast_activations():
    # the gradient of a sum: one row for all tokens (stride 0)
    row = randn(1, 1, 32, seed=3)
    dy = row.expand(2, 400, 32)
    ids = ids_of(2, 400, 50)
    out = torch.empty(2, 50, 32, device="cuda")
    B.Embedding(50, 32, 400, clients=2).grad(dy, ids, out)
    total, size, count = grad64(dy, ids, 50, 1.0)
    assert bool(((out.double() - total).abs() <= (count + 3) * 2 ** -24 * size).all())


@pytest.mark.parametrize("tokens,vocab", [(600_000, 5000), (524_289, 300_000)])
def test_grad_of_long_texts(tokens, vocab):
    # several tokens' tiles a CTA in the wide sort (256 tiles at most), two and three passes
    dy, ids = randn(1, tokens, 4, seed=1), ids_of(1, tokens, vocab, seed=3)
    out = torch.empty(1, vocab, 4, device="cuda")
    plan = B.Embedding(vocab, 4, tokens)
    plan.grad(dy, ids, out)
    total, size, count = grad64(dy, ids, vocab, 1.0)
    assert bool(((out.double() - total).abs() <= (count + 3) * 2 ** -24 * size).all())
    for n in (524_288, 2049, 2048):     # fewer than the plan was made for, with more tiles or none
        plan.grad(dy[:, :n], ids[:, :n], out)
        total, size, count = grad64(dy[:, :n], ids[:, :n], vocab, 1.0)
        assert bool(((out.double() - total).abs() <= (count + 3) * 2 ** -24 * size).all())


@pytest.mark.parametrize("n", [31, 32, 33, 63, 64, 65, 95, 96, 97, 127, 128, 129, 4000])
def test_grad_of_one_frequent_token(n):
    # n equal ids behind k others: the groups of 32 sorted tokens begin anywhere in the run
    for k in (0, 1, 17, 31):
        ids = torch.cat([torch.arange(k, device="cuda"), torch.full((n,), 40, device="cuda", dtype=torch.int64)])
        ids = ids[torch.randperm(n + k, device="cuda", generator=gen(n))][None]
        dy = randn(1, n + k, 24, seed=n + k)
        out = torch.empty(1, 64, 24, device="cuda")
        B.Embedding(64, 24, n + k).grad(dy, ids, out)
        total, size, count = grad64(dy, ids, 64, 1.0)
        assert bool(((out.double() - total).abs() <= (count + 3) * 2 ** -24 * size).all())


def test_grad_without_tokens_and_with_only_padding():
    out = torch.full((2, 30, 12), 4.0, device="cuda")
    plan = B.Embedding(30, 12, 5, clients=2)
    none = torch.empty(2, 0, dtype=torch.int64, device="cuda")
    plan.grad(torch.empty(2, 0, 12, device="cuda"), none, out, accumulate=True)
    assert bool((out == 4).all())
    plan.grad(torch.empty(2, 0, 12, device="cuda"), none, out)
    assert bool((out == 0).all())
    out.fill_(4.0)
    pad = torch.full((2, 5), -1, device="cuda", dtype=torch.int64)
    plan.grad(torch.full((2, 5, 12), float("nan"), device="cuda"), pad, out)     # what is masked is not read
    assert bool((out == 0).all())
    act = torch.full((2, 5, 12), 4.0, device="cuda")
    plan.lookup(torch.full((2, 30, 12), float("nan"), device="cuda"), pad, act)
    assert bool((act == 0).all())


def test_grad_of_non_finite_activations_stays_in_its_row():
    dy = randn(1, 100, 16, seed=4)
    dy[0, 10] = float("inf")
    ids = torch.arange(100, device="cuda")[None] % 37
    out = torch.empty(1, 40, 16, device="cuda")
    B.Embedding(40, 16, 100).grad(dy, ids, out)
    assert bool(out[0, 10].isinf().all()) and bool(out[0, torch.arange(40, device="cuda") != 10].isfinite().all())


def test_grad_is_the_derivative_of_the_lookup():
    # along any direction: <dy, lookup(E + h D) - lookup(E - h D)> / 2h = <grad, D>, exactly linear in E
    clients, tokens, vocab, dim = 2, 60, 25, 8
    plan = B.Embedding(vocab, dim, tokens, clients=clients)
    table, d, dy = randn(clients, vocab, dim, seed=1), randn(clients, vocab, dim, seed=2), randn(clients, tokens, dim, seed=3)
    ids = ids_of(clients, tokens, vocab)
    h = 0.25
    outs = []
    for s in (1, -1):
        out = torch.empty(clients, tokens, dim, device="cuda")
        plan.lookup(table + s * h * d, ids, out, scale=1.5)
        outs.append(out.double())
    slope = float((dy.double() * (outs[0] - outs[1])).sum()) / (2 * h)
    grad = torch.empty_like(table)
    plan.grad(dy, ids, grad, scale=1.5)
    # each difference is off by some 2^-23 of values up to 3, over 2 h, at 960 places
    assert abs(slope - float((grad.double() * d.double()).sum())) <= 960 * 2 ** -23 * 10 / (2 * h)


def test_table_past_32_bits_of_offset():
    # clients' tables that start more than 2^32 elements into the weights
    free = torch.cuda.mem_get_info()[0]
    if free < 30 << 30:
        pytest.skip("needs 30 GB of free memory")
    vocab, dim, ld = 1000, 64, (1 << 32) + 4096
    store = torch.empty(ld + vocab * dim, device="cuda", dtype=BF16)
    table = store.as_strided((2, vocab, dim), (ld, dim, 1))
    table.copy_(randn(2, vocab, dim, seed=5))
    ids = ids_of(2, 300, vocab)
    out = torch.empty(2, 300, dim, device="cuda")
    plan = B.Embedding(vocab, dim, 300, clients=2)
    plan.lookup(table, ids, out)
    valid = (ids >= 0) & (ids < vocab)
    want = table[torch.arange(2, device="cuda")[:, None], torch.where(valid, ids, 0)].float() * valid[..., None]
    assert torch.equal(out, want)
    plan.grad(out, ids, table)
    total, size, count = grad64(out, ids, vocab, 1.0)
    assert bool(((table.double() - total).abs() <= (count + 3) * 2 ** -24 * size + U[BF16] * total.abs()).all())


# ---- together -----------------------------------------------------------------------------------------------------

def test_rounds_of_a_language_model():
    from examples.language_model_round import train

    losses = train(rounds=25)
    # from chance (log 300 = 5.7) the loss falls although a fifth of the clients send ten times the opposite
    assert 5.0 < losses[0] < 6.5 and losses[-1] < 0.5 * losses[0]


def test_a_wait_that_ran_out_is_reported():
    # the kernels note it in the workspace's first word; the next call clears it
    plan = B.Orthogonalizer(20, 20)
    g, out = randn(1, 20, 20), torch.empty(1, 20, 20, device="cuda")
    plan.orthogonalize(g, out)
    plan.check()
    plan.workspace[:4] = torch.tensor([1, 0, 0, 0], dtype=torch.uint8)
    with pytest.raises(B.BraceError) as err:
        plan.check()
    assert err.value.status == B.ERR_TIMEOUT
    plan.orthogonalize(g, out)
    plan.check()
