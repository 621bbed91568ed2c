"""Forms of the matrix operators that sizes alone do not reach: large clusters, and what pairs of CTAs make of types, strides,
packed bits, replicas and matrices that are not finite.  References and bounds are those of test_gpu_operators.py."""

import pytest
import torch

from paper_2501_17392_b200 import brace as B
from tests.test_gpu_operators import AUTO, BF16, F16, F32, TOL, U, bound, direction64, gen, muon64, randn, rel, signs

pytestmark = pytest.mark.gpu

# one launch by 9 to 16 CTAs: a short side up to 128, a long one of 1025 to 2048 (two planes) or 2049 to 4096 (one)
LARGE_CLUSTERS = [(B.ORTHO_SINGLE, s) for s in [(1, 128, 1025), (2, 100, 1290), (1, 1500, 128), (3, 17, 1990), (1, 2048, 128),
                                                (1, 2048, 1), (1, 128, 2048)]]
LARGE_CLUSTERS += [(B.ORTHO_HALF, s) for s in [(1, 128, 2050), (2, 2700, 64), (1, 90, 3333), (3, 4096, 128), (1, 128, 4096)]]


@pytest.mark.parametrize("precision,shape", LARGE_CLUSTERS)
def test_clusters_of_9_to_16(precision, shape):
    b, r, c = shape
    g = randn(b, r, c, seed=r + c)
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


@pytest.mark.parametrize("shape", [(12, 128, 2048), (30, 1100, 30)])
def test_more_large_clusters_than_fit_at_once(shape):
    b, r, c = shape
    g = randn(b, r, c, seed=5)
    out = torch.empty_like(g)
    plan = B.Orthogonalizer(r, c, batch=b)
    plan.orthogonalize(g, out)
    plan.check()
    want = direction64(g)
    for e in range(b):
        assert rel(out[e], want[e]) <= bound(B.ORTHO_SINGLE, F32)


@pytest.mark.parametrize("tg", [F32, BF16, F16, torch.int32])
@pytest.mark.parametrize("tw", [F32, BF16, F16])
@pytest.mark.parametrize("shape", [(2, 120, 1800), (1, 1777, 99)])
def test_muon_step_in_large_clusters(shape, tg, tw):
    offset = 45 if tg == torch.int32 else 0
    n = shape[0] * shape[1] * shape[2]
    if tg == torch.int32:
        g = torch.randint(-2 ** 31, 2 ** 31, ((offset + n + 31) // 32,), device="cuda", generator=gen(1)).int()
        gf = signs(g, offset, shape)
    else:
        g = gf = randn(*shape, seed=1).to(tg)
    m, w = randn(*shape, seed=2, scale=3.0), randn(*shape, seed=3, scale=0.05).to(tw)
    want_m, want_w, step = muon64(gf, m, w, 0.03, 0.9, True, 0.1, 1.5)
    plan = B.Orthogonalizer(shape[1], shape[2], batch=shape[0])
    plan.muon_step(g, m, w, 0.03, beta=0.9, weight_decay=0.1, scale=1.5, bit_offset=offset)
    plan.check()
    assert rel(m, want_m) <= 2 ** -23
    limit = TOL[AUTO[tw]] * step.norm() + (4 * U[F32] + U[tw]) * (want_w.norm() + step.norm())
    assert float((w.double() - want_w).norm()) <= float(limit)


def test_large_clusters_keep_bad_matrices_to_themselves():
    g = randn(4, 100, 1900, seed=1)
    g[1] = 0
    g[2, 99, 1899] = float("nan")
    out = torch.empty_like(g)
    B.Orthogonalizer(100, 1900, batch=4).orthogonalize(g, out)
    want = direction64(g)
    assert rel(out[0], want[0]) <= bound(B.ORTHO_SINGLE, F32) and rel(out[3], want[3]) <= bound(B.ORTHO_SINGLE, F32)
    assert bool((out[1] == 0).all()) and bool(out[2].isnan().all())


def test_expanded_tensors_are_not_written():
    # one matrix in memory for several: read, but not written
    plan, g = B.Orthogonalizer(40, 60, batch=2), randn(2, 40, 60, seed=1)
    one = randn(1, 40, 60, seed=2)
    before, shared = one.clone(), one.expand(2, 40, 60)
    m, w = torch.zeros_like(g), torch.zeros_like(g)
    for call in (lambda: plan.orthogonalize(g, shared), lambda: plan.muon_step(g, shared, w, 0.1),
                 lambda: plan.muon_step(g, m, shared, 0.1), lambda: plan.muon_step(g, m, w[None].expand(3, 2, 40, 60), 0.1)):
        with pytest.raises(B.BraceError) as err:
            call()
        assert err.value.status == B.ERR_INVALID_ARG
    torch.cuda.synchronize()
    assert torch.equal(one, before) and not m.any() and not w.any()
    out = torch.empty_like(g)
    plan.orthogonalize(shared, out)
    assert torch.equal(out[0], out[1]) and rel(out[0], direction64(one)[0]) <= bound(B.ORTHO_SINGLE, F32)
    # three copies of the weights that begin as one
    copies = torch.empty(3, 2, 40, 60, device="cuda")
    plan.muon_step(shared, m, w[None].expand(3, 2, 40, 60), 0.1, weights_out=copies, nesterov=False)
    assert rel(copies, -0.1 * direction64(one).expand(3, 2, 40, 60)) <= bound(B.ORTHO_SINGLE, F32)


@pytest.mark.parametrize("b,r,c", [(1, 40, 60), (2, 0, 7), (0, 5, 5)])
def test_check_of_a_plan_that_has_computed_nothing(b, r, c):
    dirty = torch.full((1 << 20,), 0xFF, device="cuda", dtype=torch.uint8)
    plan = B.Orthogonalizer(r, c, batch=b, workspace=dirty)
    plan.check()
    t = torch.zeros(b, r, c, device="cuda")
    if not t.numel():
        plan.orthogonalize(t, t)
        plan.check(torch.cuda.current_stream())
        plan.muon_step(t, t, t, 0.1)
        plan.check()
    else:
        plan.orthogonalize(t, torch.empty_like(t))
        plan.check()
        plan.workspace[:4] = 0xFF       # and then it is the workspace that says it
        with pytest.raises(B.BraceError):
            plan.check()


def guarded(need, fill, seed=0):
    """A workspace of exactly `need` bytes with `fill` in it (None: random bytes) between guard bytes."""
    store = torch.randint(0, 256, (need + 1024,), device="cuda", generator=gen(seed)).to(torch.uint8)
    if fill is not None:
        store[512:512 + need] = fill
    guards = torch.cat([store[:512], store[512 + need:]])
    return store, store[512:512 + need], guards


def intact(store, need, guards):
    return torch.equal(torch.cat([store[:512], store[512 + need:]]), guards)


# 0xff: NaN in every operand, and no position in range; 0x7c: infinities and large numbers
FILLS = [0xFF, 0x7C, None]


@pytest.mark.parametrize("shape", [(1, 40, 60), (1, 100, 1500), (1, 130, 130), (2, 300, 130), (1, 161, 700), (3, 513, 770),
                                   (1, 1030, 2070), (1, 1500, 1500), (1, 2083, 1811)])
@pytest.mark.parametrize("precision", [B.ORTHO_HALF, B.ORTHO_SINGLE])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_what_the_workspace_held_does_not_matter(shape, precision, dtype):
    b, r, c = shape
    params, g = B.ortho_params(precision=precision), randn(b, r, c, seed=r)
    need = B.ortho_workspace_bytes(b, r, c, params, {F32: B.TYPE_F32, BF16: B.TYPE_BF16}[dtype])
    want = torch.empty(b, r, c, device="cuda", dtype=dtype)
    B.Orthogonalizer(r, c, batch=b, params=params, workspace=torch.zeros(need, device="cuda", dtype=torch.uint8)).orthogonalize(g, want)
    assert rel(want, direction64(g)) <= bound(precision, dtype)
    for fill in FILLS:
        store, workspace, guards = guarded(need, fill)
        out = torch.empty_like(want)
        plan = B.Orthogonalizer(r, c, batch=b, params=params, workspace=workspace)
        plan.orthogonalize(g, out)
        plan.check()
        assert torch.equal(out, want) and intact(store, need, guards)


@pytest.mark.parametrize("clients,tokens,vocab,dim", [(1, 2048, 300, 40), (2, 2049, 5000, 24), (3, 5001, 900, 33),
                                                      (1, 70000, 3, 8), (1, 300_000, 70_000, 4)])
def test_what_the_gradients_workspace_held_does_not_matter(clients, tokens, vocab, dim):
    dy = randn(clients, tokens, dim, seed=1)
    u = torch.rand(clients, tokens, device="cuda", generator=gen(2), dtype=torch.float64)
    ids = ((vocab + 1.0) ** u).long() - 2           # few frequent ids, many without a token, -1 for none
    need = int(B.lib().brace_embedding_workspace_bytes(clients, tokens, vocab, dim))
    want = torch.empty(clients, vocab, dim, device="cuda")
    B.Embedding(vocab, dim, tokens, clients=clients, workspace=torch.zeros(need, device="cuda", dtype=torch.uint8)).grad(dy, ids, want)
    for fill in FILLS:
        store, workspace, guards = guarded(need, fill)
        out = torch.full_like(want, 9.0)
        B.Embedding(vocab, dim, tokens, clients=clients, workspace=workspace).grad(dy, ids, out)
        assert torch.equal(out, want) and intact(store, need, guards)
    # positions in range that belong to other ids
    store, workspace, guards = guarded(need, 0)
    n = need // 4
    workspace[:4 * n].view(torch.int32).copy_(torch.arange(n, device="cuda", dtype=torch.int32) % tokens)
    out = torch.full_like(want, 9.0)
    B.Embedding(vocab, dim, tokens, clients=clients, workspace=workspace).grad(dy, ids, out)
    assert torch.equal(out, want) and intact(store, need, guards)


def test_tensors_on_the_host_are_refused():
    plan, g, h = B.Orthogonalizer(4, 6), torch.zeros(1, 4, 6, device="cuda"), torch.zeros(1, 4, 6)
    bits = torch.zeros(1, dtype=torch.int32)
    emb = B.Embedding(10, 8, 5)
    t, i, a = torch.zeros(1, 10, 8, device="cuda"), torch.zeros(1, 5, dtype=torch.int64, device="cuda"), torch.zeros(1, 5, 8, device="cuda")
    calls = [lambda: plan.orthogonalize(h, g), lambda: plan.orthogonalize(g, h), lambda: plan.orthogonalize(bits, g),
             lambda: plan.muon_step(h, g, g, 0.1), lambda: plan.muon_step(g, h, g, 0.1), lambda: plan.muon_step(g, g, h, 0.1),
             lambda: plan.muon_step(g, g, g, 0.1, momentum_out=h), lambda: plan.muon_step(g, g, g, 0.1, weights_out=h),
             lambda: B.Orthogonalizer(4, 6, device="cpu").orthogonalize(g, torch.empty_like(g)),
             lambda: B.Embedding(10, 8, 5, device="cpu").grad(a, i, t)]
    for op in (lambda x, y, z: emb.lookup(x, y, z), lambda x, y, z: emb.grad(z, y, x)):
        calls += [lambda op=op: op(t.cpu(), i, a), lambda op=op: op(t, i.cpu(), a), lambda op=op: op(t, i, a.cpu())]
    for call in calls:
        with pytest.raises(ValueError, match="GPU"):
            call()
    torch.cuda.synchronize()


# ---- pairs of CTAs -------------------------------------------------------------------------------------------------
# Products by pairs of CTAs: float32 and float16 results from a short side of 1600 on, bfloat16 ones and HALF from some
# 1400 (tiles of 256 x 128 and, from 2000 or in batches, 256 x 256).

PAIRS = [(1, 1610, 1700), (1, 2100, 1650), (2, 2048, 2048)]


@pytest.mark.parametrize("shape", PAIRS)
@pytest.mark.parametrize("precision", [B.ORTHO_HALF, B.ORTHO_SINGLE])
def test_float16_results_by_pairs(shape, precision):
    b, r, c = shape
    g = randn(b, r, c, seed=r).half()
    out = torch.empty_like(g)
    plan = B.Orthogonalizer(r, c, batch=b, params=B.ortho_params(precision=precision))
    plan.orthogonalize(g, out)
    plan.check()
    want = direction64(g)
    for e in range(b):
        # entries of some 0.02: subnormal ones lose half of 2^-24 at most
        assert rel(out[e], want[e]) <= bound(precision, F16) + 2.0 ** -25 * (r * c) ** 0.5 / float(want[e].norm())


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("precision", [B.ORTHO_HALF, B.ORTHO_SINGLE])
@pytest.mark.parametrize("shape", [(1700, 1610), (2050, 2303)])
def test_bad_matrices_by_pairs(shape, precision, dtype):
    g = randn(4, *shape, seed=1)
    g[0, -1, -1] = float("nan")
    g[1] = 0
    g[2, 0, 300] = float("inf")
    out = torch.empty(4, *shape, device="cuda", dtype=dtype)
    plan = B.Orthogonalizer(*shape, batch=4, params=B.ortho_params(precision=precision))
    plan.orthogonalize(g, out)
    plan.check()
    assert bool(out[0].isnan().all()) and bool(out[2].isnan().all()) and bool((out[1] == 0).all())
    assert rel(out[3], direction64(g[3:])[0]) <= bound(precision, dtype) + 2.0 ** -25 * 46


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("shape,gap,at", [((1650, 1611), 3, 5), ((2049, 2110), 1, 1), ((2304, 2048), 7, 3)])
def test_odd_strides_by_pairs(shape, gap, at, dtype):
    (r, c), b = shape, 2
    ld = c + gap
    st = ld * (r + 2) + 1
    flat = randn(b * st + 16, seed=5).to(dtype)
    g = flat.as_strided((b, r, c), (st, ld, 1), at)
    store = torch.full((b * st + 16,), 9.0, device="cuda", dtype=dtype)
    out = store.as_strided((b, r, c), (st, ld, 1), at + 2)
    B.Orthogonalizer(r, c, batch=b).orthogonalize(g, out)
    want = direction64(g)
    assert rel(out, want) <= bound(AUTO[dtype], dtype) + 2.0 ** -25 * 46
    out.fill_(9.0)
    assert bool((store == 9.0).all())


@pytest.mark.parametrize("tw", [F32, BF16, F16])
@pytest.mark.parametrize("shape,offset", [((2, 1611, 1700), 45), ((1, 2111, 2050), 7)])
def test_muon_step_from_packed_bits_by_pairs(shape, offset, tw):
    n = shape[0] * shape[1] * shape[2]
    words = torch.randint(-2 ** 31, 2 ** 31, ((offset + n + 31) // 32,), device="cuda", generator=gen(1)).int()
    m, w = randn(*shape, seed=2, scale=3.0), randn(*shape, seed=3, scale=0.05).to(tw)
    want_m, want_w, step = muon64(signs(words, offset, shape), m, w, 0.03, 0.9, False, 0.1, 1.5)
    plan = B.Orthogonalizer(shape[1], shape[2], batch=shape[0])
    plan.muon_step(words, m, w, 0.03, beta=0.9, nesterov=False, weight_decay=0.1, scale=1.5, bit_offset=offset)
    plan.check()
    assert rel(m, want_m) <= 2 ** -23
    limit = TOL[AUTO[tw]] * step.norm() + (4 * U[F32] + U[tw]) * (want_w.norm() + step.norm()) + 2.0 ** -25 * n ** 0.5
    assert float((w.double() - want_w).norm()) <= float(limit)


@pytest.mark.parametrize("n,shape,at,gap", [(7, (60, 70), 3, 77), (5, (300, 200), 0, 64), (12, (1700, 130), 1, 5),
                                            (4, (1620, 1700), 13, 3), (6, (120, 1500), 2, 2)])
@pytest.mark.parametrize("tw", [F32, BF16])
def test_many_replicas(n, shape, at, gap, tw):
    # weights are rows of clients' parameter vectors, from odd elements on; what lies between them stays
    r, c = shape
    ld = r * c + gap + at
    rows = randn(n, ld, seed=11).to(tw)
    before = rows.clone()
    w, w0 = rows.as_strided((n, 1, r, c), (ld, r * c, c, 1), at), before.as_strided((n, 1, r, c), (ld, r * c, c, 1), at)
    m, g = randn(1, r, c, seed=12), randn(1, r, c, seed=13)
    _, want, step = muon64(g, m, w0, 0.02, 0.95, True, 0.01, 0.3)
    plan = B.Orthogonalizer(r, c)
    other = torch.empty(n, 1, r, c, device="cuda", dtype=tw)
    plan.muon_step(g, m.clone(), w, 0.02, weight_decay=0.01, scale=0.3, weights_out=other)
    assert torch.equal(rows, before)
    plan.muon_step(g, m, w, 0.02, weight_decay=0.01, scale=0.3)
    plan.check()
    assert torch.equal(w, other)
    for k in range(n):
        limit = TOL[AUTO[tw]] * step.norm() + (4 * U[F32] + U[tw]) * (want[k].norm() + step.norm())
        assert float((w[k].double() - want[k]).norm()) <= float(limit)
    w.zero_()
    w0.zero_()
    assert torch.equal(rows, before)
