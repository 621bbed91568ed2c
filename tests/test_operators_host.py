"""Argument checks of the language-model operators and of their binding.  Nothing is launched here: every call below is
refused, or has nothing to do, before the library touches a GPU."""

import ctypes as C

import pytest
import torch

from paper_2501_17392_b200 import brace as B
from paper_2501_17392_b200 import build as brace_build

BAD, UNSUPPORTED, WORKSPACE = B.ERR_INVALID_ARG, B.ERR_UNSUPPORTED, B.ERR_WORKSPACE
P = 1 << 20        # an address that is aligned and never read


@pytest.fixture(scope="module", autouse=True)
def _built():
    brace_build.build()


def test_ortho_defaults_and_workspace():
    p = B.ortho_params()
    assert (p.steps, round(p.a, 4), round(p.b, 4), round(p.c, 4), p.precision) == (5, 3.4445, -4.775, 2.0315, 0)
    assert B.lib().brace_ortho_default_params(None) == BAD
    half = B.ortho_workspace_bytes(1, 512, 512, p, B.TYPE_BF16)
    assert 0 < half < B.ortho_workspace_bytes(1, 512, 512, p, B.TYPE_F32) == B.ortho_workspace_bytes(1, 512, 512, p, B.TYPE_F16)
    assert B.ortho_workspace_bytes(0, 4, 4, p) > 0
    for args in [(-1, 4, 4), (1, -4, 4), (1, 4, -4)]:
        assert B.ortho_workspace_bytes(*args, p) == 0
    assert B.ortho_workspace_bytes(1, 4, 4, p, B.TYPE_BITS) == 0
    assert B.ortho_workspace_bytes(40000, 4, 4, p) == 0


def ortho(batch=1, rows=8, cols=8, params=None, g=P, gt=0, ldg=8, sg=64, bit=0, o=P, ot=0, ldo=8, so=64, ws=P, nbytes=1 << 40):
    params = B.ortho_params() if params is None else params
    return B.lib().brace_orthogonalize(batch, rows, cols, params, g, gt, ldg, sg, bit, o, ot, ldo, so, ws, nbytes, None)


def test_orthogonalize_refuses():
    for bad in [dict(batch=-1), dict(rows=-1), dict(cols=-1), dict(g=None), dict(o=None), dict(ldg=7), dict(ldo=7),
                dict(gt=4), dict(gt=-1), dict(ot=3), dict(ot=9), dict(g=P + 2), dict(o=P + 1), dict(gt=1, g=P + 1),
                dict(gt=3, bit=-1)]:
        assert ortho(**bad) == BAD, bad
    assert ortho(ws=None) == WORKSPACE and ortho(nbytes=100) == WORKSPACE and ortho(ws=P + 128) == WORKSPACE
    assert ortho(batch=40000) == UNSUPPORTED
    assert ortho(rows=1 << 20, cols=1 << 20, ldg=1 << 20, ldo=1 << 20) == UNSUPPORTED
    assert ortho(batch=0) == ortho(rows=0) == ortho(cols=0) == B.OK


@pytest.mark.parametrize("over", [dict(steps=0), dict(steps=-3), dict(a=float("nan")), dict(b=float("inf")),
                                  dict(eps=0.0), dict(eps=float("nan")), dict(eps=-1.0), dict(precision=3),
                                  dict(precision=-1), dict(a=5.0, b=0.0, c=0.0), dict(a=2.0, b=0.0, c=0.0),
                                  dict(a=3.0, b=4.0, c=1.0), dict(a=1.0, b=-8.0, c=8.0)])
def test_orthogonalize_refuses_coefficients_that_diverge(over):
    p = B.ortho_params(**over)
    assert ortho(params=p) == BAD and B.ortho_workspace_bytes(1, 8, 8, p) == 0


@pytest.mark.parametrize("over", [dict(), dict(steps=64), dict(a=1.5, b=-0.5, c=0.0), dict(a=1.875, b=-1.25, c=0.375),
                                  dict(a=2.0, b=-1.5, c=0.5), dict(steps=1, a=1.0, b=0.0, c=0.0)])
def test_usual_coefficients_are_accepted(over):
    assert B.ortho_workspace_bytes(1, 8, 8, B.ortho_params(**over)) > 0


def muon(**over):
    s = B.Muon()
    for k, t in B.Muon._fields_:
        setattr(s, k, P if t is C.c_void_p else 64 if k.startswith("stride") else 8 if k.startswith("ld_") else 0)
    s.replicas, s.beta, s.lr, s.scale = 1, 0.9, 0.1, 1.0
    sizes = dict(batch=1, rows=8, cols=8, ws=P, nbytes=1 << 40)
    for k, v in over.items():
        if k in sizes:
            sizes[k] = v
        else:
            setattr(s, k, v)
    return B.lib().brace_muon_step(sizes["batch"], sizes["rows"], sizes["cols"], B.ortho_params(), s, sizes["ws"],
                                   sizes["nbytes"], None)


def test_muon_step_refuses():
    for bad in [dict(batch=-1), dict(d_grad=None), dict(d_momentum=None), dict(d_momentum_out=None), dict(d_weights=None),
                dict(d_weights_out=None), dict(ld_grad=7), dict(ld_momentum=7), dict(ld_momentum_out=7),
                dict(ld_weights=7), dict(ld_weights_out=7), dict(grad_type=7), dict(weights_type=3),
                dict(weights_type=-1), dict(replicas=0), dict(beta=float("nan")), dict(lr=float("inf")),
                dict(weight_decay=float("nan")), dict(scale=float("nan")), dict(d_momentum=P + 2),
                dict(d_weights=P + 2), dict(grad_type=3, bit_offset=-5)]:
        assert muon(**bad) == BAD, bad
    assert B.lib().brace_muon_step(1, 8, 8, B.ortho_params(), None, P, 1 << 40, None) == BAD
    assert muon(ws=None) == WORKSPACE and muon(nbytes=10) == WORKSPACE
    assert muon(rows=0) == B.OK


def test_one_place_is_not_written_for_several():
    # a stride of 0 is a matrix for all: what is read may be that, what is written may not
    assert ortho(batch=2, so=0) == BAD
    assert muon(batch=2, stride_momentum_out=0) == BAD and muon(batch=2, stride_weights_out=0) == BAD
    assert muon(replicas=2, replica_weights=64, replica_weights_out=0) == BAD
    assert muon(replicas=2, replica_weights=64, replica_weights_out=64, ws=None) == WORKSPACE   # past those checks
    assert ortho(so=0, ws=None) == WORKSPACE and ortho(batch=2, sg=0, ws=None) == WORKSPACE
    assert muon(batch=2, stride_grad=0, stride_momentum=0, stride_weights=0, ws=None) == WORKSPACE
    assert muon(replicas=2, replica_weights=0, replica_weights_out=64, ws=None) == WORKSPACE


def embedding(grad, **over):
    e = B.EmbeddingArgs()
    e.clients, e.dim, e.tokens, e.vocab = 2, 8, 5, 10
    e.d_table = e.d_ids = e.d_act = P
    e.ld_table = e.ld_act = 8
    e.stride_table, e.stride_act, e.stride_ids, e.id_bytes, e.scale = 80, 40, 5, 8, 1.0
    ws, nbytes = over.pop("ws", P), over.pop("nbytes", 1 << 40)
    for k, v in over.items():
        setattr(e, k, v)
    return B.lib().brace_embedding_grad(e, ws, nbytes, None) if grad else B.lib().brace_embedding_lookup(e, None)


@pytest.mark.parametrize("grad", [False, True])
def test_embedding_refuses(grad):
    for bad in [dict(clients=-1), dict(clients=70000), dict(dim=0), dict(tokens=-1), dict(tokens=1 << 31), dict(vocab=0),
                dict(vocab=1 << 31), dict(d_table=None), dict(d_ids=None), dict(d_act=None), dict(ld_table=7),
                dict(ld_act=7), dict(table_type=3), dict(act_type=-1), dict(id_bytes=2), dict(scale=float("nan")),
                dict(d_table=P + 2), dict(d_ids=P + 4), dict(act_type=1, d_act=P + 1)]:
        assert embedding(grad, **bad) == BAD, bad
    assert embedding(grad, clients=0) == B.OK
    assert embedding(grad, dim=1 << 23, ld_table=1 << 23, ld_act=1 << 23) == UNSUPPORTED
    # what is written must not be the same place for several clients, what is read may be
    assert embedding(grad, **({"stride_table": 0} if grad else {"stride_act": 0})) == BAD
    if grad:
        assert embedding(True, ws=None) == WORKSPACE and embedding(True, nbytes=8) == WORKSPACE
        assert embedding(True, ws=P + 64) == WORKSPACE
        assert embedding(True, tokens=0, accumulate=1, d_ids=None, d_act=None) == B.OK
        assert B.lib().brace_embedding_grad(None, P, 1 << 40, None) == BAD
    else:
        assert embedding(False, tokens=0) == B.OK
        assert embedding(False, ld_act=0) == BAD
        assert B.lib().brace_embedding_lookup(None, None) == BAD


def test_embedding_workspace():
    f = B.lib().brace_embedding_workspace_bytes
    assert f(2, 5, 10, 8) >= 2 * 10 * 8 and f(0, 0, 1, 1) > 0
    assert f(1, 1, 10, 8) < f(1, 3000, 10, 8) < f(2, 3000, 10, 8)
    for bad in [(-1, 5, 10, 8), (2, -5, 10, 8), (2, 5, 0, 8), (2, 5, 10, 0)]:
        assert f(*bad) == 0
    # a workspace for so many tokens serves any fewer
    edge = 256 * 2048
    sizes = [f(3, t, 5000, 8) for t in (0, 1, 2048, 2049, 4096, 4097, 5000, edge - 1, edge, edge + 1, edge + 2048, 2 * edge,
                                        2 * edge + 1, 10 * edge)]
    assert sizes == sorted(sizes)
    # far past 32 bits
    assert f(16, 1 << 30, 1 << 20, 4096) > 16 * (1 << 30) * 8


def test_binding_checks_shapes_types_and_strides():
    o = B.Orthogonalizer(4, 6, batch=2, device="cpu")
    g = torch.zeros(2, 4, 6)
    for bad in [torch.zeros(2, 6, 4), torch.zeros(4, 6), torch.zeros(2, 4, 6, dtype=torch.float64),
                torch.zeros(2, 6, 4).transpose(1, 2), torch.zeros(1, dtype=torch.int32),
                torch.zeros(2, 8, dtype=torch.int32)]:
        with pytest.raises(ValueError):
            o.orthogonalize(bad, g)
    with pytest.raises(ValueError):
        o.orthogonalize(torch.zeros(2, dtype=torch.int32), g, bit_offset=17)    # 48 bits from there on
    with pytest.raises(ValueError):
        o.orthogonalize(g, torch.zeros(2, 4, 6, dtype=torch.int32))
    with pytest.raises(ValueError):
        o.muon_step(g, g.half(), g, 0.1)
    with pytest.raises(ValueError):
        o.muon_step(g, g, g, 0.1, weights_out=g.half())
    with pytest.raises(ValueError):
        o.muon_step(g, g, torch.zeros(3, 2, 4, 6), 0.1, weights_out=torch.zeros(2, 2, 4, 6))
    e = B.Embedding(10, 8, 5, clients=2, device="cpu")
    table, ids, act = torch.zeros(2, 10, 8), torch.zeros(2, 5, dtype=torch.int64), torch.zeros(2, 5, 8)
    for t, i, a in [(table[:, :9], ids, act), (table[0], ids, act[:, :4]), (table, ids[:, :4], act),
                    (table, ids.float(), act), (table, torch.zeros(2, 6, dtype=torch.int64), torch.zeros(2, 6, 8)),
                    (table.double(), ids, act), (table, ids, act.double()),
                    (table, torch.zeros(5, 2, dtype=torch.int64).t(), act),
                    (torch.zeros(2, 8, 10).transpose(1, 2), ids, act), (table, torch.zeros((), dtype=torch.int64), act)]:
        with pytest.raises(ValueError):
            e.lookup(t, i, a)
    with pytest.raises(ValueError):
        e.grad(act, ids, table[0])          # one gradient for two clients
    with pytest.raises(B.BraceError) as err:
        B.Embedding(10, 8, 5, clients=2, device="cpu", grad=False).grad(act, ids, table, stream=_NoStream())
    assert err.value.status == WORKSPACE


class _NoStream:
    cuda_stream = 0


def test_binding_takes_tensors_of_one_gpu_only():
    # the kernels would read host memory; nothing may get as far as a launch
    o, g = B.Orthogonalizer(4, 6, batch=2, device="cpu"), torch.zeros(2, 4, 6)
    bits = torch.zeros(2, dtype=torch.int32)
    e = B.Embedding(10, 8, 5, clients=2, device="cpu")
    table, ids, act = torch.zeros(2, 10, 8), torch.zeros(2, 5, dtype=torch.int64), torch.zeros(2, 5, 8)
    for call in (lambda: o.orthogonalize(g, g.clone(), stream=_NoStream()), lambda: o.orthogonalize(bits, g, stream=_NoStream()),
                 lambda: o.muon_step(g, g.clone(), g.clone(), 0.1, stream=_NoStream()),
                 lambda: e.lookup(table, ids, act, stream=_NoStream()), lambda: e.grad(act, ids, table, stream=_NoStream())):
        with pytest.raises(ValueError, match="GPU"):
            call()
