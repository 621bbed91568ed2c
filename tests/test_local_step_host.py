"""Argument checks of the operators of a client's local step and of their binding.  Nothing is launched here: every call
below is refused, or has nothing to do, before the library touches a GPU."""

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


# ---- layer norm

def norm(grad=False, ws=P, nbytes=1 << 40, **over):
    e = B.LayerNormArgs()
    for k, t in B.LayerNormArgs._fields_:
        setattr(e, k, P if t is C.c_void_p else 64 if k.startswith("stride") else 8 if k.startswith("ld_") else 0)
    e.clients, e.dim, e.rows, e.eps = 2, 8, 4, 1e-5
    for k, v in over.items():
        setattr(e, k, v)
    if grad:
        return B.lib().brace_layer_norm_grad(e, ws, nbytes, None)
    return B.lib().brace_layer_norm_forward(e, None)


def test_norm_refuses():
    common = [dict(clients=-1), dict(clients=70000), dict(rows=-1), dict(rows=1 << 31), dict(dim=0), dict(dim=-5),
              dict(x_type=3), dict(y_type=-1), dict(weight_type=4), dict(d_x=None), dict(d_y=None), dict(d_x=P + 2),
              dict(y_type=1, d_y=P + 1), dict(d_weight=P + 1), dict(ld_x=7), dict(ld_y=7)]
    for bad in common + [dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(ld_y=0),
                         dict(d_bias=P + 2), dict(d_mean=P + 1), dict(stride_y=0), dict(stride_stats=3)]:
        assert norm(**bad) == BAD, bad
    for bad in common + [dict(d_mean=None), dict(d_rstd=None), dict(d_dx=None), dict(ld_dx=7), dict(ld_dx=0),
                         dict(grad_type=3), dict(d_dweight=P + 2), dict(d_dbias=P + 1), dict(stride_dx=0),
                         dict(stride_dweight=0), dict(stride_dbias=0)]:
        assert norm(True, **bad) == BAD, bad
    assert norm(dim=(1 << 22) + 1, ld_x=1 << 23, ld_y=1 << 23) == UNSUPPORTED
    assert norm(True, ws=None) == norm(True, nbytes=0) == norm(True, ws=P + 128) == WORKSPACE
    assert norm(clients=0) == norm(rows=0) == norm(True, clients=0) == norm(True, rows=0, accumulate=1) == B.OK
    assert B.lib().brace_layer_norm_forward(None, None) == B.lib().brace_layer_norm_grad(None, P, 1, None) == BAD


def test_norm_workspace():
    f = B.lib().brace_layer_norm_workspace_bytes
    assert f(-1, 1, 1) == f(1, -1, 1) == f(1, 1, 0) == f(70000, 1, 1) == f(1, 1 << 31, 1) == f(1, 1, (1 << 22) + 1) == 0
    assert f(0, 0, 1) >= 256
    for d in (1, 64, 333, 768, 8192, 10000):
        sizes = [f(3, n, d) for n in (0, 1, 10, 100, 1000, 10000, 100000)]
        assert sizes == sorted(sizes)        # one for many rows serves fewer


def test_norm_binding_refuses():
    p = B.LayerNorm(8, 4, clients=2, device="cpu")
    x, v, s = torch.zeros(2, 4, 8), torch.zeros(2, 8), torch.zeros(2, 4)
    for args in [(x[:, :, :7], x), (x, x[:1]), (x.double(), x), (x, x.long()), (torch.zeros(2, 5, 8), torch.zeros(2, 5, 8)),
                 (x.mT.contiguous().mT, x), (x[0, 0], x[0, 0])]:
        with pytest.raises(ValueError):
            p.forward(*args)
    for kw in [dict(weight=v[:, :7]), dict(weight=v.double()), dict(weight=v, bias=v.half()), dict(mean=s.half()),
               dict(mean=s[:, :3]), dict(mean=s, rstd=torch.zeros(2, 8)[:, :4]), dict(mean=s.mT.contiguous().mT)]:
        with pytest.raises(ValueError):
            p.forward(x, x, **kw)
    for kw in [dict(dweight=v[0]), dict(dbias=v[:1]), dict(dweight=v, dbias=v.half())]:
        with pytest.raises(ValueError):
            p.grad(x, x, s, s, x, **kw)
    with pytest.raises(ValueError):
        p.grad(x, x, s, s, x.half())
    with pytest.raises(ValueError):      # the host's memory
        p.forward(x, x)
    with pytest.raises(B.BraceError):
        B.LayerNorm(8, 4, clients=2, grad=False, device="cpu").grad(x, x, s, s, x)


# ---- clipping

def tensor(**over):
    t = B.TensorArgs(P, P + 4096, 2, 8, 8, 64, 8, 64, 0, 0)
    for k, v in over.items():
        setattr(t, k, v)
    return t


def clip(*tensors, clients=2, max_norm=1.0, eps=1e-6, nonfinite=0, norms=P, ws=P, nbytes=1 << 40, count=None):
    a = (B.TensorArgs * max(len(tensors), 1))(*tensors)
    return B.lib().brace_gradient_clip(clients, a, len(tensors) if count is None else count, max_norm, eps, nonfinite,
                                       norms, ws, nbytes, None)


def gradient_norm(*tensors, clients=2, norms=P, ws=P, nbytes=1 << 40):
    return B.lib().brace_gradient_norm(clients, (B.TensorArgs * len(tensors))(*tensors), len(tensors), norms, ws, nbytes, None)


def test_clip_refuses():
    for bad in [dict(rows=-1), dict(cols=-1), dict(in_type=3), dict(d_in=None), dict(d_in=P + 2), dict(ld_in=7)]:
        assert clip(tensor(**bad)) == gradient_norm(tensor(**bad)) == BAD, bad
    for bad in [dict(out_type=-1), dict(d_out=None), dict(d_out=P + 1), dict(ld_out=7), dict(stride_out=0),
                dict(d_out=P, out_type=1), dict(d_out=P, ld_out=9), dict(d_out=P, stride_out=128)]:
        assert clip(tensor(**bad)) == BAD, bad
    for bad in [dict(clients=-1), dict(max_norm=-1.0), dict(max_norm=float("nan")), dict(max_norm=float("inf")),
                dict(eps=-1e-6), dict(eps=float("nan")), dict(nonfinite=2), dict(nonfinite=-1), dict(norms=P + 2),
                dict(count=-1)]:
        assert clip(tensor(), **bad) == BAD, bad
    assert clip(tensor(), tensor(cols=1 << 45, ld_in=1 << 45, ld_out=1 << 45, rows=4)) == UNSUPPORTED
    assert clip(tensor(), ws=None) == clip(tensor(), nbytes=8) == clip(tensor(), ws=P + 64) == WORKSPACE
    assert gradient_norm(tensor(), norms=None) == BAD and gradient_norm(tensor(), ws=None) == WORKSPACE
    assert clip(tensor(), clients=0) == gradient_norm(tensor(), clients=0) == B.OK
    assert B.lib().brace_gradient_clip(1, None, 3, 1.0, 0.0, 0, P, P, 1 << 40, None) == BAD


@pytest.mark.parametrize("count", [2, 341, 1000])
def test_clip_refuses_two_tensors_of_one_place(count):
    """Both would be clipped there, in no order.  Empty tensors are written nowhere."""
    apart = [tensor(d_in=P + 4096 * i, d_out=P + 4096 * i) for i in range(count)]
    assert clip(*apart, apart[0], nbytes=8) == BAD
    assert gradient_norm(*apart, apart[0], nbytes=8) == WORKSPACE
    assert clip(*apart, tensor(rows=0, d_out=P), nbytes=8) == WORKSPACE


def test_clip_workspace():
    f = B.lib().brace_clip_workspace_bytes
    one = (B.TensorArgs * 1)(tensor())
    assert f(2, one, 1) > 0 and f(-1, one, 1) == f(2, one, -1) == f(2, None, 1) == 0
    assert f(2, (B.TensorArgs * 1)(tensor(rows=-1)), 1) == f(2, (B.TensorArgs * 1)(tensor(in_type=7)), 1) == 0
    assert f(2, (B.TensorArgs * 1)(tensor(rows=1 << 40, cols=1 << 40)), 1) == 0


def test_clip_binding_refuses():
    x = torch.zeros(2, 4, 6)
    for args in [([],), ([x], [x, x]), ([x, x[:1]],), ([x], [x[:, :3]]), ([x.double()],), ([x.long()],),
                 ([torch.tensor(1.0)],), ([torch.zeros(2, 4, 6, 8)[:, ::2, ::2, ::2]],)]:
        with pytest.raises(ValueError):
            B.GradientClip(*args)
    p = B.GradientClip([x, torch.zeros(2, 0), torch.zeros(2, 6, 4).mT])
    for norms in (torch.zeros(3), torch.zeros(2).half(), torch.zeros(4)[::2]):
        with pytest.raises(ValueError):
            p.norms(norms)
    with pytest.raises(ValueError):      # the host's memory
        p.clip(1.0)


# ---- attention

def attention(grad=False, ws=P, nbytes=1 << 40, **over):
    e = B.WindowAttentionArgs()
    e.batch, e.tokens, e.heads, e.kv_heads, e.dim, e.window, e.sinks, e.type, e.scale = 2, 16, 4, 2, 8, 5, 1, 0, 0.3
    e.d_lse, e.head_lse, e.stride_lse = P, 16, 64
    for name in ("q", "k", "v", "out", "dout", "dq", "dk", "dv"):
        h = getattr(e, name)
        h.d, h.ld, h.head, h.stride = P, 32, 8, 512
    for k, v in over.items():
        if "_" in k and k.split("_")[0] in ("q", "k", "v", "out", "dout", "dq", "dk", "dv"):
            setattr(getattr(e, k.split("_")[0]), k.split("_")[1], v)
        else:
            setattr(e, k, v)
    if grad:
        return B.lib().brace_window_attention_grad(e, ws, nbytes, None)
    return B.lib().brace_window_attention_forward(e, None)


def test_attention_refuses():
    common = [dict(batch=-1), dict(tokens=-1), dict(heads=-1), dict(kv_heads=-1), dict(kv_heads=0), dict(kv_heads=3),
              dict(dim=0), dict(window=0), dict(window=-4), dict(sinks=-1), dict(type=3), dict(type=-1),
              dict(scale=float("nan")), dict(scale=float("inf")), dict(d_lse=P + 2), dict(d_lengths=P + 1),
              dict(head_lse=15), dict(stride_lse=8)]
    common += [{f"{t}_{k}": v} for t in ("q", "k", "v", "out") for k, v in (("d", None), ("d", P + 2), ("ld", -1), ("head", -8), ("stride", -1))]
    for bad in common + [dict(out_ld=7), dict(out_head=0), dict(out_stride=0)]:
        assert attention(**bad) == BAD, bad
    for bad in common + [dict(d_lse=None)] + [{f"{t}_{k}": v} for t in ("dq", "dk", "dv") for k, v in
                                              (("d", None), ("d", P + 1), ("ld", 7), ("head", 0), ("stride", 0), ("ld", -8))]:
        assert attention(True, **bad) == BAD, bad
    assert attention(True, dout_d=None) == attention(True, dout_ld=-1) == BAD
    for kw in (dict(dim=257), dict(batch=70000), dict(heads=70000, kv_heads=70000)):
        assert attention(**kw) == attention(True, **kw) == UNSUPPORTED
    assert attention(True, ws=None) == attention(True, nbytes=16) == attention(True, ws=P + 16) == WORKSPACE
    for kw in (dict(batch=0), dict(tokens=0), dict(heads=0)):
        assert attention(**kw) == attention(True, **kw) == B.OK
    assert B.lib().brace_window_attention_forward(None, None) == B.lib().brace_window_attention_grad(None, P, 1, None) == BAD


def test_attention_workspace():
    f = B.lib().brace_window_attention_workspace_bytes
    assert f(1, 100, 4, 2, 64, 0) > 0 and f(0, 0, 0, 0, 1, 0) >= 256
    for bad in [(-1, 1, 1, 1, 1, 0), (1, -1, 1, 1, 1, 0), (1, 1, -1, 1, 1, 0), (1, 1, 3, 2, 1, 0), (1, 1, 1, 0, 1, 0),
                (1, 1, 1, 1, 0, 0), (1, 1, 1, 1, 1, -1), (1, 1, 1, 1, 257, 0), (70000, 1, 1, 1, 1, 0)]:
        assert f(*bad) == 0, bad
    for kw in (dict(b=1), dict(b=3)):
        sizes = [f(kw["b"], n, 4, 2, 64, 4) for n in (0, 1, 100, 128, 129, 1000, 10000)]
        assert sizes == sorted(sizes)        # one for many tokens serves fewer


def test_attention_binding_refuses():
    p = B.WindowAttention(4, 8, 16, batch=2, kv_heads=2, device="cpu")
    q, k = torch.zeros(2, 16, 4, 8), torch.zeros(2, 16, 2, 8)
    lse = torch.zeros(2, 4, 16)
    for args in [(q[:1], k, k, q), (q, q, k, q), (q, k, k[:, :5], q), (q, k, k, k), (q.double(),) * 4, (q, k.half(), k, q),
                 (q, k, k, q.half()), (torch.zeros(2, 17, 4, 8), k, k, q), (q[..., :7], k, k, q), (q[0], k, k, q),
                 (q.mT.contiguous().mT, k, k, q)]:
        with pytest.raises(ValueError):
            p.forward(*args)
    for kw in [dict(lse=lse.half()), dict(lse=lse[:, :2]), dict(lse=lse.mT.contiguous().mT), dict(lengths=torch.zeros(2)),
               dict(lengths=torch.zeros(3, dtype=torch.int32)), dict(lengths=torch.zeros(4, dtype=torch.int32)[::2])]:
        with pytest.raises(ValueError):
            p.forward(q, k, k, q, **kw)
    with pytest.raises(ValueError):
        p.grad(k, q, k, k, q, lse, q, k, k)
    with pytest.raises(ValueError):      # the host's memory
        p.forward(q, k, k, q, lse=lse)
    with pytest.raises(B.BraceError):
        B.WindowAttention(4, 8, 16, batch=2, kv_heads=2, grad=False, device="cpu").grad(q, q, k, k, q, lse, q, k, k)
