"""Cases, plain forms and 64-bit values of the operators inside a client's local step and before the ring.

Three kinds, in the order in which a round of a federated language model uses them:

* ``norm`` and ``norm_grad``  layer norm of all clients' activations with each client's own weights (pieces of its row
  of the weights), and its gradients, those of the weights written into the client's row of updates;
* ``attn`` and ``attn_grad``  causal attention with a sliding window and a few first tokens that stay visible, and its
  gradients;
* ``clip``  every client's gradient norm over all of its tensors, and the gradients clipped into the update matrix.

``own`` chooses between the plain form in elementary torch operations and the library's calls.
"""

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}

EPS = 1e-5        # of the layer norm
CLIP_EPS = 1e-6   # of the clipping


def listed():
    return [
        # a short text through one small layer: latency counts
        dict(name="norm_small", op="norm", clients=1, rows=33, dim=64, type="f32", out="f32"),
        # the local batches of 16 clients, float32 residual stream, bf16 into the layer's matrices
        dict(name="norm_batch", op="norm", clients=16, rows=8192, dim=768, type="f32", out="bf16"),
        # odd everywhere: rows that start at any address, weights at an odd coordinate of the client's row
        dict(name="norm_grad_odd", op="norm_grad", clients=3, rows=5001, dim=333, type="f32", out="f32"),
        # backward of 16 clients' batches in bf16, the weights' gradients into 16 rows of updates
        dict(name="norm_grad_batch", op="norm_grad", clients=16, rows=8192, dim=768, type="bf16", out="bf16"),
        # a short text, float32, four heads, window longer than the text
        dict(name="attn_short", op="attn", batch=1, tokens=33, heads=4, kv_heads=4, dim=16, window=64, sinks=1,
             ragged=False, type="f32"),
        # one long text: 12 heads of 64, a window of an eighth of it and 4 sinks
        dict(name="attn_long", op="attn", batch=1, tokens=8192, heads=12, kv_heads=12, dim=64, window=1024, sinks=4,
             ragged=False, type="bf16"),
        # a padded batch of texts, shared key and value heads, short window
        dict(name="attn_shared", op="attn", batch=16, tokens=1000, heads=8, kv_heads=2, dim=128, window=256, sinks=16,
             ragged=True, type="f16"),
        # backward of a small padded batch in float32, no size a multiple of anything
        dict(name="attn_grad_odd", op="attn_grad", batch=3, tokens=501, heads=6, kv_heads=2, dim=40, window=100,
             sinks=3, ragged=True, type="f32"),
        # backward of a batch of long texts, 16 heads on 4
        dict(name="attn_grad_long", op="attn_grad", batch=4, tokens=4096, heads=16, kv_heads=4, dim=128, window=1024,
             sinks=4, ragged=False, type="bf16"),
        # one client's small model: a byte-level table and one layer, nine tensors
        dict(name="clip_small", op="clip", clients=1, vocab=256, dim=64, layers=1, type="f32", out="f32", clip=True),
        # the update matrix as the ring takes it, one row of 11,689,512 coordinates for each of 50 clients
        dict(name="clip_rows", op="clip", clients=50, vocab=11689512, dim=1, layers=0, type="f32", out="f32", clip=True),
        # the gradients of 8 clients' models as the backward pass leaves them: 41 bf16 tensors each, into the rows
        dict(name="clip_model", op="clip", clients=8, vocab=50000, dim=768, layers=5, type="bf16", out="f32", clip=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm_grad", "attn", "attn_grad", "clip"])
    types = ["f32", "bf16", "f16"]
    if kind in ("norm", "norm_grad"):
        while True:
            case = dict(op=kind, clients=rng.choice([1, 1, _log(rng, 2, 16)]), rows=_log(rng, 1, 32768),
                        dim=_log(rng, 1, 16384) if rng.random() < 0.5 else 8 * _log(rng, 1, 1024),
                        type=rng.choice(types), out=rng.choice(types))
            if case["clients"] * case["rows"] * case["dim"] <= 16 * 8192 * 768:
                return case
    if kind == "clip":
        while True:
            case = dict(op="clip", clients=_log(rng, 1, 50), vocab=_log(rng, 1, 4000000), dim=_log(rng, 1, 1024),
                        layers=rng.choice([0, 1, rng.randint(2, 24)]), type=rng.choice(types), out=rng.choice(types),
                        clip=rng.random() < 0.8)
            if case["clients"] * _coordinates(case) <= 400e6:
                return case
    top = work(dict(op="attn_grad", batch=4, tokens=4096, heads=16, kv_heads=4, dim=128, window=1024, sinks=4,
                    ragged=False, type="bf16"))["flops"]
    while True:
        kv = _log(rng, 1, 16)
        tokens = _log(rng, 1 if kind == "attn" else 16, 8192)
        case = dict(op=kind, batch=rng.choice([1, 1, _log(rng, 2, 32)]), tokens=tokens,
                    heads=kv * rng.choice([1, 1, 2, 3, 4, 8]), kv_heads=kv,
                    dim=rng.choice([16, 32, 64, 64, 128, 128, 8 * rng.randint(1, 16), rng.randint(1, 128)]),
                    window=rng.choice([_log(rng, 1, 2 * tokens), max(1, tokens // 8)]),
                    sinks=rng.choice([0, 1, 4, _log(rng, 1, 128)]), ragged=rng.random() < 0.4, type=rng.choice(types))
        if kind == "attn_grad" and case["window"] + case["sinks"] < 2:
            continue        # a token that sees itself alone has no gradient but its value's
        # the plain form holds every pair of tokens
        if work(case)["flops"] <= top and case["batch"] * case["heads"] * tokens * tokens <= 1.08e9:
            return case


def _lengths(case, turn=0):
    """Tokens of each sequence: all of them, or between half and all; another seed turns them round."""
    n, b = case["tokens"], case["batch"]
    full = [n - (i * 37 + 11) % (n // 2 + 1) if case["ragged"] and i else n for i in range(b)]
    return full[turn % b:] + full[:turn % b]


def _shapes(case):
    """The tensors of a client's model: the table, and for each layer two vectors, four square matrices, two wide ones."""
    d = case["dim"]
    return [(case["vocab"], d)] + case["layers"] * [(d,), (d,), (d, d), (d, d), (d, d), (d, d), (2 * d, d), (d, 2 * d)]


def _coordinates(case):
    return sum(math.prod(s) for s in _shapes(case))


def work(case):
    """Bytes of each input once and each output once, operations on the pairs of tokens that see each other."""
    if case["op"] in ("norm", "norm_grad"):
        rows = case["clients"] * case["rows"]
        n, vectors = rows * case["dim"], case["clients"] * case["dim"] * 4
        if case["op"] == "norm":
            return {"bytes": n * (SIZE[case["type"]] + SIZE[case["out"]]) + 2 * vectors + 8 * rows, "flops": 8 * n}
        return {"bytes": n * (2 * SIZE[case["type"]] + SIZE[case["out"]]) + 3 * vectors + 8 * rows, "flops": 14 * n}
    if case["op"] == "clip":
        n = case["clients"] * _coordinates(case)
        return {"bytes": n * (SIZE[case["type"]] + (SIZE[case["out"]] if case["clip"] else 0)) + 4 * case["clients"],
                "flops": 3 * n if case["clip"] else 2 * n}
    lengths, w = _lengths(case), case["window"]
    pairs = 0
    for n in lengths:
        m = min(n, w)
        pairs += m * (m + 1) // 2 + (n - m) * w                        # the window
        k = min(case["sinks"], n - m)
        pairs += k * (k + 1) // 2 + (n - m - k) * k                    # sinks behind it
    dim, size = case["dim"], SIZE[case["type"]]
    q, k = sum(lengths) * case["heads"], sum(lengths) * case["kv_heads"]
    if case["op"] == "attn":
        return {"bytes": 2 * (q + k) * dim * size + 4 * q, "flops": 4 * pairs * case["heads"] * dim}
    return {"bytes": 4 * (q + k) * dim * size + 4 * q, "flops": 10 * pairs * case["heads"] * dim}


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000003 + 29)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, device="cuda", generator=g)


def prepare(case, seed):
    g = _gen(seed)
    s = {"case": case}
    if case["op"] in ("norm", "norm_grad"):
        _prepare_norm(s, case, g)
    elif case["op"] == "clip":
        _prepare_clip(s, case, g)
    else:
        _prepare_attention(s, case, g, seed)
    return s


def _prepare_norm(s, case, g):
    c, n, d = case["clients"], case["rows"], case["dim"]
    # activations: every row with a level and a spread of its own, a few coordinates much larger than the others
    x = _randn(g, c, n, d) * (0.5 + torch.rand(c, n, 1, device="cuda", generator=g))
    x += 0.3 * _randn(g, c, n, 1)
    x *= torch.where(torch.rand(d, device="cuda", generator=g) < 0.01, 6.0, 1.0)
    s["x"] = x.to(TYPES[case["type"]])
    # weight and bias lie one after the other in the client's row of weights
    ld = (77 + 2 * d + 127) // 128 * 128
    rows = _randn(g, c, ld) * 0.1
    s["weight"], s["bias"] = rows[:, 77:77 + d], rows[:, 77 + d:77 + 2 * d]
    s["weight"] += 1
    if case["op"] == "norm":
        s["y"] = torch.empty(c, n, d, dtype=TYPES[case["out"]], device="cuda")
        s["mean"], s["rstd"] = (torch.empty(c, n, device="cuda") for _ in range(2))
    else:
        x = s["x"].double()
        s["mean"] = x.mean(-1).float()
        s["rstd"] = (x.var(-1, correction=0) + EPS).rsqrt().float()
        s["dy"] = (_randn(g, c, n, d) * 1e-2).to(TYPES[case["out"]])
        s["dx"] = torch.empty_like(s["x"])
        updates = torch.zeros(c, ld, device="cuda")
        s["dweight"], s["dbias"] = updates[:, 77:77 + d], updates[:, 77 + d:77 + 2 * d]
    if own:
        from paper_2501_17392_b200 import brace

        s["plan"] = brace.LayerNorm(d, n, clients=c, eps=EPS, grad=case["op"] == "norm_grad")


def _prepare_clip(s, case, g):
    c, d = case["clients"], _coordinates(case)
    # clients' gradients differ in size; the last one, a Byzantine client, sends ten times its own
    size = 1e-3 * 4 ** (2 * torch.rand(c, device="cuda", generator=g) - 1)
    size[-1] *= -10
    ld = (d + 127) // 128 * 128
    s["updates"] = torch.zeros(c, ld, dtype=TYPES[case["out"]], device="cuda")
    s["tensors"], s["pieces"], at = [], [], 0
    for shape in _shapes(case):
        n = math.prod(shape)
        lead = ld if not case["layers"] else n          # one tensor alone is the clients' rows themselves
        x = _randn(g, c, lead).mul_(size[:, None]).to(TYPES[case["type"]])
        s["tensors"].append(x.as_strided((c, *shape), (lead, *torch.empty(shape, device="meta").stride())))
        s["pieces"].append(s["updates"].as_strided((c, *shape), (ld, *s["tensors"][-1].stride()[1:]), at))
        at += n
    s["max_norm"] = 1e-3 * math.sqrt(d)
    s["norms"] = torch.empty(c, device="cuda")
    if own:
        from paper_2501_17392_b200 import brace

        s["plan"] = brace.GradientClip(s["tensors"], s["pieces"])


def _prepare_attention(s, case, g, seed):
    b, n, h, k, d = (case[x] for x in ("batch", "tokens", "heads", "kv_heads", "dim"))
    dtype = TYPES[case["type"]]
    # queries, keys and values as one projection leaves them, side by side in a token's row
    qkv = _randn(g, b, n, h + 2 * k, d)
    qkv[:, :, :h] *= 1.5
    qkv = qkv.to(dtype)
    s["q"], s["k"], s["v"] = qkv[:, :, :h], qkv[:, :, h:h + k], qkv[:, :, h + k:]
    s["scale"] = 1 / math.sqrt(d)
    s["lengths"] = torch.tensor(_lengths(case, seed), dtype=torch.int32, device="cuda") if case["ragged"] else None
    if case["op"] == "attn":
        s["out"] = torch.empty(b, n, h, d, dtype=dtype, device="cuda")
        s["lse"] = torch.empty(b, h, n, device="cuda")
    else:
        s["out"], s["lse"] = _plain_attn(s, case).values()
        s["dout"] = (_randn(g, b, n, h, d) * 1e-2).to(dtype)
        grads = torch.empty_like(qkv)
        s["dq"], s["dk"], s["dv"] = grads[:, :, :h], grads[:, :, h:h + k], grads[:, :, h + k:]
    if own:
        from paper_2501_17392_b200 import brace

        s["plan"] = brace.WindowAttention(h, d, n, batch=b, kv_heads=k, window=case["window"], sinks=case["sinks"],
                                          grad=case["op"] == "attn_grad")


def run(s):
    case = s["case"]
    return (_own if own else _plain)[case["op"]](s, case)


# ---- the plain forms: elementary torch operations in 32 bits, rounded once at the end


def _plain_norm(s, case):
    x = s["x"].float()
    mean = x.sum(-1, keepdim=True) / case["dim"]
    x = x - mean
    rstd = 1 / ((x * x).sum(-1, keepdim=True) / case["dim"] + EPS).sqrt()
    y = x * rstd * s["weight"][:, None] + s["bias"][:, None]
    return {"y": y.to(TYPES[case["out"]]), "mean": mean[..., 0], "rstd": rstd[..., 0]}


def _plain_norm_grad(s, case):
    dy, rstd = s["dy"].float(), s["rstd"][..., None]
    xh = (s["x"].float() - s["mean"][..., None]) * rstd
    g = dy * s["weight"][:, None]
    dx = rstd * (g - g.sum(-1, keepdim=True) / case["dim"] - xh * ((g * xh).sum(-1, keepdim=True) / case["dim"]))
    return {"dx": dx.to(TYPES[case["type"]]), "dweight": (dy * xh).sum(1), "dbias": dy.sum(1)}


def _sees(case, device):
    """Which of its tokens each token sees."""
    i = torch.arange(case["tokens"], device=device)
    back = i[:, None] - i
    return (back >= 0) & ((back < case["window"]) | (i < case["sinks"]))


def _scores(s, case):
    """[batch, kv head, heads of it, query, key], -inf where the key is not seen."""
    b, n, k, d = (case[x] for x in ("batch", "tokens", "kv_heads", "dim"))
    q = s["q"].float().reshape(b, n, k, -1, d).permute(0, 2, 3, 1, 4)
    keys = s["k"].float().permute(0, 2, 3, 1)[:, :, None]
    sees = _sees(case, q.device)[None]
    if s["lengths"] is not None:
        here = torch.arange(n, device=q.device) < s["lengths"][:, None]
        sees = sees & here[:, None, :] & here[:, :, None]
    return q, (q @ keys * s["scale"]).masked_fill_(~sees[:, None, None], -math.inf)


def _as_tokens(x, case):
    """[batch, kv head, heads of it, token, dim] as [batch, token, head, dim]."""
    return x.permute(0, 3, 1, 2, 4).reshape(case["batch"], case["tokens"], -1, case["dim"])


def _plain_attn(s, case):
    score = _scores(s, case)[1]
    top = score.amax(-1, keepdim=True).clamp_min(-3e38)      # of a row behind the sequence's end too
    p = (score - top).exp()
    total = p.sum(-1, keepdim=True)
    v = s["v"].float().permute(0, 2, 1, 3)[:, :, None]
    out = p @ v / torch.where(total > 0, total, 1.0)
    lse = (top + total.log())[..., 0].flatten(1, 2)
    return {"out": _as_tokens(out, case).to(TYPES[case["type"]]), "lse": lse}


def _plain_attn_grad(s, case):
    b, n, h, k, d = (case[x] for x in ("batch", "tokens", "heads", "kv_heads", "dim"))
    q, score = _scores(s, case)
    lse = s["lse"].view(b, k, h // k, n, 1)
    p = (score - torch.where(lse > -math.inf, lse, 0.0)).exp()
    dout = s["dout"].float().reshape(b, n, k, -1, d).permute(0, 2, 3, 1, 4)
    dv = (p.mT @ dout).sum(2)
    ds = dout @ s["v"].float().permute(0, 2, 3, 1)[:, :, None]
    ds = p * (ds - (p * ds).sum(-1, keepdim=True)) * s["scale"]
    dq = ds @ s["k"].float().permute(0, 2, 1, 3)[:, :, None]
    dk = (ds.mT @ q).sum(2)
    return {"dq": _as_tokens(dq, case).to(s["q"].dtype), "dk": dk.transpose(1, 2).to(s["q"].dtype),
            "dv": dv.transpose(1, 2).to(s["q"].dtype)}


def _plain_clip(s, case):
    total = torch.zeros(case["clients"], dtype=torch.float64, device="cuda")
    for x in s["tensors"]:      # as many as the model has
        x = x.flatten(1).float()
        total += (x * x).sum(1, dtype=torch.float64)
    norms = total.sqrt().float()
    if not case["clip"]:
        return norms
    factor = (s["max_norm"] / (norms + CLIP_EPS)).clamp(max=1.0)
    for x, piece in zip(s["tensors"], s["pieces"]):
        piece.copy_(x.float() * factor.view(-1, *[1] * (x.dim() - 1)))
    return {"norms": norms, "updates": s["updates"]}


_plain = {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "attn": _plain_attn, "attn_grad": _plain_attn_grad,
          "clip": _plain_clip}


# ---- the library's calls


def _own_norm(s, case):
    s["plan"].forward(s["x"], s["y"], weight=s["weight"], bias=s["bias"], mean=s["mean"], rstd=s["rstd"])
    return {x: s[x] for x in ("y", "mean", "rstd")}


def _own_norm_grad(s, case):
    s["plan"].grad(s["dy"], s["x"], s["mean"], s["rstd"], s["dx"], weight=s["weight"], dweight=s["dweight"],
                   dbias=s["dbias"])
    return {x: s[x] for x in ("dx", "dweight", "dbias")}


def _own_attn(s, case):
    s["plan"].forward(s["q"], s["k"], s["v"], s["out"], lse=s["lse"], lengths=s["lengths"])
    return {x: s[x] for x in ("out", "lse")}


def _own_attn_grad(s, case):
    s["plan"].grad(s["dout"], s["q"], s["k"], s["v"], s["out"], s["lse"], s["dq"], s["dk"], s["dv"],
                   lengths=s["lengths"])
    return {x: s[x] for x in ("dq", "dk", "dv")}


def _own_clip(s, case):
    if not case["clip"]:
        s["plan"].norms(s["norms"])
        return s["norms"]
    s["plan"].clip(s["max_norm"], norms=s["norms"], eps=CLIP_EPS)
    return {"norms": s["norms"], "updates": s["updates"]}


_own = {"norm": _own_norm, "norm_grad": _own_norm_grad, "attn": _own_attn, "attn_grad": _own_attn_grad,
        "clip": _own_clip}


# ---- the definitions in 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "clip":
        total = sum(torch.linalg.vector_norm(x.flatten(1), dim=1, dtype=torch.float64) ** 2 for x in s["tensors"])
        if not case["clip"]:
            return total ** 0.5
        factor = torch.minimum(torch.ones_like(total), s["max_norm"] / (total ** 0.5 + CLIP_EPS))
        updates = torch.zeros(s["updates"].shape, dtype=torch.float64, device="cuda")
        at = 0
        for x in s["tensors"]:
            n = x[0].numel()
            torch.mul(x.flatten(1), factor[:, None], out=updates[:, at:at + n])
            at += n
        return {"norms": total ** 0.5, "updates": updates}
    if case["op"] in ("norm", "norm_grad"):
        return _exact_norm(s, case)
    return _exact_attention(s, case)


def _exact_norm(s, case):
    x = s["x"].double().requires_grad_(case["op"] == "norm_grad")
    weight, bias = (s[k].double().requires_grad_(case["op"] == "norm_grad") for k in ("weight", "bias"))
    var, mean = torch.var_mean(x, -1, correction=0, keepdim=True)
    y = torch.addcmul(bias[:, None], (x - mean) / (var + EPS) ** 0.5, weight[:, None])
    if case["op"] == "norm":
        return {"y": y, "mean": mean[..., 0], "rstd": (var + EPS)[..., 0] ** -0.5}
    dx, dweight, dbias = torch.autograd.grad(y, (x, weight, bias), s["dy"].double())
    return {"dx": dx, "dweight": dweight, "dbias": dbias}


def _exact_attention(s, case):
    """Sequence by sequence and head by head: the softmax over the keys seen, its gradients by differentiation."""
    grad = case["op"] == "attn_grad"
    q, k, v = (s[x].double().requires_grad_(grad) for x in ("q", "k", "v"))
    got = {x: torch.zeros(s[x].shape, dtype=torch.float64, device="cuda") for x in (("dq", "dk", "dv") if grad else ("out", "lse"))}
    if not grad:
        got["lse"] -= math.inf
    share = case["heads"] // case["kv_heads"]
    for b in range(case["batch"]):
        n = case["tokens"] if s["lengths"] is None else int(s["lengths"][b])
        hidden = ~_sees({**case, "tokens": n}, q.device)
        for h in range(case["heads"]):
            one = [t[b, :n, at].detach().requires_grad_(grad) for t, at in ((q, h), (k, h // share), (v, h // share))]
            score = torch.masked_fill(torch.einsum("id,jd->ij", one[0], one[1]) * s["scale"], hidden, -math.inf)
            out = torch.softmax(score, -1) @ one[2]
            if grad:
                dq, dk, dv = torch.autograd.grad(out, one, s["dout"][b, :n, h].double())
                got["dq"][b, :n, h] = dq
                got["dk"][b, :n, h // share] += dk
                got["dv"][b, :n, h // share] += dv
            else:
                got["out"][b, :n, h] = out
                got["lse"][b, h, :n] = torch.logsumexp(score, -1)
    return got
