"""Cases, plain forms and 64-bit values of the language-model operators beside the aggregation round.

Four operators, in the order in which one training round of a federated language model uses them:

* ``lookup``  rows of a client's embedding table for its tokens, times a scale (start of a local step);
* ``grad``    the gradient of that table, written into the client's row of the update matrix (end of it);
* ``ortho``   an update matrix replaced by its Newton-Schulz orthogonalisation;
* ``muon``    the server side of the round: momentum of the aggregate (floats, or the packed consensus bits
  that the round leaves), orthogonalised, applied to the weights with decoupled weight decay.

``own`` chooses between the plain form in elementary torch operations and the library's calls.
"""

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2, "bits": 0.125}

#: Newton-Schulz: quintic coefficients and steps of the usual orthogonalised-momentum optimiser.
A, B, C, STEPS, EPS = 3.4445, -4.7750, 2.0315, 5, 1e-7
BETA, LR, DECAY = 0.95, 0.02, 0.01
PAD = -1  # a token id that stands for no token


def listed():
    return [
        # one small matrix, as a probe or a head's projection has it: fifteen dependent products, latency counts
        dict(name="ortho_small", op="ortho", batch=1, rows=128, cols=128, type="bf16", out="bf16"),
        # the matrices of a small model's layers at once, no size a multiple of anything, full float32
        dict(name="ortho_ragged", op="ortho", batch=6, rows=257, cols=1001, type="f32", out="f32"),
        # one wide matrix, 1:4
        dict(name="ortho_wide", op="ortho", batch=1, rows=1024, cols=4096, type="bf16", out="bf16"),
        # the largest square matrix of a mid-sized model
        dict(name="ortho_large", op="ortho", batch=1, rows=4096, cols=4096, type="f32", out="bf16"),
        # the round's own output: packed consensus bits of twelve square matrices, float32 weights
        dict(name="muon_bits", op="muon", batch=12, rows=768, cols=768, type="bits", out="f32"),
        # a tall matrix trained in bf16 from a bf16 gradient
        dict(name="muon_tall", op="muon", batch=1, rows=4096, cols=1024, type="bf16", out="bf16"),
        # float32 gradient (the plain-sum round) and float32 weights
        dict(name="muon_f32", op="muon", batch=1, rows=2048, cols=2048, type="f32", out="f32"),
        # one token, as generation asks for it
        dict(name="lookup_one", op="lookup", clients=1, tokens=1, vocab=50000, dim=768, type="f32", out="bf16"),
        # the local batches of 16 clients, each with a table of its own (a row of the weights)
        dict(name="lookup_batch", op="lookup", clients=16, tokens=8192, vocab=50000, dim=768, type="f32", out="bf16"),
        # a short text on a byte-level vocabulary
        dict(name="grad_small", op="grad", clients=1, tokens=33, vocab=256, dim=64, type="f32", out="f32"),
        # odd everywhere: the table starts at an odd coordinate of each client's update
        dict(name="grad_odd", op="grad", clients=3, tokens=5001, vocab=10007, dim=333, type="f32", out="f32"),
        # 16 clients' batches into the 16 rows of the update matrix: mostly rows that no token touches
        dict(name="grad_large", op="grad", clients=16, tokens=8192, vocab=50000, dim=768, type="bf16", out="f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["ortho", "muon", "lookup", "grad"])
    if op in ("ortho", "muon"):
        top = work(dict(op="ortho", batch=1, rows=4096, cols=4096, type="f32", out="bf16"))["flops"]
        while True:
            short = _log(rng, 16, 4096)
            long = min(8192, int(short * rng.choice([1, 1, rng.uniform(1, 2), rng.uniform(2, 8)])))
            batch = rng.choice([1, 1, _log(rng, 2, 24)])
            rows, cols = (short, long) if rng.random() < 0.6 else (long, short)
            kind = rng.choice(["f32", "bf16", "f16"] if op == "ortho" else ["f32", "bf16", "bits"])
            out = rng.choice(["f32", "bf16", "f16"] if op == "ortho" else ["f32", "bf16"])
            case = dict(op=op, batch=batch, rows=rows, cols=cols, type=kind, out=out)
            if 3072 not in (rows, cols) and work(case)["flops"] <= top:
                return case
    while True:
        case = dict(op=op, clients=rng.choice([1, 1, _log(rng, 2, 16)]), tokens=_log(rng, 1, 65536),
                    vocab=_log(rng, 256, 130000), dim=_log(rng, 32, 4096), type=rng.choice(["f32", "bf16", "f16"]),
                    out=rng.choice(["f32", "bf16"]))
        if case["tokens"] * case["clients"] > 131072 or case["dim"] == 3072 or case["vocab"] == 3072:
            continue
        if work(case)["bytes"] <= 2.5e9 and case["clients"] * case["vocab"] * case["dim"] <= 700e6:
            return case


def work(case):
    """Bytes of each input once and each output once; the products' operations with symmetric results counted by half."""
    if case["op"] in ("ortho", "muon"):
        n = case["batch"] * case["rows"] * case["cols"]
        m, k = sorted((case["rows"], case["cols"]))
        flops = case["batch"] * STEPS * (m * (m + 1) * k + m * (m + 1) * m + 2 * m * m * k)
        if case["op"] == "ortho":
            return {"bytes": n * (SIZE[case["type"]] + SIZE[case["out"]]), "flops": flops}
        return {"bytes": n * (SIZE[case["type"]] + 2 * 4 + 2 * SIZE[case["out"]]), "flops": flops}
    rows = case["clients"] * case["tokens"]
    if case["op"] == "lookup":
        # of each client's tokens the distinct ones have to be read: about this many of a log-uniform draw
        seen = case["clients"] * _distinct(case["tokens"], case["vocab"])
        return {"bytes": rows * (8 + case["dim"] * SIZE[case["out"]]) + seen * case["dim"] * SIZE[case["type"]],
                "flops": rows * case["dim"]}
    return {"bytes": rows * (8 + case["dim"] * SIZE[case["type"]]) + case["clients"] * case["vocab"] * case["dim"] * SIZE[case["out"]],
            "flops": rows * case["dim"]}


def _distinct(tokens, vocab):
    """Expected number of distinct ids in `tokens` draws of id = floor(vocab ** u), u uniform."""
    span, cells = math.log(vocab), 400
    got = 0.0
    for i in range(cells):  # ids in cells of equal probability
        lo, hi = vocab ** (i / cells), vocab ** ((i + 1) / cells)
        ids = max(hi - lo, 1e-9)
        p = 1 / cells / max(ids, 1)
        got += max(ids, 1) * -math.expm1(tokens * math.log1p(-min(p, 0.999999))) if ids >= 1 else ids
    return min(got, tokens, vocab) if span > 0 else 1


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000003 + 17)
    return g


def _update(case, g):
    """An update as training gives it: a few strong directions over noise of full rank."""
    b, r, c = case["batch"], case["rows"], case["cols"]
    k = max(1, min(16, r, c))
    u = torch.randn(b, r, k, device="cuda", generator=g)
    v = torch.randn(b, k, c, device="cuda", generator=g)
    x = torch.randn(b, r, c, device="cuda", generator=g)
    return x.add_(u @ v, alpha=0.3).mul_(1e-3)


def _tokens(case, g):
    """Token ids with a Zipf-like tail in an order that is not their frequency's; about one in forty is padding."""
    u = torch.rand(case["clients"], case["tokens"], device="cuda", generator=g, dtype=torch.float64)
    rank = (case["vocab"] ** u).long().sub_(1).clamp_(0, case["vocab"] - 1)
    ids = torch.randperm(case["vocab"], device="cuda", generator=g)[rank]
    pad = torch.rand(ids.shape, device="cuda", generator=g) < 0.025
    return torch.where(pad & (case["tokens"] > 1), PAD, ids)


def _scale(case):
    """The usual factor of an orthogonalised step: sqrt(max(1, rows / cols))."""
    return math.sqrt(max(1.0, case["rows"] / case["cols"]))


def prepare(case, seed):
    g = _gen(seed)
    s = {"case": case}
    if case["op"] in ("ortho", "muon"):
        x = _update(case, g)
        if case["type"] == "bits":
            n, at = x.numel(), 77  # the matrices start inside the packed vector, as layers do
            bit = torch.zeros((n + at + 31) // 32 * 32, dtype=torch.int64, device="cuda")
            bit[at:at + n] = (x.flatten() > 0).long()
            words = (bit.view(-1, 32) << torch.arange(32, device="cuda")).sum(1)
            s["grad"], s["offset"] = torch.where(words >= 1 << 31, words - (1 << 32), words).int(), at
        else:
            s["grad"], s["offset"] = x.to(TYPES[case["type"]]), 0
        if case["op"] == "muon":
            size = 1.0 if case["type"] == "bits" else 1e-3
            s["momentum"] = torch.randn(x.shape, device="cuda", generator=g).mul_(3 * size)
            s["weights"] = torch.randn(x.shape, device="cuda", generator=g).mul_(0.02).to(TYPES[case["out"]])
        if own:
            from paper_2501_17392_b200 import brace

            s["plan"] = brace.Orthogonalizer(case["rows"], case["cols"], batch=case["batch"])
            s["out"] = torch.empty(x.shape, dtype=TYPES[case["out"]], device="cuda")
            s["momentum_out"] = torch.empty_like(x) if case["op"] == "muon" else None
        return s
    c, v, d = case["clients"], case["vocab"], case["dim"]
    s["ids"] = _tokens(case, g)
    # a table is a part of the client's row of weights or of updates; rows are padded to 128 coordinates
    at = 77 if d % 4 else 128
    ld = (at + v * d + 127) // 128 * 128
    if case["op"] == "lookup":
        rows = torch.randn(c, ld, device="cuda", generator=g).mul_(0.02).to(TYPES[case["type"]])
        s["table"], s["scale"] = rows.as_strided((c, v, d), (ld, d, 1), at), math.sqrt(d)
    else:
        s["dy"] = torch.randn(c, case["tokens"], d, device="cuda", generator=g).mul_(1e-2).to(TYPES[case["type"]])
        s["scale"] = math.sqrt(d)
    if own:
        from paper_2501_17392_b200 import brace

        s["plan"] = brace.Embedding(v, d, case["tokens"], clients=c, grad=case["op"] == "grad")
        if case["op"] == "lookup":
            s["out"] = torch.empty(c, case["tokens"], d, dtype=TYPES[case["out"]], device="cuda")
        else:
            s["out"] = torch.zeros(c, ld, dtype=TYPES[case["out"]], device="cuda").as_strided((c, v, d), (ld, d, 1), at)
    return s


def run(s):
    case = s["case"]
    return (_own if own else _plain)[case["op"]](s, case)


# ---- the plain forms: elementary torch operations in 32 bits, rounded once at the end


def _direction(x):
    """x times a polynomial of its Gram matrix, STEPS times over, from unit Frobenius norm."""
    x = x / (x.square().sum((-2, -1), keepdim=True).sqrt() + EPS)
    turn = x.shape[-2] > x.shape[-1]
    x = x.mT if turn else x
    for _ in range(STEPS):
        gram = x @ x.mT
        x = A * x + (B * gram + C * (gram @ gram)) @ x
    return x.mT if turn else x


def _signs(words, offset, shape):
    """+1 or -1 for each of the packed bits, least significant first."""
    n = math.prod(shape)
    k = torch.arange(offset, offset + n, device=words.device)
    return (((words[k >> 5] >> (k & 31)) & 1) * 2 - 1).float().view(shape)


def _plain_ortho(s, case):
    return _direction(s["grad"].float()).to(TYPES[case["out"]])


def _plain_muon(s, case):
    g = _signs(s["grad"], s["offset"], s["momentum"].shape) if case["type"] == "bits" else s["grad"].float()
    momentum = BETA * s["momentum"] + g
    step = _direction(g + BETA * momentum)
    w = (1 - LR * DECAY) * s["weights"].float() - LR * _scale(case) * step
    return {"momentum": momentum, "weights": w.to(TYPES[case["out"]])}


def _plain_lookup(s, case):
    ids, table = s["ids"], s["table"]
    valid = (ids >= 0) & (ids < case["vocab"])
    client = torch.arange(case["clients"], device=ids.device)[:, None]
    rows = table[client, torch.where(valid, ids, 0)].float() * s["scale"]
    return torch.where(valid[..., None], rows, 0.0).to(TYPES[case["out"]])


def _plain_grad(s, case):
    ids, v, d = s["ids"], case["vocab"], case["dim"]
    valid = (ids >= 0) & (ids < v)
    client = torch.arange(case["clients"], device=ids.device)[:, None]
    dy = torch.where(valid[..., None], s["dy"].float(), 0.0)
    total = torch.zeros(case["clients"] * v, d, device=ids.device)
    total.index_add_(0, torch.where(valid, client * v + ids, 0).flatten(), dy.view(-1, d))
    return (total * s["scale"]).to(TYPES[case["out"]]).view(case["clients"], v, d)


_plain = {"ortho": _plain_ortho, "muon": _plain_muon, "lookup": _plain_lookup, "grad": _plain_grad}


# ---- the library's calls


def _own_ortho(s, case):
    s["plan"].orthogonalize(s["grad"], s["out"])
    return s["out"]


def _own_muon(s, case):
    s["plan"].muon_step(s["grad"], s["momentum"], s["weights"], LR, beta=BETA, weight_decay=DECAY, scale=_scale(case),
                        bit_offset=s["offset"], momentum_out=s["momentum_out"], weights_out=s["out"])
    return {"momentum": s["momentum_out"], "weights": s["out"]}


def _own_lookup(s, case):
    s["plan"].lookup(s["table"], s["ids"], s["out"], scale=s["scale"])
    return s["out"]


def _own_grad(s, case):
    s["plan"].grad(s["dy"], s["ids"], s["out"], scale=s["scale"])
    return s["out"]


_own = {"ortho": _own_ortho, "muon": _own_muon, "lookup": _own_lookup, "grad": _own_grad}


# ---- the definitions in 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("ortho", "muon"):
        if case["type"] == "bits":
            bits = (s["grad"].long()[:, None] >> torch.arange(32, device="cuda")) & 1
            n = case["batch"] * case["rows"] * case["cols"]
            x = (2 * bits.flatten()[s["offset"]:s["offset"] + n] - 1).double()
            x = x.view(case["batch"], case["rows"], case["cols"])
        else:
            x = s["grad"].double()
        if case["op"] == "ortho":
            return _exact_direction(x)
        momentum = s["momentum"].double() * BETA + x
        step = _exact_direction(momentum * BETA + x) * (LR * _scale(case))
        return {"momentum": momentum, "weights": s["weights"].double() * (1 - LR * DECAY) - step}
    if case["op"] == "lookup":
        ids, table = s["ids"], s["table"]
        got = torch.zeros(case["clients"], case["tokens"], case["dim"], dtype=torch.float64, device="cuda")
        for c in range(case["clients"]):
            here = torch.nonzero((ids[c] >= 0) & (ids[c] < case["vocab"]))[:, 0]
            got[c, here] = table[c].index_select(0, ids[c, here]).double() * s["scale"]
        return got
    got = torch.zeros(case["clients"], case["vocab"], case["dim"], dtype=torch.float64, device="cuda")
    for c in range(case["clients"]):
        ids = s["ids"][c]
        here = torch.nonzero((ids >= 0) & (ids < case["vocab"]))[:, 0]
        order = here[torch.argsort(ids[here], stable=True)]
        key, count = torch.unique_consecutive(ids[order], return_counts=True)
        for part in torch.arange(case["dim"], device="cuda").split(256):
            run_sum = torch.cumsum(s["dy"][c][order][:, part].double(), 0)
            upto = run_sum[count.cumsum(0) - 1] if len(key) else run_sum[:0]
            got[c, key[:, None], part] = torch.diff(upto, dim=0, prepend=torch.zeros_like(upto[:1])) * s["scale"]
    return got


def _exact_direction(x):
    """The same polynomial with the Gram matrix of the other side, by Horner's rule."""
    x = x / (torch.linalg.matrix_norm(x, keepdim=True) + EPS)
    turn = x.shape[-2] < x.shape[-1]
    y = x.mT.contiguous() if turn else x
    for _ in range(STEPS):
        s = y.mT @ y
        p = torch.eye(s.shape[-1], dtype=s.dtype, device=s.device) * B + C * s
        y = A * y + y @ (s @ p)
    return y.mT if turn else y
