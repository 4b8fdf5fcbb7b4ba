"""Steps of a training rank beside AdamW: the orthogonalised update of its matrices, and its embedding with the gradient.

  op             orthogonalize  every matrix G of a list -> O(G), in bf16
                 muon           momentum, O of it, and the weights' update, over a list of matrices
                 lookup         rows of an embedding table for a batch of tokens, scaled
                 embed_grad     the table's gradient from the rows' gradients, written anew or added to what is there

O(G) is five steps of X <- a X + b (X X^T) X + c (X X^T)^2 X from X = G / |G|, |G| the root of the sum of squares (of a zero matrix:
zero).  It moves all singular values near 1.  With h = factor * gradient, m <- beta m + (1 - beta) h, G = beta m + (1 - beta) h (m the
new one), p <- p - lr (s O(G) + decay p), s = 0.2 sqrt(max(rows, columns)): an update of about 0.2 lr per element.

A rank of a model whose vocabulary is split holds the rows [first, first + rows): other tokens look up zeros and give no gradient.
"""
import math

import numpy as np
import torch

own = False

F32, BF16, I32, I64, F64 = torch.float32, torch.bfloat16, torch.int32, torch.int64, torch.float64
A, B, C = 3.4445, -4.7750, 2.0315
STEPS = 5
LR, BETA, DECAY = 2e-4, 0.95, 0.1
TYPES = {"bf16": BF16, "f32": F32}


def listed():
    return [
        # Three small matrices: launches and latency.
        dict(name="small_orthogonalize", op="orthogonalize", shapes="64x64 33x200 200x7", grad="f32"),
        # Matrices of odd sizes, tall and wide: adapters, convolutions, projections of unusual widths.
        dict(name="odd_orthogonalize", op="orthogonalize", count=40, lo=65, hi=1500, sizes_seed=1, grad="bf16"),
        # One large matrix, gradients accumulated in fp32: a whole MLP projection of an 8B-parameter model.
        dict(name="mlp_orthogonalize", op="orthogonalize", shapes="14336x4096", grad="f32"),
        # A unit test's model: the matrices of two layers.
        dict(name="tiny_muon", op="muon", shapes="2*768x256 2*256x256", param="master", grad="f32"),
        # A model of 24 layers of width 1024.
        dict(name="medium_muon", op="muon", shapes="96*1024x1024 24*4096x1024 24*1024x4096", param="bf16", grad="bf16"),
        # A tensor-parallel rank of half the layers of an 8B-parameter model, weights with fp32 masters.
        dict(name="llama8b_tp8pp2_muon", op="muon", shapes="16*512x4096 32*128x4096 16*4096x512 32*1792x4096 16*4096x1792",
             param="master", grad="bf16"),
        # A few tokens: latency.
        dict(name="tiny_lookup", op="lookup", vocab=2048, first=0, rows=2048, dim=256, tokens=128, index="i64", table="f32", out="bf16"),
        # A batch of a rank that holds an eighth of the vocabulary.
        dict(name="llama8b_tp8_lookup", op="lookup", vocab=128256, first=16032, rows=16032, dim=4096, tokens=32768, index="i64",
             table="bf16", out="bf16"),
        dict(name="tiny_embed_grad", op="embed_grad", vocab=2048, first=0, rows=2048, dim=256, tokens=512, index="i64", out="bf16",
             grad="f32", add=False),
        # A small language model, gradients accumulated in fp32 over micro-batches.
        dict(name="gpt2s_embed_grad", op="embed_grad", vocab=50257, first=0, rows=50257, dim=768, tokens=32768, index="i64", out="bf16",
             grad="f32", add=True),
        dict(name="llama8b_tp8_embed_grad", op="embed_grad", vocab=128256, first=0, rows=16032, dim=4096, tokens=65536, index="i32",
             out="bf16", grad="bf16", add=False),
        # Very many tokens of a small alphabet (bytes), a third of them the same one, rows of odd length.
        dict(name="bytes_embed_grad", op="embed_grad", vocab=259, first=0, rows=259, dim=321, tokens=500001, index="i32", out="f32",
             grad="f32", add=False, same=0.33),
    ]


def _log(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))


def draw(rng):
    """Lists of 1 to 100 matrices of 1 to 6,000 rows and columns; tables of up to 130,000 rows of 1 to 5,000 elements, 1 to a
    million tokens."""
    op = rng.choice(["orthogonalize", "muon", "muon", "lookup", "embed_grad", "embed_grad"])
    if op in ("orthogonalize", "muon"):
        case = dict(op=op, count=_log(rng, 1, 100), lo=rng.choice([1, 16, 100, 129]), hi=_log(rng, 200, 6000), sizes_seed=rng.randrange(1 << 30),
                    grad=rng.choice(["bf16", "f32"]))
        if op == "muon":
            case.update(param=rng.choice(["master", "master", "bf16", "f32"]))
        while work(case)["flops"] > 6e12:
            case["count"], case["hi"] = case["count"] // 2 + 1, case["hi"] * 3 // 4
        return case
    vocab = _log(rng, 50, 130000)
    parts = rng.choice([1, 1, 2, 8])
    rows = -(-vocab // parts)
    first = rng.randrange(parts) * rows
    rows = max(1, min(rows, vocab - first))
    dim = _log(rng, 1, 5000) if rng.random() < 0.4 else 8 * _log(rng, 2, 600)
    case = dict(op=op, vocab=vocab, first=first, rows=rows, dim=dim, tokens=max(1, min(_log(rng, 1, 1000000), 200000000 // dim)),
                index=rng.choice(["i32", "i64"]), out=rng.choice(["bf16", "f32"]))
    if op == "lookup":
        return dict(case, table=rng.choice(["bf16", "f32"]))
    return dict(case, grad=rng.choice(["bf16", "f32"]), add=rng.random() < 0.5, same=rng.choice([0.0, 0.0, 0.1, 0.6]))


# ---------------------------------------------------------------- sizes, from the case alone


def _shapes(case):
    """(count, rows, columns) of the groups of equal matrices."""
    if "shapes" in case:
        groups = []
        for part in case["shapes"].split():
            count, _, size = part.rpartition("*")
            rows, _, cols = size.partition("x")
            groups.append((int(count or 1), int(rows), int(cols)))
        return groups
    r = np.random.default_rng(case["sizes_seed"])
    lo, hi = math.log(case["lo"]), math.log(case["hi"])
    return [(1, *(max(1, int(math.exp(x))) for x in lo + r.random(2) * (hi - lo))) for _ in range(case["count"])]


def _chances(case):
    """The chance of each token of the vocabulary: as 1 / rank, and `same` of them one token of the slice."""
    v = np.arange(case["vocab"])
    p = (np.log(v + 2) - np.log(v + 1)) / math.log(case["vocab"] + 1)
    same = case.get("same", 0.0)
    p *= 1 - same
    p[case["first"] + case["rows"] // 3] += same
    return p


def _rows_met(case):
    """How many tokens fall into the slice, and how many of its rows they meet, on average."""
    p = _chances(case)[case["first"]:case["first"] + case["rows"]]
    return case["tokens"] * float(p.sum()), float((-np.expm1(case["tokens"] * np.log1p(-np.minimum(p, 1 - 1e-12)))).sum())


# ---------------------------------------------------------------- inputs


class _State:
    """What a program has in hand before the call."""


def _matrices(case, gen, scale):
    """One buffer of all matrices.  Gradients have a part of low rank, as large as their noise, and rows of different sizes."""
    parts = []
    for count, m, n in _shapes(case):
        r = max(1, min(m, n) // 16)
        x = torch.randn(count, m, n, generator=gen, device="cuda")
        x += torch.randn(count, m, r, generator=gen, device="cuda") @ torch.randn(count, r, n, generator=gen, device="cuda") / math.sqrt(r)
        x *= torch.exp(0.3 * torch.randn(count, m, 1, generator=gen, device="cuda"))
        parts.append(x.mul_(scale).view(-1))
    return torch.cat(parts)


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    b = {}
    if case["op"] in ("orthogonalize", "muon"):
        b["grad"] = _matrices(case, gen, 1e-3).to(TYPES[case["grad"]])
        if case["op"] == "muon":
            b["m"] = _matrices(case, gen, 4e-4)
            b["weight"] = (torch.randn(b["m"].numel(), generator=gen, device="cuda") * 0.02).to(F32 if case["param"] == "f32" else BF16)
            if case["param"] == "master":
                b["master"] = b["weight"].float()
            # the record of a clipping that another call has done
            b["factor"] = float(torch.rand(1, generator=gen, device="cuda", dtype=F64)) * 0.5 + 0.25
        return b
    n, dim = case["tokens"], case["dim"]
    ends = torch.from_numpy(np.cumsum(_chances(case))).cuda()
    tokens = torch.searchsorted(ends, torch.rand(n, generator=gen, device="cuda", dtype=F64) * ends[-1])
    b["tokens"] = tokens.clamp_(max=case["vocab"] - 1).to(I64 if case["index"] == "i64" else I32)
    b["scale"] = math.sqrt(dim) if case["op"] == "lookup" else 0.125
    if case["op"] == "lookup":
        b["table"] = (torch.randn(case["rows"], dim, generator=gen, device="cuda") * 0.02).to(TYPES[case["table"]])
    else:
        b["out"] = (torch.randn(n, dim, generator=gen, device="cuda") * 1e-3).to(TYPES[case["out"]])
        b["grad"] = (torch.randn(case["rows"], dim, generator=gen, device="cuda") * 1e-3).to(TYPES[case["grad"]])
    return b


def _views(case, flat):
    views, at = [], 0
    for count, m, n in _shapes(case):
        for _ in range(count):
            views.append(flat[at:at + m * n].view(m, n))
            at += m * n
    return views


def prepare(case, seed):
    s = _State()
    s.case, s.b = case, _inputs(case, seed)
    if case["op"] == "orthogonalize":
        s.b["update"] = torch.zeros(s.b["grad"].numel(), dtype=BF16, device="cuda")
    elif case["op"] == "lookup":
        s.b["out"] = torch.zeros(case["tokens"], case["dim"], dtype=TYPES[case["out"]], device="cuda")
    elif case["op"] == "muon":
        s.record = torch.zeros(2, dtype=I64, device="cuda")  # norm and factor in fp32, the count of non-finite gradients
        s.record.view(F32)[0] = 2.0
        s.record.view(F32)[1] = s.b["factor"]
    if own:
        _plans(s)
    return s


# ---------------------------------------------------------------- the framework's calls


def _plans(s):
    from paper_2509_03047_gb300 import flashrec as fr

    case, b = s.case, s.b
    if case["op"] in ("orthogonalize", "muon"):
        lists = {k: _views(case, b[k]) for k in ("weight", "grad", "m", "master", "update") if k in b}
        names = {"weight": "weights", "grad": "grads", "m": "momenta", "master": "masters", "update": "updates"}
        scales = [0.2 * math.sqrt(max(g.shape)) for g in lists["grad"]] if case["op"] == "muon" else None
        s.plan = fr.MuonPlan(update_scale=scales, **{names[k]: x for k, x in lists.items()})
        s.hyper = fr.muon(lr=LR, beta=BETA, weight_decay=DECAY, nesterov=True, coefficients=[(A, B, C)] * STEPS)
    else:
        s.plan = fr.EmbedPlan(case["rows"], case["dim"], case["tokens"], first=case["first"])


def _run_own(s):
    case, b = s.case, s.b
    if case["op"] == "orthogonalize":
        s.plan.orthogonalize(s.hyper)
        return {"update": b["update"]}
    if case["op"] == "muon":
        s.plan.step(s.hyper, s.record)
        return {k: b[k] for k in ("weight", "master", "m") if k in b}
    if case["op"] == "lookup":
        s.plan.lookup(b["table"], b["tokens"], scale=b["scale"], out=b["out"])
        return {"out": b["out"]}
    s.plan.grad(b["out"], b["tokens"], b["grad"], scale=b["scale"], accumulate=case["add"])
    return {"grad": b["grad"]}


# ---------------------------------------------------------------- the plain form


def _orthogonal(x):
    """Of a stack of matrices in fp32, with no more rows than columns in the products."""
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2)
    norm = x.square().sum((1, 2), keepdim=True, dtype=F64).sqrt().float()
    x = torch.where(norm > 0, x / norm, 0.0)
    for _ in range(STEPS):
        gram = x @ x.transpose(1, 2)
        x = A * x + (B * gram + C * (gram @ gram)) @ x
    return x.transpose(1, 2) if tall else x


def _run_plain(s):
    case, b = s.case, s.b
    if case["op"] in ("orthogonalize", "muon"):
        at = 0
        for count, m, n in _shapes(case):
            here = slice(at, at + count * m * n)
            at += count * m * n
            g = b["grad"][here].float().view(count, m, n)
            if case["op"] == "orthogonalize":
                b["update"][here] = _orthogonal(g).reshape(-1).to(BF16)
                continue
            h = g * s.record.view(F32)[1]
            u = b["m"][here].view(count, m, n)
            u.copy_(u * BETA + h * (1 - BETA))
            o = _orthogonal(u * BETA + h * (1 - BETA)).reshape(-1)
            p = (b["master"] if "master" in b else b["weight"])[here].float()
            p = p - LR * (0.2 * math.sqrt(max(m, n)) * o + DECAY * p)
            if "master" in b:
                b["master"][here] = p
            b["weight"][here] = p.to(b["weight"].dtype)
        return {"update": b["update"]} if case["op"] == "orthogonalize" else {k: b[k] for k in ("weight", "master", "m") if k in b}
    at = b["tokens"].long() - case["first"]
    inside = (at >= 0) & (at < case["rows"])
    if case["op"] == "lookup":
        rows = b["table"][torch.where(inside, at, 0)].float() * b["scale"]
        b["out"].copy_(torch.where(inside[:, None], rows, 0.0))
        return {"out": b["out"]}
    # (in 64 bits: one token may stand for a third of a million rows)
    total = torch.zeros(case["rows"] + 1, case["dim"], dtype=F64, device="cuda")
    total.index_add_(0, torch.where(inside, at, case["rows"]), b["out"].double())
    total = total[:-1] * b["scale"]
    b["grad"].copy_(total + b["grad"].double() if case["add"] else total)
    return {"grad": b["grad"]}


def run(s):
    return _run_own(s) if own else _run_plain(s)


# ---------------------------------------------------------------- what it cannot do without


def work(case):
    if case["op"] in ("orthogonalize", "muon"):
        n = sum(count * m * k for count, m, k in _shapes(case))
        # products with a symmetric result need half of it; with r the smaller side and k the larger: r r k, r r r, 2 r r k
        flops = sum(count * STEPS * (3 * min(m, k) ** 2 * max(m, k) + min(m, k) ** 3) for count, m, k in _shapes(case))
        grad = TYPES[case["grad"]].itemsize
        if case["op"] == "orthogonalize":
            return {"bytes": n * (grad + 2), "flops": flops}
        return {"bytes": n * (grad + 8 + {"master": 4 + 4 + 2, "bf16": 4, "f32": 8}[case["param"]]), "flops": flops}
    inside, met = _rows_met(case)
    dim, index = case["dim"], 8 if case["index"] == "i64" else 4
    out = TYPES[case["out"]].itemsize
    if case["op"] == "lookup":
        return {"bytes": case["tokens"] * (index + dim * out) + met * dim * TYPES[case["table"]].itemsize, "flops": inside * dim}
    grad = TYPES[case["grad"]].itemsize
    written = 2 * met if case["add"] else case["rows"]
    return {"bytes": case["tokens"] * index + inside * dim * out + written * dim * grad, "flops": inside * dim}


# ---------------------------------------------------------------- from the definition, in 64 bits


def _exact_orthogonal(g):
    """By the polynomial on the singular values of G itself: with G = U S V^T, O = U p(S) V^T, and p(S) S^-1 a polynomial in G G^T."""
    side = min(g.shape)
    x = g if g.shape[0] == side else g.T
    norm = math.sqrt(float((x * x).sum()))
    if norm == 0.0:
        return torch.zeros_like(g)
    x = x / norm
    one = torch.eye(side, dtype=F64, device=g.device)
    for _ in range(STEPS):
        s = x @ x.T
        x = (A * one + s @ (B * one + C * s)) @ x
    return x if g.shape[0] == side else x.T


def exact(case, seed):
    b = _inputs(case, seed)
    if case["op"] in ("orthogonalize", "muon"):
        g = b["grad"].double()
        if case["op"] == "muon":
            # (the program's factor is an fp32 number in the record)
            h = g * float(np.float32(b["factor"]))
            u = BETA * b["m"].double() + (1 - BETA) * h
            g = BETA * u + (1 - BETA) * h
        o = torch.cat([_exact_orthogonal(x).reshape(-1) for x in _views(case, g)])
        if case["op"] == "orthogonalize":
            return {"update": o}
        scale = torch.cat([x.new_full((x.numel(),), 0.2 * math.sqrt(max(x.shape))) for x in _views(case, g)])
        p = (b["master"] if "master" in b else b["weight"]).double()
        p = p - LR * (scale * o + DECAY * p)
        return dict({"weight": p, "m": u}, **({"master": p} if "master" in b else {}))
    tokens, first, rows = b["tokens"].long(), case["first"], case["rows"]
    if case["op"] == "lookup":
        padded = torch.cat([b["table"].double(), torch.zeros(1, case["dim"], dtype=F64, device="cuda")])
        return {"out": padded[torch.where((tokens < first) | (tokens >= first + rows), rows, tokens - first)] * b["scale"]}
    # sums of the sorted tokens' rows: differences of running sums at the tokens' ends (in 64 bits, of fewer columns at a time)
    order = torch.argsort(tokens, stable=True)
    ends = torch.searchsorted(tokens[order].contiguous(), torch.arange(first, first + rows + 1, device="cuda"))
    total = torch.zeros(rows, case["dim"], dtype=F64, device="cuda")
    for at in range(0, case["dim"], 512):
        run_ = torch.nn.functional.pad(b["out"][:, at:at + 512][order].double().cumsum(0), (0, 0, 1, 0))
        total[:, at:at + 512] = run_[ends[1:]] - run_[ends[:-1]]
    total *= b["scale"]
    return {"grad": total + b["grad"].double() if case["add"] else total}
