"""The optimizer step over a training rank's whole state, as a program that trains and recovers calls it: what is measured.

Per parameter a rank holds a weight, perhaps an fp32 master of it, a gradient, and two Adam moments in fp32 or in 8 bits.

  op        clip       norm of all gradients, the count of non-finite ones and the factor that clips them
            adamw      the step; its 8-bit moments are also read back as the values that they stand for
            clip_adamw both, as a training step makes them
            convert    fp32 moments to 8 bits, and those read back as values
  param     master     bf16 weight with an fp32 master;  bf16, f32: the weight alone
  layout    model      transformer shapes, one allocation per buffer: every tensor starts aligned, many end oddly
            fragments  thousands of tensors of sizes spread from `lo` to `hi` elements, each its own allocation
            flat       ZeRO / FSDP flat groups: tensors of odd sizes back to back in one buffer of each kind

A tensor list lies in one buffer of each kind here, zeros between its tensors, so that the plain form is a few operations over
whole buffers.  Zero gradient, moments and weight stay zero in a step, and add nothing to a norm or a block's maximum.

8-bit moments, per block of 256 elements from the tensor's start: one byte E, the exponent of the block's largest value, and per
element a code c.  With base = 8 (E - 15) for the first moment (a sign and 7 bits of c), 8 (E - 31) for the second (8 bits of c),
the value of c > 0 is the fp32 number of bit pattern (c + base) << 20, and c = 0 is zero.  Bits below 2^20 round to nearest even,
or up with a probability: the element's 16 random bits, a function of seed, step, tensor and index, are added above bit 4.
"""
import math

import numpy as np
import torch

own = False

F32, BF16, U8, I32, I64 = torch.float32, torch.bfloat16, torch.uint8, torch.int32, torch.int64
BLOCK = 256
LR, BETA1, BETA2, EPS, DECAY = 3e-4, 0.9, 0.95, 1e-8, 0.1


def listed():
    return [
        # A unit test's model: launches and latency, the norm alone and a whole training step's update.
        dict(name="tiny_clip", op="clip", layout="model", hidden=128, layers=4, vocab=2048, grad="bf16", nonfinite=0),
        dict(name="tiny_clip_adamw", op="clip_adamw", layout="model", hidden=128, layers=4, vocab=2048, param="master",
             grad="f32", bits=32, nonfinite=0),
        # The norm of a tensor-parallel rank's gradients of an 8B-parameter model, three of them not finite (an overflowed loss scale).
        dict(name="llama8b_tp8_clip", op="clip", layout="model", hidden=4096, ffn=14336, layers=32, vocab=128256, tp=8, grad="bf16",
             nonfinite=3),
        # A small language model, gradients accumulated in fp32.
        dict(name="gpt2s_adamw", op="adamw", layout="model", hidden=768, layers=12, vocab=50257, param="master", grad="f32", bits=32),
        # Flat groups with odd sizes, tensors that start at any element: clipped step.
        dict(name="flat_clip_adamw", op="clip_adamw", layout="flat", tensors=400, lo=1001, hi=1000003, sizes_seed=1, param="master",
             grad="bf16", bits=32, nonfinite=0),
        # An fp32 optimizer partition in very many small tensors.
        dict(name="fragments_adamw", op="adamw", layout="fragments", tensors=20000, lo=256, hi=131072, sizes_seed=0, param="f32",
             grad="f32", bits=32),
        # A rank of an 8B-parameter model, the whole update of a training step.
        dict(name="llama8b_tp8_clip_adamw", op="clip_adamw", layout="model", hidden=4096, ffn=14336, layers=32, vocab=128256, tp=8,
             param="master", grad="bf16", bits=32, nonfinite=0),
        # 8-bit moments: a small model, a model whose bf16 weights have no master, and a rank of an 8B model.
        dict(name="tiny_adamw8", op="adamw", layout="model", hidden=128, layers=4, vocab=2048, param="master", grad="bf16", bits=8,
             rounding="random"),
        dict(name="gpt2s_adamw8", op="adamw", layout="model", hidden=768, layers=12, vocab=50257, param="bf16", grad="bf16", bits=8,
             rounding="random"),
        dict(name="llama8b_tp8_adamw8", op="adamw", layout="model", hidden=4096, ffn=14336, layers=32, vocab=128256, tp=8,
             param="master", grad="bf16", bits=8, rounding="random"),
        # A run that goes over to 8-bit moments: many small tensors, and a small model.
        dict(name="fragments_convert", op="convert", layout="fragments", tensors=2000, lo=1, hi=100000, sizes_seed=2,
             rounding="nearest"),
        dict(name="gpt2s_convert", op="convert", layout="model", hidden=768, layers=12, vocab=50257, rounding="random"),
    ]


def _log(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi))))


def draw(rng):
    """Another call on another list: 3,000 to 700 million elements, at most 10,000 tensors of one element and more."""
    op = rng.choice(["clip", "adamw", "adamw", "adamw", "clip_adamw", "clip_adamw", "convert"])
    case = dict(op=op)
    if op != "convert":
        case.update(grad=rng.choice(["bf16", "f32"]))
    if op.startswith("clip"):
        case.update(nonfinite=rng.choice([0, 0, 0, 1, 40]))
    if op.endswith("adamw"):
        case.update(param=rng.choice(["master", "master", "bf16", "f32"]), bits=32 if op == "clip_adamw" else rng.choice([8, 8, 32]))
    if op == "convert" or case.get("bits") == 8:
        case.update(rounding=rng.choice(["nearest", "random", "random"]))
    total = _log(rng, 3000, 700000000)
    layout = rng.choice(["model", "fragments"] if "rounding" in case else ["model", "fragments", "flat"])
    case.update(layout=layout)
    if layout == "model":
        hidden = 8 * _log(rng, 2, 256)
        layers = max(1, min(48, total // (14 * hidden * hidden)))
        return dict(case, hidden=hidden, layers=layers, vocab=max(7, min(128256, (total - 12 * layers * hidden * hidden) // hidden)))
    lo, hi = rng.choice([1, 255, 1001]), 1 + min(_log(rng, 2000, 8000000), total)
    mean = (hi - lo) / math.log(hi / lo) if hi > lo else lo
    return dict(case, tensors=int(max(1, min(total / mean, 10000))), lo=min(lo, hi), hi=hi, sizes_seed=rng.randrange(1 << 30))


# ---------------------------------------------------------------- the tensor list, from the case alone


def _sizes(case):
    """Elements of every tensor, and whether it decays (matrices do, norms and biases do not)."""
    if case["layout"] != "model":
        r = np.random.default_rng(case["sizes_seed"])
        a, b = math.log(case["lo"]), math.log(case["hi"])
        sizes = np.maximum(1, np.exp(a + r.random(case["tensors"]) * (b - a)).astype(np.int64))
        return sizes, np.ones(len(sizes), bool)
    h, layers, vocab, tp = case["hidden"], case["layers"], case["vocab"], case.get("tp", 1)
    f = case.get("ffn", 4 * h)
    if tp > 1:  # gated MLP, grouped queries with one key-value head of 128 per rank, untied head
        layer = [h, h // tp * h, 128 * h, 128 * h, h * (h // tp), h, f // tp * h, f // tp * h, h * (f // tp)]
        sizes = [vocab // tp * h] + layer * layers + [h, vocab // tp * h]
    else:
        layer = [h, h, 3 * h * h, 3 * h, h * h, h, h, h, h * f, f, f * h, h]
        sizes = [vocab * h] + layer * layers + [h, h]
    sizes = np.array(sizes, np.int64)
    return sizes, sizes > f


def _places(case):
    """(sizes, first elements in the buffers, elements of a buffer, lr factors, decay factors)."""
    sizes, decays = _sizes(case)
    room = sizes if case["layout"] == "flat" else -(-sizes // BLOCK) * BLOCK
    ends = np.cumsum(room)
    lr = np.ones(len(sizes), np.float32)
    lr[0] = 0.5  # the embedding learns at half the rate
    return sizes, ends - room, int(-(-ends[-1] // BLOCK) * BLOCK), lr, decays.astype(np.float32)


# ---------------------------------------------------------------- inputs


class _State:
    """What a program has in hand before the call."""


def _kinds(case):
    """Types of the buffers that the case has."""
    kinds = {}
    if case["op"] != "convert":
        kinds["grad"] = BF16 if case["grad"] == "bf16" else F32
    if case["op"].endswith("adamw"):
        kinds["weight"] = F32 if case["param"] == "f32" else BF16
        if case["param"] == "master":
            kinds["master"] = F32
    if case["op"] != "clip":
        kinds["m"] = kinds["v"] = F32
    return kinds


def _inputs(case, seed):
    """Buffers of gradients, weights and moments as training has them: magnitudes differ from block to block, one block in ten
    (rows of an embedding that no token has met) has no gradient and no moments."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kinds = _kinds(case)
    sizes, starts, total, _, _ = _places(case)
    gaps = np.diff(np.append(starts, total)) - sizes
    inside = torch.tensor([1.0, 0.0], device="cuda").repeat(len(sizes)).repeat_interleave(
        torch.from_numpy(np.stack([sizes, gaps], 1).reshape(-1)).cuda(), output_size=total)
    blocks = (total // BLOCK, 1)
    size = torch.exp(torch.randn(blocks, generator=gen, device="cuda") * 1.5) * 1e-3
    size *= torch.rand(blocks, generator=gen, device="cuda") > 0.1

    def noise(scale):
        x = torch.randn(total, generator=gen, device="cuda")
        x.view(-1, BLOCK).mul_(scale)
        return x.mul_(inside)

    b = {}
    if "grad" in kinds:
        b["grad"] = noise(size).to(kinds["grad"])
    if "weight" in kinds:
        b["weight"] = noise(0.02).to(kinds["weight"])
        if "master" in kinds:
            b["master"] = b["weight"].float()
    if "m" in kinds:
        b["m"] = noise(0.3 * size)
        b["v"] = noise(size).square_().mul_(0.7)
    for k in range(case.get("nonfinite", 0)):
        t, at = torch.randint(0, 1 << 30, (2,), generator=gen, device="cuda").tolist()
        t %= len(sizes)
        b["grad"][int(starts[t]) + at % int(sizes[t])] = (math.nan, math.inf, -math.inf)[k % 3]
    # A step without a clip of its own uses a record that another call has left: the factor of an accumulated, clipped gradient.
    factor = float(torch.rand(1, generator=gen, device="cuda", dtype=torch.float64)) * 0.5 + 0.25
    return b, factor


def _bits(x):
    return x.view(I32)


def prepare(case, seed):
    s = _State()
    s.case, s.step, s.seed = case, 1 + seed % 1000, seed
    b, factor = _inputs(case, seed)
    sizes, starts, total, s.lr, s.decay = _places(case)
    s.sizes, s.starts = sizes, starts
    s.max_norm = 1.0 if case.get("nonfinite") or seed % 4 else math.inf
    s.loss_scale = 0.125
    s.record = torch.zeros(2, dtype=I64, device="cuda")  # norm and factor in fp32, the count of non-finite gradients
    s.norm, s.factor, s.nonfinite = s.record.view(F32)[0:1], s.record.view(F32)[1:2], s.record[1:2]
    s.norm.fill_(2.0)
    s.factor.fill_(factor)
    s.rounding = case.get("rounding", "nearest")
    if case.get("bits") == 8:
        m, v = b.pop("m"), b.pop("v")
        b["m_code"], b["m_exp"] = _encode(m, True, _half(m))
        b["v_code"], b["v_exp"] = _encode(v, False, _half(v))
    if case["op"] == "convert":
        b["m_code"], b["v_code"] = (torch.zeros(total, dtype=U8, device="cuda") for _ in range(2))
        b["m_exp"], b["v_exp"] = (torch.zeros(total // BLOCK, dtype=U8, device="cuda") for _ in range(2))
    if case["op"] == "convert" or case.get("bits") == 8:
        b["m_value"], b["v_value"] = (torch.zeros(total, device="cuda") for _ in range(2))
    s.b = b
    ends = starts + sizes
    s.views = {k: [x[i:j] for i, j in zip(starts.tolist(), ends.tolist())] for k, x in b.items() if not k.endswith("_exp")}
    for k in ("m_exp", "v_exp"):
        if k in b:
            s.views[k] = [b[k][i:j] for i, j in zip((starts // BLOCK).tolist(), (-(-ends // BLOCK)).tolist())]
    if own:
        _plans(s)
    return s


# ---------------------------------------------------------------- the framework's calls


def _plans(s):
    from paper_2509_03047_gb300 import flashrec as fr

    s.fr, v = fr, s.views
    eight = dict(m=v.get("m_code"), v=v.get("v_code"), m_exp=v.get("m_exp"), v_exp=v.get("v_exp"))
    moments = eight if s.case.get("bits") == 8 else dict(m=v.get("m"), v=v.get("v"))
    if s.case["op"] == "clip":
        s.plan = fr.OptPlan(grads=v["grad"])
    elif s.case["op"] == "convert":
        s.plan, s.plan8 = fr.OptPlan(**moments), fr.OptPlan(**eight)
    else:
        s.plan = fr.OptPlan(v["weight"], v["grad"], masters=v.get("master"), lr_scale=s.lr, decay_scale=s.decay, **moments)
    if "m_value" in v:
        s.values = fr.OptPlan(m=v["m_value"], v=v["v_value"])
    s.round_how = fr.FR_ROUND_RANDOM if s.rounding == "random" else fr.FR_ROUND_NEAREST
    s.hyper = fr.fr_adamw(LR, BETA1, BETA2, EPS, DECAY, s.step, s.seed, s.round_how)


def _run_own(s):
    fr, op = s.fr, s.case["op"]
    if op == "convert":
        fr.fr_opt_convert(s.plan.handle, s.plan8.handle, s.round_how, s.seed)
        fr.fr_opt_convert(s.plan8.handle, s.values.handle)
        return {"m": s.b["m_value"], "v": s.b["v_value"]}
    if op.startswith("clip"):
        fr.fr_grad_clip(s.plan.handle, s.max_norm, s.loss_scale, s.record)
        if op == "clip":
            return {"norm": s.norm, "factor": s.factor, "nonfinite": s.nonfinite}
    fr.fr_adamw_step(s.plan.handle, s.hyper, s.record)
    if s.case["bits"] == 8:
        fr.fr_opt_convert(s.plan.handle, s.values.handle)
    return _outputs(s)


def _outputs(s):
    out = {k: s.b[k] for k in ("weight", "master") if k in s.b}
    out.update({k: s.b.get(k + "_value", s.b.get(k)) for k in ("m", "v")})
    if s.case["op"] == "clip_adamw":
        out.update(norm=s.norm, factor=s.factor, nonfinite=s.nonfinite)
    return out


# ---------------------------------------------------------------- the plain form


def _half(x):
    """What rounding to nearest even adds below bit 20."""
    return ((_bits(x) >> 20) & 1) + 0x7FFFF


def _encode(x, signed, r):
    """Codes and block exponents of fp32 moments; r: what the rounding adds below bit 20, at most 0xFFFFF."""
    mag = (_bits(x) & 0x7FFFFFFF).view(-1, BLOCK)
    top, span = mag.amax(1, keepdim=True).clamp_(max=0x7F800000), 15 if signed else 31
    e = ((top + 0xFFFFF) >> 23).clamp_(min=span + 1)
    c = ((mag + r.view(-1, BLOCK)) >> 20) - ((e - span) << 3)
    c = c.clamp_(min=0) if signed else torch.where(mag > 0, c.clamp_(min=1), 0)
    c = torch.where(e == 255, 0, c)
    if signed:
        c |= torch.where((_bits(x).view(-1, BLOCK) < 0) & (c > 0), 128, 0)
    return c.to(U8).view(-1), e.to(U8).view(-1)


def _decode(code, exp, signed):
    c, e = code.view(-1, BLOCK).int(), exp.view(-1, 1).int()
    span = 15 if signed else 31
    mag = c & 127 if signed else c
    x = ((mag + ((e.clamp(min=span + 1) - span) << 3)) << 20).view(F32)
    x = torch.where(mag > 0, x, 0.0)
    if signed:
        x = torch.where(c > 127, -x, x)
    return torch.where(e == 255, math.nan, x).view(-1)


def _mix(z):
    """The output function of splitmix64 (Steele, Lea, Flood 2014) on int64 tensors."""
    z = (z ^ ((z >> 30) & 0x3FFFFFFFF)) * -0x40A7B892E31B1A47
    z = (z ^ ((z >> 27) & 0x1FFFFFFFFF)) * -0x6B2FB644ECCEEE15
    return z ^ ((z >> 31) & 0x1FFFFFFFF)


def _random(s, step):
    """Two tensors of 32 random bits, as int64: per element, and per pair of elements (its high half for the first, its low half
    for the second)."""
    low = 0xFFFFFFFF
    room = torch.from_numpy(-(-s.sizes // BLOCK)).cuda()
    tensors = torch.arange(len(s.sizes), device="cuda")
    key = _mix(_mix(_mix(torch.tensor(s.seed, device="cuda")) + step) + tensors * -0x61C8864680B583EB)
    key = key.repeat_interleave(room).view(-1, 1)
    first = (torch.cumsum(room, 0) - room).repeat_interleave(room).view(-1, 1)
    blocks = torch.arange(first.numel(), device="cuda").view(-1, 1) - first
    p = blocks * (BLOCK // 2) + torch.arange(BLOCK // 2, device="cuda")
    u = ((p & low) * 0x9E3779B1 + ((key & low) ^ ((p >> 32) * 0x85EBCA77))) & low
    u ^= u >> 16
    u = (u * 2891336453 + ((key >> 32) & low)) & low
    u ^= u >> 15
    return torch.stack([(u * 1597334677) & low, (u * 741103597) & low], 2).view(-1), (u * 747796405 & low).view(-1)


def _per_element(s, per_tensor, total):
    spans = torch.from_numpy(np.diff(np.append(s.starts, total))).cuda()
    return torch.from_numpy(per_tensor).cuda().repeat_interleave(spans, output_size=total)


def _run_plain(s):
    op, b = s.case["op"], s.b
    if op == "convert":
        rnd = _random(s, 0)[0] if s.rounding == "random" else None
        for k, signed, shift in (("m", True, 0), ("v", False, 16)):
            r = _half(b[k]) if rnd is None else (((rnd >> shift) & 0xFFFF) << 4).int()
            code, exp = _encode(b[k], signed, r)
            b[k + "_code"].copy_(code)
            b[k + "_exp"].copy_(exp)
            b[k + "_value"].copy_(_decode(code, exp, signed))
        return {"m": b["m_value"], "v": b["v_value"]}
    if op.startswith("clip"):
        g = b["grad"].float()
        bad = ~g.isfinite()
        s.nonfinite.copy_(bad.sum())
        s.norm.copy_(g.masked_fill(bad, 0.0).square().sum().sqrt() * s.loss_scale)
        s.factor.copy_(torch.where(s.nonfinite > 0, 0.0, s.loss_scale * (s.max_norm / s.norm).clamp(max=1.0)))
        del g, bad
        if op == "clip":
            return {"norm": s.norm, "factor": s.factor, "nonfinite": s.nonfinite}
    eight, total = s.case["bits"] == 8, b["grad"].numel()
    m = _decode(b["m_code"], b["m_exp"], True) if eight else b["m"]
    v = _decode(b["v_code"], b["v_exp"], False) if eight else b["v"]
    p = b["master"] if "master" in b else b["weight"].float()
    h = b["grad"].float() * s.factor
    m2 = m * BETA1 + h * (1 - BETA1)
    v2 = v * BETA2 + (h * h) * (1 - BETA2)
    below = v2.sqrt() * (1 / math.sqrt(1 - BETA2 ** s.step)) + EPS
    u = (m2 / below) * (1 / (1 - BETA1 ** s.step)) + p * (_per_element(s, s.decay, total) * DECAY)
    p2 = p - u * (_per_element(s, s.lr, total) * LR)
    del h, below, u
    go = s.nonfinite == 0
    rnd, rnd_w = _random(s, s.step) if s.rounding == "random" else (None, None)
    if "master" in b:
        b["master"].copy_(torch.where(go, p2, p))
        w = p2.to(b["weight"].dtype)
    elif b["weight"].dtype == BF16 and rnd is not None:
        r = torch.stack([rnd_w >> 16, rnd_w & 0xFFFF], 1).view(-1).int()
        w = ((_bits(p2) + r) & -0x10000).view(F32).to(BF16)
    else:
        w = p2.to(b["weight"].dtype)
    b["weight"].copy_(torch.where(go, w, b["weight"]))
    del p, p2, w
    for k, new, signed, shift in (("m", m2, True, 0), ("v", v2, False, 16)):
        if eight:
            r = _half(new) if rnd is None else (((rnd >> shift) & 0xFFFF) << 4).int()
            code, exp = _encode(new, signed, r)
            b[k + "_code"].copy_(torch.where(go, code, b[k + "_code"]))
            b[k + "_exp"].copy_(torch.where(go, exp, b[k + "_exp"]))
            b[k + "_value"].copy_(_decode(b[k + "_code"], b[k + "_exp"], signed))
        else:
            b[k].copy_(torch.where(go, new, b[k]))
    return _outputs(s)


def run(s):
    return _run_own(s) if own else _run_plain(s)


# ---------------------------------------------------------------- what it cannot do without


def work(case):
    sizes, _, _, _, _ = _places(case)
    n, blocks = int(sizes.sum()), int((-(-sizes // BLOCK)).sum())
    kinds, op = _kinds(case), case["op"]
    grad = kinds["grad"].itemsize * n if "grad" in kinds else 0
    if op == "clip":
        return {"bytes": grad + 16, "flops": 2 * n}
    if op == "convert":  # values in, codes and exponents out, values out
        return {"bytes": (8 + 2 + 8) * n + 2 * blocks, "flops": 6 * n}
    weight = 8 + 2 if case["param"] == "master" else 2 * kinds["weight"].itemsize
    moments = 16 * n if case["bits"] == 32 else (2 * 2 + 8) * n + 2 * 2 * blocks
    return {"bytes": grad + weight * n + moments + 16, "flops": (16 if case["bits"] == 32 else 24) * n + (2 * n if op == "clip_adamw" else 0)}


# ---------------------------------------------------------------- from the definition, in 64 bits


def _exact_key(seed, step, tensor):
    """The random rule's 64-bit key of a tensor, in Python's integers."""
    full = (1 << 64) - 1

    def mix(z):
        z = ((z ^ z >> 30) * 0xBF58476D1CE4E5B9) & full
        z = ((z ^ z >> 27) * 0x94D049BB133111EB) & full
        return z ^ z >> 31

    return mix((mix((mix(seed) + step) & full) + tensor * 0x9E3779B97F4A7C15) & full)


def _exact_random(seed, step, tensor, n):
    """(first moments', second moments') random fractions of a step, multiples of 2^-16, of one tensor's n elements."""
    key = _exact_key(seed, step, tensor)
    i = torch.arange(n, device="cuda")
    pair, odd = i.div(2, rounding_mode="floor"), i % 2
    u = (pair * 0x9E3779B1 + (key % 2 ** 32)) % 2 ** 32  # (a pair's index is below 2^32 here)
    u = u ^ u.div(2 ** 16, rounding_mode="floor")
    u = (u * 2891336453 + key // 2 ** 32) & 0xFFFFFFFF
    u = u ^ u.div(2 ** 15, rounding_mode="floor")
    h = (u * torch.where(odd == 1, 741103597, 1597334677)) & 0xFFFFFFFF
    return (h & 0xFFFF).double() / 2 ** 16, (h >> 16).double() / 2 ** 16


def _exact_eight(x, span, up):
    """Values that a tensor's moments x stand for in 8 bits.  On the scale q of eighths of a binade (8 times the biased exponent,
    plus 8 times the fraction) codes are the whole numbers from 1 to 8 span + 7 above the block's base; up: what is added to q
    before it is cut off, None for the nearest."""
    n = x.numel()
    x = torch.nn.functional.pad(x, (0, -n % BLOCK)).view(-1, BLOCK)
    frac, ex = torch.frexp(x.abs())
    q = torch.where(x == 0, 0.0, (ex + 126) * 8.0 + (2 * frac - 1) * 8)
    top = ((q.amax(1, keepdim=True) + (1 - 2.0 ** -20)) / 8).floor().clamp(min=span + 1)
    base = 8 * (top - span)
    c = (torch.round(q) if up is None else (q + torch.nn.functional.pad(up, (0, -n % BLOCK)).view(-1, BLOCK)).floor()) - base
    c = torch.where((c < 1) & (x > 0) & (span == 31), 1.0, c)
    k = c + base
    value = torch.ldexp(1 + (k % 8) / 8, (k / 8).floor() - 127)
    return (torch.where(c < 1, 0.0, value) * x.sign()).view(-1)[:n]


def exact(case, seed):
    b, factor = _inputs(case, seed)
    sizes, starts, total, lr, decay = _places(case)
    op, step = case["op"], 1 + seed % 1000
    out = {}
    if op.startswith("clip"):
        g = b["grad"].double()
        bad = ~g.isfinite()
        norm = 0.125 * float(g[~bad].square().sum().sqrt())
        most = 1.0 if case["nonfinite"] or seed % 4 else math.inf
        count = int(bad.sum())
        factor = 0.0 if count else 0.125 * min(1.0, most / norm if norm else 1.0)
        out = {"norm": torch.tensor([norm], dtype=torch.float64), "factor": torch.tensor([factor], dtype=torch.float64),
               "nonfinite": None}
        del g, bad
        if op == "clip":
            return out
        if count:
            return dict(out, **{k: b[k].double() for k in ("weight", "master", "m", "v") if k in b})
    if case.get("bits") == 8:  # the state that a step starts from: rounded to nearest
        for k, signed in (("m", True), ("v", False)):
            b[k] = _decode(*_encode(b[k], signed, _half(b[k])), signed)
    new = {k: torch.zeros(total, dtype=torch.float64, device="cuda") for k in ("weight", "m", "v") if k in b}
    for t, (at, n) in enumerate(zip(starts.tolist(), sizes.tolist())):
        here = slice(at, at + n)
        m, v = b["m"][here].double(), b["v"][here].double()
        if op != "convert":
            h = b["grad"][here].double() * float(np.float32(factor))
            m = BETA1 * m + (1 - BETA1) * h
            v = BETA2 * v + (1 - BETA2) * h * h
            p = (b["master"] if "master" in b else b["weight"])[here].double()
            direction = (m / (1 - BETA1 ** step)) / ((v / (1 - BETA2 ** step)).sqrt() + EPS)
            new["weight"][here] = p - LR * float(lr[t]) * (direction + DECAY * float(decay[t]) * p)
        if "rounding" in case:
            up_m, up_v = _exact_random(seed, 0 if op == "convert" else step, t, n) if case["rounding"] == "random" else (None, None)
            m, v = _exact_eight(m, 15, up_m), _exact_eight(v, 31, up_v)
        new["m"][here], new["v"][here] = m, v
    if "master" in b:
        new["master"] = new["weight"]
    return dict(new, **out)
