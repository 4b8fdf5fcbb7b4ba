"""The optimizer step on the GPU against its definition (tests/optim_reference.py):
moments, codes and exponents bit for bit, parameters and norms within bounds
that count the fp32 roundings."""
import math

import numpy as np
import pytest
import torch

import optim_reference as ref
from gpu_helpers import GUARD_BYTES

pytestmark = pytest.mark.gpu

fr = pytest.importorskip("paper_2509_03047_gb300.flashrec")

SIZES = [1, 0, 255, 256, 257, 7, 1000, 4099, 65549, 8192]
FILL = 0xA5


@pytest.fixture(autouse=True)
def _free_memory():
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


class Buffers:
    """One kind of buffer for a list of tensors, each `shift` elements past a 512-byte boundary of one allocation filled
    with a pattern that must survive between them."""

    def __init__(self, arrays, shift=0):
        item = arrays[0].dtype.itemsize
        self.spans, at = [], 0
        for i, a in enumerate(arrays):
            lead = item * (shift + (i if shift else 0) % 5)
            self.spans.append((at + lead, a.nbytes))
            at += -(-(lead + a.nbytes + GUARD_BYTES) // 512) * 512
        self.whole = torch.full((at,), FILL, dtype=torch.uint8, device="cuda")
        kind = {"uint16": torch.bfloat16, "float32": torch.float32, "uint8": torch.uint8}[str(arrays[0].dtype)]
        self.dtype, self.tensors = arrays[0].dtype, []
        for (a, n), x in zip(self.spans, arrays):
            raw = self.whole[a:a + n]
            if n:
                raw.copy_(torch.from_numpy(x.view(np.uint8).copy()))
            self.tensors.append(raw.view(kind) if n else torch.empty(0, dtype=kind, device="cuda"))

    def get(self):
        self.check()
        host = self.whole.cpu().numpy()
        return [host[a:a + n].view(self.dtype) for a, n in self.spans]

    def check(self):
        mask = np.ones(self.whole.numel(), bool)
        for a, n in self.spans:
            mask[a:a + n] = False
        assert (self.whole.cpu().numpy()[mask] == FILL).all(), "bytes outside the tensors were written"


def _state(seed, sizes, param, grad, bits):
    """Host arrays by kind; magnitudes differ between blocks, some blocks are zero."""
    r = np.random.default_rng(seed)
    out = {k: [] for k in ("weight", "grad", "m", "v")}
    for n in sizes:
        k = -(-n // 256)
        size = np.repeat(np.exp(r.normal(size=k) * 3) * 1e-3 * (r.random(k) > 0.15), 256)[:n].astype(np.float32)
        f = lambda: r.normal(size=n).astype(np.float32)  # noqa: E731
        out["grad"].append(f() * size * (r.random(n) > 0.05))
        out["m"].append(f() * size * 0.3)
        out["v"].append((f() * size) ** 2)
        out["weight"].append(f() * np.float32(0.02))
    bf = lambda xs: [ref.f32_to_bf16(x) for x in xs]  # noqa: E731
    if grad == "bf16":
        out["grad"] = bf(out["grad"])
    if param != "f32":
        out["weight"] = bf(out["weight"])
    if param == "master":
        out["masters"] = [ref.bf16_to_f32(x) + np.float32(1e-5) for x in out["weight"]]
    if bits == 8:
        for k in ("m", "v"):
            pairs = [ref.encode(x, k) for x in out[k]]
            out[k], out[k + "_exp"] = [c for c, _ in pairs], [e for _, e in pairs]
    return out


def _wide(x):
    return ref.bf16_to_f32(x) if x.dtype == np.uint16 else x


def _plan(host, shift, **more):
    b = {k: Buffers(v, 0 if k.endswith("_exp") else shift) for k, v in host.items()}
    names = {"weight": "weights", "grad": "grads"}
    return b, fr.OptPlan(**{names.get(k, k): x.tensors for k, x in b.items()}, **more)


def _record(scale, nonfinite=0):
    r = torch.zeros(2, dtype=torch.int64, device="cuda")
    r.view(torch.float32)[1] = scale
    r[1] = nonfinite
    return r


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("rounding", ["nearest", "random"])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("grad", ["bf16", "f32"])
@pytest.mark.parametrize("param", ["master", "bf16", "f32"])
def test_step_is_its_definition(param, grad, bits, rounding, shift):
    host = _state(11, SIZES, param, grad, bits)
    lr_scale = [1.0 + 0.5 * (i % 3) for i in range(len(SIZES))]
    decay_scale = [float(i % 2) for i in range(len(SIZES))]
    b, plan = _plan(host, shift, lr_scale=lr_scale, decay_scale=decay_scale)
    h, scale = ref.Numbers(), 0.37109375
    how = fr.FR_ROUND_RANDOM if rounding == "random" else fr.FR_ROUND_NEAREST
    hyper = fr.fr_adamw(h.lr, h.beta1, h.beta2, h.eps, h.weight_decay, h.step, h.seed, how)
    plan.step(hyper, _record(scale))
    torch.cuda.synchronize()
    got = {k: x.get() for k, x in b.items()}
    for i, n in enumerate(SIZES):
        if n == 0:
            continue
        rm, rv, rw = ref.random_bits(h.seed, h.step, i, np.arange(n)) if rounding == "random" else (None, None, None)
        old = {k: host[k][i] for k in ("m", "v")}
        if bits == 8:
            old = {k: ref.decode(host[k][i], host[k + "_exp"][i], k).astype(np.float32) for k in old}
        p, g = _wide(host.get("masters", host["weight"])[i]), _wide(host["grad"][i])
        m2, v2 = ref.moments(h, old["m"], old["v"], g, scale)
        p64, m64, v64, p_err, m_err, v_err = ref.step64(h, p, old["m"], old["v"], g, scale, lr_scale[i], decay_scale[i])
        assert (np.abs(m2 - m64) <= m_err).all() and (np.abs(v2 - v64) <= v_err).all()
        if bits == 8:
            for k, x, r in (("m", m2, rm), ("v", v2, rv)):
                codes, exps = ref.encode(x, k, r)
                assert np.array_equal(got[k + "_exp"][i], exps), (k, i)
                assert np.array_equal(got[k][i], codes), (k, i)
        else:
            assert np.array_equal(got["m"][i].view(np.uint32), m2.view(np.uint32)), i
            assert np.array_equal(got["v"][i].view(np.uint32), v2.view(np.uint32)), i
        if param == "master":
            new = got["masters"][i]
            assert (np.abs(new - p64) <= p_err).all(), i
            assert np.array_equal(got["weight"][i], ref.f32_to_bf16(new)), i
        elif param == "f32":
            assert (np.abs(got["weight"][i] - p64) <= p_err).all(), i
        else:  # between the roundings of both ends of what p may be
            new = _wide(got["weight"][i])
            for end, ok in ((p64 - p_err, np.less_equal), (p64 + p_err, np.greater_equal)):
                x = end.astype(np.float32)
                x = np.nextafter(x, np.float32(-np.inf) if ok is np.less_equal else np.float32(np.inf))
                if rounding == "random":
                    edge = ((x.view(np.uint32).astype(np.int64) + rw) >> 16).astype(np.uint16)
                else:
                    edge = ref.f32_to_bf16(x)
                assert ok(_wide(edge), new).all(), i


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("shift", [0, 1])
def test_step_leaves_every_byte_when_a_gradient_is_not_finite(bits, shift):
    host = _state(5, SIZES, "master", "bf16", bits)
    host["grad"][8][60000] = 0x7F80  # Inf
    b, plan = _plan(host, shift)
    before = {k: x.whole.clone() for k, x in b.items()}
    rec = plan.clip(max_norm=1.0)
    plan.step(fr.fr_adamw(1e-2, 0.9, 0.95, 1e-8, 0.1, 1, 0, 0), rec)
    norm, scale, bad = fr.clip_view(rec)
    assert int(bad) == 1 and float(scale) == 0.0 and math.isfinite(float(norm))
    for k, x in b.items():
        assert torch.equal(x.whole, before[k]), k


def test_nonfinite_gradients_without_a_record_follow_the_formula():
    host = _state(6, [1000], "f32", "f32", 32)
    for i, x in ((3, np.nan), (300, np.inf), (301, -np.inf), (999, 3e38)):
        host["grad"][0][i] = x
    b, plan = _plan(host, 0)
    h = ref.Numbers()
    plan.step(fr.fr_adamw(h.lr, h.beta1, h.beta2, h.eps, h.weight_decay, h.step, h.seed, 0))
    m2, v2 = ref.moments(h, host["m"][0], host["v"][0], host["grad"][0])
    got = {k: x.get()[0] for k, x in b.items()}
    for name, want in (("m", m2), ("v", v2)):
        assert np.array_equal(got[name], want, equal_nan=True), name
    w = got["weight"]
    assert np.isnan(w[[3, 300, 301]]).all() and np.isfinite(np.delete(w, [3, 300, 301])).all()
    assert abs(w[999] - host["weight"][0][999] * (1 - h.lr * h.weight_decay)) < 1e-6  # v overflowed: no step


def test_eight_bit_block_with_a_nonfinite_moment_reads_as_nan_and_stays_so():
    host = _state(7, [700], "f32", "f32", 8)
    host["grad"][0][300] = np.inf
    b, plan = _plan(host, 0)
    hyper = fr.fr_adamw(1e-2, 0.9, 0.95, 1e-8, 0.0, 1, 0, 0)
    plan.step(hyper)
    assert b["m_exp"].get()[0].tolist()[1] == 255 and b["v_exp"].get()[0].tolist()[1] == 255
    assert 255 not in (b["m_exp"].get()[0][0], b["m_exp"].get()[0][2])
    values = [torch.empty(700, device="cuda") for _ in range(2)]
    out = fr.OptPlan(m=values[:1], v=values[1:])
    plan.convert_to(out)
    for x in values:
        assert torch.isnan(x[256:512]).all() and torch.isfinite(x[:256]).all() and torch.isfinite(x[512:]).all()
    b["grad"].tensors[0].zero_()
    plan.step(hyper)
    plan.convert_to(out)
    assert torch.isnan(values[0][256:512]).all() and torch.isfinite(values[0][:256]).all()


# ---------------------------------------------------------------- the norm

def _clip(grads, shift, max_norm=math.inf, grad_scale=1.0):
    b = Buffers(grads, shift)
    plan = fr.OptPlan(grads=b.tensors)
    rec = torch.full((48,), FILL, dtype=torch.uint8, device="cuda")
    plan.clip(max_norm, grad_scale, out=rec[16:32])
    assert (rec[:16] == FILL).all() and (rec[32:] == FILL).all()
    b.check()
    return [x.item() for x in fr.clip_view(rec[16:32])]


def _grads(kind, sizes, seed=0):
    r = np.random.default_rng(seed)
    gs = []
    for n in sizes:
        x = r.normal(size=n).astype(np.float32)
        if kind == "huge":
            x = x * np.float32(1e30)
        elif kind == "tiny":
            x = x * np.float32(1e-28)
        elif kind == "subnormal":
            x = x * np.float32(1e-40)
        elif kind == "zero":
            x = x * 0
        elif kind == "mixed":
            x = x * np.exp(r.normal(size=n) * 20).astype(np.float32)
            x[~np.isfinite(x)] = 1.0
        elif kind == "nonfinite":
            for v in (np.nan, np.inf, -np.inf):
                if n:
                    x[r.integers(0, n)] = v
        elif kind == "constant":
            x[:] = np.float32(0.1)
        gs.append(x)
    return gs


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["plain", "huge", "tiny", "subnormal", "zero", "mixed", "nonfinite", "constant"])
def test_norm_is_its_definition(kind, dtype, shift):
    gs = _grads(kind, SIZES + [300001])
    if dtype == "bf16":
        with np.errstate(all="ignore"):
            gs = [np.where(np.isfinite(x), ref.f32_to_bf16(x), (x.view(np.uint32) >> 16).astype(np.uint16) | 0x40 * np.isnan(x)).astype(np.uint16)
                  for x in gs]
    norm, scale, bad = ref.norm64([_wide(x) for x in gs], 0.75, 0.5)
    got_norm, got_scale, got_bad = _clip(gs, shift, 0.75, 0.5)
    # A lane adds at most 64 squares in each of two fp32 sums, whose pairs and everything above them are exact to 2^-40: 64 u of
    # the sum of squares, half of that of the norm; and the rounding to fp32.
    tol = 33 * ref.U
    assert got_bad == bad and (bad > 0) == (kind == "nonfinite")
    # (an fp32 result below 2^-126 is rounded to a multiple of 2^-149)
    assert abs(got_norm - norm) <= tol * norm + 2.0 ** -149
    assert abs(got_scale - scale) <= tol * scale


def test_norm_mixes_types_and_takes_empty_lists():
    f, h = _grads("plain", [1000, 5]), [ref.f32_to_bf16(x) for x in _grads("plain", [300, 70000], 1)]
    tensors = Buffers(f).tensors + Buffers(h).tensors
    rec = fr.OptPlan(grads=tensors).clip()
    norm, scale, bad = ref.norm64(f + [_wide(x) for x in h], math.inf, 1.0)
    assert abs(float(fr.clip_view(rec)[0]) - norm) <= 33 * ref.U * norm and float(fr.clip_view(rec)[1]) == 1.0
    for empty in ([], [torch.empty(0, device="cuda")]):
        rec = fr.OptPlan(grads=empty).clip(max_norm=1.0, grad_scale=0.25)
        assert [x.item() for x in fr.clip_view(rec)] == [0.0, 0.25, 0]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norm_has_the_same_bits_at_every_alignment(dtype):
    gs = _grads("mixed", SIZES + [1000003, 70000])
    if dtype == "bf16":
        gs = [ref.f32_to_bf16(x) for x in gs]
    want = _clip(gs, 0)
    for shift in range(1, 8):
        assert _clip(gs, shift) == want, shift


# ---------------------------------------------------------------- replicas, streams, lengths

@pytest.mark.parametrize("param,bits,rounding", [("master", 32, 0), ("bf16", 8, 1), ("master", 8, 1), ("f32", 8, 0)])
def test_replicas_at_other_addresses_stay_bit_identical(param, bits, rounding):
    sizes = SIZES + [300007]
    host = _state(21, sizes, param, "bf16", bits)
    runs = []
    for shift in (0, 1, 3):
        b, plan = _plan(host, shift)
        hyper = fr.fr_adamw(1e-2, 0.9, 0.95, 1e-8, 0.1, 0, 99, rounding)
        rec = plan.new_clip()
        for t in range(1, 6):
            hyper.step = t
            plan.clip(0.5, 1.0, out=rec)
            plan.step(hyper, rec)
        runs.append({k: x.get() for k, x in b.items()})
    for other in runs[1:]:
        for k in runs[0]:
            for x, y in zip(runs[0][k], other[k]):
                assert x.tobytes() == y.tobytes(), k


@pytest.mark.parametrize("bits", [32, 8])
def test_calls_back_to_back_and_from_a_graph_equal_calls_with_waits(bits):
    """Each kernel may start while the one before ends: the record that a step reads, the states that a step and a conversion read
    are the ones of the call before, with nothing between them."""
    host = _state(31, [200000, 77, 5000], "master", "f32", bits)

    def calls(b, plan, out, stream, wait):
        rec = plan.new_clip()
        for t in range(1, 5):
            for g in b["grad"].tensors:
                g.mul_(1.5)
            plan.clip(0.5, 1.0, out=rec, stream=stream)
            if wait:
                torch.cuda.synchronize()
            plan.step(fr.fr_adamw(1e-2, 0.9, 0.95, 1e-8, 0.1, t, 5, 1), rec, stream=stream)
            if wait:
                torch.cuda.synchronize()
            if bits == 8:
                plan.convert_to(out, stream=stream)
            if wait:
                torch.cuda.synchronize()

    results = []
    for how in ("wait", "back to back", "graph"):
        b, plan = _plan(host, 0)
        values = [torch.zeros(n, device="cuda") for n in (200000, 77, 5000) * 2]
        out = fr.OptPlan(m=values[:3], v=values[3:])
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        torch.cuda.synchronize()
        if how == "graph":
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                calls(b, plan, out, s, False)
            g.replay()
        else:
            with torch.cuda.stream(s):
                calls(b, plan, out, s, how == "wait")
        torch.cuda.synchronize()
        results.append(([x.whole for x in b.values()], values))
    for state, values in results[1:]:
        assert all(torch.equal(x, y) for x, y in zip(state, results[0][0]))
        assert all(torch.equal(x, y) for x, y in zip(values, results[0][1]))


@pytest.mark.parametrize("as_handle", [False, True])
def test_a_record_made_for_another_stream_is_not_filled_later(as_handle):
    """The current stream is busy while a norm runs on another one, which has a record of its own: whatever fills that must
    not wait for the current stream's work and come after the norm."""
    _, plan = _plan(_state(33, [5000, 300], "master", "f32", 32), 0)
    want = plan.clip(0.5, 1.0)
    torch.cuda.synchronize()
    s, busy = torch.cuda.Stream(), torch.empty(1 << 30, dtype=torch.uint8, device="cuda")
    for _ in range(100):  # 15 ms and more
        busy.fill_(1)
    got = plan.clip(0.5, 1.0, stream=s.cuda_stream if as_handle else s)
    torch.cuda.synchronize()
    assert torch.equal(got.view(torch.uint8), want.view(torch.uint8)) and float(fr.clip_view(want)[0]) > 0


def test_offsets_past_32_bits():
    """A bf16 tensor of 2^33 + 777 elements with 8-bit moments (52 GB): its last blocks, where a pair's index passes 2^32,
    against the definition, and the norm of gradients that are zero but there."""
    n, tail = (1 << 33) + 777, 2048 + 777 - 256 * 3
    if torch.cuda.mem_get_info()[0] < 70 << 30:
        pytest.skip("needs 70 GB")
    weight, grad = (torch.zeros(n, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    m, v = (torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in range(2))
    m_exp, v_exp = (torch.zeros(-(-n // 256), dtype=torch.uint8, device="cuda") for _ in range(2))
    r = np.random.default_rng(3)
    start = n - tail
    assert start % 256 == 0 and start < 1 << 33 < n
    w0, g0 = (ref.f32_to_bf16(r.normal(size=tail).astype(np.float32) * s) for s in (0.02, 1e-3))
    weight[start:].copy_(torch.from_numpy(w0.view(np.int16)).view(torch.bfloat16))
    grad[start:].copy_(torch.from_numpy(g0.view(np.int16)).view(torch.bfloat16))
    plan = fr.OptPlan([weight], [grad], [m], [v], m_exp=[m_exp], v_exp=[v_exp])
    rec = plan.clip()
    norm = ref.norm64([_wide(g0)], math.inf, 1.0)[0]
    assert abs(float(fr.clip_view(rec)[0]) - norm) <= 33 * ref.U * norm
    h = ref.Numbers(step=1, seed=123)
    plan.step(fr.fr_adamw(h.lr, h.beta1, h.beta2, h.eps, 0.0, h.step, h.seed, fr.FR_ROUND_RANDOM))
    rm, rv, _ = ref.random_bits(h.seed, h.step, 0, np.arange(start, n, dtype=np.uint64))
    m2, v2 = ref.moments(h, np.zeros(tail), np.zeros(tail), _wide(g0))
    for got, exp, k, x, rnd in ((m, m_exp, "m", m2, rm), (v, v_exp, "v", v2, rv)):
        codes, exps = ref.encode(x, k, rnd)
        assert np.array_equal(got[start:].cpu().numpy(), codes) and np.array_equal(exp[start // 256:].cpu().numpy(), exps)
    h.weight_decay = 0.0
    p64, _, _, p_err, _, _ = ref.step64(h, _wide(w0), np.zeros(tail), np.zeros(tail), _wide(g0))
    new = weight[start:].double().cpu().numpy()
    assert (np.abs(new - p64) <= 2.0 ** -7 * np.abs(p64) + p_err).all()  # one step of bf16 at most
    assert not weight[:start:4097].any() and not m[:start].any()


# ---------------------------------------------------------------- conversion

def _convert_plan(host8, n):
    b = {k: Buffers([x]) for k, x in host8.items()}
    return b, fr.OptPlan(**{k: x.tensors for k, x in b.items()})


def test_every_code_under_every_exponent_reads_as_its_meaning():
    codes = np.tile(np.arange(256, dtype=np.uint8), 256)
    exps = np.arange(256, dtype=np.uint8)
    _, src = _convert_plan({"m": codes, "v": codes, "m_exp": exps, "v_exp": exps}, codes.size)
    out = [torch.empty(codes.size, device="cuda") for _ in range(2)]
    src.convert_to(fr.OptPlan(m=out[:1], v=out[1:]))
    for k, x in zip("mv", out):
        want = ref.decode(codes, exps, k)
        got = x.cpu().numpy()
        assert np.array_equal(got, want.astype(np.float32), equal_nan=True) and np.array_equal(got.astype(np.float64), want, equal_nan=True)


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("rounding", [0, 1])
@pytest.mark.parametrize("spread", [0.0, 1.0, 12.0, 40.0])
def test_coding_is_its_definition(spread, rounding, shift):
    r = np.random.default_rng(17)
    host = {"m": [], "v": []}
    for n in SIZES:
        x = r.normal(size=(2, n)) * np.exp(r.normal(size=(2, n)) * spread)
        x = np.clip(x, -1e38, 1e38).astype(np.float32)
        x[:, ::7] = 0
        host["m"].append(x[0].copy())
        host["v"].append(np.abs(x[1]))
        if n > 600:
            host["m"][-1][256:512] = 0
            host["v"][-1][256:512] = 0
            host["v"][-1][3] = -1.0  # no second moment is negative: read as zero
            host["m"][-1][600], host["v"][-1][600] = np.float32(1e-42), np.float32(3e-44)
        if n > 5000:
            host["m"][-1][4100], host["v"][-1][4400], host["v"][-1][4700] = np.nan, np.inf, -np.nan
            host["m"][-1][4400] = np.float32(3.4e38)  # above the largest code's binade: as if infinite
    b, src = _plan(host, shift)
    e = {k: [np.zeros(-(-n // 256), np.uint8) for n in SIZES] for k in ("m_exp", "v_exp")}
    c = {k: [np.full(n, 9, np.uint8) for n in SIZES] for k in ("m", "v")}
    b8, dst = _plan({**c, **e}, shift)
    src.convert_to(dst, rounding, 1234)
    got = {k: x.get() for k, x in b8.items()}
    for i, n in enumerate(SIZES):
        if n == 0:
            continue
        rnd = ref.random_bits(1234, 0, i, np.arange(n)) if rounding else (None, None, None)
        for k, q in zip("mv", rnd):
            codes, exps = ref.encode(host[k][i], k, q)
            assert np.array_equal(got[k + "_exp"][i], exps), (k, i)
            assert np.array_equal(got[k][i], codes), (k, i)
    # and back: within half a step (an eighth of a binade's start, or the whole step at random) above the smallest code
    bv, back = _plan({k: [np.zeros(n, np.float32) for n in SIZES] for k in "mv"}, shift)
    dst.convert_to(back)
    for i, n in enumerate(SIZES):
        for k in "mv":
            if n == 0:
                continue
            value = bv[k].get()[i]
            assert np.array_equal(value.astype(np.float64), ref.decode(got[k][i], got[k + "_exp"][i], k), equal_nan=True)
            x = np.where((host[k][i] < 0) & (k == "v"), 0, host[k][i]).astype(np.float64)
            low = 2.0 ** (np.maximum(got[k + "_exp"][i].astype(int), ref.SPAN[k] + 1) - 127.0 - ref.SPAN[k])
            low = np.repeat(low, 256)[:n]
            fine = np.repeat(got[k + "_exp"][i] < 255, 256)[:n]
            step = (1 / 8 if rounding else 1 / 16) * np.abs(x)
            assert (np.abs(value - x)[fine] <= (step + 1.25 * low)[fine]).all()
            if k == "v":
                assert ((value > 0) == (x > 0))[fine].all()


def test_random_rounding_is_unbiased_and_new_at_every_step():
    """One block of equal second moments, coded under 4,096 seeds: the mean of the values is the moment, within 5 standard
    errors of a rounding whose two outcomes are a step apart."""
    n, seeds = 256, 512
    x = np.linspace(1.0, 1.875, n).astype(np.float32)
    m = Buffers([x])
    src = fr.OptPlan(m=m.tensors, v=m.tensors)
    codes = [torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in range(2)]
    exps = [torch.zeros(1, dtype=torch.uint8, device="cuda") for _ in range(2)]
    dst = fr.OptPlan(m=codes[:1], v=codes[1:], m_exp=exps[:1], v_exp=exps[1:])
    values = [torch.zeros(n, device="cuda") for _ in range(2)]
    back = fr.OptPlan(m=values[:1], v=values[1:])
    total = [np.zeros(n), np.zeros(n)]
    seen = set()
    for s in range(seeds):
        src.convert_to(dst, fr.FR_ROUND_RANDOM, s)
        dst.convert_to(back)
        for k in range(2):
            total[k] += values[k].cpu().numpy()
        seen.add(codes[0].cpu().numpy().tobytes())
    assert len(seen) == seeds
    frac = (x.astype(np.float64) * 8) % 1
    for k in range(2):
        err = total[k] / seeds - x
        sd = np.sqrt(frac * (1 - frac) / seeds) / 8 + 2.0 ** -16
        assert (np.abs(err) <= 5 * sd).all()
        assert abs(err.mean()) <= 5 * np.sqrt((sd ** 2).mean() / n)


# ---------------------------------------------------------------- refusals

def _refused(status, call, *args, **kw):
    with pytest.raises(fr.FlashrecError) as e:
        call(*args, **kw)
    assert e.value.status == status, fr.fr_last_error()


def test_refusals():
    import ctypes

    n = 300
    f = lambda: torch.zeros(n, device="cuda")  # noqa: E731
    h = lambda: torch.zeros(n, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    u = lambda k=n: torch.zeros(k, dtype=torch.uint8, device="cuda")  # noqa: E731
    whole = fr.OptPlan([h()], [h()], [f()], [f()], masters=[f()])
    ok = fr.fr_adamw(1e-3, 0.9, 0.99, 1e-8, 0.0, 1, 0, 0)
    whole.step(ok)
    # numbers out of range
    for field, bad in [("lr", -1.0), ("lr", math.nan), ("beta1", 1.0), ("beta1", -0.1), ("beta2", 1.0), ("beta2", math.nan),
                       ("eps", 0.0), ("eps", math.inf), ("eps", 1e-60), ("weight_decay", -0.5), ("weight_decay", math.inf), ("step", 0),
                       ("rounding", 2), ("reserved", 1)]:
        x = fr.fr_adamw(1e-3, 0.9, 0.99, 1e-8, 0.0, 1, 0, 0)
        setattr(x, field, bad)
        _refused(fr.FR_ERR_INVALID_ARG, whole.step, x)
    for norm, scale in [(0.0, 1.0), (-1.0, 1.0), (math.nan, 1.0), (1.0, 0.0), (1.0, math.inf), (1.0, -1.0), (1.0, math.nan)]:
        _refused(fr.FR_ERR_INVALID_ARG, whole.clip, norm, scale)
    # a plan without what the call needs
    grads = fr.OptPlan(grads=[f()])
    grads.clip()
    _refused(fr.FR_ERR_INVALID_ARG, grads.step, ok)
    moments = fr.OptPlan(m=[f()], v=[f()])
    _refused(fr.FR_ERR_INVALID_ARG, moments.clip)
    _refused(fr.FR_ERR_INVALID_ARG, moments.convert_to, grads)
    partial = fr.OptPlan([f(), f()], [f(), None], [f(), f()], [f(), f()])
    _refused(fr.FR_ERR_INVALID_ARG, partial.step, ok)
    _refused(fr.FR_ERR_INVALID_ARG, partial.clip)
    # conversions
    eight = fr.OptPlan(m=[u()], v=[u()], m_exp=[u(2)], v_exp=[u(2)])
    _refused(fr.FR_ERR_INVALID_ARG, moments.convert_to, moments)
    _refused(fr.FR_ERR_INVALID_ARG, eight.convert_to, eight)
    _refused(fr.FR_ERR_INVALID_ARG, moments.convert_to, eight, 2)
    _refused(fr.FR_ERR_PLAN_MISMATCH, moments.convert_to, fr.OptPlan(m=[u(299)], v=[u(299)], m_exp=[u(2)], v_exp=[u(2)]))
    mixed = fr.OptPlan(m=[f(), u()], v=[f(), u()], m_exp=[None, u(2)], v_exp=[None, u(2)])
    _refused(fr.FR_ERR_INVALID_ARG, fr.OptPlan(m=[f(), f()], v=[f(), f()]).convert_to, mixed)
    # lists that do not fit together, caught before the library
    for bad in [dict(weights=[f()], grads=[torch.zeros(299, device="cuda")]), dict(m=[u()], v=[u()], m_exp=[u(1)], v_exp=[u(2)]),
                dict(m=[f()], v=[u()]), dict(weights=[f()], grads=[f(), f()]), dict(grads=[torch.zeros(n)]),
                dict(grads=[torch.zeros(n, 2, device="cuda")[:, 0]]), dict(grads=[torch.zeros(n, dtype=torch.float16, device="cuda")]),
                dict(grads=[f()], lr_scale=[1.0, 2.0]), dict()]:
        with pytest.raises(ValueError):
            fr.OptPlan(**bad)
    # and by it
    def create(**fields):
        a, b, c, d = f(), f(), f(), f()
        t = fr.fr_opt_tensor(a.data_ptr(), b.data_ptr(), None, c.data_ptr(), d.data_ptr(), None, None, n, fr.FR_DT_F32, fr.FR_DT_F32,
                             fr.FR_DT_F32, 0, 1.0, 1.0)
        for k, x in fields.items():
            setattr(t, k, x)
        handle = ctypes.c_void_p()
        st = fr.lib.fr_opt_create(ctypes.byref(t), 1, ctypes.byref(handle))
        assert (st == fr.FR_OK) == bool(handle.value)
        fr.lib.fr_opt_destroy(handle)
        return st

    p = f().data_ptr()
    assert create() == fr.FR_OK
    for bad in [dict(weight_dtype=0), dict(weight_dtype=7), dict(grad_dtype=0), dict(state_dtype=fr.FR_DT_BF16), dict(flags=1),
                dict(m=None), dict(v=None), dict(m_exp=p), dict(state_dtype=0), dict(state_dtype=0, m_exp=p), dict(master=p),
                dict(weight=None, master=p), dict(lr_scale=math.nan), dict(decay_scale=math.inf), dict(n=1 << 60)]:
        assert create(**bad) == fr.FR_ERR_INVALID_ARG, bad
    for bad in [dict(weight=p + 2), dict(grad=p + 1), dict(m=p + 1), dict(v=p + 3),
                dict(weight=p, weight_dtype=fr.FR_DT_BF16, master=p + 2)]:
        assert create(**bad) == fr.FR_ERR_ALIGNMENT, bad
    # records
    for rec in (torch.zeros(8, dtype=torch.uint8, device="cuda"), torch.zeros(16, dtype=torch.uint8)):
        with pytest.raises(ValueError):
            whole.clip(out=rec)
    odd = torch.zeros(20, dtype=torch.uint8, device="cuda")[4:]
    _refused(fr.FR_ERR_INVALID_ARG, whole.clip, out=odd)
    _refused(fr.FR_ERR_INVALID_ARG, whole.step, ok, odd)
    assert fr.lib.fr_grad_clip(None, 1.0, 1.0, p, None) == fr.FR_ERR_INVALID_ARG
    assert fr.lib.fr_grad_clip(whole.handle, 1.0, 1.0, None, None) == fr.FR_ERR_INVALID_ARG
    assert fr.lib.fr_adamw_step(whole.handle, None, None, None) == fr.FR_ERR_INVALID_ARG
    assert fr.lib.fr_opt_create(None, 1, ctypes.byref(ctypes.c_void_p())) == fr.FR_ERR_INVALID_ARG
    assert fr.lib.fr_opt_create(None, 0, None) == fr.FR_ERR_INVALID_ARG
    assert fr.lib.fr_opt_info(None, None, None, None) == fr.FR_ERR_INVALID_ARG
    assert fr.fr_opt_info(whole.handle) == (1, n, 2)


def test_empty_lists_do_nothing():
    e = torch.empty(0, device="cuda")
    for plan in (fr.OptPlan([], [], [], []), fr.OptPlan([e], [e], [e], [e])):
        plan.step(fr.fr_adamw(1e-3, 0.9, 0.99, 1e-8, 0.0, 1, 0, 0))
        assert plan.n_elems == 0 and plan.n_blocks == 0
    torch.cuda.synchronize()
