"""The orthogonalised update on the GPU against its definition in 64 bits (tests/muon_reference.py): momenta bit for bit, O
and the weights within bounds that count the fp16 roundings of the products and each type's own."""
import numpy as np
import pytest
import torch

import muon_reference as mref
import optim_reference as ref
from test_gpu_optim import Buffers, _record, _wide

pytestmark = pytest.mark.gpu

fr = pytest.importorskip("paper_2509_03047_gb300.flashrec")

SHAPES = [(1, 1), (1, 300), (300, 1), (0, 5), (64, 64), (33, 200), (200, 7), (128, 128), (129, 257), (257, 129), (130, 1000),
          (1000, 130), (5, 0), (384, 640), (7, 7), (256, 128), (520, 260)]
SMALL = [(33, 200), (0, 5), (200, 7), (129, 130), (1, 70)]


@pytest.fixture(autouse=True)
def _free_memory():
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def _views(b, shapes):
    return [t.view(s) for t, s in zip(b.tensors, shapes)]


def _near(got, want, rel, note):
    """2-norms over the matrix."""
    err = np.linalg.norm((got.astype(np.float64) - want).ravel())
    assert err <= rel * np.linalg.norm(want.ravel()) + 1e-300, (note, err / np.linalg.norm(want.ravel()), rel)


def _orthogonalize(gs, grad="f32", update="f32", shift=0, coefficients=mref.USUAL, products=0, **more):
    """(gradients as the library reads them, its updates)"""
    shapes = [g.shape for g in gs]
    flat = [g.ravel() if grad == "f32" else ref.f32_to_bf16(g.ravel()) for g in gs]
    b = Buffers(flat, shift)
    u = Buffers([np.zeros(g.size, np.float32 if update == "f32" else np.uint16) for g in gs], shift)
    plan = fr.MuonPlan(grads=_views(b, shapes), updates=_views(u, shapes), **more)
    plan.orthogonalize(fr.muon(coefficients=coefficients, products=products))
    torch.cuda.synchronize()
    b.check()
    return [_wide(x).reshape(s) for x, s in zip(flat, shapes)], [_wide(x).reshape(s) for x, s in zip(u.get(), shapes)]


def _bound(kind, shape, coefficients=mref.USUAL, products=0):
    """Of O in an output of this type, its own rounding included."""
    split = kind == "f32" and products == fr.FR_MUON_BY_TYPE
    return mref.bound(coefficients, split, shape) + (2.0 ** -8 if kind == "bf16" else 2.0 ** -24)


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("grad,update", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
def test_orthogonalize_is_its_definition(grad, update, shift):
    rng = np.random.default_rng(5)
    scale = [1.0 + i % 3 for i in range(len(SHAPES))]
    gs, got = _orthogonalize([mref.matrix(rng, *s) for s in SHAPES], grad, update, shift, update_scale=scale)
    for g, o, x in zip(gs, got, scale):
        if g.size:
            _near(o, x * mref.orthogonal(g), _bound(update, g.shape), g.shape)


@pytest.mark.parametrize("products", [0, 1])
@pytest.mark.parametrize("kind", ["lowrank", "decay", "spiky"])
def test_hard_spectra(kind, products):
    rng = np.random.default_rng(6)
    gs, got = _orthogonalize([mref.matrix(rng, *s, kind) for s in [(128, 128), (300, 700), (700, 300), (512, 512)]], products=products)
    for g, o in zip(gs, got):
        _near(o, mref.orthogonal(g), _bound("f32", g.shape, products=products), (kind, g.shape))


@pytest.mark.parametrize("grad", ["f32", "bf16"])
def test_products_of_one_half(grad):
    rng = np.random.default_rng(5)
    gs, got = _orthogonalize([mref.matrix(rng, *s) for s in SHAPES], grad, products=fr.FR_MUON_ONE)
    for g, o in zip(gs, got):
        if g.size:
            _near(o, mref.orthogonal(g), _bound("f32", g.shape, products=fr.FR_MUON_ONE), g.shape)


def test_a_list_of_both_kinds():
    """Matrices with fp32 outputs and others in one plan: each as alone."""
    rng = np.random.default_rng(18)
    shapes = [(200, 300), (300, 130), (64, 64), (257, 256)]
    gs = [torch.from_numpy(mref.matrix(rng, *s)).cuda() for s in shapes]
    kinds = [torch.float32, torch.bfloat16, torch.bfloat16, torch.float32]
    outs = [torch.zeros(s, dtype=k, device="cuda") for s, k in zip(shapes, kinds)]
    fr.MuonPlan(grads=gs, updates=outs).orthogonalize()
    for g, o in zip(gs, outs):
        alone = torch.zeros_like(o)
        fr.MuonPlan(grads=[g], updates=[alone]).orthogonalize()
        assert torch.equal(alone, o)


@pytest.mark.parametrize("coefficients", [((1.5, -0.5, 0.0),) * 10, ((2.0, -1.5, 0.5),), ((3.4445, -4.7750, 2.0315),) * 2,
                                          ((0.0, 0.0, 0.0),), ((1.0, 0.0, 0.0),) * 3, ((-1.0, 0.25, 0.0),) * 3])
def test_other_polynomials(coefficients):
    rng = np.random.default_rng(7)
    gs, got = _orthogonalize([mref.matrix(rng, *s) for s in [(130, 300), (300, 130), (64, 64)]], coefficients=coefficients)
    for g, o in zip(gs, got):
        _near(o, mref.orthogonal(g, coefficients), _bound("f32", g.shape, coefficients), (coefficients, g.shape))


def test_scales_of_a_matrix_and_its_empty_and_nonfinite_ones():
    """O does not depend on the matrix's size, from subnormals to the largest numbers; zeros give zeros, a non-finite
    element NaNs in its matrix alone."""
    rng = np.random.default_rng(8)
    base = mref.matrix(rng, 130, 70)
    base /= np.abs(base).max()
    gs = [base * np.float32(s) for s in (3e38, 1e20, 1.0, 1e-20, 2.0 ** -126)]
    tiny = (rng.integers(-40, 40, size=(130, 70)) * 2.0 ** -149).astype(np.float32)
    one = np.zeros((130, 70), np.float32)
    one[129, 69] = 2.0 ** -149
    bad = base.copy()
    bad[77, 3] = np.nan
    worse = base.copy()
    worse[0, 0] = -np.inf
    gs += [tiny, one, np.zeros_like(base), bad, worse, base]
    _, got = _orthogonalize(gs)
    for g, o in zip(gs, got):
        if np.isfinite(g).all():
            _near(o, mref.orthogonal(g), _bound("f32", g.shape), float(np.abs(g).max()))
        else:
            assert np.isnan(o).all()


def _mix(p, x, h):
    """beta x + (1 - beta) h, each operation rounded to fp32"""
    beta, rest = np.float32(p["beta"]), np.float32(1.0 - p["beta"])
    return (x * beta + h * rest).astype(np.float32)


class Step:
    """A list's buffers, its plan, and what a step makes of them by the definition."""

    def __init__(self, shapes, param, grad, shift=0, seed=3, **numbers):
        rng = np.random.default_rng(seed)
        self.shapes, self.param = shapes, param
        gs = [mref.matrix(rng, *s) for s in shapes]
        host = {"grad": [g.ravel() if grad == "f32" else ref.f32_to_bf16(g.ravel()) for g in gs],
                "momentum": [mref.matrix(rng, *s).ravel() * np.float32(0.4) for s in shapes]}
        w = [(rng.normal(size=g.size) * 0.02).astype(np.float32) for g in gs]
        host["weight"] = w if param == "f32" else [ref.f32_to_bf16(x) for x in w]
        if param == "master":
            host["master"] = [ref.bf16_to_f32(x) + np.float32(1e-5) for x in host["weight"]]
        self.host = host
        self.b = {k: Buffers(v, shift) for k, v in host.items()}
        self.factors = {"lr_scale": [1.0 + 0.5 * (i % 2) for i in range(len(shapes))],
                        "decay_scale": [float(i % 3 != 1) for i in range(len(shapes))],
                        "update_scale": [0.2 * max(1, *s) ** 0.5 for s in shapes]}
        names = {"grad": "grads", "momentum": "momenta", "weight": "weights", "master": "masters"}
        self.plan = fr.MuonPlan(**{names[k]: _views(x, shapes) for k, x in self.b.items()}, **self.factors)
        self.p = dict(dict(lr=3e-3, beta=0.95, weight_decay=0.1, nesterov=True, step=3, seed=9), **numbers)

    def hyper(self, **more):
        return fr.muon(**dict(self.p, **more))

    def get(self):
        return {k: [_wide(x).reshape(s) if k != "weight" or self.param == "f32" else x.reshape(s) for x, s in zip(b.get(), self.shapes)]
                for k, b in self.b.items()}

    def check(self, scale):
        got, p = self.get(), self.p
        for i, s in enumerate(self.shapes):
            if 0 in s:
                continue
            h = (_wide(self.host["grad"][i]) * np.float32(scale)).astype(np.float32)
            m = _mix(p, self.host["momentum"][i], h)
            assert np.array_equal(got["momentum"][i].ravel().view(np.uint32), m.view(np.uint32)), s
            g = (_mix(p, m, h) if p["nesterov"] else m).reshape(s)
            old = _wide(self.host["master" if self.param == "master" else "weight"][i]).astype(np.float64).reshape(s)
            f = {k: x[i] for k, x in self.factors.items()}
            u = f["update_scale"] * mref.orthogonal(g)
            want = old - p["lr"] * f["lr_scale"] * (u + p["weight_decay"] * f["decay_scale"] * old)
            new = got["master" if self.param == "master" else "weight"][i]
            if new.dtype == np.uint16:
                new = ref.bf16_to_f32(new)
            # the update's own error, the sum's in fp32 (products, sums and lr: four roundings), a bf16 weight's rounding
            # (at random: a whole step)
            bound = mref.bound(split=self.param != "bf16" and not p.get("products"), shape=s)
            slack = p["lr"] * f["lr_scale"] * bound * np.linalg.norm(u) + 4 * 2.0 ** -24 * np.linalg.norm(old)
            if self.param == "bf16":
                slack += (2.0 ** -7 if p.get("rounding") else 2.0 ** -8) * np.linalg.norm(want)
            assert np.linalg.norm(new.astype(np.float64) - want) <= slack, (s, np.linalg.norm(new - want) / slack)
            if self.param == "master":
                assert np.array_equal(got["weight"][i], ref.f32_to_bf16(got["master"][i].ravel()).reshape(s))
        self.b["grad"].check()


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("grad", ["bf16", "f32"])
@pytest.mark.parametrize("param", ["master", "bf16", "f32"])
def test_step_is_its_definition(param, grad, nesterov, shift):
    s = Step(SHAPES, param, grad, shift, nesterov=nesterov)
    s.plan.step(s.hyper(), _record(0.37109375))
    torch.cuda.synchronize()
    s.check(0.37109375)


@pytest.mark.parametrize("param", ["master", "f32"])
def test_step_with_products_of_one_half(param):
    s = Step(SHAPES, param, "bf16", products=fr.FR_MUON_ONE)
    s.plan.step(s.hyper(), _record(0.5))
    torch.cuda.synchronize()
    s.check(0.5)


def test_step_without_a_record_and_without_momentum():
    s = Step(SMALL, "master", "f32", beta=0.0, nesterov=False)
    s.plan.step(s.hyper())
    torch.cuda.synchronize()
    s.check(1.0)


@pytest.mark.parametrize("shift", [0, 1])
def test_random_rounding_of_weights_is_near_and_unbiased(shift):
    s = Step([(256, 512), (3, 5)], "bf16", "bf16", shift, rounding=fr.FR_ROUND_RANDOM)
    s.plan.step(s.hyper(), _record(1.0))
    torch.cuda.synchronize()
    s.check(1.0)
    # the same step with fp32 weights, by the same products, gives what was rounded
    f = Step([(256, 512), (3, 5)], "f32", "bf16", shift, products=fr.FR_MUON_ONE)
    for t, x in zip(f.b["weight"].tensors, s.host["weight"]):
        t.copy_(torch.from_numpy(ref.bf16_to_f32(x)))
    f.plan.step(f.hyper(), _record(1.0))
    torch.cuda.synchronize()
    exact = f.get()["weight"][0].astype(np.float64).ravel()
    got = ref.bf16_to_f32(s.get()["weight"][0].ravel()).astype(np.float64)
    step = np.exp2(np.floor(np.log2(np.abs(exact))) - 7)
    off = (got - exact) / step
    assert np.abs(off).max() <= 1.0
    # of n independent roundings: a variance of at most 1/4 each; five standard deviations
    assert abs(off.mean()) <= 5 * 0.5 / np.sqrt(off.size)


@pytest.mark.parametrize("param", ["master", "bf16", "f32"])
def test_step_leaves_every_byte_when_a_gradient_is_not_finite(param):
    s = Step(SMALL, param, "bf16", 1)
    before = s.get()
    s.plan.step(s.hyper(), _record(0.5, nonfinite=1))
    torch.cuda.synchronize()
    after = s.get()
    for k in before:
        for a, b in zip(before[k], after[k]):
            assert a.tobytes() == b.tobytes()
    s.plan.step(s.hyper(), _record(0.5))  # the plan's own counters are as they were
    torch.cuda.synchronize()
    s.check(0.5)


@pytest.mark.parametrize("param,rounding", [("master", 0), ("bf16", 1)])
def test_replicas_at_other_addresses_stay_bit_identical(param, rounding):
    a, b = (Step(SHAPES, param, "bf16", shift, rounding=rounding) for shift in (0, 1))
    for step in (1, 2, 3):
        for s in (a, b):
            s.plan.step(s.hyper(step=step), _record(0.7))
    torch.cuda.synchronize()
    x, y = a.get(), b.get()
    for k in x:
        for p, q in zip(x[k], y[k]):
            assert p.tobytes() == q.tobytes(), k


def test_a_matrix_gives_the_same_bits_in_any_list():
    rng = np.random.default_rng(12)
    some = [mref.matrix(rng, *s) for s in [(300, 200), (64, 700), (513, 129)]]
    _, alone = _orthogonalize(some[1:2])
    _, among = _orthogonalize([some[0], some[2], some[1], some[0]])
    assert alone[0].tobytes() == among[2].tobytes()


def test_calls_back_to_back_and_from_a_graph_equal_calls_with_waits():
    want = Step(SMALL, "master", "bf16")
    for _ in range(3):
        want.plan.step(want.hyper(), _record(0.5))
        torch.cuda.synchronize()
    quick = Step(SMALL, "master", "bf16")
    record, stream = _record(0.5), torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        quick.plan.step(quick.hyper(), record, stream=stream)
    graphed = Step(SMALL, "master", "bf16")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        graphed.plan.step(graphed.hyper(), record)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    a, b, c = want.get(), quick.get(), graphed.get()
    for k in a:
        for x, y, z in zip(a[k], b[k], c[k]):
            assert x.tobytes() == y.tobytes() == z.tobytes(), k


def test_two_plans_on_two_streams():
    rng = np.random.default_rng(14)
    gs = [mref.matrix(rng, 400, 300), mref.matrix(rng, 300, 500)]
    _, want = zip(*[_orthogonalize([g]) for g in gs])
    streams = [torch.cuda.Stream() for _ in gs]
    dev = [torch.from_numpy(g).cuda() for g in gs]
    outs = [torch.zeros_like(g) for g in dev]
    plans = [fr.MuonPlan(grads=[g], updates=[o]) for g, o in zip(dev, outs)]
    torch.cuda.synchronize()
    for _ in range(4):
        for p, s in zip(plans, streams):
            p.orthogonalize(stream=s)
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert o.cpu().numpy().tobytes() == w[0].tobytes()


@pytest.mark.parametrize("shape", [(1, 1 << 20), (1 << 18, 2), (1500, 3000), (2049, 1025)])
def test_long_and_large(shape):
    rng = np.random.default_rng(15)
    gs, got = _orthogonalize([mref.matrix(rng, *shape, "half" if min(shape) > 2 else "plain")], "bf16", "bf16")
    _near(got[0], mref.orthogonal(gs[0]), _bound("bf16", shape), shape)


@pytest.mark.parametrize("shape", [(1, 1 << 20), (1500, 3000), (2049, 1025)])
def test_long_and_large_in_fp32(shape):
    rng = np.random.default_rng(16)
    gs, got = _orthogonalize([mref.matrix(rng, *shape, "half" if min(shape) > 2 else "plain")])
    _near(got[0], mref.orthogonal(gs[0]), _bound("f32", shape), shape)


def test_empty_lists_do_nothing():
    fr.MuonPlan(grads=[], updates=[]).orthogonalize()
    e = [torch.empty(0, 4, device="cuda")]
    plan = fr.MuonPlan(e, e, e)
    plan.step(fr.muon(lr=1.0))
    assert plan.n_elems == 0
    torch.cuda.synchronize()


def test_a_matrix_gives_the_same_bits_in_a_long_list():
    """One whose phases fill the SMs has wider tiles."""
    rng = np.random.default_rng(19)
    g = mref.matrix(rng, 700, 520)
    for update in ("bf16", "f32"):
        _, alone = _orthogonalize([g], update=update)
        _, among = _orthogonalize([g] * 40, update=update)
        for o in among:
            assert alone[0].tobytes() == o.tobytes()


@pytest.mark.parametrize("param", ["master", "bf16"])
def test_a_long_list_from_a_graph(param):
    """More tiles than go through all iterations in one launch."""
    shapes = [(600, 700)] * 30 + [(1024, 1100)] * 12 + [(300, 200)] * 40
    eager, graphed = (Step(shapes, param, "bf16") for _ in range(2))
    record, graph = _record(0.5), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        graphed.plan.step(graphed.hyper(), record)
    eager.plan.step(eager.hyper(), record)
    graph.replay()
    torch.cuda.synchronize()
    assert eager.plan.sync_status() == graphed.plan.sync_status() == fr.FR_OK
    a, b = eager.get(), graphed.get()
    for k in a:
        for x, y in zip(a[k], b[k]):
            assert x.tobytes() == y.tobytes()
    eager.check(0.5)


def test_refused_calls_leave_everything():
    s = Step(SMALL, "bf16", "bf16")
    before = s.get()
    for change in (dict(lr=-1.0), dict(lr=float("nan")), dict(beta=1.0), dict(step=0), dict(coefficients=[(16.0, 0.0, 0.0)]), dict(rounding=2),
                   dict(products=2), dict(weight_decay=float("inf"))):
        with pytest.raises(fr.FlashrecError):
            s.plan.step(s.hyper(**change))
    with pytest.raises(fr.FlashrecError, match="update"):
        s.plan.orthogonalize()
    with pytest.raises(ValueError):
        s.plan.step(s.hyper(), torch.zeros(2, dtype=torch.int64))
    torch.cuda.synchronize()
    after = s.get()
    for k in before:
        for x, y in zip(before[k], after[k]):
            assert x.tobytes() == y.tobytes()
